"""The backward pass reads staged keys and values after every wavefront has written its part of them: what earlier kernels
left in the LDS (here NaN, from attention over keys that are NaN) never shows."""
import pytest
import torch

import test_gpu_draft_attn as attn
import test_gpu_qcache as base

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2609_31093_amd import pisa


@pytest.mark.parametrize("C", [32, 64, 96, 128])
@pytest.mark.parametrize("d", [64, 128])
def test_lds_left_by_others(C, d):
    N, K = 5000, 12
    p = base.problem(1, 4, 2, N, N, d, C, 2, K, 1, "bf16")
    q, k, v, d_o = (base.normal((1, h, N, d), i, "bf16") for i, h in enumerate((4, 2, 2, 4)))
    idx = pisa.select(p, q, k, pisa.build_pyramid(p, k))
    o, lse = pisa.sparse_attn_fwd(p, q, k, v, idx)
    # 2048 wavefronts with keys of NaN in their LDS, 64 KB a workgroup
    far = attn.problem((2, 16, 8, 128, 4000, 128, 64, 2, 16, "bf16", 0))
    bad = tuple(torch.full((2, 8, 4128, 128), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    fill = [far, bad, base.normal((2, 16, 128, 128), 5, "bf16"), attn.selection(far, 4), *attn.drafted(far, 6, "bf16"), attn.trees(2, 128, 7)]
    first = None
    for _ in range(12):
        attn.attend(*fill)
        got = pisa.sparse_attn_bwd(p, q, k, v, idx, o, lse, d_o)
        assert all(bool(torch.isfinite(x).all()) for x in got)
        first = got if first is None else first
        assert torch.equal(got[0], first[0])  # dq is summed in order
        for x, y in zip(got[1:], first[1:]):
            # up to n = 2 * 5000 terms that atomics add in any order, 2 n 2^-24 of their magnitudes, and a step of bf16
            assert (x.double() - y.double()).norm() <= 2.0 ** -6 * y.double().norm()
