"""Weights of drafted tokens' attention against 64 bits where values nearly cancel, so that the result's own rounding does
not hide how far the weights are off.

Tolerance: that of test_gpu_draft_attn.py, with weights off by 2^-16 for bf16 values (two bf16 terms) and 2^-21 for 8-bit
ones in bf16 problems: a first fp16 term is off by 2^-11 of the weight at most, a second by 2^-11 of that, or by 2^-25 where
it is a subnormal number, 2^-39 of the largest weight; twice 2^-22 leaves room for both."""
import math

import numpy as np
import pytest
import torch

import test_gpu_draft_attn as attn
import test_gpu_qcache as base

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2609_31093_amd import pisa


def opposite(B, Hkv, n, d, seed, dtype):
    """n rows, an even number: each value's negative follows it."""
    x = base.normal((B, Hkv, n // 2, 1, d), seed, dtype)
    return torch.cat((x, -x), 3).flatten(2, 3).contiguous()


@pytest.mark.parametrize("eight", [False, True], ids=["raw", "8bit"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,C,n,T", [(128, 64, 2, 40), (64, 64, 2, 40), (64, 32, 6, 33), (128, 96, 4, 17)])
def test_values_that_cancel(eight, dtype, d, C, n, T):
    """Every row sees a few cached keys, or a few drafted ones, of nearly equal logits."""
    B, H, Hkv = 2, 8, 2
    p = base.problem(B, H, Hkv, T, n + T, d, C, 2, 3, 1, dtype, 0)
    k, v = base.normal((B, Hkv, n, d), 1, dtype), opposite(B, Hkv, n, d, 2, dtype)
    if eight:
        cache = pisa.make_qcache(p)
        pisa.qcache_append(base.at(p, n), cache, k, v, 0)
    else:
        cache = tuple(torch.nn.functional.pad(x, (0, 0, 0, T)).contiguous() for x in (k, v))
    q = base.normal((B, H, T, d), 3, dtype) * 0.02
    k_new, v_new = base.normal((B, Hkv, T, d), 4, dtype), opposite(B, Hkv, T + T % 2, d, 5, dtype)[:, :, :T].contiguous()
    idx = torch.full((B, Hkv, T, 3), -1, dtype=torch.int32, device="cuda")
    mask = torch.zeros((B, T, 1), dtype=torch.int64, device="cuda")
    idx[:, :, ::2, 1] = 0             # even rows: the cached keys
    mask[:, 1::2] = (1 << n) - 1      # odd rows: the first n drafted ones
    o = attn.attend(p, cache, q, idx, k_new, v_new, mask)[0].double().cpu().numpy()

    held = attn.stored(p, cache)
    new = tuple(x.double().cpu().numpy() for x in (k_new, v_new))
    q64, G, wide = q.double().cpu().numpy(), H // Hkv, 0
    for b, h, r in np.ndindex(B, H, T):
        kt, vt = ((held, new)[r % 2][i][b, h // G, :n] for i in range(2))
        z = kt @ q64[b, h, r] / math.sqrt(d)
        w = np.exp(z - z.max())
        w /= w.sum()
        want = w @ vt
        delta = (d + 5) * 2.0 ** -24 * (abs(kt) @ abs(q64[b, h, r])).max() / math.sqrt(d)
        rel = math.expm1(2 * delta) + 2.0 ** -21 + 2.0 ** -23 * (z.max() - z).max()
        # drafted values are bf16 over an 8-bit cache too
        term = 0.0 if dtype == "f32" else 2.0 ** -21 if eight and r % 2 == 0 else 2.0 ** -16
        half = 2.0 ** -8 if dtype == "bf16" else 0.0
        tol = (2 * rel + term + 2 * n * 2.0 ** -23) * (w @ abs(vt)) + (half + 2.0 ** -22) * abs(want)
        off = abs(o[b, h, r] - want) - tol
        assert (off <= 0).all(), (b, h, r, off.max(), tol.max())
        wide += int((tol < 2.0 ** -13 * (w @ abs(vt))).sum())
    # most results tell a weight that is off by 2^-12 from one that is not
    assert wide > 0.2 * o.size
