"""More rows of queries and keys than the workgroups of one launch, which go on to other rows: each row's norm and gradient
are those of a call with few rows.

Tolerance.  The compiler may fuse products and sums otherwise in another iteration of a loop, so two calls agree within twice
the tolerance of test_gpu_norm_rope.py, here by the largest values of a head (d of them, w and dy its weights and its output's
gradient, inv = 1 / sqrt(mean(x^2) + eps)).  Outputs: a turned pair's |a| + |b| is at most 2 sqrt(2) of the head's largest
output, so (2^-19 + 2^-21) 3 max|y|.  Gradients: e <= 2^-20 max|dy|, |u| <= sqrt(2) max|dy|, and by Cauchy's inequality, with
inv |x|_2 <= sqrt(d), what follows |x| inv^2 / d is at most |x| inv <= sqrt(d) times its largest term: inv (1 + sqrt(d)) max|w|
max|dy| (2^-20 + sqrt(2) 2^-17), which is below inv (1 + sqrt(d)) max|w| max|dy| 2^-16.  bf16 results another 2^-8 of
themselves."""
import pytest
import torch

import test_gpu_norm_rope as norm

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2609_31093_amd import pisa


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout,rot", [("half", 42), ("half", 64), ("interleaved", 42)])
def test_rows_of_long_calls(dtype, layout, rot):
    B, H, N, d, part = 2, 2, 70011, 64, 9000
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k, gq, gk = (torch.randn((B, h, N, d), generator=gen, device="cuda").to(norm.TYPES[dtype]) for h in (H, 1, H, 1))
    w = norm.weights(d, 2, dtype, 0.0)
    pos = torch.arange(N, dtype=torch.int32, device="cuda") * 3 % 50021

    def both(q, k, gq, gk, pos):
        r = pisa.make_rope(B, H, 1, q.shape[2], d, rot=rot, layout=layout, dtype=dtype)
        m = pisa.make_qk_norm(r, w, w)
        return (*pisa.norm_rope_fwd(r, m, q, k, pos), *pisa.norm_rope_bwd(r, m, q, k, gq, gk, pos))

    whole = both(q, k, gq, gk, pos)
    sums = [torch.zeros(d, dtype=torch.float64, device="cuda") for _ in range(2)]
    for i in range(0, N, part):
        few = both(*(x[:, :, i:i + part] for x in (q, k, gq, gk)), pos[i:i + part].contiguous())
        for j, (x, dy) in enumerate(((q, gq), (k, gk))):
            y, dx, x, dy = few[j].double(), few[2 + j].double(), x[:, :, i:i + part].double(), dy[:, :, i:i + part].double()
            inv = 1 / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt()
            tol_y = (2.0 ** -19 + 2.0 ** -21) * 3 * y.abs().amax(-1, keepdim=True)
            tol_dx = inv * (1 + d ** 0.5) * w.double().abs().max() * dy.abs().amax(-1, keepdim=True) * 2.0 ** -16
            for got, want, tol in ((whole[j], y, tol_y), (whole[2 + j], dx, tol_dx)):
                off = (got[:, :, i:i + part].double() - want).abs()
                assert (off <= 2 * (tol + (2.0 ** -8 * want.abs() if dtype == "bf16" else 0))).all(), off.max()
        for s, b in zip(sums, few[4:]):
            s += b.double()
    # sums of n values: off by 2^-24 of what they sum for each addition of a chain, here at most n / 64 rows of a thread
    # and the parts' 2^10 on either side; |u x r| is below 60
    for a, s, h in zip(whole[4:], sums, (H, 1)):
        assert ((a.double() - s).abs() <= 2 * (B * h * N / 64 + 1024) * 2.0 ** -24 * 60 * B * h * N).all()
