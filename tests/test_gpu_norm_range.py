"""Norms of queries and keys whose values, weights or gradients lie far from 1: what the formula's result has within the
type's range comes out, though products of two of its factors are beyond it.  Reference and tolerances of
test_gpu_norm_rope.py, all of them relative.  A gradient's last product, r times a normal number, may be a subnormal one,
whose rounding is off by half of its step whatever its size: 2^-150, and in bf16 2^-134 on top of it."""
import numpy as np
import pytest
import torch

import test_gpu_norm_rope as norm

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2609_31093_amd import pisa


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout,rot", [("half", 128), ("half", 90), ("interleaved", 64)])
@pytest.mark.parametrize("x,w,dy,eps", [(1e-17, 1e25, 1e-5, 1e-30), (1e18, 1e-25, 1.0, 1e-5), (1e17, 1e12, 1e12, 1e-5), (1e17, 1.0, 1e-15, 1e-5),
                                        (1e-12, 1.0, 1e-12, 1e-20)])
def test_far_from_one(dtype, layout, rot, x, w, dy, eps):
    B, H, N, d = 1, 2, 33, 128
    r = pisa.make_rope(B, H, H, N, d, rot=rot, layout=layout, dtype=dtype, pos0=3)
    weight = norm.normal((d,), 1, dtype, 0.25 * w) + w
    m = pisa.make_qk_norm(r, weight, None, eps=eps)
    q, g = norm.normal((B, H, N, d), 2, dtype, x), norm.normal((B, H, N, d), 3, dtype, dy)
    y, _ = pisa.norm_rope_fwd(r, m, q)
    dx, _, dw, _ = pisa.norm_rope_bwd(r, m, q, None, g, None)
    pos, x64, w64, eps = np.broadcast_to(3 + np.arange(N), (B, N)), norm.numbers(q), norm.numbers(weight), float(np.float32(eps))
    want, size, _ = norm.forward(x64, w64, pos, r, layout, eps)
    norm.near(y, want, (2.0 ** -19 + 2.0 ** -21) * size, dtype)
    want, want_w, tol, tol_w = norm.backward(x64, w64, norm.numbers(g), pos, r, layout, eps)
    norm.near(dx, want, tol + 2.0 ** -150 + (2.0 ** -134 if dtype == "bf16" else 0.0), dtype)
    norm.near(dw, want_w, tol_w)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_zeros(dtype):
    """The largest weights that an offset gives, at the smallest eps."""
    r = pisa.make_rope(1, 2, 1, 20, 64, dtype=dtype)
    m = pisa.make_qk_norm(r, torch.zeros(64, device="cuda"), None, eps=1e-30, offset=1e30)
    q = torch.zeros((1, 2, 20, 64), dtype=norm.TYPES[dtype], device="cuda")
    q[:, :, ::2] = norm.normal((1, 2, 10, 64), 1, dtype)
    y, _ = pisa.norm_rope_fwd(r, m, q)
    assert bool((y[:, :, 1::2] == 0).all()) and bool(torch.isfinite(y).all()) and bool((y[:, :, ::2].abs() > 1e27).any())
