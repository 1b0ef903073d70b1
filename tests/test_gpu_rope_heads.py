"""Rotations large enough that a thread takes two or four heads: groups of heads that begin with queries and end with keys
(whose strides differ), and last groups that are short."""
import numpy as np
import pytest
import torch

import test_gpu_rope as base

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2609_31093_amd import pisa


def heads_per_thread(B, N, d, heads):
    """As the launcher's rule has it."""
    groups = -(-B * N * (d // 16) // 256) * heads
    return 4 if groups >= 4096 else 2 if groups >= 2048 else 1


@pytest.mark.parametrize("turn", ["fwd", "bwd"])
@pytest.mark.parametrize("layout,rot", [("half", 64), ("half", 50), ("interleaved", 64), ("interleaved", 50)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,share", [(1001, 1), (3001, 2), (6001, 4)])
def test_groups_of_heads(turn, layout, rot, dtype, N, share):
    B, H, Hkv, d = 1, 41, 6, 64
    assert heads_per_thread(B, N, d, H + Hkv) == share and (H % share or share == 1) and ((H + Hkv) % share or share == 1)
    r = pisa.make_rope(B, H, Hkv, N, d, rot=rot, layout=layout, dtype=dtype, scaling="parts", factor=4.0, pos0=777)
    fn, sign = (pisa.rope_fwd, 1) if turn == "fwd" else (pisa.rope_bwd, -1)
    q, k = base.normal((B, H, N, d), 1, dtype), base.normal((B, Hkv, N, d), 2, dtype)
    want_q, want_k = fn(r, q, k)
    pos = 777 + np.arange(N)[None]
    base.check(want_q, q, pos, r, layout, sign, dtype)
    base.check(want_k, k, pos, r, layout, sign, dtype)
    # queries out of a packed projection into another, keys from [B, heads, N, d] into rows of heads, and the other way
    # round; then all of it in place
    packed = torch.full((B, N, H + 2 * Hkv, d), 7.0, dtype=base.TYPES[dtype], device="cuda")
    view = lambda x, lo, n: x[:, :, lo:lo + n].transpose(1, 2)  # noqa: E731
    view(packed, 0, H).copy_(q)
    view(packed, H + Hkv, Hkv).copy_(k)
    other = torch.full_like(packed, 7.0)
    fn(r, view(packed, 0, H), k, None, view(other, Hkv, H), view(other, 0, Hkv))
    assert torch.equal(view(other, Hkv, H), want_q) and torch.equal(view(other, 0, Hkv), want_k)
    assert bool((other[:, :, H + Hkv:] == 7).all())
    yq, yk = fn(r, q, view(packed, H + Hkv, Hkv))
    assert torch.equal(yq, want_q) and torch.equal(yk, want_k)
    fn(r, view(packed, 0, H), view(packed, H + Hkv, Hkv), None, view(packed, 0, H), view(packed, H + Hkv, Hkv))
    assert torch.equal(view(packed, 0, H), want_q) and torch.equal(view(packed, H + Hkv, Hkv), want_k)
    assert bool((packed[:, :, H:H + Hkv] == 7).all())


@pytest.mark.parametrize("N", [1500, 3000])
def test_groups_of_heads_with_positions(N):
    """Two sequences at positions of their own, groups of two and of four heads, one side alone."""
    B, H, Hkv, d = 2, 41, 6, 64
    assert heads_per_thread(B, N, d, H + Hkv) == N // 750
    pos = np.random.default_rng(3).integers(-(1 << 20), 1 << 20, (B, N)).astype(np.int32)
    r = pisa.make_rope(B, H, Hkv, N, d, dtype="f32")
    q, k = base.normal((B, H, N, d), 1, "f32"), base.normal((B, Hkv, N, d), 2, "f32")
    given = torch.from_numpy(pos).cuda()
    yq, yk = pisa.rope_fwd(r, q, k, given)
    base.check(yq, q, pos, r, "half", 1, "f32")
    base.check(yk, k, pos, r, "half", 1, "f32")
    assert torch.equal(pisa.rope_fwd(r, q, None, given)[0], yq) and torch.equal(pisa.rope_fwd(r, None, k, given)[1], yk)
