"""Rotary positions on the GPU against their formula in 64 bits.

Tolerance of a turned value a cos - b sin, amplitude A: the angle's fraction of a turn is rounded to 32 bits (2^-26
turns, 2^-23.3 radians), sine and cosine are off by at most 2 ulp (2^-23), each of the scale, the two products and the
sum by 2^-24 of |a| + |b|: in all below 2^-21 A (|a| + |b|), and bf16 outputs by another 2^-8 of themselves.
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2609_31093_amd import pisa

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def formula(x, pos, freq, amplitude, layout, sign):
    """(turned x, bound of |a| + |b| of each value), in 64 bits; x [B, h, N, d], pos [B, N]."""
    x = x.double().cpu().numpy()
    pairs = len(freq)
    angle = pos[:, None, :, None].astype(np.float64) * np.asarray(freq)
    c, s = amplitude * np.cos(angle), sign * amplitude * np.sin(angle)
    i = np.arange(pairs)
    a, b = (i, i + pairs) if layout == "half" else (2 * i, 2 * i + 1)
    y, size = x.copy(), np.zeros_like(x)
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    size[..., a] = size[..., b] = abs(x[..., a]) + abs(x[..., b])
    return y, size


def check(got, x, pos, r, layout, sign, dtype):
    pairs = r.rot // 2
    want, size = formula(x, pos, list(r.freq)[:pairs], r.amplitude, layout, sign)
    tol = 2.0 ** -21 * abs(r.amplitude) * size + (2.0 ** -8 * abs(want) if dtype == "bf16" else 0)
    got = got.double().cpu().numpy()
    assert np.array_equal(got[..., r.rot:], want[..., r.rot:]), "values behind the rotated ones are copied"
    off = abs(got - want) - tol
    assert (off <= 0).all(), off.max()


def normal(shape, seed, dtype):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal(shape).astype(np.float32)).to(TYPES[dtype]).cuda()


@pytest.mark.parametrize("turn", ["fwd", "bwd"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,Hkv,N,d,rot,scaling,pos0", [
    (1, 1, 1, 1, 64, 64, "none", 0),
    (2, 4, 2, 37, 128, 128, "parts", 1000),
    (1, 3, 1, 130, 64, 50, "linear", 0),          # halves that fit no vector
    (2, 2, 2, 5, 128, 2, "none", 12345),
    (1, 2, 1, 33, 64, 62, "base", 7),
    (1, 2, 2, 19, 128, 126, "none", 1 << 20),     # far positions
    (3, 2, 1, 65, 128, 64, "parts", -40),         # positions on both sides of 0
])
def test_values(turn, layout, dtype, B, H, Hkv, N, d, rot, scaling, pos0):
    r = pisa.make_rope(B, H, Hkv, N, d, rot=rot, layout=layout, dtype=dtype, scaling=scaling,
                       factor=1.0 if scaling == "none" else 4.0, pos0=pos0)
    q, k = normal((B, H, N, d), 1, dtype), normal((B, Hkv, N, d), 2, dtype)
    fn = pisa.rope_fwd if turn == "fwd" else pisa.rope_bwd
    yq, yk = fn(r, q, k)
    pos = np.broadcast_to(pos0 + np.arange(N), (B, N))
    sign = 1 if turn == "fwd" else -1
    check(yq, q, pos, r, layout, sign, dtype)
    check(yk, k, pos, r, layout, sign, dtype)


@pytest.mark.parametrize("layout,rot", [("half", 128), ("half", 90), ("interleaved", 90)])
@pytest.mark.parametrize("shared", [True, False])
def test_positions_of_their_own(layout, rot, shared):
    B, H, Hkv, N, d = 3, 2, 1, 41, 128
    rng = np.random.default_rng(3)
    pos = rng.integers(-(1 << 30), 1 << 30, (N,) if shared else (B, N)).astype(np.int32)
    r = pisa.make_rope(B, H, Hkv, N, d, rot=rot, layout=layout, dtype="f32")
    q, k = normal((B, H, N, d), 4, "f32"), normal((B, Hkv, N, d), 5, "f32")
    yq, yk = pisa.rope_fwd(r, q, k, torch.from_numpy(pos).cuda())
    pos = np.broadcast_to(pos, (B, N))
    check(yq, q, pos, r, layout, 1, "f32")
    check(yk, k, pos, r, layout, 1, "f32")


@pytest.mark.parametrize("layout,rot", [("half", 128), ("half", 90), ("half", 64), ("interleaved", 90)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strided_tensors_in_place_and_one_side(layout, rot, dtype):
    """A packed projection [B, N, H + 2 Hkv, d]: its views as inputs, in place, into a cache, and one side alone; what
    lies between the rows stays as it was."""
    B, H, Hkv, N, d = 2, 3, 2, 29, 128
    r = pisa.make_rope(B, H, Hkv, N, d, rot=rot, layout=layout, dtype=dtype, pos0=11)
    packed = normal((B, N, H + 2 * Hkv, d), 6, dtype)
    view = lambda x, lo, n: x[:, :, lo:lo + n].transpose(1, 2)  # noqa: E731
    q, k = view(packed, 0, H), view(packed, H, Hkv)
    want_q, want_k = pisa.rope_fwd(r, q.contiguous(), k.contiguous())
    yq, yk = pisa.rope_fwd(r, q, k)
    assert torch.equal(yq, want_q) and torch.equal(yk, want_k)
    only, none = pisa.rope_fwd(r, q)
    assert torch.equal(only, want_q) and none is None
    none, only = pisa.rope_fwd(r, None, k)
    assert torch.equal(only, want_k) and none is None
    cache = torch.full((B, Hkv, 64, d), 7.0, dtype=TYPES[dtype], device="cuda")
    pisa.rope_fwd(r, None, k, k_out=cache[:, :, 20:20 + N])
    assert torch.equal(cache[:, :, 20:20 + N], want_k)
    assert bool((cache[:, :, :20] == 7).all()) and bool((cache[:, :, 20 + N:] == 7).all())
    whole = packed.clone()
    pisa.rope_fwd(r, view(whole, 0, H), view(whole, H, Hkv), q_out=view(whole, 0, H), k_out=view(whole, H, Hkv))
    assert torch.equal(view(whole, 0, H), want_q) and torch.equal(view(whole, H, Hkv), want_k)
    assert torch.equal(whole[:, :, H + Hkv:], packed[:, :, H + Hkv:])
    shared = normal((1, 1, N, d), 7, dtype)  # a broadcast input
    y, _ = pisa.rope_fwd(r, shared.expand(B, H, N, d))
    assert torch.equal(y, pisa.rope_fwd(r, shared.expand(B, H, N, d).contiguous())[0])


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_gradient_against_differences_and_the_transposed_map(layout):
    """The map is linear: <w, f(x + e) - f(x)> = <grad, e>, exactly but for rounding."""
    B, H, Hkv, N, d = 1, 2, 1, 9, 64
    r = pisa.make_rope(B, H, Hkv, N, d, rot=48, layout=layout, dtype="f32", scaling="parts", factor=4.0, pos0=100)
    q, k, wq, wk = (normal((B, h, N, d), s, "f32") for s, h in ((1, H), (2, Hkv), (3, H), (4, Hkv)))
    gq, gk = pisa.rope_bwd(r, wq, wk)
    for x, w, g, side in ((q, wq, gq, 0), (k, wk, gk, 1)):
        run = lambda z: (pisa.rope_fwd(r, z, None) if side == 0 else pisa.rope_fwd(r, None, z))[side].double()  # noqa: E731
        rng = np.random.default_rng(8)
        for _ in range(8):
            e = torch.zeros_like(x)
            at = tuple(int(rng.integers(n)) for n in x.shape)
            e[at] = 1.0
            got = (w.double() * (run(x + e) - run(x))).sum().item()
            # two values change by A (|a| + |b| + 1) 2^-21 at most, and x + e is rounded (2^-24 of |x| + 1 < 8)
            tol = 4 * 2.0 ** -21 * r.amplitude * (x.abs().max().item() * 2 + 2) * w.abs().max().item()
            assert abs(got - g[at].item()) <= tol


def test_special_values_stay_in_their_pair():
    B, H, N, d = 1, 1, 4, 128
    r = pisa.make_rope(B, H, 1, N, d, rot=100, dtype="f32")
    x = normal((B, H, N, d), 9, "f32")
    x[0, 0, 1, 3], x[0, 0, 2, 120], x[0, 0, 3, 60] = float("nan"), float("inf"), float("inf")
    y, _ = pisa.rope_fwd(r, x)
    bad = ~torch.isfinite(y)
    want = torch.zeros_like(bad)
    want[0, 0, 1, [3, 53]] = True
    want[0, 0, 2, 120] = True
    want[0, 0, 3, [10, 60]] = True
    assert torch.equal(bad, want) and y[0, 0, 2, 120] == float("inf")


def test_many_heads_and_rows_past_one_workgroup():
    B, H, Hkv, N, d = 1, 40, 7, 1001, 64
    r = pisa.make_rope(B, H, Hkv, N, d, layout="interleaved", dtype="bf16")
    q, k = normal((B, H, N, d), 10, "bf16"), normal((B, Hkv, N, d), 11, "bf16")
    yq, yk = pisa.rope_fwd(r, q, k)
    pos = np.arange(N)[None]
    check(yq, q, pos, r, "interleaved", 1, "bf16")
    check(yk, k, pos, r, "interleaved", 1, "bf16")


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_offsets_past_32_bits(layout):
    """2.5e9 values: heads and rows at the far end as on their own."""
    H, N, d = 64, 300001, 128
    q = torch.randn((1, H, N, d), device="cuda", dtype=torch.bfloat16)
    r = pisa.make_rope(1, H, 1, N, d, layout=layout)
    pisa.rope_fwd(r, q, q_out=(out := torch.empty_like(q)))
    for h in (0, 33, 63):
        one = pisa.make_rope(1, 1, 1, 500, d, layout=layout, pos0=N - 500)
        want, _ = pisa.rope_fwd(one, q[:, h:h + 1, N - 500:])
        assert torch.equal(out[:, h:h + 1, N - 500:], want)
    check(out[:, 63:, -3:], q[:, 63:, -3:], np.arange(N - 3, N)[None], r, layout, 1, "bf16")


def test_wrapper_refusals():
    r = pisa.make_rope(1, 2, 1, 8, 64, dtype="bf16")
    q = torch.zeros((1, 2, 8, 64), dtype=torch.bfloat16, device="cuda")
    for bad in (q.cpu(), q.float(), q[:, :1], torch.zeros((1, 2, 8, 128), dtype=torch.bfloat16, device="cuda")[..., ::2]):
        with pytest.raises(ValueError):
            pisa.rope_fwd(r, bad)
    with pytest.raises(ValueError):
        pisa.rope_fwd(r, q, positions=torch.zeros(8, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        pisa.rope_fwd(r, q, k_out=q)
    odd = torch.zeros((1, 2, 8, 66), dtype=torch.bfloat16, device="cuda")[..., :64]  # rows 132 bytes apart
    with pytest.raises(pisa.PisaError):
        pisa.rope_fwd(r, odd)


def test_another_stream():
    r = pisa.make_rope(1, 2, 1, 513, 64, dtype="bf16")
    q = normal((1, 2, 513, 64), 12, "bf16")
    want, _ = pisa.rope_fwd(r, q)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    out = torch.empty_like(q)
    pisa.rope_fwd(r, q, q_out=out, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    assert math.isfinite(out.float().sum().item())


def test_positions_leave_the_descriptor_alone():
    """One descriptor serves calls with positions per batch, shared ones and none, whichever came before."""
    B, N = 3, 41
    r = pisa.make_rope(B, 2, 1, N, 64, dtype="bf16", pos0=5)
    q, before = normal((B, 2, N, 64), 13, "bf16"), bytes(r)
    own = np.random.default_rng(14).integers(-1000, 1000, (B, N)).astype(np.int32)
    counted = np.broadcast_to(5 + np.arange(N, dtype=np.int32), (B, N))
    for pos in (own, own[0], None, own[1], own):
        given = None if pos is None else torch.from_numpy(pos).cuda()
        got, _ = pisa.rope_fwd(r, q, positions=given)
        assert bytes(r) == before
        check(got, q, counted if pos is None else np.broadcast_to(pos, (B, N)), r, "half", 1, "bf16")
