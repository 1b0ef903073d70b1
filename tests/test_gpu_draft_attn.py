"""Attention of drafted tokens on the GPU against 64 bits.

Tolerance.  A logit z is a sum of d products, each exact in 32 bits (raw fp32: off by 2^-24), so off by at most delta =
(d + 5) 2^-24 sum|q_i k_i| / sqrt(d) in any order and after its scaling; the exponent of base 2 adds the rounding of its
argument (2^-23 |z - m| with the scale's) and 2 ulp.  A weight is then off by rel = exp(2 delta) - 1 + 2^-21 + 2^-23
max|z - m|, its sum likewise, and sums of n terms by n 2^-23 (products and additions); weights that meet bf16 values are
two bf16 terms, off by another 2^-8 2^-8 at most, for 8-bit ones in bf16 problems fp16, 2^-11.  With W the sum of weight
times |value|: |o - o_ref| <= (2 rel + 2^-16 or 2^-11 [bf16] + 2 n 2^-23) W + 2^-8 |o| [bf16] + 2^-22 |o|,
lse moves by no more than its logits do, and a weight's 2^-23 |z - m| is small where |z - m| is large (|z - m| exp(z - m) <
1): |lse - lse_ref| <= delta + 2^-20 + n 2^-23 + 2^-22 max(1, |lse|).
"""
import math

import numpy as np
import pytest
import torch

import test_gpu_qcache as base

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2609_31093_amd import pisa

normal = base.normal


def stored(p, cache):
    """Keys and values [B, Hkv, M C, d] in 64 bits that a cache (a pair of tensors, or 8-bit) stands for."""
    if isinstance(cache, tuple):
        return tuple(x.double().cpu().numpy() for x in cache)
    k = base.values(cache.k) * cache.k_scale.double().cpu().numpy()[..., None, None]
    v = base.values(cache.v).swapaxes(-1, -2) * cache.v_scale.double().cpu().numpy()[..., None, None]
    return tuple(x.reshape(p.B, p.Hkv, -1, p.d) for x in (k, v))


def bits_of(mask, T):
    """[B or 1, T, T] truth values of a mask."""
    m = mask.cpu().numpy().view(np.uint64)
    m = m if m.ndim == 3 else m[None]
    j = np.arange(T)
    return ((m[..., j // 64] >> (j % 64).astype(np.uint64)) & np.uint64(1)).astype(bool)


def reference(p, cache, q, idx, k_new, v_new, mask, alone=None, terms=2.0 ** -16):
    """(o, lse, bound of o's error, of lse's) in 64 bits; `alone` lists the rows whose largest logit is 50 above the next
    however both are off, for which o is that key's value; `terms`: how far weights for bf16 values are off."""
    C, d, G, T, n = p.C, p.d, p.H // p.Hkv, p.Nq, p.N - p.Nq
    M = -(-n // C)
    kk, vv = stored(p, cache)
    kn, vn, q64 = (x.double().cpu().numpy() for x in (k_new, v_new, q))
    sel = idx.cpu().numpy()
    see = bits_of(mask, T)
    o, lse = np.zeros((p.B, p.H, T, d)), np.full((p.B, p.H, T), -np.inf)
    tol_o, tol_l = np.zeros_like(o), np.zeros_like(lse)
    half, own_w, weight = (2.0 ** -8, terms, terms if isinstance(cache, tuple) else 2.0 ** -11) \
        if p.dtype == pisa.PISA_DTYPE_BF16 else (0, 0, 0)
    for b in range(p.B):
        for hk in range(p.Hkv):
            for r in range(T):
                blocks = [j for j in sel[b, hk, r] if 0 <= j < M]
                tok = np.concatenate([np.arange(j * C, min((j + 1) * C, n)) for j in blocks] or [np.zeros(0, int)]).astype(int)
                own = np.flatnonzero(see[b if len(see) > 1 else 0, r])
                kt = np.concatenate((kk[b, hk, tok], kn[b, hk, own]))
                vt = np.concatenate((vv[b, hk, tok], vn[b, hk, own]))
                if not len(kt):
                    continue
                # drafted rows are bf16 over an 8-bit cache too
                wt = np.concatenate((np.full(len(tok), weight), np.full(len(own), own_w)))
                for h in range(hk * G, (hk + 1) * G):
                    z = kt @ q64[b, h, r] / math.sqrt(d)
                    m = z.max()
                    w = np.exp(z - m)
                    N, total = len(kt), w.sum()
                    w /= total
                    o[b, h, r], lse[b, h, r] = w @ vt, m + math.log(total)
                    delta = (d + 5) * 2.0 ** -24 * (abs(kt) @ abs(q64[b, h, r])).max() / math.sqrt(d)
                    if alone is not None:
                        if N == 1 or m - np.partition(z, -2)[-2] > 50 + 4 * delta:
                            alone.append((b, h, r))
                        rel = 0.0
                    else:
                        rel = math.expm1(2 * delta) + 2.0 ** -21 + 2.0 ** -23 * (m - z).max()
                    tol_o[b, h, r] = (w * (2 * rel + wt + 2 * N * 2.0 ** -23)) @ abs(vt) + (half + 2.0 ** -22) * abs(o[b, h, r])
                    tol_l[b, h, r] = delta + 2.0 ** -20 + N * 2.0 ** -23 + 2.0 ** -22 * max(1, abs(lse[b, h, r]))
    return o, lse, tol_o, tol_l


def check(p, cache, q, idx, k_new, v_new, mask, o, lse):
    want_o, want_l, tol_o, tol_l = reference(p, cache, q, idx, k_new, v_new, mask)
    got_o, got_l = o.double().cpu().numpy(), lse.double().cpu().numpy()
    empty = np.isneginf(want_l)
    assert np.array_equal(np.isneginf(got_l), empty) and (got_o[empty] == 0).all()
    off = abs(got_o - want_o) - tol_o
    assert (off <= 0).all(), (off.max(), np.argwhere(off > 0)[:3])
    off = abs(got_l[~empty] - want_l[~empty]) - tol_l[~empty]
    assert (off <= 0).all(), off.max()


def selection(p, seed, alike=0.7, empty=0.1):
    """Distinct blocks per row, most of them its neighbours' too; padding of every kind, blocks of drafted rows, empty rows."""
    rng = np.random.default_rng(seed)
    M, have = -(-p.N // p.C), -(-(p.N - p.Nq) // p.C)
    idx = np.full((p.B, p.Hkv, p.Nq, p.K), -1, np.int32)
    for b in range(p.B):
        for h in range(p.Hkv):
            common = rng.permutation(M)
            for r in range(p.Nq):
                if rng.random() < empty:
                    idx[b, h, r] = rng.choice([-1, -2 ** 31, have, 2 ** 31 - 1], p.K)
                    continue
                row = common if rng.random() < alike else rng.permutation(M)
                row = list(rng.permutation(row[:p.K])[:int(rng.integers(1, p.K + 1))])
                row += [int(rng.choice([-1, -7, have, M + 3, 2 ** 31 - 1])) for _ in range(p.K - len(row))]
                # M + 3 and the like may come twice: they are nothing
                idx[b, h, r] = rng.permutation(row)
    return torch.from_numpy(idx).cuda()


def trees(B, T, seed, drop=0.1):
    """Masks of random trees, some rows without any bit; bits past the last token set."""
    rng = np.random.default_rng(seed)
    parents = np.array([[-1 if i == 0 or rng.random() < 0.1 else int(rng.integers(max(0, i - 8), i)) for i in range(T)] for _ in range(B)])
    mask = pisa.draft_layout(torch.from_numpy(parents.astype(np.int32)).cuda(), 0)[0]
    m = mask.cpu().numpy().view(np.uint64)
    m[rng.random((B, T)) < drop] = 0
    if T % 64:
        m[..., -1] |= ~np.uint64(0) << np.uint64(T % 64)
    return torch.from_numpy(m.view(np.int64)).cuda()


def drafted(p, seed, dtype):
    """Rows of heads, and a slice of a packed projection."""
    k = normal((p.B, p.Nq, p.Hkv, p.d), seed, dtype).transpose(1, 2)
    return k, normal((p.B, p.Nq, 3 * p.Hkv, p.d), seed + 1, dtype)[:, :, 2 * p.Hkv:].transpose(1, 2)


def make(p, eight, seed, dtype, spread=0.5):
    """A cache of N - Nq rows, what lies behind them NaN (8-bit: as appending leaves it)."""
    n, cap = p.N - p.Nq, p.Ncap or p.N
    k, v = normal((p.B, p.Hkv, max(n, 1), p.d), seed, dtype, spread), normal((p.B, p.Hkv, max(n, 1), p.d), seed + 1, dtype, spread)
    if eight:
        cache = pisa.make_qcache(p)
        if n:
            pisa.qcache_append(base.at(p, n), cache, k[:, :, :n], v[:, :, :n], 0)
        return cache
    held = tuple(torch.full((p.B, p.Hkv, cap, p.d), float("nan"), dtype=base.TYPES[dtype], device="cuda") for _ in range(2))
    for x, y in zip(held, (k, v)):
        x[:, :, :n] = y[:, :, :n]
    return held


def attend(p, cache, q, idx, k_new, v_new, mask, **kw):
    if isinstance(cache, tuple):
        return pisa.draft_attn_fwd(p, q, *cache, idx, k_new, v_new, mask, **kw)
    return pisa.qcache_draft_attn_fwd(p, cache, q, idx, k_new, v_new, mask, **kw)


SHAPES = [
    # B, H, Hkv, T, n, d, C, g, K, dtype, room behind the drafted rows
    (1, 1, 1, 1, 0, 128, 64, 2, 4, "bf16", 0),          # nothing cached
    (1, 2, 1, 5, 0, 64, 32, 2, 4, "f32", 3),
    (2, 4, 2, 40, 1, 128, 64, 2, 4, "bf16", 0),         # one cached token
    (1, 8, 8, 1, 2000, 128, 64, 2, 16, "bf16", 64),     # one drafted token
    (1, 8, 8, 16, 2047, 128, 64, 2, 16, "bf16", 64),
    (2, 8, 2, 25, 777, 128, 64, 2, 8, "bf16", 7),
    (1, 16, 1, 33, 500, 64, 32, 2, 8, "bf16", 0),       # a row to a tile
    (1, 9, 1, 7, 300, 128, 96, 2, 5, "bf16", 0),        # 16 / 9
    (1, 3, 1, 40, 333, 128, 96, 2, 3, "bf16", 400),     # five rows of three heads
    (2, 5, 1, 64, 900, 64, 128, 4, 5, "bf16", 0),
    (1, 6, 1, 65, 1500, 128, 256, 3, 4, "bf16", 0),
    (1, 2, 2, 130, 1000, 64, 64, 2, 4, "f32", 1),
    (1, 6, 2, 33, 450, 128, 32, 2, 6, "f32", 0),
    (1, 16, 1, 6, 1100, 128, 160, 2, 4, "f32", 30),
    (1, 1, 1, 300, 3000, 64, 32, 2, 40, "bf16", 0),
    (1, 1, 1, 1024, 100, 64, 32, 2, 3, "bf16", 0),
    (2, 8, 2, 3, 3000, 128, 128, 4, 30, "bf16", 100),   # splits
    (1, 4, 1, 2, 4100, 64, 32, 2, 100, "f32", 0),
    (1, 2, 2, 20, 8000, 128, 224, 2, 12, "bf16", 0),
    (3, 4, 4, 8, 640, 128, 64, 2, 10, "f32", 0),        # blocks that end where the cache does
    (2, 16, 16, 200, 700, 64, 64, 2, 6, "bf16", 0),
    (4, 16, 4, 128, 513, 128, 64, 2, 8, "bf16", 0),
]


def problem(shape):
    B, H, Hkv, T, n, d, C, g, K, dtype, room = shape
    return base.problem(B, H, Hkv, T, n + T, d, C, g, K, 1, dtype, n + T + room)


@pytest.mark.parametrize("eight", [False, True], ids=["raw", "8bit"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_attention(shape, eight):
    p, dtype = problem(shape), shape[9]
    cache, q = make(p, eight, 1, dtype), normal((p.B, p.H, p.Nq, p.d), 3, dtype)
    new, idx, mask = drafted(p, 5, dtype), selection(p, 4), trees(p.B, p.Nq, 6)
    o, lse = attend(p, cache, q, idx, *new, mask)
    check(p, cache, q, idx, *new, mask, o, lse)
    # one mask for the batch; what is given is written, and nothing around the workspace
    size = (pisa.pisa_qcache_draft_attn_workspace_bytes if eight else pisa.pisa_draft_attn_workspace_bytes)(p)
    band = torch.full((size + 8192,), 0xFF, dtype=torch.uint8, device="cuda")
    o2, lse2 = torch.full_like(q, 7.0), torch.full_like(lse, 7.0)
    got = attend(p, cache, q, idx, *(x.contiguous() for x in new), mask[0], o=o2, lse=lse2, ws=band[4096:4096 + size])
    assert got[0] is o2 and got[1] is lse2
    assert torch.equal(o2[0], o[0]) and torch.equal(lse2[0], lse[0])
    want = attend(p, cache, q, idx, *new, mask[:1].expand(p.B, -1, -1).contiguous())
    assert torch.equal(o2, want[0]) and torch.equal(lse2, want[1])
    assert bool((band[:4096] == 0xFF).all()) and bool((band[4096 + size:] == 0xFF).all())


@pytest.mark.parametrize("eight", [False, True], ids=["raw", "8bit"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_see_one_side_or_nothing(eight, dtype):
    p = problem((2, 4, 2, 20, 200, 128, 64, 2, 4, dtype, 0))
    cache, q, new = make(p, eight, 1, dtype), normal((2, 4, 20, 128), 3, dtype), drafted(p, 5, dtype)
    idx, mask = selection(p, 4, empty=0.0), trees(2, 20, 6, drop=0.0)
    nothing, none = torch.full_like(idx, -1), torch.zeros_like(mask)
    for i, m in ((idx, none), (nothing, mask), (nothing, none)):
        check(p, cache, q, i, *new, m, *attend(p, cache, q, i, *new, m))
    o, lse = attend(p, cache, q, nothing, *new, none)
    assert bool((o == 0).all()) and bool((lse == -math.inf).all())


@pytest.mark.parametrize("eight", [False, True], ids=["raw", "8bit"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hkv,T,K", [(2, 2, 24, 4), (8, 2, 40, 4), (16, 1, 5, 30)])
def test_hidden_values(eight, dtype, H, Hkv, T, K):
    """NaN and infinities in blocks, rows and drafted tokens that some rows see: the others' results keep their bits."""
    d, C, n = 128, 32, 1000
    p = problem((1, H, Hkv, T, n, d, C, 2, K, dtype, 50))
    cache, q, new = make(p, eight, 1, dtype), normal((1, H, T, d), 3, dtype), tuple(x.contiguous() for x in drafted(p, 5, dtype))
    idx, mask = selection(p, 4, alike=0.5), trees(1, T, 6)
    want = attend(p, cache, q, idx, *new, mask)
    at, own = [(70, 5), (500, 9), (999, 127)], [(2, 3), (T - 1, 90)]
    if eight:
        cache.v[:, :, at[0][0] // C, at[0][1], at[0][0] % C] = 0x7F
        cache.k[:, :, at[1][0] // C, at[1][0] % C, at[1][1]] = 0xFF
        cache.v[:, :, at[2][0] // C, at[2][1], at[2][0] % C] = 0xFF
    else:
        cache[1][:, :, at[0][0], at[0][1]] = math.inf
        cache[0][:, :, at[1][0], at[1][1]] = math.nan
        cache[1][:, :, at[2][0], at[2][1]] = math.nan
    new[1][:, :, own[0][0], own[0][1]] = -math.inf
    new[0][:, :, own[1][0], own[1][1]] = math.nan
    o, lse = attend(p, cache, q, idx, *new, mask)
    bits = torch.from_numpy(bits_of(mask, T)).cuda()[0]
    sees = torch.zeros((Hkv, T), dtype=torch.bool, device="cuda")
    for x, _ in at:
        sees |= (idx[0] == x // C).any(-1)
    for j, _ in own:
        sees |= bits[:, j][None]
    free = ~sees.repeat_interleave(H // Hkv, 0)
    assert bool(free.any()) and bool(sees.any())
    assert torch.equal(o[0][free], want[0][0][free]) and torch.equal(lse[0][free], want[1][0][free])
    assert not torch.isfinite(o[0][~free]).all(-1).any()
    only = (idx[0] == at[0][0] // C).any(-1) & ~(idx[0] == at[1][0] // C).any(-1) & ~bits[:, own[1][0]][None]
    only = only.repeat_interleave(H // Hkv, 0)
    assert not torch.isfinite(o[0][only][:, at[0][1]]).any() and torch.equal(lse[0][only], want[1][0][only])


@pytest.mark.parametrize("eight", [False, True], ids=["raw", "8bit"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size,value", [(2.0 ** 20, 1.0), (2.0 ** 50, 1.0), (1.0, 2.0 ** 126), (1.0, 2.0 ** -60)])
def test_range(eight, dtype, size, value):
    """Logits and values from tiny to the type's largest."""
    p = problem((1, 4, 2, 12, 300, 64, 32, 2, 5, dtype, 0))
    q, idx, mask = normal((1, 4, 12, 64), 3, dtype) * size, selection(p, 4), trees(1, 12, 6)
    k, v = normal((1, 2, 300, 64), 1, dtype), torch.clamp(normal((1, 2, 300, 64), 2, dtype), -1.9, 1.9) * value
    new = normal((1, 2, 12, 64), 5, dtype), torch.clamp(normal((1, 2, 12, 64), 6, dtype), -1.9, 1.9) * value
    if eight:
        cache = pisa.make_qcache(p)
        pisa.qcache_append(base.at(p, 300), cache, k, v, 0)
    else:
        cache = tuple(torch.nn.functional.pad(x, (0, 0, 0, 12)).contiguous() for x in (k, v))
    o, lse = attend(p, cache, q, idx, *new, mask)
    if size == 1.0:
        check(p, cache, q, idx, *new, mask, o, lse)
        return
    alone = []
    want, want_l, tol_o, tol_l = reference(p, cache, q, idx, *new, mask, alone)
    got, got_l = o.double().cpu().numpy(), lse.double().cpu().numpy()
    seen = ~np.isneginf(want_l)
    assert np.isfinite(got).all() and (abs(got_l - want_l)[seen] <= tol_l[seen]).all()
    assert len(alone) > 10
    for at in alone:  # (what is not the first key's weighs less than n e^-50)
        assert (abs(got[at] - want[at]) <= tol_o[at] + 1e-19).all()


@pytest.mark.parametrize("eight", [False, True], ids=["raw", "8bit"])
def test_captured_and_on_another_stream(eight):
    """Two graphs with workspaces of their own, replayed with other inputs, and eager calls on a side stream between them."""
    p = problem((1, 8, 2, 12, 3000, 128, 64, 2, 16, "bf16", 64))
    cache, q, new = make(p, eight, 1, "bf16"), normal((1, 8, 12, 128), 3, "bf16"), drafted(p, 5, "bf16")
    idx, mask = selection(p, 4), trees(1, 12, 6)
    size = (pisa.pisa_qcache_draft_attn_workspace_bytes if eight else pisa.pisa_draft_attn_workspace_bytes)(p)
    assert size > 0, "a call in two launches"
    attend(p, cache, q, idx, *new, mask)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = attend(p, cache, q, idx, *new, mask)
        graphs.append((graph, out))
    side = torch.cuda.Stream()
    for i in range(4):
        q.copy_(normal((1, 8, 12, 128), 20 + i, "bf16"))
        idx.copy_(selection(p, 30 + i))
        mask.copy_(trees(1, 12, 40 + i))
        want = attend(p, cache, q, idx, *new, mask)
        check(p, cache, q, idx, *new, mask, *want)
        torch.cuda.synchronize()
        got = attend(p, cache, q, idx, *new, mask, stream=side)
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        for graph, out in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for _, out in graphs:
            for a, b in zip(out, want):
                assert torch.equal(a, b)


@pytest.mark.parametrize("eight", [False, True], ids=["raw", "8bit"])
def test_one_workspace_for_a_growing_cache(eight):
    """Lengths whose tiles are spread over one workgroup and over several, with what an earlier call left."""
    need = pisa.pisa_qcache_draft_attn_workspace_bytes if eight else pisa.pisa_draft_attn_workspace_bytes
    ws = None
    for n in (0, 40, 700, 5000, 1500, 64):
        p = problem((1, 8, 2, 12, n, 128, 64, 2, 16, "bf16", 64))
        ws = torch.full((need(p),), 0xFF, dtype=torch.uint8, device="cuda") if ws is None else ws
        assert need(p) == ws.numel() > 0
        cache, q, new = make(p, eight, 1, "bf16"), normal((1, 8, 12, 128), 3, "bf16"), drafted(p, 5, "bf16")
        idx, mask = selection(p, n), trees(1, 12, 6)
        check(p, cache, q, idx, *new, mask, *attend(p, cache, q, idx, *new, mask, ws=ws))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_drafted_rows_far_apart(dtype):
    """Strides of drafted rows around the one up to which 32-bit offsets serve."""
    p = problem((1, 2, 1, 70, 100, 64, 32, 2, 3, dtype, 0))
    cache, q, idx, mask = make(p, False, 1, dtype), normal((1, 2, 70, 64), 3, dtype), selection(p, 4), trees(1, 70, 6)
    new = drafted(p, 5, dtype)
    want = attend(p, cache, q, idx, *new, mask)
    for stride in ((1 << 24) - 8, 1 << 24, (1 << 24) + 8):
        wide = torch.empty((70, stride), dtype=base.TYPES[dtype], device="cuda")
        views = [wide[:, 64 * i:64 * (i + 1)][None, None] for i in range(2)]
        for x, y in zip(views, new):
            x.copy_(y)
        got = attend(p, cache, q, idx, *views, mask)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        got = attend(p, cache, q, idx, new[0], views[1], mask)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        del wide, views


def test_many_tiles_past_one_launch():
    """More tiles than the 2^22 that one launch takes: 5000 sequences of 1024 rows, a row to a tile, 9 heads on 1."""
    B, H, T, d = 5000, 9, 1024, 64
    p = base.problem(B, H, 1, T, T + 32, d, 32, 2, 3, 1, "bf16", T + 32)
    assert pisa.pisa_draft_attn_workspace_bytes(p) == 0
    q = normal((1, H, 1, d), 1, "bf16").expand(B, H, T, d).contiguous()
    k = torch.zeros((B, 1, T + 32, d), dtype=torch.bfloat16, device="cuda")
    v = torch.ones_like(k)
    new = normal((1, 1, T, d), 2, "bf16").expand(B, 1, T, d)
    idx = torch.full((B, 1, T, 3), -1, dtype=torch.int32, device="cuda")
    mask = torch.zeros((T, T // 64), dtype=torch.int64, device="cuda")
    i = torch.arange(T, device="cuda")
    mask[i, i // 64] = torch.ones_like(i) << (i % 64)  # each row itself alone
    o, lse = attend(p, (k, v), q, idx, new, new, mask)
    assert torch.equal(o, new.expand(B, H, T, d)) and bool(torch.isfinite(lse).all())


def test_long_cache():
    """A cache whose offsets pass 2^31 elements, its last block short."""
    n, T, d, C = 65535 * 256 - 40 - 77, 40, 128, 256
    p = base.problem(1, 4, 2, T, n + T, d, C, 2, 6, 1, "bf16", 0)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    k, v = (torch.randn((1, 2, n + T, d), generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    q, new = normal((1, 4, T, d), 3, "bf16"), drafted(p, 5, "bf16")
    M, rng = -(-n // C), np.random.default_rng(2)
    idx = np.stack([np.stack([np.append(rng.permutation(M - 1)[:5], M - 1) for _ in range(T)]) for _ in range(2)])[None]
    idx, mask = torch.from_numpy(idx.astype(np.int32)).cuda(), trees(1, T, 6)
    o, lse = attend(p, (k, v), q, idx, *new, mask)
    # the same blocks out of a short cache
    used = torch.unique(idx)
    at = {int(j): i for i, j in enumerate(used)}
    assert max(at) == M - 1
    short = [torch.cat([x[:, :, j * C:(j + 1) * C] for j in at], 2)[:, :, :(len(at) - 1) * C + n - (M - 1) * C] for x in (k, v)]
    del k, v
    ns = short[0].shape[2]
    ps = base.problem(1, 4, 2, T, ns + T, d, C, 2, 6, 1, "bf16", 0)
    cache = tuple(torch.nn.functional.pad(x, (0, 0, 0, T)).contiguous() for x in short)
    small = torch.tensor([at[int(j)] for j in idx.flatten()], dtype=torch.int32, device="cuda").view_as(idx)
    check(ps, cache, q, small, *new, mask, o, lse)


@pytest.mark.parametrize("eight", [False, True], ids=["raw", "8bit"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_longest_list(eight, dtype):
    """As many blocks as a tile can select together, out of as many as there are: the list that leaves a unit least room."""
    T, d, C, K = 20, 64, 32, 128
    n = 65535 * C - T
    p = base.problem(1, 1, 1, T, n + T, d, C, 2, K, 1, dtype, 0)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    k, v = (torch.randn((1, 1, n + T, d), generator=gen, device="cuda").to(base.TYPES[dtype]) for _ in range(2))
    if eight:
        cache = pisa.make_qcache(p)
        pisa.qcache_append(base.at(p, n), cache, k[:, :, :n], v[:, :, :n], 0)
    q, new, mask = normal((1, 1, T, d), 3, dtype), drafted(p, 5, dtype), trees(1, T, 6)
    M, rng = -(-n // C), np.random.default_rng(2)
    order = rng.permutation(M - 1)[:T * K].reshape(T, K)
    order[:, 0] = M - 1
    idx = torch.from_numpy(order.astype(np.int32))[None, None].contiguous().cuda()
    o, lse = attend(p, cache if eight else (k, v), q, idx, *new, mask)
    # each row's blocks out of a short cache of their own
    for r in (0, 7, 15, 16, 19):
        at = idx[0, 0, r].sort().values.long()
        ns = (K - 1) * C + n - (M - 1) * C
        ps = base.problem(1, 1, 1, T, ns + T, d, C, 2, K, 1, dtype, K * C + T)
        if eight:
            short = pisa.make_qcache(ps)
            for f in ("k", "v", "k_scale", "v_scale"):
                getattr(short, f)[:, :, :K] = getattr(cache, f)[:, :, at]
        else:
            short = tuple(torch.nn.functional.pad(x[:, :, :M * C].unflatten(2, (M, C))[:, :, at].flatten(2, 3)[:, :, :ns], (0, 0, 0, C + T + K * C - ns - C))
                          for x in (k, v))
        only = torch.full_like(idx, -1)
        only[0, 0, r] = torch.arange(K, device="cuda")
        want_o, want_l, tol_o, tol_l = (x[:, :, r] for x in reference(ps, short, q, only, *new, mask))
        assert (abs(o[:, :, r].double().cpu().numpy() - want_o) <= tol_o).all()
        assert (abs(lse[:, :, r].double().cpu().numpy() - want_l) <= tol_l).all()


@pytest.mark.parametrize("eight", [False, True], ids=["raw", "8bit"])
def test_wrapper_refuses(eight):
    p = problem((1, 4, 2, 12, 300, 64, 32, 2, 5, "bf16", 10))
    cache, q, new = make(p, eight, 1, "bf16"), normal((1, 4, 12, 64), 3, "bf16"), drafted(p, 5, "bf16")
    good = dict(q=q, idx=selection(p, 4), k_new=new[0], v_new=new[1], mask=trees(1, 12, 6))
    attend(p, cache, **good)
    for bad in (dict(q=q.float()), dict(q=q[:, :3].contiguous()), dict(q=q.cpu()), dict(q=q.transpose(1, 2)), dict(idx=good["idx"].long()),
                dict(idx=good["idx"][..., :4].contiguous()), dict(k_new=new[0][:, :, :5]), dict(v_new=new[1].float()),
                dict(mask=good["mask"].int()), dict(mask=good["mask"][:, :5].contiguous()), dict(o=q.float()),
                dict(lse=torch.zeros((1, 4, 11), device="cuda"))):
        with pytest.raises(ValueError):
            attend(p, cache, **{**good, **bad})
    with pytest.raises(pisa.PisaError):
        attend(p, cache, **good, o=q)
    big = problem((1, 4, 2, 12, 3000, 64, 32, 2, 60, "bf16", 10))
    with pytest.raises(pisa.PisaError):
        attend(big, make(big, eight, 1, "bf16"), **{**good, "idx": selection(big, 4)}, ws=torch.empty(256, dtype=torch.uint8, device="cuda"))
    if not eight:
        with pytest.raises(ValueError):
            attend(p, (cache[0][:, :, :300], cache[1]), **good)
