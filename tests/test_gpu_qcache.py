"""The 8-bit cache on the GPU: its codes against e4m3 written out, its attention against 64 bits.

Codes, scales, raw rows and the pyramid are compared for equality: powers of two scale exactly, so a code is the nearest
e4m3 value (ties to even) and nothing else.

Tolerance of the attention.  Keys and values are exact in what they stand for.  A logit is a sum of d products, exact in
32 bits (8 bits times 24 at most), so off by at most delta = (d + 4) 2^-24 sum|q_i k_i| / sqrt(d) in any order and after
its scaling; the exponent of base 2 adds the rounding of its argument (2^-24 |z - m| / ln 2) and 2 ulp.  A weight is then
off by w = exp(2 delta) - 1 + 2^-21 + 2^-23 max|z - m| relative, its sum likewise, and sums of n terms by n 2^-24; weights
of bf16 queries by another 2^-11 (fp16; they reach down to 2^-28 of the largest before they lose bits, which n 2^-24
covers).  With W the sum of weight times |value|: |o - o_ref| <= (2 w + 2^-11 [bf16] + 2 n 2^-24) W + 2^-8 |o| [bf16] +
2^-23 |o|, |lse - lse_ref| <= delta + w + n 2^-24 + 2^-22 max(1, |lse|).
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2609_31093_amd import pisa

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}

# value of each e4m3 code 0..127 (127 is NaN)
E4M3 = np.array([(c & 7) * 2.0 ** -9 if c < 8 else (8 + (c & 7)) * 2.0 ** ((c >> 3) - 10) for c in range(127)] + [np.nan])


def values(codes):
    c = codes.cpu().numpy().astype(np.int64)
    return np.where(c & 128, -1.0, 1.0) * E4M3[c & 127]


def quantise(x):
    """(codes, scale) of one block in 64 bits."""
    fine = np.isfinite(x)
    big = abs(np.where(fine, x, 0)).max()
    e = -100
    while big > 448 * 2.0 ** e:
        e += 1
    y = abs(np.where(fine, x, 0)) / 2.0 ** e
    hi = np.searchsorted(E4M3[:127], y).clip(0, 126)
    lo = (hi - 1).clip(0)
    dl, dh = y - E4M3[lo], E4M3[hi] - y
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    code = np.where(np.signbit(x), code | 128, code)
    return np.where(fine, code, 127), 2.0 ** e


def normal(shape, seed, dtype, spread=0.0):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal(shape).astype(np.float32)
    if spread:
        x *= np.exp(spread * rng.standard_normal(shape[:2] + (1, shape[3]))).astype(np.float32)
    return torch.from_numpy(x).to(TYPES[dtype]).cuda()


def problem(B, H, Hkv, Nq, N, d, C, g, K, causal, dtype, cap=0):
    return pisa.make_problem(B, H, Hkv, Nq, N, d, C, g, K, causal, dtype, Ncap=cap)


def new_pyramid(p):
    return torch.full((p.B, p.Hkv, pisa.pisa_pyramid_layout(p)[1], p.d), float("nan"), device="cuda")


def at(p, n):
    q = pisa.Problem(*[getattr(p, f) for f, _ in pisa.Problem._fields_])
    q.N, q.Nq, q.Ncap = n, 1, p.Ncap or p.N
    return q


def append_in(p, cache, k, v, steps, pyr=None):
    n = 0
    for new in steps:
        pisa.qcache_append(at(p, n + new), cache, k[:, :, n:n + new], v[:, :, n:n + new], n, pyr)
        n += new
    assert n == p.N


def check_cache(p, cache, k, v):
    C, M = p.C, -(-p.N // p.C)
    for x, codes, scale, raw in ((k, cache.k, cache.k_scale, cache.k_open), (v, cache.v, cache.v_scale, cache.v_open)):
        x64 = x.double().cpu().numpy()
        c, s = codes.cpu().numpy(), scale.double().cpu().numpy()
        for b in range(p.B):
            for h in range(p.Hkv):
                for j in range(M):
                    rows = x64[b, h, j * C:min(p.N, (j + 1) * C)]
                    want, e = quantise(rows)
                    got = c[b, h, j].T if codes is cache.v else c[b, h, j]
                    assert s[b, h, j] == e, (b, h, j)
                    same = (got[:len(rows)] == want) | (np.isnan(E4M3[want & 127]) & (got[:len(rows)] & 127 == 127))
                    assert same.all(), (b, h, j, np.argwhere(~same)[:3], got[:len(rows)][~same][:3], want[~same][:3])
                    assert (got[len(rows):] == 0).all(), "codes of tokens that do not exist"
        n = p.N - (M - 1) * C
        assert torch.equal(raw[:, :, :n].view(torch.uint8), x[:, :, (M - 1) * C:].contiguous().view(torch.uint8))


CACHES = [
    # B, Hkv, N, d, C, g, dtype, cap, appended at a time
    (1, 1, 1, 128, 64, 2, "bf16", 0, [[1]]),
    (2, 3, 200, 64, 32, 2, "bf16", 0, [[200], [1, 31, 1, 64, 103], [32, 32, 136], [199, 1]]),
    (1, 2, 1000, 128, 64, 4, "f32", 1111, [[1000], [999, 1], [64] * 15 + [40], [130, 1, 1, 868]]),
    (1, 1, 700, 128, 256, 2, "bf16", 0, [[700], [255, 2, 256, 187], [512, 188]]),
    (2, 1, 301, 64, 96, 3, "f32", 302, [[301], [96, 96, 96, 13], [100, 100, 100, 1]]),
    (1, 2, 1089, 64, 32, 16, "bf16", 2000, [[1089], [512, 1, 576], [513, 576], [1088, 1]]),
    (1, 1, 1025, 64, 32, 2, "bf16", 4000, [[1025], [512, 513], [32] * 32 + [1], [544, 481]]),
]


@pytest.mark.parametrize("B,Hkv,N,d,C,g,dtype,cap,orders", CACHES)
def test_append_in_any_steps(B, Hkv, N, d, C, g, dtype, cap, orders):
    p = problem(B, Hkv, Hkv, 1, N, d, C, g, 4, 1, dtype, cap)
    k, v = normal((B, Hkv, N, d), 1, dtype, 0.7), normal((B, Hkv, N, d), 2, dtype, 0.7)
    full = normal((B, Hkv, cap or N, d), 1, dtype)
    full[:, :, :N] = k
    want_pyr = new_pyramid(p)
    pisa.pisa_build_pyramid(p, full, want_pyr)
    for order in orders:
        cache, pyr = pisa.make_qcache(p), new_pyramid(p)
        append_in(p, cache, k, v, order, pyr)
        check_cache(p, cache, k, v)
        assert torch.equal(torch.nan_to_num(pyr, 7.0), torch.nan_to_num(want_pyr, 7.0)), order
        bare = pisa.make_qcache(p)
        append_in(p, bare, k, v, order)
        assert torch.equal(bare.k, cache.k) and torch.equal(bare.v, cache.v)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_every_magnitude(dtype, d):
    """Blocks whose largest value sits at, just below and just above a scale's border, from tiny to the type's largest;
    zeros, subnormals, infinities, NaN; values half way between two codes."""
    C = 32
    tops = [0.0, 1e-45, 1e-40, 2.0 ** -126, 448 * 2.0 ** -100, 448 * 2.0 ** -99, 1.0, 448.0, 3.3e38]
    tops += [float(np.float32(448 * s) * np.float32(1 + t)) for s in (1.0, 2.0 ** 9, 2.0 ** -20) for t in (-2.0 ** -9, 2.0 ** -7)]
    rng = np.random.default_rng(5)
    blocks = []
    for top in tops:
        x = rng.uniform(-1, 1, (C, d)) * top
        x[0, 0], x[5, 7] = top, -top
        blocks.append(x)
    halves = (E4M3[:126] + E4M3[1:127]) / 2  # each rounds to the even code of its two
    x = np.zeros((C, d))
    x.flat[:126], x.flat[126:252], x.flat[252] = halves, -halves, 448.0
    blocks += [x, x * 2.0 ** -30]
    x = rng.standard_normal((C, d))
    x[1, 1], x[2, 2], x[3, 3] = np.inf, -np.inf, np.nan
    blocks += [x, np.full((C, d), np.nan), np.full((C, d), -0.0)]
    k = torch.from_numpy(np.concatenate(blocks).astype(np.float32)).to(TYPES[dtype]).cuda()[None, None]
    N = k.shape[2]
    p = problem(1, 1, 1, 1, N, d, C, 2, 4, 1, dtype)
    cache = pisa.make_qcache(p)
    pisa.qcache_append(p, cache, k, k, 0)
    check_cache(p, cache, k, k)


def test_strided_rows_and_untouched_neighbours():
    """Rows out of a packed projection; blocks before the first changed one, blocks past the last and rows of the raw
    buffer past the last stay as they were, and so does what lies around every buffer."""
    B, Hkv, N, d, C, cap = 2, 2, 150, 64, 32, 320
    p = problem(B, Hkv, Hkv, 1, N, d, C, 2, 4, 1, "bf16", cap)
    packed = normal((B, N, 3 * Hkv, d), 3, "bf16")
    k, v = packed[:, :, :Hkv].transpose(1, 2), packed[:, :, 2 * Hkv:].transpose(1, 2)
    want = pisa.make_qcache(p)
    pisa.qcache_append(p, want, k.contiguous(), v.contiguous(), 0)
    raws = {}

    def guarded(shape, dtype):
        n = int(np.prod(shape)) * torch.empty((), dtype=dtype).element_size()
        raw = torch.full((n + 8192,), 0xA5, dtype=torch.uint8, device="cuda")
        raws[len(raws)] = (raw, n)
        return raw[4096:4096 + n].view(dtype).reshape(shape)
    M = pisa.pisa_qcache_blocks(p)
    cache = pisa.QCache(guarded((B, Hkv, M, C, d), torch.uint8), guarded((B, Hkv, M, d, C), torch.uint8),
                        guarded((B, Hkv, M), torch.float32), guarded((B, Hkv, M), torch.float32),
                        guarded((B, Hkv, C, d), torch.bfloat16), guarded((B, Hkv, C, d), torch.bfloat16))
    append_in(p, cache, k, v, [70, 60, 20])
    used = -(-N // C)
    for got, ref in ((cache.k, want.k), (cache.v, want.v), (cache.k_scale, want.k_scale), (cache.v_scale, want.v_scale)):
        assert torch.equal(got[:, :, :used], ref[:, :, :used])
        assert bool((got[:, :, used:].contiguous().view(torch.uint8) == 0xA5).all())
    # one row for every token and head
    one, same = normal((1, 1, 1, d), 5, "bf16").expand(B, Hkv, N, d), (pisa.make_qcache(p), pisa.make_qcache(p))
    pisa.qcache_append(p, same[0], one, one, 0)
    pisa.qcache_append(p, same[1], one.contiguous(), one.contiguous(), 0)
    assert torch.equal(same[0].k, same[1].k) and torch.equal(same[0].v, same[1].v) and torch.equal(same[0].v_open, same[1].v_open)
    before = cache.k[:, :, :4].clone()
    pisa.qcache_append(p, cache, k[:, :, 140:], v[:, :, 140:], 140)
    assert torch.equal(cache.k[:, :, :4], before) and torch.equal(cache.k[:, :, 4], want.k[:, :, 4])
    for raw, n in raws.values():
        assert bool((raw[:4096] == 0xA5).all()) and bool((raw[4096 + n:] == 0xA5).all())


# -------------------------------------------------------------- attention ---

def reference(p, cache, q, idx, rows=None, more=0.0):
    """(o, lse, bound of o's error, of lse's) in 64 bits, of the given rows (default: all; others stay 0); `more`: another
    relative error of what is summed."""
    C, d, G, M = p.C, p.d, p.H // p.Hkv, -(-p.N // p.C)
    kk = values(cache.k) * cache.k_scale.double().cpu().numpy()[..., None, None]
    vv = values(cache.v).swapaxes(-1, -2) * cache.v_scale.double().cpu().numpy()[..., None, None]
    q64, sel = q.double().cpu().numpy(), idx.cpu().numpy()
    o = np.zeros((p.B, p.H, p.Nq, d))
    lse = np.full((p.B, p.H, p.Nq), -np.inf)
    tol_o, tol_l = np.zeros_like(o), np.zeros_like(lse)
    half, weight = (2.0 ** -8, 2.0 ** -11) if p.dtype == pisa.PISA_DTYPE_BF16 else (0.0, 0.0)
    for b in range(p.B):
        for hk in range(p.Hkv):
            for r in range(p.Nq) if rows is None else rows:
                t = p.N - p.Nq + r if p.causal else p.N - 1
                blocks = [j for j in sel[b, hk, r] if 0 <= j < M]
                tok = np.concatenate([np.arange(j * C, min((j + 1) * C, t + 1)) for j in blocks] or [np.zeros(0, int)]).astype(int)
                if not len(tok):
                    continue
                kt, vt = kk[b, hk].reshape(-1, d)[tok], vv[b, hk].reshape(-1, d)[tok]
                for h in range(hk * G, (hk + 1) * G):
                    z = kt @ q64[b, h, r] / math.sqrt(d)
                    m = z.max()
                    w = np.exp(z - m)
                    n, total = len(tok), w.sum()
                    w /= total
                    o[b, h, r], lse[b, h, r] = w @ vt, m + math.log(total)
                    delta = (d + 4) * 2.0 ** -24 * (abs(kt) @ abs(q64[b, h, r])).max() / math.sqrt(d)
                    rel = math.expm1(2 * delta) + 2.0 ** -21 + 2.0 ** -23 * (m - z).max()
                    tol_o[b, h, r] = (2 * rel + weight + more + 2 * n * 2.0 ** -24) * (w @ abs(vt)) + (half + 2.0 ** -23) * abs(o[b, h, r])
                    tol_l[b, h, r] = delta + rel + n * 2.0 ** -24 + 2.0 ** -22 * max(1, abs(lse[b, h, r]))
    return o, lse, tol_o, tol_l


def check_attention(p, cache, q, idx, o, lse, rows=None):
    want_o, want_l, tol_o, tol_l = reference(p, cache, q, idx, rows)
    got_o, got_l = o.double().cpu().numpy(), lse.double().cpu().numpy()
    if rows is not None:
        want_o, want_l, tol_o, tol_l, got_o, got_l = (x[:, :, rows] for x in (want_o, want_l, tol_o, tol_l, got_o, got_l))
    empty = np.isneginf(want_l)
    assert np.array_equal(np.isneginf(got_l), empty) and (got_o[empty] == 0).all()
    off = abs(got_o - want_o) - tol_o
    assert (off <= 0).all(), (off.max(), np.argwhere(off > 0)[:3])
    off = abs(got_l[~empty] - want_l[~empty]) - tol_l[~empty]
    assert (off <= 0).all(), off.max()


def random_selection(p, seed, padding=True):
    """Distinct blocks per row: the row's own one, others at random (some after the row), padding of every kind."""
    rng = np.random.default_rng(seed)
    M = -(-p.N // p.C)
    idx = np.full((p.B, p.Hkv, p.Nq, p.K), -1, np.int32)
    for b in range(p.B):
        for h in range(p.Hkv):
            for r in range(p.Nq):
                own = (p.N - p.Nq + r) // p.C
                rest = rng.permutation([j for j in range(M) if j != own])
                n = int(rng.integers(1, min(p.K, M) + 1)) if padding else min(p.K, M)
                row = [own, *rest[:n - 1]]
                row += [int(rng.choice([-1, -7, M, M + 3, 2 ** 31 - 1, -2 ** 31])) for _ in range(p.K - n)] if padding else [-1] * (p.K - n)
                idx[b, h, r] = rng.permutation(row)
    return torch.from_numpy(idx).cuda()


SHAPES = [
    # B, H, Hkv, Nq, N, d, C, g, K, causal, dtype, cap
    (1, 1, 1, 1, 1, 128, 64, 2, 4, 1, "bf16", 0),
    (1, 1, 1, 1, 1, 64, 32, 2, 1, 0, "f32", 0),
    (1, 8, 8, 1, 2000, 128, 64, 2, 16, 1, "bf16", 2112),
    (2, 8, 2, 1, 777, 128, 64, 2, 8, 1, "bf16", 0),
    (1, 16, 1, 3, 500, 64, 32, 2, 8, 1, "bf16", 0),
    (1, 3, 1, 40, 333, 128, 96, 2, 3, 1, "bf16", 400),
    (2, 5, 1, 7, 900, 64, 128, 4, 5, 1, "bf16", 0),
    (1, 4, 2, 5, 1500, 128, 256, 3, 4, 1, "bf16", 0),
    (1, 2, 2, 65, 1000, 64, 64, 2, 4, 1, "f32", 0),
    (1, 6, 2, 9, 450, 128, 32, 2, 6, 1, "f32", 0),
    (1, 16, 1, 2, 1100, 128, 160, 2, 4, 0, "f32", 1300),
    (1, 4, 4, 70, 70, 64, 32, 2, 3, 0, "bf16", 0),
    (1, 4, 2, 300, 300, 128, 64, 2, 5, 1, "bf16", 0),
    (1, 2, 1, 2, 4100, 64, 32, 2, 120, 1, "bf16", 0),
    # from few rows, whose units are spread over workgroups, to many, one wavefront each; 16 heads to a KV head
    (1, 16, 1, 1, 1000, 128, 64, 2, 8, 1, "bf16", 0),
    (1, 16, 1, 2, 3000, 128, 64, 2, 16, 1, "bf16", 0),
    (2, 8, 2, 3, 3000, 128, 128, 4, 30, 1, "bf16", 3100),
    (2, 8, 2, 2, 2500, 128, 128, 4, 20, 0, "f32", 0),
    (1, 4, 4, 40, 1500, 64, 64, 2, 16, 1, "bf16", 0),
    (1, 2, 2, 128, 900, 64, 32, 2, 12, 1, "f32", 0),
    (1, 3, 3, 300, 600, 64, 32, 2, 7, 1, "bf16", 0),
    (1, 7, 1, 5, 1234, 128, 192, 2, 6, 1, "bf16", 1500),
    (1, 2, 2, 33, 800, 64, 224, 2, 3, 1, "f32", 0),
]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_attention(shape):
    B, H, Hkv, Nq, N, d, C, g, K, causal, dtype, cap = shape
    p = problem(*shape)
    k, v = normal((B, Hkv, N, d), 1, dtype, 0.5), normal((B, Hkv, N, d), 2, dtype, 0.5)
    q = normal((B, H, Nq, d), 3, dtype)
    cache = pisa.make_qcache(p)
    pisa.qcache_append(p, cache, k, v, 0)
    idx = random_selection(p, 4)
    o, lse = pisa.qcache_attn_fwd(p, cache, q, idx)
    check_attention(p, cache, q, idx, o, lse)


# Rows enough to be grouped by block.  Their partials are normalised and rounded to fp16 before they are weighted and
# summed: another 2^-11 of W.
GROUPED = [
    (1, 1, 1, 2500, 2600, 128, 64, 2, 16, 1, "bf16", 0),
    (1, 4, 1, 3500, 9000, 128, 64, 2, 16, 1, "bf16", 9100),
    (2, 6, 2, 1500, 2100, 64, 64, 2, 32, 1, "bf16", 0),
    (1, 4, 4, 2300, 2300, 64, 32, 2, 30, 1, "bf16", 0),
    (1, 5, 1, 2200, 4000, 128, 128, 4, 16, 1, "bf16", 0),
    (1, 2, 2, 1200, 3333, 128, 96, 2, 16, 0, "bf16", 0),
    (1, 3, 1, 1500, 2500, 64, 256, 2, 16, 1, "bf16", 0),
    (1, 9, 1, 6500, 6600, 128, 128, 2, 50, 0, "bf16", 0),
]


def quick_selection(p, seed):
    """random_selection for many rows: distinct blocks of the whole cache, some of them padding."""
    M = -(-p.N // p.C)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    order = torch.rand((p.B, p.Hkv, p.Nq, M), generator=gen, device="cuda").argsort(-1)[..., :p.K].int()
    order = torch.nn.functional.pad(order, (0, p.K - order.shape[-1]), value=-1)
    drop = torch.rand(order.shape, generator=gen, device="cuda")
    order = torch.where(drop < 0.1, -1, torch.where(drop < 0.15, M + 5, order))
    order[:, :, ::97] = -1
    return order.int().contiguous()


def sample(p, seed, n=40):
    rng = np.random.default_rng(seed)
    return sorted({0, 1, 97, p.Nq - 1, p.Nq - 2, *rng.integers(0, p.Nq, n).tolist()})


def check_grouped(p, cache, q, idx, o, lse, rows):
    want_o, want_l, tol_o, tol_l = (x[:, :, rows] for x in reference(p, cache, q, idx, rows, more=2.0 ** -11))
    got_o, got_l = o[:, :, rows].double().cpu().numpy(), lse[:, :, rows].double().cpu().numpy()
    empty = np.isneginf(want_l)
    assert np.array_equal(np.isneginf(got_l), empty) and (got_o[empty] == 0).all()
    off = abs(got_o - want_o) - tol_o
    assert (off <= 0).all(), (off.max(), np.argwhere(off > 0)[:3])
    assert (abs(got_l[~empty] - want_l[~empty]) <= tol_l[~empty]).all()


@pytest.mark.parametrize("shape", GROUPED, ids=str)
def test_many_rows(shape):
    B, H, Hkv, Nq, N, d, C, g, K, causal, dtype, cap = shape
    p = problem(*shape)
    few = problem(*shape[:3], 1, *shape[4:])
    assert pisa.pisa_qcache_attn_workspace_bytes(p) > B * H * Nq * K * d * 2 > pisa.pisa_qcache_attn_workspace_bytes(few)
    k, v = normal((B, Hkv, N, d), 1, dtype, 0.5), normal((B, Hkv, N, d), 2, dtype, 0.5)
    q = normal((B, H, Nq, d), 3, dtype)
    cache = pisa.make_qcache(p)
    pisa.qcache_append(p, cache, k, v, 0)
    idx = quick_selection(p, 4)
    o, lse = torch.full_like(q, 7.0), torch.full((B, H, Nq), 7.0, device="cuda")
    nb = pisa.pisa_qcache_attn_workspace_bytes(p)
    band = torch.full((nb + 8192,), 0xA5, dtype=torch.uint8, device="cuda")
    pisa.pisa_qcache_attn_fwd(p, cache, q, idx, o, lse, band[4096:], nb)
    check_grouped(p, cache, q, idx, o, lse, sample(p, 5))
    assert bool((band[:4096] == 0xA5).all()) and bool((band[-4096:] == 0xA5).all())
    assert torch.isfinite(o).all()
    o2 = torch.empty_like(o)
    pisa.pisa_qcache_attn_fwd(p, cache, q, idx, o2, None, band[4096:], nb)
    assert torch.equal(o2, o)


@pytest.mark.parametrize("C", [64, 128])
def test_many_rows_hidden_tokens(C):
    """Values that are NaN or infinite, and keys: rows before them are as without them, rows after them NaN where they
    attend them."""
    B, H, Hkv, Nq, N, d, K = 1, 2, 1, 4000, 4000, 128, 16
    p = problem(B, H, Hkv, Nq, N, d, C, 2, K, 1, "bf16")
    k, v, q = normal((B, Hkv, N, d), 1, "bf16"), normal((B, Hkv, N, d), 2, "bf16"), normal((B, H, Nq, d), 3, "bf16")
    idx = quick_selection(p, 4)
    rows = torch.arange(N, device="cuda")
    idx[..., 0] = (rows // C).int()  # every row its own block
    idx[..., 1:] = torch.where(idx[..., 1:] == idx[..., :1], -1, idx[..., 1:])
    clean, dirty = pisa.make_qcache(p), pisa.make_qcache(p)
    pisa.qcache_append(p, clean, k, v, 0)
    want = pisa.qcache_attn_fwd(p, clean, q, idx)
    at = [130, 131, 1000, 3999]
    pisa.qcache_append(p, dirty, k, v, 0)
    dirty.v[0, 0, at[0] // C, 5, at[0] % C] = 0x7F
    dirty.v[0, 0, at[1] // C, 77, at[1] % C] = 0xFF
    dirty.k[0, 0, at[2] // C, at[2] % C, 9] = 0x7F
    dirty.v[0, 0, at[3] // C, :, at[3] % C] = 0x7F
    o, lse = pisa.qcache_attn_fwd(p, dirty, q, idx)
    sees = torch.zeros((Nq, len(at)), dtype=torch.bool, device="cuda")
    for i, x in enumerate(at):
        sees[:, i] = (idx[0, 0] == x // C).any(-1) & (rows >= x)
    free = ~sees.any(-1)
    assert torch.equal(o[:, :, free], want[0][:, :, free]) and torch.equal(lse[:, :, free], want[1][:, :, free])
    nan = torch.isnan(o[0])
    assert bool(nan[:, sees[:, 0], 5].all()) and bool(nan[:, sees[:, 1], 77].all())
    assert bool(nan[:, sees[:, 2]].all()) and bool(nan[:, sees[:, 3]].all()) and bool(torch.isnan(lse[0][:, sees[:, 2]]).all())
    only = sees[:, 0] & ~sees[:, 1] & ~sees[:, 2] & ~sees[:, 3]
    assert int(nan[:, only].sum()) == 2 * int(only.sum())  # one dimension of each head


def test_many_rows_in_passes():
    """Partials past the bound of one pass."""
    p = problem(1, 32, 8, 9000, 9000, 128, 64, 2, 16, 1, "bf16")
    k, v = normal((1, 8, 9000, 128), 1, "bf16"), normal((1, 8, 9000, 128), 2, "bf16")
    q = torch.randn((1, 32, 9000, 128), device="cuda").bfloat16()
    cache = pisa.make_qcache(p)
    pisa.qcache_append(p, cache, k, v, 0)
    idx = quick_selection(p, 4)
    assert pisa.pisa_qcache_attn_workspace_bytes(p) < 9000 * 8 * 16 * 4 * 260
    o, lse = pisa.qcache_attn_fwd(p, cache, q, idx)
    check_grouped(p, cache, q, idx, o, lse, [5, 8063, 8064, 8065, 8066, 8067, 8999])


def test_rows_past_one_launch():
    """4.2 million rows, a wavefront each: two launches."""
    B, Hkv, Nq, N, d, C = 64, 64, 1026, 1026, 64, 32
    p = problem(B, Hkv, Hkv, Nq, N, d, C, 2, 1, 0, "f32")
    assert pisa.pisa_qcache_attn_workspace_bytes(p) == 0
    cache = pisa.make_qcache(p)
    k = torch.randn((B, Hkv, N, d), device="cuda", dtype=torch.float32)
    pisa.qcache_append(p, cache, k, k, 0)
    idx = torch.randint(0, 33, (B, Hkv, Nq, 1), dtype=torch.int32, device="cuda")
    o = torch.full((B, Hkv, Nq, d), 7.0, dtype=torch.float32, device="cuda")
    lse = torch.full((B, Hkv, Nq), 7.0, device="cuda")
    pisa.pisa_qcache_attn_fwd(p, cache, k, idx, o, lse)
    assert bool((o != 7).any(-1).all()) and bool((lse != 7).all())
    part = problem(1, 2, 2, Nq, N, d, C, 2, 1, 0, "f32")
    for b, h in ((0, 0), (63, 62)):
        cut = lambda x: x[b:b + 1, h:h + 2].contiguous()  # noqa: E731
        small = pisa.QCache(*(cut(x) for x in (cache.k, cache.v, cache.k_scale, cache.v_scale)))
        check_attention(part, small, cut(k), cut(idx), cut(o), cut(lse), [0, 1, 1023, 1024, 1025])


@pytest.mark.parametrize("Nq", [1, 33])
def test_rows_that_see_nothing(Nq):
    """Nothing selected, only blocks after the row, only padding: 0 and -inf, and other rows as ever."""
    p = problem(1, 4, 2, Nq, 640, 128, 64, 2, 4, 1, "bf16")
    k, v, q = normal((1, 2, 640, 128), 1, "bf16"), normal((1, 2, 640, 128), 2, "bf16"), normal((1, 4, Nq, 128), 3, "bf16")
    cache = pisa.make_qcache(p)
    pisa.qcache_append(p, cache, k, v, 0)
    idx = random_selection(p, 5)
    idx[0, 0, 0] = -1
    if Nq > 1:
        idx[0, 1, 1] = torch.tensor([10, 99, -3, 12])
        idx[0, 0, 5] = torch.tensor([9, -1, -1, -1]) if 640 - Nq + 5 < 576 else torch.tensor([-1, -1, -1, 10])
    o = torch.full_like(q, 7.0)
    lse = torch.full((1, 4, Nq), 7.0, device="cuda")
    nb = pisa.pisa_qcache_attn_workspace_bytes(p)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda") if nb else None
    pisa.pisa_qcache_attn_fwd(p, cache, q, idx, o, lse, ws, nb)
    check_attention(p, cache, q, idx, o, lse)
    o2 = torch.full_like(q, 7.0)
    pisa.pisa_qcache_attn_fwd(p, cache, q, idx, o2, None, ws, nb)
    assert torch.equal(o2, o)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_hidden_tokens_are_not_used(dtype):
    """NaN and infinite keys and values after a row's position, and NaN codes past N, change nothing."""
    B, H, Hkv, Nq, N, d, C = 1, 4, 2, 4, 200, 64, 64
    cap = 320
    k, v = normal((B, Hkv, N, d), 1, dtype), normal((B, Hkv, N, d), 2, dtype)
    q = normal((B, H, Nq, d), 3, dtype)
    p = problem(B, H, Hkv, Nq, N, d, C, 2, 4, 1, dtype, cap)
    idx = torch.tensor([0, 1, 2, 3], dtype=torch.int32, device="cuda").expand(B, Hkv, Nq, 4).contiguous()
    clean = pisa.make_qcache(p)
    pisa.qcache_append(p, clean, k, v, 0)
    want = pisa.qcache_attn_fwd(p, clean, q, idx)
    dirty = pisa.make_qcache(p)
    pisa.qcache_append(p, dirty, k, v, 0)
    dirty.k[:, :, 3, N - 3 * C:] = 0x7F
    dirty.v[:, :, 3, :, N - 3 * C:] = 0xFF
    dirty.k[:, :, 4:], dirty.v[:, :, 4:] = 0x7F, 0x7F
    got = pisa.qcache_attn_fwd(p, dirty, q, idx)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    # the last token alone is broken: the rows before it do not see it, the last row does
    bad_k, bad_v = k.clone(), v.clone()
    bad_k[:, :, -1], bad_v[:, :, -1] = float("nan"), float("inf")
    broken = pisa.make_qcache(p)
    pisa.qcache_append(p, broken, bad_k, bad_v, 0)
    o, lse = pisa.qcache_attn_fwd(p, broken, q, idx)
    assert torch.isfinite(o[:, :, :-1]).all() and torch.isfinite(lse[:, :, :-1]).all()
    assert torch.isnan(o[:, :, -1]).all()


def test_logits_far_apart():
    """Weights from 1 to 0 within a row, and a block whose logits are far below another's."""
    p = problem(1, 2, 1, 2, 512, 128, 64, 2, 8, 1, "f32")
    k, v, q = normal((1, 1, 512, 128), 1, "f32"), normal((1, 1, 512, 128), 2, "f32"), normal((1, 2, 2, 128), 3, "f32")
    k[:, :, 64:128] *= 300
    k[:, :, 300] *= 40
    cache = pisa.make_qcache(p)
    pisa.qcache_append(p, cache, k, v, 0)
    idx = torch.arange(8, dtype=torch.int32, device="cuda").expand(1, 1, 2, 8).contiguous()
    o, lse = pisa.qcache_attn_fwd(p, cache, q, idx)
    check_attention(p, cache, q, idx, o, lse)


def test_agrees_with_the_attention_over_what_the_codes_stand_for():
    """The same rows through pisa_sparse_attn_fwd on code * scale, which is exact in bf16: two roundings of the weights
    to bf16 (2^-8 each of the summed weights times values) and two of the output apart."""
    B, H, Hkv, Nq, N, d, C, K = 2, 8, 2, 200, 1500, 128, 64, 8
    p = problem(B, H, Hkv, Nq, N, d, C, 2, K, 1, "bf16")
    k, v, q = normal((B, Hkv, N, d), 1, "bf16", 0.5), normal((B, Hkv, N, d), 2, "bf16"), normal((B, H, Nq, d), 3, "bf16")
    cache = pisa.make_qcache(p)
    pisa.qcache_append(p, cache, k, v, 0)
    idx = random_selection(p, 6, padding=False)
    kk = (torch.from_numpy(values(cache.k)).cuda() * cache.k_scale[..., None, None]).flatten(2, 3)[:, :, :N]
    vv = (torch.from_numpy(values(cache.v)).cuda() * cache.v_scale[..., None, None]).transpose(-1, -2).flatten(2, 3)[:, :, :N]
    o, lse = pisa.qcache_attn_fwd(p, cache, q, idx)
    o2, lse2 = pisa.sparse_attn_fwd(p, q, kk.bfloat16().contiguous(), vv.bfloat16().contiguous(), idx)
    assert torch.equal(kk.bfloat16().double(), kk) and torch.equal(vv.bfloat16().double(), vv)
    top = vv.abs().max().item()
    assert (o.float() - o2.float()).abs().max().item() <= 4 * 2.0 ** -8 * top
    assert (lse - lse2).abs().max().item() <= 1e-4


def test_guards_and_streams():
    """Outputs and workspace between guard bands, on another stream."""
    B, H, Hkv, Nq, N, d, C, K = 1, 12, 4, 3, 3000, 128, 64, 16
    p = problem(B, H, Hkv, Nq, N, d, C, 2, K, 1, "bf16")
    k, v, q = normal((B, Hkv, N, d), 1, "bf16"), normal((B, Hkv, N, d), 2, "bf16"), normal((B, H, Nq, d), 3, "bf16")
    cache = pisa.make_qcache(p)
    pisa.qcache_append(p, cache, k, v, 0)
    idx = random_selection(p, 7)
    want_o, want_l = pisa.qcache_attn_fwd(p, cache, q, idx)
    torch.cuda.synchronize()
    nb = pisa.pisa_qcache_attn_workspace_bytes(p)
    bands = [torch.full((n + 8192,), 0xA5, dtype=torch.uint8, device="cuda") for n in (want_o.numel() * 2, want_l.numel() * 4, nb)]
    o, lse = bands[0][4096:-4096].view(torch.bfloat16).view_as(want_o), bands[1][4096:-4096].view(torch.float32).view_as(want_l)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    pisa.pisa_qcache_attn_fwd(p, cache, q, idx, o, lse, bands[2][4096:] if nb else None, nb, side)
    side.synchronize()
    assert torch.equal(o, want_o) and torch.equal(lse, want_l)
    for x in bands:
        assert bool((x[:4096] == 0xA5).all()) and bool((x[-4096:] == 0xA5).all())


def test_offsets_past_32_bits():
    """A cache of 4.3 GB of keys: rows that attend its last blocks, and an append to its last one."""
    Hkv, d, C, M, K, Nq = 8, 128, 64, 65535, 8, 3
    N = M * C
    p = problem(1, 16, Hkv, Nq, N, d, C, 2, K, 0, "bf16")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    codes = lambda shape: torch.randint(0, 0x70, shape, generator=gen, device="cuda", dtype=torch.uint8)  # noqa: E731
    scale = lambda: 2.0 ** torch.randint(-6, -3, (1, Hkv, M), generator=gen, device="cuda").float()  # noqa: E731
    raw = normal((1, Hkv, C, d), 2, "bf16")
    big = pisa.QCache(codes((1, Hkv, M, C, d)), codes((1, Hkv, M, d, C)), scale(), scale(), raw.clone(), raw.clone())
    q = normal((1, 16, Nq, d), 3, "bf16")
    blocks = torch.stack([torch.tensor([M - 1 - j * 7 - h for j in range(K)], device="cuda") for h in range(Hkv)])
    idx = blocks[None, :, None].expand(1, Hkv, Nq, K).int().contiguous()
    o, lse = pisa.qcache_attn_fwd(p, big, q, idx)
    small_p = problem(1, 16, Hkv, Nq, K * C, d, C, 2, K, 0, "bf16")
    h = torch.arange(Hkv, device="cuda")[:, None]
    small = pisa.QCache(*(x[0][h, blocks][None].contiguous() for x in (big.k, big.v, big.k_scale, big.v_scale)))
    order = torch.arange(K, dtype=torch.int32, device="cuda").expand(1, Hkv, Nq, K).contiguous()
    want = pisa.qcache_attn_fwd(small_p, small, q, order)
    assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
    check_attention(small_p, small, q, order, o, lse)
    new = normal((1, Hkv, 3, d), 4, "bf16")
    before = big.k[:, :, :M - 1].sum(dtype=torch.int64)
    pisa.qcache_append(p, big, new, new, N - 3)
    rows = torch.cat((raw[:, :, :C - 3], new), 2)
    last = pisa.QCache(*(x[:, :, M - 1:].contiguous() for x in (big.k, big.v, big.k_scale, big.v_scale)), big.k_open, big.v_open)
    check_cache(problem(1, Hkv, Hkv, 1, C, d, C, 2, 4, 1, "bf16"), last, rows, rows)
    assert big.k[:, :, :M - 1].sum(dtype=torch.int64) == before


# ------------------------------------------------------- together, as used ---

def test_a_sequence_from_prompt_to_tokens():
    """Rotary positions, append, block selection from the pyramid, attention: a prompt and then tokens one by one, out
    of packed projections, as a serving loop runs them; the cache at the end is that of one append."""
    B, H, Hkv, d, C, g, K, n0, steps, cap = 2, 8, 2, 128, 64, 2, 4, 517, 70, 704
    rng = np.random.default_rng(11)
    packed = torch.from_numpy(rng.standard_normal((B, n0 + steps, H + 2 * Hkv, d)).astype(np.float32)).bfloat16().cuda()
    p_all = problem(B, H, Hkv, 1, n0 + steps, d, C, g, K, 1, "bf16", cap)
    cache, pyr = pisa.make_qcache(p_all), new_pyramid(p_all)
    keys, n = [], 0
    for new in [n0] + [1] * steps:
        p = problem(B, H, Hkv, new, n + new, d, C, g, K, 1, "bf16", cap)
        x = packed[:, n:n + new]
        r = pisa.make_rope(B, H, Hkv, new, d, pos0=n, scaling="parts", factor=4.0, ctx=256)
        q, k = pisa.rope_fwd(r, x[:, :, :H].transpose(1, 2), x[:, :, H:H + Hkv].transpose(1, 2))
        pisa.qcache_append(p, cache, k, x[:, :, H + Hkv:].transpose(1, 2), n, pyr)
        idx = pisa.select_flat_bsa(p, q, pyr)
        o, lse = pisa.qcache_attn_fwd(p, cache, q, idx)
        keys.append(k)
        if new > 1 or n in (n0, n0 + 58, n0 + 59, n0 + steps - 1):
            if new > 1:  # the last rows of the prompt
                tail = problem(B, H, Hkv, 5, n + new, d, C, g, K, 1, "bf16", cap)
                check_attention(tail, cache, q[:, :, -5:].contiguous(), idx[:, :, -5:].contiguous(), o[:, :, -5:], lse[:, :, -5:])
            else:
                check_attention(p, cache, q, idx, o, lse)
        n += new
    k = torch.cat(keys, 2)
    check_cache(p_all, cache, k, packed[:, :, H + Hkv:].transpose(1, 2).contiguous())
    full = torch.zeros((B, Hkv, cap, d), dtype=torch.bfloat16, device="cuda")
    full[:, :, :n] = k
    want = new_pyramid(p_all)
    pisa.pisa_build_pyramid(p_all, full, want)
    assert torch.equal(torch.nan_to_num(pyr, 7.0), torch.nan_to_num(want, 7.0))


def test_a_cache_that_grows():
    """Appends across a growth: as in buffers that were large enough from the start."""
    B, Hkv, d, C, g, n, cap = 2, 2, 64, 32, 2, 500, 480
    k, v = normal((B, Hkv, n, d), 1, "bf16"), normal((B, Hkv, n, d), 2, "bf16")
    p = problem(B, Hkv, Hkv, 1, 470, d, C, g, 4, 1, "bf16", cap)
    cache, pyr = pisa.make_qcache(p), new_pyramid(p)
    pisa.qcache_append(p, cache, k[:, :, :470], v[:, :, :470], 0, pyr)
    bigger = pisa.pisa_cache_capacity(cap, n, C)
    p, cache, pyr = pisa.grow_qcache(p, bigger, cache, pyr)
    p = problem(B, Hkv, Hkv, 1, n, d, C, g, 4, 1, "bf16", bigger)
    pisa.qcache_append(p, cache, k[:, :, 470:], v[:, :, 470:], 470, pyr)
    check_cache(p, cache, k, v)
    want = pisa.make_qcache(p), new_pyramid(p)
    pisa.qcache_append(p, want[0], k, v, 0, want[1])
    levels = torch.isfinite(want[1])
    assert torch.equal(pyr[levels], want[1][levels])
    with pytest.raises(ValueError):
        pisa.grow_qcache(p, n - 1, cache)


def test_graph_replays_match_eager():
    """One generated token (rotary positions, append, attention) captured and replayed on new inputs, with the program's
    own work between the replays."""
    B, H, Hkv, N, d, C, g, K = 2, 8, 2, 1000, 128, 64, 2, 8
    p = problem(B, H, Hkv, 1, N, d, C, g, K, 1, "bf16", 1024)
    k0, v0 = normal((B, Hkv, N - 1, d), 1, "bf16"), normal((B, Hkv, N - 1, d), 2, "bf16")
    cache, pyr = pisa.make_qcache(p), new_pyramid(p)
    pisa.qcache_append(at(p, N - 1), cache, k0, v0, 0, pyr)
    idx = random_selection(p, 8)
    r = pisa.make_rope(B, H, Hkv, 1, d)
    x = normal((B, 1, H + 2 * Hkv, d), 9, "bf16")
    pos = torch.full((B, 1), N - 1, dtype=torch.int32, device="cuda")
    q, k = torch.empty((B, H, 1, d), dtype=torch.bfloat16, device="cuda"), torch.empty((B, Hkv, 1, d), dtype=torch.bfloat16, device="cuda")
    o, lse = torch.empty_like(q), torch.empty((B, H, 1), device="cuda")
    nb = pisa.pisa_qcache_attn_workspace_bytes(p)
    ws = torch.empty(max(nb, 1), dtype=torch.uint8, device="cuda")

    def step():
        pisa.rope_fwd(r, x[:, :, :H].transpose(1, 2), x[:, :, H:H + Hkv].transpose(1, 2), pos, q, k)
        pisa.qcache_append(p, cache, k, x[:, :, H + Hkv:].transpose(1, 2), N - 1, pyr)
        pisa.pisa_qcache_attn_fwd(p, cache, q, idx, o, lse, ws, nb)
    inputs = [normal((B, 1, H + 2 * Hkv, d), 20 + i, "bf16") for i in range(4)]
    eager = []
    for y in inputs:
        x.copy_(y)
        step()
        torch.cuda.synchronize()
        eager.append([t.clone() for t in (o, lse, cache.k, cache.v, cache.k_scale, pyr)])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in (2, 0, 3, 1, 1):
        x.copy_(inputs[i])
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip((o, lse, cache.k, cache.v, cache.k_scale, pyr), eager[i]):
            assert torch.equal(torch.nan_to_num(got.float(), 7.0), torch.nan_to_num(want.float(), 7.0)), i
        (torch.randn(1000, device="cuda") @ torch.randn(1000, device="cuda")).item()


def test_two_graphs_share_a_workspace():
    """Many rows and few rows of one cache, captured on their own with one workspace, replayed in turn with eager work
    between."""
    H, Hkv, N, d, C, K = 8, 4, 3000, 128, 64, 16
    k, v = normal((1, Hkv, N, d), 1, "bf16"), normal((1, Hkv, N, d), 2, "bf16")
    runs = []
    for Nq in (3000, 2):
        p = problem(1, H, Hkv, Nq, N, d, C, 2, K, 1, "bf16")
        runs.append([p, normal((1, H, Nq, d), 3, "bf16"), quick_selection(p, Nq), torch.empty((1, H, Nq, d), dtype=torch.bfloat16, device="cuda"),
                     torch.empty((1, H, Nq), device="cuda")])
    cache = pisa.make_qcache(runs[0][0])
    pisa.qcache_append(runs[0][0], cache, k, v, 0)
    need = [pisa.pisa_qcache_attn_workspace_bytes(x[0]) for x in runs]
    assert min(need) > 0
    ws = torch.empty(max(need), dtype=torch.uint8, device="cuda")
    call = lambda x: pisa.pisa_qcache_attn_fwd(x[0], cache, *x[1:], ws, ws.numel())  # noqa: E731
    graphs = []
    for x in runs:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call(x)
        torch.cuda.current_stream().wait_stream(side)
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call(x)
    for i, n in enumerate((0, 1, 1, 0, 1, 0)):
        x = runs[n]
        x[1].copy_(normal(x[1].shape, 30 + i, "bf16"))
        call(x)
        torch.cuda.synchronize()
        want = [t.clone() for t in x[3:]]
        x[3].fill_(7)
        x[4].fill_(7)
        graphs[n].replay()
        torch.cuda.synchronize()
        assert torch.equal(x[3], want[0]) and torch.equal(x[4], want[1]), i


def test_wrapper_refusals():
    p = problem(1, 2, 1, 1, 100, 64, 32, 2, 4, 1, "bf16")
    cache = pisa.make_qcache(p)
    k = torch.zeros((1, 1, 100, 64), dtype=torch.bfloat16, device="cuda")
    for bad in (k.cpu(), k.float(), k[:, :, :99], k[..., ::2]):
        with pytest.raises(ValueError):
            pisa.qcache_append(p, cache, bad, k, 0)
    with pytest.raises(ValueError):
        pisa.qcache_append(p, cache, k, k, 0, torch.zeros((1, 1, 3, 64), device="cuda"))
    with pytest.raises(ValueError):
        pisa.qcache_append(problem(1, 2, 1, 1, 100, 64, 32, 2, 4, 1, "f32"), cache, k.float(), k.float(), 0)
    with pytest.raises(ValueError):
        pisa.qcache_append(problem(1, 2, 1, 1, 130, 64, 32, 2, 4, 1, "bf16"), cache, k[:, :, :30], k[:, :, :30], 100)
    q, idx = torch.zeros((1, 2, 1, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((1, 1, 1, 4), dtype=torch.int32, device="cuda")
    for bad_q, bad_idx in ((q.float(), idx), (q, idx.long()), (q[:, :1], idx), (q, idx[..., :3])):
        with pytest.raises(ValueError):
            pisa.qcache_attn_fwd(p, cache, bad_q, bad_idx)
    with pytest.raises(ValueError):
        pisa.QCache(cache.k, cache.k, cache.k_scale, cache.v_scale)
    with pytest.raises(ValueError):
        pisa.QCache(cache.k.cpu(), cache.v.cpu(), cache.k_scale.cpu(), cache.v_scale.cpu())
