"""Trees of drafted tokens on the GPU: masks and positions against a walk up the parents; accepted rows appended to a cache,
bit for bit what copies and an append in order leave."""
import numpy as np
import pytest
import torch

import test_gpu_qcache as base

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2609_31093_amd import pisa


def walked(parents, n):
    """(mask bits [B, T, T], positions) by the definition."""
    B, T = parents.shape
    bits, pos = np.zeros((B, T, T), bool), np.full((B, T), n, np.int64)
    for b in range(B):
        for i in range(T):
            if parents[b, i] < -1:
                continue
            j, seen = i, set()
            while 0 <= j < T and j not in seen:
                seen.add(j)
                j = parents[b, j]
            bits[b, i, list(seen)] = True
            pos[b, i] = n + (T - 1 if 0 <= j < T else len(seen) - 1)
    return bits, pos


def unpack(mask, T):
    m = mask.cpu().numpy().view(np.uint64)
    j = np.arange(T)
    assert m.shape[-1] == -(-T // 64)
    rest = np.arange(T, m.shape[-1] * 64)
    assert ((m[..., rest // 64] >> (rest % 64).astype(np.uint64)) & np.uint64(1) == 0).all(), "bits past the last token"
    return ((m[..., j // 64] >> (j % 64).astype(np.uint64)) & np.uint64(1)).astype(bool)


def check_layout(parents, n):
    parents = np.asarray(parents, np.int32)
    mask, pos = pisa.draft_layout(torch.from_numpy(parents).cuda(), n)
    bits, want = walked(parents, n)
    assert np.array_equal(unpack(mask, parents.shape[1]), bits)
    assert np.array_equal(pos.cpu().numpy(), want)


@pytest.mark.parametrize("T", [1, 2, 3, 63, 64, 65, 128, 129, 777, 1023, 1024])
def test_layout(T):
    rng = np.random.default_rng(T)
    i = np.arange(T)
    chain, star = i - 1, np.where(i == 0, -1, 0)
    back = i[::-1] * 0 + np.where(i == T - 1, -1, i + 1)                   # parents behind their children
    tree = np.array([-1] + [int(rng.integers(max(0, x - 8), x)) for x in range(1, T)])
    forest = np.where(rng.random(T) < 0.1, -1, tree)
    order = rng.permutation(T)
    mixed = np.empty(T, int)
    mixed[order] = np.where(tree < 0, -1, order[tree])                      # the tree's tokens in any order
    check_layout([chain, star, back, tree, forest, mixed], 20010)


@pytest.mark.parametrize("T", [1, 5, 70, 1024])
def test_layout_of_odd_parents(T):
    """Tokens that pad (and children of them), parents out of range, circles and ways into them."""
    rng = np.random.default_rng(T)
    wild = rng.integers(-3, T + 3, (4, T))
    wild[1] = rng.choice([-2, -2 ** 31, -1, 0, T, 2 ** 31 - 1], T)
    wild[2] = (np.arange(T) + 1) % T          # one circle of all
    wild[3] = np.arange(T)                    # every token its own parent
    check_layout(wild, 0)
    check_layout(wild, 2 ** 31 - 1 - T)


def test_layout_of_part_of_a_batch():
    """Sequences of a batch on their own, which begin at any multiple of a value's size; their masks into attention."""
    parents = torch.randint(-1, 7, (4, 7), dtype=torch.int32, device="cuda")
    mask, pos = pisa.draft_layout(parents, 50)
    p = base.problem(1, 2, 1, 7, 57, 64, 32, 2, 3, 1, "bf16")
    x = [base.normal((1, h, n, 64), i, "bf16") for i, (h, n) in enumerate(((2, 7), (1, 57), (1, 57), (1, 7), (1, 7)))]
    idx = torch.tensor([0, 1, -1], dtype=torch.int32, device="cuda").expand(1, 1, 7, 3).contiguous()
    for b in range(1, 4):
        got = pisa.draft_layout(parents[b:b + 1], 50)
        assert torch.equal(got[0][0], mask[b]) and torch.equal(got[1][0], pos[b])
        a = pisa.draft_attn_fwd(p, x[0], x[1], x[2], idx, x[3], x[4], mask[b])
        c = pisa.draft_attn_fwd(p, x[0], x[1], x[2], idx, x[3], x[4], mask[b].clone())
        assert torch.equal(a[0], c[0]) and torch.equal(a[1], c[1])


def test_layout_without_positions_captured():
    parents = torch.tensor([[-1, 0, 1, 1, 0], [-1, -1, -2, 2, 3]], dtype=torch.int32, device="cuda")
    mask = torch.full((2, 5, 1), -1, dtype=torch.int64, device="cuda")
    pisa.pisa_draft_layout(2, 5, parents, 7, mask)
    assert torch.equal(mask, pisa.draft_layout(parents, 7)[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = pisa.draft_layout(parents, 7)
    for i in range(3):
        parents.copy_(torch.randint(-2, 5, (2, 5)).int())
        want = pisa.draft_layout(parents, 7)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


# ------------------------------------------------------------------ append ---

APPENDS = [
    # B, Hkv, n_old, T, m, d, C, g, dtype, cap
    (1, 1, 0, 1, 1, 64, 32, 2, "bf16", 40),
    (1, 2, 0, 200, 150, 128, 64, 2, "f32", 300),       # into an empty cache
    (2, 2, 130, 16, 5, 128, 64, 2, "bf16", 400),       # within a block
    (2, 2, 126, 16, 5, 128, 64, 2, "f32", 400),        # past a border
    (1, 3, 128, 64, 9, 64, 64, 4, "bf16", 400),        # from the border on
    (4, 4, 2044, 64, 40, 64, 32, 2, "bf16", 3000),     # a new level
    (1, 1, 63, 1024, 1000, 128, 256, 2, "bf16", 1500),
    (2, 1, 500, 300, 257, 64, 96, 3, "f32", 800),
    (1, 2, 4000, 8, 1, 128, 32, 16, "bf16", 4100),
]


def start(p, n_old, T, dtype):
    k, v = base.normal((p.B, p.Hkv, max(n_old, 1), p.d), 1, dtype, 0.7), base.normal((p.B, p.Hkv, max(n_old, 1), p.d), 2, dtype, 0.7)
    # drafted rows: keys as rows of heads, values as a slice of a packed projection
    k_new = base.normal((p.B, T, p.Hkv, p.d), 3, dtype).transpose(1, 2)
    v_new = base.normal((p.B, T, 3 * p.Hkv, p.d), 4, dtype)[:, :, 2 * p.Hkv:].transpose(1, 2)
    return k[:, :, :n_old], v[:, :, :n_old], k_new, v_new


def chosen(B, T, m, seed):
    """Rows in order, in any order, one row for all, and entries outside (which are read as the nearest inside)."""
    rng = np.random.default_rng(seed)
    ordered = np.stack([np.sort(rng.permutation(T)[:m]) for _ in range(B)])
    shuffled = np.stack([rng.permutation(T)[:m] for _ in range(B)])
    wild = rng.choice([-1, -2 ** 31, 0, T // 2, T - 1, T, 2 ** 31 - 1], (B, m))
    return [torch.from_numpy(x.astype(np.int32)).cuda() for x in (ordered, shuffled, np.full((B, m), T // 3), wild)]


def gathered(x, rows):
    at = rows.long().clamp(0, x.shape[2] - 1)[:, None, :, None].expand(-1, x.shape[1], -1, x.shape[3])
    return x.gather(2, at)


@pytest.mark.parametrize("shape", APPENDS, ids=str)
def test_raw_append(shape):
    B, Hkv, n_old, T, m, d, C, g, dtype, cap = shape
    N = n_old + m
    p = base.problem(B, Hkv, Hkv, 1, N, d, C, g, 4, 1, dtype, cap)
    k, v, k_new, v_new = start(p, n_old, T, dtype)
    for rows in [None, *chosen(B, T, m, 5)]:
        new = [x[:, :, :m] if rows is None else gathered(x, rows) for x in (k_new, v_new)]
        cache = [torch.full((B, Hkv, cap, d), 7.0, dtype=base.TYPES[dtype], device="cuda") for _ in range(2)]
        for x, y in zip(cache, (k, v)):
            x[:, :, :n_old] = y
        pyr = base.new_pyramid(p)
        if n_old:
            pisa.pisa_build_pyramid(base.at(p, n_old), cache[0], pyr)
        bare = [x.clone() for x in cache]
        pisa.cache_append_rows(p, *cache, k_new, v_new, rows, n_old, pyr)
        pisa.cache_append_rows(p, *bare, k_new, v_new, rows, n_old)
        for x, y, old, z in zip(cache, new, (k, v), bare):
            assert torch.equal(x[:, :, :n_old], old) and torch.equal(x[:, :, n_old:N], y) and torch.equal(x, z)
            assert bool((x[:, :, N:] == 7.0).all()), "rows behind the last one"
        want = base.new_pyramid(p)
        pisa.pisa_build_pyramid(p, cache[0], want)
        used = torch.isfinite(want)  # nodes of the N tokens
        assert torch.equal(pyr[used], want[used])


@pytest.mark.parametrize("shape", APPENDS, ids=str)
def test_8bit_append(shape):
    B, Hkv, n_old, T, m, d, C, g, dtype, cap = shape
    N = n_old + m
    p = base.problem(B, Hkv, Hkv, 1, N, d, C, g, 4, 1, dtype, cap)
    k, v, k_new, v_new = start(p, n_old, T, dtype)
    for rows in [None, *chosen(B, T, m, 6)]:
        got, want = pisa.make_qcache(p), pisa.make_qcache(p)
        trees = base.new_pyramid(p), base.new_pyramid(p)
        for cache, pyr in zip((got, want), trees):
            if n_old:
                pisa.qcache_append(base.at(p, n_old), cache, k, v, 0, pyr)
        pisa.qcache_append_rows(p, got, k_new, v_new, rows, n_old, trees[0])
        new = [x[:, :, :m].contiguous() if rows is None else gathered(x, rows) for x in (k_new, v_new)]
        pisa.qcache_append(p, want, *new, n_old, trees[1])
        for f in ("k", "v", "k_scale", "v_scale", "k_open", "v_open"):
            assert torch.equal(getattr(got, f), getattr(want, f)), f
        assert torch.equal(torch.nan_to_num(trees[0], 7.0), torch.nan_to_num(trees[1], 7.0))


@pytest.mark.parametrize("d,C,dtype", [(64, 32, "f32"), (128, 128, "bf16")])
@pytest.mark.parametrize("g", [2, 3, 4, 16])
def test_two_blocks_at_every_count(d, C, dtype, g):
    """Appends that change the last two blocks, of as many blocks as have them under one node or two at each level."""
    cap = 40 * C
    k, v = base.normal((1, 1, cap, d), 1, dtype), base.normal((1, 1, cap, d), 2, dtype)
    for M in range(2, 38):
        for n_old, N in (((M - 1) * C - 3, (M - 1) * C + 2), ((M - 2) * C + 1, M * C), ((M - 2) * C, (M - 1) * C + 1)):
            if n_old == 0:
                continue
            p = base.problem(1, 1, 1, 1, N, d, C, g, 3, 1, dtype, cap)
            want = base.new_pyramid(p)
            pisa.pisa_build_pyramid(p, k, want)
            used = torch.isfinite(want)
            trees = [base.new_pyramid(p) for _ in range(2)]
            held = [x.clone() for x in (k, v)]
            for x in held:
                x[:, :, n_old:] = float("nan")
            cache = pisa.make_qcache(p)
            pisa.qcache_append(base.at(p, n_old), cache, k[:, :, :n_old], v[:, :, :n_old], 0, trees[0])
            pisa.pisa_build_pyramid(base.at(p, n_old), held[0], trees[1])
            new = [x[:, :, n_old:N] for x in (k, v)]
            pisa.qcache_append(p, cache, *new, n_old, trees[0])
            pisa.cache_append_rows(p, *held, *new, None, n_old, trees[1])
            for tree in trees:
                assert torch.equal(tree[used], want[used]) and not torch.isfinite(tree[~used]).any(), (M, n_old, N)
            assert torch.equal(held[0][:, :, :N], k[:, :, :N]) and torch.equal(held[1][:, :, :N], v[:, :, :N])
    p = base.problem(1, 1, 1, 1, N, d, C, g, 3, 1, dtype, cap)
    base.check_cache(p, cache, k[:, :, :N], v[:, :, :N])


@pytest.mark.parametrize("eight", [False, True])
def test_append_nothing(eight):
    p = base.problem(2, 1, 1, 1, 100, 64, 32, 2, 4, 1, "bf16", 200)
    k, v, k_new, v_new = start(p, 100, 8, "bf16")
    cache = pisa.make_qcache(p)
    pisa.qcache_append(p, cache, k, v, 0)
    none = torch.empty((2, 0), dtype=torch.int32, device="cuda")
    if eight:
        was = cache.k.clone()
        pisa.qcache_append_rows(p, cache, k_new, v_new, none, 100)
        assert torch.equal(cache.k, was)
    else:
        raw = torch.full((2, 1, 200, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        pisa.cache_append_rows(p, raw, raw.clone(), k_new, v_new, none, 100)
        assert bool((raw == 7.0).all())


@pytest.mark.parametrize("eight", [False, True])
def test_append_captured(eight):
    """A graph of an append, with other accepted rows at each replay."""
    B, Hkv, n_old, T, m, d, C, cap = 2, 2, 126, 16, 5, 64, 64, 300
    p = base.problem(B, Hkv, Hkv, 1, n_old + m, d, C, 2, 4, 1, "bf16", cap)
    k, v, k_new, v_new = start(p, n_old, T, "bf16")
    rows = torch.zeros((B, m), dtype=torch.int32, device="cuda")

    def fresh():
        pyr = base.new_pyramid(p)
        if eight:
            cache = pisa.make_qcache(p)
            pisa.qcache_append(base.at(p, n_old), cache, k, v, 0, pyr)
            held = [cache.k, cache.v, cache.k_scale, cache.v_scale, cache.k_open, cache.v_open, pyr]
            return held, lambda s=None: pisa.qcache_append_rows(p, cache, k_new, v_new, rows, n_old, pyr, stream=s)
        held = [torch.full((B, Hkv, cap, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        for x, y in zip(held, (k, v)):
            x[:, :, :n_old] = y
        pisa.pisa_build_pyramid(base.at(p, n_old), held[0], pyr)
        return [*held, pyr], lambda s=None: pisa.cache_append_rows(p, *held, k_new, v_new, rows, n_old, pyr, stream=s)
    held, call = fresh()
    first = [x.clone() for x in held]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    side = torch.cuda.Stream()
    for i in range(4):
        rows.copy_(chosen(B, T, m, i)[i % 2])
        for x, y in zip(held, first):
            x.copy_(y)
        want, eager = fresh()
        torch.cuda.synchronize()
        eager(side if i % 2 else None)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(held, want):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_wrapper_refuses():
    p = base.problem(1, 1, 1, 1, 100, 64, 32, 2, 4, 1, "bf16", 200)
    k, v, k_new, v_new = start(p, 100, 8, "bf16")
    raw = torch.zeros((1, 1, 200, 64), dtype=torch.bfloat16, device="cuda")
    rows = torch.zeros((1, 4), dtype=torch.int32, device="cuda")
    good = dict(k_new=k_new, v_new=v_new, rows=rows, n_old=96)
    for bad in (dict(rows=rows.long()), dict(rows=rows[:, :3].contiguous()), dict(rows=rows.cpu()), dict(k_new=k_new.float()),
                dict(k_new=k_new[:, :, :5]), dict(v_new=v_new[0]), dict(pyramid=torch.zeros((1, 1, 3, 64), device="cuda"))):
        with pytest.raises(ValueError):
            pisa.cache_append_rows(p, raw, raw.clone(), **{**good, **bad})
        with pytest.raises(ValueError):
            pisa.qcache_append_rows(p, pisa.make_qcache(p), **{**good, **bad})
    with pytest.raises(ValueError):
        pisa.cache_append_rows(p, raw[:, :, :150], raw, **good)
    with pytest.raises(pisa.PisaError):
        pisa.cache_append_rows(p, raw, raw, **good)
    with pytest.raises(ValueError):
        pisa.draft_layout(rows[0], 5)
    with pytest.raises(ValueError):
        pisa.draft_layout(rows.cpu(), 5)
    with pytest.raises(pisa.PisaError):
        pisa.draft_layout(torch.zeros((1, 1025), dtype=torch.int32, device="cuda"), 5)
