"""Operators around drafted tokens: norms with rotary positions, trees of drafts, their attention, what is kept of them.

A case is a dict of plain values.  Its "op" says what one pass is:

  norm    root-mean-square norm of each head of queries and keys with learned weights and their rotary positions, as
          projected ([B, N, heads, d]), into [B, heads, N, d]; "bwd": the gradients of both and of the weights
  layout  ancestor masks and positions of B trees of T drafted tokens, from each token's parent
  attend  attention of T drafted tokens over their selected blocks of n cached tokens and over their ancestors among
          the drafted ones, whose keys and values are not in the cache; "cache": "raw" (the problem's type) or "8bit"
  keep    the accepted rows of T drafted ones, m for each sequence, into the cache behind its first n_old, and its mean
          pyramid with them

Layout of the 8-bit cache: keys [B, Hkv, M, C, d] and values [B, Hkv, M, d, C] in e4m3 (bytes), a power of two per block
and head as scale, and the raw rows of the last block.
"""
import math

import torch

own = False

E4M3_MAX = 448.0
LEAST_EXP = -100
EPS = 1e-6


def _norm(name, bwd, B, H, Hkv, N, d, rot, layout, offset, pos0, ragged, dtype="bf16"):
    c = dict(op="norm", bwd=bwd, B=B, H=H, Hkv=Hkv, N=N, d=d, rot=rot, layout=layout, offset=offset, pos0=pos0,
             ragged=ragged, dtype=dtype)
    return dict(c, name=name) if name else c


def _layout(name, B, T, n):
    c = dict(op="layout", B=B, T=T, n=n)
    return dict(c, name=name) if name else c


def _attend(name, cache, B, H, Hkv, T, n, d, C, g, K, empty=False, dtype="bf16"):
    c = dict(op="attend", cache=cache, B=B, H=H, Hkv=Hkv, T=T, n=n, cap=n + T + C, d=d, C=C, g=g, K=K, empty=empty,
             dtype=dtype)
    return dict(c, name=name) if name else c


def _keep(name, cache, B, Hkv, n_old, T, m, d, C, g, dtype="bf16"):
    c = dict(op="keep", cache=cache, B=B, Hkv=Hkv, n_old=n_old, T=T, m=m, cap=n_old + T + C, d=d, C=C, g=g, dtype=dtype)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One token of each of eight sequences, at positions of their own: the latency of a generated token.
        _norm("norm-token-batch", False, 8, 16, 4, 1, 128, 128, "half", 0.0, 20010, True),
        # Gradients of a short prompt in 32 bits, an odd length, a part of the head whose halves fit no vector.
        _norm("norm-bwd-fp32-4k", True, 1, 2, 2, 4099, 64, 50, "interleaved", 0.0, 0, False, "f32"),
        # Gradients of a grouped-query layer's prompt, half of each head rotated, weights stored around zero.
        _norm("norm-bwd-gqa-30k", True, 1, 16, 4, 30011, 128, 64, "half", 1.0, 0, False),
        # The headline prompt.
        _norm("norm-prompt-128k", False, 1, 8, 8, 131072, 128, 128, "half", 0.0, 0, False),
        # The trees of a batch, before the drafted tokens' layers run.
        _layout("layout-batch", 8, 25, 20010),
        # The widest tree.
        _layout("layout-wide", 2, 777, 131072),
        # A small tree in 32 bits; the second sequence of the batch is padding and sees nothing.
        _attend("attend-fp32-4k", "raw", 2, 2, 2, 13, 4001, 64, 64, 2, 4, empty=True, dtype="f32"),
        # A tree over the 8-bit cache of the headline prompt, a head of its own per KV head.
        _attend("attend-8bit-128k", "8bit", 1, 8, 8, 16, 131071, 128, 64, 2, 16),
        # A wider tree over an unquantised cache, four heads per KV head.
        _attend("attend-raw-gqa-32k", "raw", 1, 16, 4, 64, 32749, 128, 64, 2, 16),
        # Many drafted tokens over the longest cache: wide blocks, a wide budget.
        _attend("attend-8bit-512k", "8bit", 1, 8, 2, 256, 523776, 128, 128, 4, 32),
        # What one verified tree leaves in the 8-bit cache of the headline prompt.
        _keep("keep-8bit-128k", "8bit", 1, 8, 131070, 16, 5, 128, 64, 2),
        # The same for a batch over unquantised caches, past a block's border.
        _keep("keep-raw-batch-20k", "raw", 4, 4, 20028, 64, 9, 128, 64, 2),
    ]


# Query heads per KV head, head dim, block, fan-out, budget, KV heads to choose from, longest sequence.
FAMILIES = {
    "mha": (1, 128, 64, 2, 16, (4, 8), 131072),
    "gqa": (4, 128, 64, 2, 16, (2, 4, 8), 65536),
    "wide": (16, 64, 64, 2, 8, (1, 2), 131072),
    "long": (4, 128, 128, 4, 32, (1, 2), 524288),
    "small": (1, 64, 32, 2, 4, (2, 4), 8192),
}


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    G, d, C, g, K, heads, hi = FAMILIES[rng.choice(tuple(FAMILIES))]
    Hkv, op = rng.choice(heads), rng.choice(("norm", "norm", "layout", "attend", "attend", "attend", "keep"))
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if op == "norm":
        bwd, B = rng.random() < 0.5, rng.choice((1, 2, 8))
        most = (30011 * 20 if bwd else 131072 * 16) // (B * Hkv * (G + 1)) // (2 if dtype == "f32" else 1)
        N = _spread(rng, 1, min(hi, most))
        rot = rng.choice((d, d, d // 2, 2 * rng.randrange(2, d // 2 + 1)))
        return _norm(None, bwd, B, G * Hkv, Hkv, N, d, rot, rng.choice(("half", "interleaved")), rng.choice((0.0, 1.0)),
                     rng.choice((0, rng.randrange(1 << 20))), rng.random() < 0.5, dtype)
    if op == "layout":
        T = _spread(rng, 1, 1024)
        return _layout(None, rng.choice((1, 2, 8)) if T < 512 else 1, T, rng.randrange(1, hi))
    B = rng.choice((1, 1, 2, 4))
    cache = rng.choice(("raw", "8bit"))
    n = _spread(rng, 3 * C, hi // B // (2 if dtype == "f32" else 1))
    if op == "keep":
        T = _spread(rng, 1, 256)
        return _keep(None, cache, B, Hkv, n, T, rng.randrange(1, 1 + min(T, 40)), d, C, g, dtype)
    T = _spread(rng, 1, min(1024, (1 << 28) // (B * Hkv * K * C * d)) // (4 if dtype == "f32" else 1))
    return _attend(None, cache, B, G * Hkv, Hkv, T, n, d, C, g, K, rng.random() < 0.25, dtype)


# ---------------------------------------------------------------- inputs ---

def _gen(seed, what):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 32 + what)
    return gen


def _normal(shape, seed, what):
    return torch.randn(shape, generator=_gen(seed, what), device="cuda", dtype=torch.float32)


def _type(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _rows(c, n, seed, what, channels):
    """n rows per KV head whose channels differ in size, as a trained layer's do."""
    x = _normal((c["B"], c["Hkv"], n, c["d"]), seed, what)
    return (x * torch.exp(0.5 * _normal((c["Hkv"], 1, c["d"]), seed, channels))).to(_type(c))


def _parents(B, T, seed):
    """Trees whose tokens follow one of the last eight, the first token their root."""
    i = torch.arange(T, device="cuda")
    back = torch.rand((B, T), generator=_gen(seed, 9), device="cuda") ** 2 * torch.clamp(i, max=8)
    return (i - 1 - back.floor().long().clamp(min=0)).clamp(min=0).masked_fill(i == 0, -1).to(torch.int32)


def _levels(n, C, g):
    """Nodes of each stored level of an n-token pyramid, leaves first."""
    sizes = [-(-n // C)]
    while sizes[-1] > 1:
        sizes.append(-(-sizes[-1] // g))
    return sizes[:-1] if len(sizes) > 1 else sizes


def _leaves(x, C):
    """[..., n, d] as [..., leaves, C, d] in 32 bits, zeros behind the last row."""
    n = x.shape[-2]
    M = -(-n // C)
    return torch.nn.functional.pad(x.float(), (0, 0, 0, M * C - n)).unflatten(-2, (M, C))


def _quantise(leaves):
    """e4m3 codes and the powers of two that they are multiples of, one per leaf."""
    big = leaves.abs().amax((-1, -2))
    m, e = torch.frexp(big / E4M3_MAX)
    e = torch.where(m == 0.5, e - 1, e).clamp(min=LEAST_EXP)
    e = torch.where(big > 0, e, torch.full_like(e, LEAST_EXP))
    scale = ((e.to(torch.int32) + 127) << 23).view(torch.float32)
    return (leaves / scale[..., None, None]).to(torch.float8_e4m3fn), scale


def _means(leaves, n, C):
    """Means of the leaves' rows, of which the last leaf has n - C * (leaves - 1)."""
    M = leaves.shape[-3]
    rows = torch.full((M, 1), float(C), device=leaves.device)
    rows[-1] = n - C * (M - 1)
    return leaves.sum(-2) / rows


def _grouped(x, first, g):
    """Means of g neighbours each, from node `first` on; the last group may be short."""
    n = x.shape[-2] - first * g
    m = -(-n // g)
    have = torch.full((m, 1), float(g), device=x.device)
    have[-1] = n - g * (m - 1)
    return torch.nn.functional.pad(x[..., first * g:, :], (0, 0, 0, m * g - n)).unflatten(-2, (m, g)).sum(-2) / have


def _pyramid_update(pyr, means, first, n, n_old, cap, C, g):
    """Level 1 from leaf `first` on, and above it what that changes or what did not exist at n_old."""
    sizes, room = _levels(n, C, g), _levels(cap, C, g)
    stored = len(_levels(n_old, C, g)) if n_old else 0
    pyr[:, :, first:sizes[0]] = means
    at = 0
    for lv in range(1, len(sizes)):
        below, at = pyr[:, :, at:at + sizes[lv - 1]], at + room[lv - 1]
        first = first // g if lv < stored else 0
        pyr[:, :, at + first:at + sizes[lv]] = _grouped(below, first, g)


def _empty_cache(c):
    B, Hkv, d, C, cap = c["B"], c["Hkv"], c["d"], c["C"], c["cap"]
    M, new = -(-cap // C), dict(device="cuda")
    s = dict(pyramid=torch.zeros((B, Hkv, sum(_levels(cap, C, c["g"])), d), **new))
    if c["cache"] == "raw":
        return dict(s, k=torch.zeros((B, Hkv, cap, d), dtype=_type(c), **new), v=torch.zeros((B, Hkv, cap, d), dtype=_type(c), **new))
    return dict(s, k=torch.zeros((B, Hkv, M, C, d), dtype=torch.uint8, **new),
                v=torch.zeros((B, Hkv, M, d, C), dtype=torch.uint8, **new),
                k_scale=torch.ones((B, Hkv, M), **new), v_scale=torch.ones((B, Hkv, M), **new),
                k_open=torch.zeros((B, Hkv, C, d), dtype=_type(c), **new),
                v_open=torch.zeros((B, Hkv, C, d), dtype=_type(c), **new))


def _append_plain(s, c, k, v, n_old, n):
    """Rows n_old .. n-1 into the cache s (k, v: those rows)."""
    C = c["C"]
    first, last = n_old // C, (n - 1) // C
    had = n_old - first * C
    for name, new in (("k", k), ("v", v)):
        if c["cache"] == "raw":
            s[name][:, :, n_old:n] = new
            raw = s[name][:, :, first * C:n]
        else:
            raw = torch.cat((s[name + "_open"][:, :, :had], new), 2)
            codes, scale = _quantise(_leaves(raw, C))
            s[name].view(torch.float8_e4m3fn)[:, :, first:last + 1] = codes.transpose(-1, -2) if name == "v" else codes
            s[name + "_scale"][:, :, first:last + 1] = scale
            s[name + "_open"][:, :, :n - last * C] = raw[:, :, (last - first) * C:]
        if name == "k":
            _pyramid_update(s["pyramid"], _means(_leaves(raw, C), n - first * C, C), first, n, n_old, c["cap"], C, c["g"])


def _select(c, q, k):
    """Blocks of each drafted row by block mean: the first, previous and own one by its place in the sequence, then the
    highest; ascending, -1 behind."""
    B, H, Hkv, T, n, C, K = (c[x] for x in ("B", "H", "Hkv", "T", "n", "C", "K"))
    M, have = -(-(n + T) // C), -(-n // C)
    mean = torch.nn.functional.pad(_means(_leaves(k, C), n, C), (0, 0, 0, M - have))
    score = torch.matmul(q.float().view(B, Hkv, H // Hkv, T, -1).sum(2), mean.transpose(-1, -2).contiguous())
    at = (torch.arange(n, n + T, device="cuda") // C)[:, None]
    j = torch.arange(M, device="cuda")
    score = score.masked_fill(j > at, -math.inf).masked_fill((j == 0) | (j == at) | (j == at - 1), math.inf)
    top = score.topk(min(K, M), dim=-1)
    idx = torch.where(top.values == -math.inf, M, top.indices).sort(-1).values
    idx = torch.nn.functional.pad(torch.where(idx == M, -1, idx), (0, K - idx.shape[-1]), value=-1).to(torch.int32)
    if c["empty"]:  # the last sequence is padding; of a single one, every seventh row selects nothing
        if B > 1:
            idx[-1] = -1
        else:
            idx[:, :, ::7] = -1
    return idx.contiguous()


def _frequencies(c):
    return [10000.0 ** (-2.0 * i / c["rot"]) for i in range(c["rot"] // 2)]


def _prepare_norm(c, seed):
    B, H, Hkv, N, d = (c[x] for x in ("B", "H", "Hkv", "N", "d"))
    s = dict(case=c, plan=None, positions=None)
    # as projected: rows of [heads, d] one after another, seen as [B, heads, N, d]
    s["q"], s["k"] = ((_normal((B, N, h, d), seed, w) * 1.5).to(_type(c)).transpose(1, 2) for w, h in enumerate((H, Hkv)))
    s["q_weight"], s["k_weight"] = ((1.0 - c["offset"] + 0.25 * _normal((d,), seed, w)).to(_type(c)) for w in (2, 3))
    if c["bwd"]:  # gradients come in [B, heads, N, d] and go back into the projections' order
        s["d_q_out"], s["d_k_out"] = (_normal((B, h, N, d), seed, w).to(_type(c)) for w, h in ((4, H), (5, Hkv)))
        s["d_q"], s["d_k"] = (torch.empty((B, N, h, d), dtype=_type(c), device="cuda").transpose(1, 2) for h in (H, Hkv))
    else:
        s["q_out"], s["k_out"] = (torch.empty((B, h, N, d), dtype=_type(c), device="cuda") for h in (H, Hkv))
    s["freq"] = torch.tensor(_frequencies(c), dtype=torch.float64, device="cuda")
    if c["ragged"]:
        start = torch.randint(0, c["pos0"] + 1, (B, 1), generator=_gen(seed, 8), device="cuda")
        s["positions"] = (start + torch.arange(N, device="cuda")).to(torch.int32)
    return s


def prepare(case, seed):
    c = dict(case)
    if c["op"] == "norm":
        return _prepare_norm(c, seed)
    s = dict(case=c, plan=None)
    if c["op"] == "layout":
        s["parents"] = _parents(c["B"], c["T"], seed)
        return s
    B, Hkv, T, d, n = c["B"], c["Hkv"], c["T"], c["d"], c["n"] if c["op"] == "attend" else c["n_old"]
    s.update(_empty_cache(c))
    k, v = _rows(c, n, seed, 0, 6), _rows(c, n, seed, 1, 7)
    _append_plain(s, c, k, v, 0, n)
    # the drafted keys as rotated, the values as projected
    s["k_new"] = _rows(c, T, seed, 2, 6)
    s["v_new"] = _rows(c, T, seed, 3, 7).transpose(1, 2).contiguous().transpose(1, 2)
    if c["op"] == "keep":
        # accepted rows: the root and m - 1 others, in order
        place = torch.rand((B, T), generator=_gen(seed, 10), device="cuda")
        place[:, 0] = -1.0
        s["rows"] = place.argsort(-1)[:, :c["m"]].sort(-1).values.to(torch.int32).contiguous()
        if c["cache"] == "8bit":
            s["k_was"], s["v_was"] = s["k_open"].clone(), s["v_open"].clone()
        return s
    # a tree's rows have one context: what they look for is mostly the same
    shared = _normal((B, c["H"], 1, d), seed, 4)
    s["q"] = (0.7 * (0.95 * shared + 0.31 * _normal((B, c["H"], T, d), seed, 5))).to(_type(c))
    s["idx"] = _select(c, s["q"], k)
    s["mask"] = _layout_plain(_parents(B, T, seed), n)[0]
    if c["empty"] and B > 1:
        s["mask"][-1] = 0
    s["o"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty((B, c["H"], T), dtype=torch.float32, device="cuda")
    return s


# ---------------------------------------------------------------- plain forms ---

def _pairs(c):
    """Dimensions of each rotated pair."""
    i = torch.arange(c["rot"] // 2, device="cuda")
    return (i, i + c["rot"] // 2) if c["layout"] == "half" else (2 * i, 2 * i + 1)


def _angles(s):
    c = s["case"]
    pos = s["positions"] if s["positions"] is not None else torch.arange(c["pos0"], c["pos0"] + c["N"], device="cuda")[None]
    angle = pos.double()[:, None, :, None] * s["freq"]
    return angle.cos().float(), angle.sin().float()


def _turn(x, a, b, cos, sin):
    y = x.clone()
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    return y


def _norm_plain(s):
    c = s["case"]
    (a, b), (cos, sin) = _pairs(c), _angles(s)
    out = {}
    for x in "qk":
        y = s[x].float()
        w = s[x + "_weight"].float() + c["offset"]
        r = torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS)
        if not c["bwd"]:
            out[x] = _turn(y * r * w, a, b, cos, sin).to(s[x].dtype)
            continue
        u = _turn(s["d_" + x + "_out"].float(), a, b, cos, -sin)
        y = y * r
        out["d_" + x + "_weight"] = (u * y).sum((0, 1, 2), dtype=torch.float64).float()
        u = u * w
        out["d_" + x] = (r * (u - y * (u * y).mean(-1, keepdim=True))).to(s[x].dtype)
    return out


def _layout_plain(parents, n):
    """(mask, positions): bit j of row i where j is i or an ancestor of it; positions by depth."""
    B, T = parents.shape
    reach = torch.zeros((B, T, T + 1), device="cuda")
    reach.scatter_(-1, torch.where(parents < 0, T, parents).long()[..., None], 1.0)
    reach = reach[..., :T] + torch.eye(T, device="cuda")
    for _ in range(max(1, (T - 1).bit_length())):  # paths of twice the length each time
        reach = torch.matmul(reach, reach).clamp(max=1.0)
    bits = torch.nn.functional.pad(reach, (0, -T % 64)).to(torch.int64).unflatten(-1, (-1, 64))
    mask = (bits << torch.arange(64, device="cuda")).sum(-1)
    return mask, (n - 1 + reach.sum(-1)).to(torch.int32)


def _attend_plain(s):
    c = s["case"]
    B, H, Hkv, T, n, d, C = (c[x] for x in ("B", "H", "Hkv", "T", "n", "d", "C"))
    M = -(-n // C)
    b, h = torch.arange(B, device="cuda").view(B, 1, 1, 1), torch.arange(Hkv, device="cuda").view(1, Hkv, 1, 1)
    idx = s["idx"].long()
    at = torch.where((idx >= 0) & (idx < M), idx, 0)
    if c["cache"] == "raw":
        k, v = (s[x][:, :, :M * C].unflatten(2, (M, C))[b, h, at].float() for x in "kv")
    else:
        k, v = (s[x][b, h, at].view(torch.float8_e4m3fn).float() * s[x + "_scale"][b, h, at][..., None, None] for x in "kv")
        v = v.transpose(-1, -2)
    token = at[..., None] * C + torch.arange(C, device="cuda")
    shown = (((idx >= 0) & (idx < M))[..., None] & (token < n)).flatten(3)[..., None, :]
    q = s["q"].float().view(B, Hkv, H // Hkv, T, d).transpose(2, 3) / math.sqrt(d)
    cached = torch.matmul(q, k.flatten(3, 4).transpose(-1, -2).contiguous()).masked_fill(~shown, -math.inf)
    j = torch.arange(T, device="cuda")
    seen = ((s["mask"][..., j // 64] >> (j % 64)) & 1).bool()[:, None, :, None]
    drafted = torch.matmul(q, s["k_new"].float()[:, :, None].transpose(-1, -2).contiguous()).masked_fill(~seen, -math.inf)
    top = torch.maximum(cached.amax(-1, keepdim=True), drafted.amax(-1, keepdim=True))
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p, r = torch.exp(cached - top), torch.exp(drafted - top)
    total = p.sum(-1, keepdim=True) + r.sum(-1, keepdim=True)
    o = torch.matmul(p, v.flatten(3, 4).contiguous()) + torch.matmul(r, s["v_new"].float()[:, :, None].contiguous())
    o = (o / torch.where(total > 0, total, torch.ones_like(total))).transpose(2, 3)
    lse = (top + torch.log(total)).squeeze(-1).transpose(2, 3)
    return o.reshape(B, H, T, d).to(s["q"].dtype), lse.reshape(B, H, T).contiguous()


def _keep_plain(s):
    c = s["case"]
    at = s["rows"].long()[:, None, :, None].expand(-1, c["Hkv"], -1, c["d"])
    k, v = (s[x].gather(2, at) for x in ("k_new", "v_new"))
    _append_plain(s, c, k, v, c["n_old"], c["n_old"] + c["m"])


# ---------------------------------------------------------------- one pass ---

def run(s):
    c = s["case"]
    if c["op"] == "norm":
        return _norm_own(s) if own else _norm_plain(s)
    if c["op"] == "layout":
        return _layout_own(s) if own else _layout_plain(s["parents"], c["n"])
    if c["op"] == "attend":
        return _attend_own(s) if own else _attend_plain(s)
    if c["cache"] == "8bit" and c["n_old"] % c["C"] and c["n_old"] // c["C"] != (c["n_old"] + c["m"] - 1) // c["C"]:
        # a pass that leaves its first block leaves other raw rows behind: put back what the next one starts from
        s["k_open"].copy_(s["k_was"])
        s["v_open"].copy_(s["v_was"])
    if own:
        _keep_own(s)
    else:
        _keep_plain(s)
    if c["cache"] == "raw":
        return {x: s[x] for x in ("k", "v", "pyramid")}
    return dict({x: s[x].view(torch.float8_e4m3fn) for x in "kv"},
                **{x: s[x] for x in ("k_scale", "v_scale", "k_open", "v_open", "pyramid")})


def _problem(c, T, N, H, K):
    from paper_2609_31093_amd import pisa

    return pisa.make_problem(c["B"], H, c["Hkv"], T, N, c["d"], c["C"], c["g"], K, True, c["dtype"], Ncap=c["cap"])


def _qcache(s):
    from paper_2609_31093_amd import pisa

    return pisa.QCache(s["k"], s["v"], s["k_scale"], s["v_scale"], s["k_open"], s["v_open"])


def _norm_own(s):
    from paper_2609_31093_amd import pisa

    c = s["case"]
    if s["plan"] is None:
        r = pisa.make_rope(c["B"], c["H"], c["Hkv"], c["N"], c["d"], rot=c["rot"], layout=c["layout"], dtype=c["dtype"],
                           pos0=c["pos0"])
        s["plan"] = r, pisa.make_qk_norm(r, s["q_weight"], s["k_weight"], eps=EPS, offset=c["offset"])
    r, m = s["plan"]
    if not c["bwd"]:
        q, k = pisa.norm_rope_fwd(r, m, s["q"], s["k"], s["positions"], s["q_out"], s["k_out"])
        return dict(q=q, k=k)
    got = pisa.norm_rope_bwd(r, m, s["q"], s["k"], s["d_q_out"], s["d_k_out"], s["positions"], s["d_q"], s["d_k"])
    return dict(zip(("d_q", "d_k", "d_q_weight", "d_k_weight"), got))


def _layout_own(s):
    from paper_2609_31093_amd import pisa

    return pisa.draft_layout(s["parents"], s["case"]["n"])


def _attend_own(s):
    from paper_2609_31093_amd import pisa

    c = s["case"]
    eight = c["cache"] == "8bit"
    if s["plan"] is None:
        p = _problem(c, c["T"], c["n"] + c["T"], c["H"], c["K"])
        nb = (pisa.pisa_qcache_draft_attn_workspace_bytes if eight else pisa.pisa_draft_attn_workspace_bytes)(p)
        s["plan"] = p, _qcache(s) if eight else None, torch.empty(max(nb, 1), dtype=torch.uint8, device="cuda")
    p, cache, ws = s["plan"]
    drafted = s["k_new"], s["v_new"], s["mask"]
    if eight:
        return pisa.qcache_draft_attn_fwd(p, cache, s["q"], s["idx"], *drafted, o=s["o"], lse=s["lse"], ws=ws)
    return pisa.draft_attn_fwd(p, s["q"], s["k"], s["v"], s["idx"], *drafted, o=s["o"], lse=s["lse"], ws=ws)


def _keep_own(s):
    from paper_2609_31093_amd import pisa

    c = s["case"]
    eight = c["cache"] == "8bit"
    if s["plan"] is None:
        s["plan"] = _problem(c, 1, c["n_old"] + c["m"], c["Hkv"], 4), _qcache(s) if eight else None
    p, cache = s["plan"]
    if eight:
        pisa.qcache_append_rows(p, cache, s["k_new"], s["v_new"], s["rows"], c["n_old"], s["pyramid"])
    else:
        pisa.cache_append_rows(p, s["k"], s["v"], s["k_new"], s["v_new"], s["rows"], c["n_old"], s["pyramid"])


# ---------------------------------------------------------------- work, exact results ---

def work(case):
    c = case
    e = 4 if c.get("dtype") == "f32" else 2
    if c["op"] == "norm":
        values, weights = c["B"] * (c["H"] + c["Hkv"]) * c["N"] * c["d"], 2 * c["d"]
        more = weights * e + (4 * c["B"] * c["N"] if c["ragged"] else 0)
        if c["bwd"]:
            return {"bytes": 3 * values * e + 4 * weights + more, "flops": 14 * values}
        return {"bytes": 2 * values * e + more, "flops": 7 * values}
    if c["op"] == "layout":
        B, T = c["B"], c["T"]
        return {"bytes": 8 * B * T + 8 * B * T * -(-T // 64), "flops": B * T * T}
    B, Hkv, T, d, C = c["B"], c["Hkv"], c["T"], c["d"], c["C"]
    block = 2 * C * d * e if c["cache"] == "raw" else 2 * C * d + 8
    if c["op"] == "attend":
        n, H = c["n"], c["H"]
        K = min(c["K"], -(-n // C))
        blocks = min(-(-n // C), int(K * T ** (1 / 3)))  # what a tree's rows select together, counted on these inputs
        rows = B * H * T
        byte = 2 * rows * d * e + 4 * rows + 4 * B * Hkv * T * c["K"] + B * T * 8 * -(-T // 64)
        return {"bytes": byte + B * Hkv * (blocks * block + 2 * T * d * e), "flops": 4 * rows * (K * C + T) * d}
    n_old, m = c["n_old"], c["m"]
    N, first = n_old + m, n_old // C
    blocks, had = (N - 1) // C + 1 - first, n_old - first * C
    nodes = sum(-(-blocks // c["g"] ** i) for i in range(len(_levels(N, C, c["g"]))))
    if c["cache"] == "raw":  # the rows out and in, and the block's other keys for its mean
        byte = 4 * m * d * e + had * d * e + 4 * nodes * d
    else:
        byte = 2 * (m + had) * d * e + 2 * (N - first * C) * d + 8 * blocks + 4 * nodes * d
        byte += 2 * min(m, N - (N - 1) // C * C) * d * e
    return {"bytes": B * Hkv * byte + 4 * B * m, "flops": 4 * B * Hkv * (m + had) * d}


def _exact_norm(c, seed):
    s = _prepare_norm(c, seed)
    rot, half = c["rot"], c["layout"] == "half"
    pos = s["positions"].double() if s["positions"] is not None else (c["pos0"] + torch.arange(c["N"], device="cuda")).double()
    turn = torch.polar(torch.ones(1, dtype=torch.float64, device="cuda"), pos.view(-1, c["N"], 1) * s["freq"])[:, None]

    def turned(x, by):
        z = x[..., :rot].unflatten(-1, (2, rot // 2)).transpose(-1, -2) if half else x[..., :rot].unflatten(-1, (rot // 2, 2))
        z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * by)
        z = z.transpose(-1, -2).flatten(-2) if half else z.flatten(-2)
        return torch.cat((z, x[..., rot:]), -1)

    out = {}
    for name in "qk":
        x, w = s[name].double(), s[name + "_weight"].double() + c["offset"]
        size = (torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / c["d"] + EPS).sqrt()
        if not c["bwd"]:
            out[name] = turned(x / size * w, turn)
            continue
        g = turned(s["d_" + name + "_out"].double(), turn.conj())
        out["d_" + name + "_weight"] = (g * x / size).sum((0, 1, 2))
        # d(x / size) by x: 1 / size - x x^T / (d size^3)
        along = (g * w * x).sum(-1, keepdim=True)
        out["d_" + name] = g * w / size - x * along / (c["d"] * size ** 3)
    return out


def _exact_attend(c, seed):
    s = prepare(c, seed)
    B, H, Hkv, T, n, d, C, K = (c[x] for x in ("B", "H", "Hkv", "T", "n", "d", "C", "K"))
    G, M = H // Hkv, -(-n // C)
    o = torch.zeros((B, Hkv, T, G, d), dtype=torch.float64, device="cuda")
    lse = torch.full((B, Hkv, T, G), -math.inf, dtype=torch.float64, device="cuda")
    q = s["q"].double().view(B, Hkv, G, T, d).transpose(2, 3)
    step = max(1, (1 << 27) // ((K * C + T) * d))
    place = torch.arange(T, device="cuda")
    for b in range(B):
        sees = ((s["mask"][b][:, place // 64] >> (place % 64)) & 1) == 1
        for h in range(Hkv):
            for r in range(0, T, step):
                i = s["idx"][b, h, r:r + step].long()
                real = (i >= 0) & (i < M)
                at = i.masked_fill(~real, 0)
                if c["cache"] == "raw":
                    k, v = (s[x][b, h, :M * C].view(M, C, d)[at].double() for x in "kv")
                else:
                    k, v = (s[x][b, h][at].view(torch.float8_e4m3fn).double() * s[x + "_scale"][b, h][at].double()[..., None, None] for x in "kv")
                    v = v.transpose(2, 3)
                token = at[..., None] * C + torch.arange(C, device="cuda")
                on = torch.cat(((real[..., None] & (token < n)).flatten(1), sees[r:r + step]), 1)
                k = torch.cat((k.flatten(1, 2), s["k_new"][b, h].double().expand(len(i), T, d)), 1)
                v = torch.cat((v.flatten(1, 2), s["v_new"][b, h].double().expand(len(i), T, d)), 1)
                z = torch.bmm(q[b, h, r:r + step].contiguous(), k.transpose(1, 2).contiguous()) / math.sqrt(d)
                z = torch.where(on[:, None], z, -math.inf)
                total = torch.logsumexp(z, -1)
                w = torch.where((total > -math.inf)[..., None], torch.exp(z - total[..., None]), 0.0)
                o[b, h, r:r + step] = torch.bmm(w, v.contiguous())
                lse[b, h, r:r + step] = total
    return o.transpose(2, 3).reshape(B, H, T, d), lse.transpose(2, 3).reshape(B, H, T)


def _exact_codes(x):
    """Nearest e4m3 multiples of each leaf's power of two, in 64 bits (ties to even), and that power."""
    big = x.abs().amax((-1, -2))
    scale = torch.full_like(big, 2.0 ** LEAST_EXP)
    for at in range(LEAST_EXP + 1, 121):
        scale = torch.where(big > E4M3_MAX * 2.0 ** (at - 1), 2.0 ** at, scale)
    y = x / scale[..., None, None]
    e = torch.frexp(y.abs().clamp(min=2.0 ** -6)).exponent.to(torch.int64)
    step = ((e - 4 + 1023) << 52).view(torch.float64)
    return torch.round(y / step) * step, scale


def _exact_keep(c, seed):
    B, C, g, n_old, N = c["B"], c["C"], c["g"], c["n_old"], c["n_old"] + c["m"]
    M, first = -(-N // C), n_old // C
    s = prepare(c, seed)
    out = {}
    for i, name in enumerate("kv"):
        fresh = torch.stack([s[name + "_new"][b][:, s["rows"][b].long()] for b in range(B)])
        raw = torch.cat((_rows(c, n_old, seed, i, 6 + i), fresh), 2).double()
        if c["cache"] == "raw":
            out[name] = s[name].double()
            out[name][:, :, :N] = raw
        else:
            rows = raw[:, :, first * C:]
            rows = torch.cat((rows, rows.new_zeros((*rows.shape[:2], M * C - N, c["d"]))), 2)
            codes, scale = _exact_codes(rows.view(B, c["Hkv"], M - first, C, c["d"]))
            out[name] = s[name].view(torch.float8_e4m3fn).double()
            out[name][:, :, first:M] = codes.transpose(-1, -2) if name == "v" else codes
            for part, values, lo, hi in (("_scale", scale, first, M), ("_open", raw[:, :, (M - 1) * C:], 0, N - (M - 1) * C)):
                out[name + part] = s[name + part].double()
                out[name + part][:, :, lo:hi] = values
        if name == "k":  # every level from the level below in 64 bits
            level = torch.stack([x.mean(2) for x in raw.split(C, 2)], 2)
            pyr, at = s["pyramid"].double(), 0
            for size, room in zip(_levels(N, C, g), _levels(c["cap"], C, g)):
                pyr[:, :, at:at + size] = level
                at += room
                level = torch.stack([x.mean(2) for x in level.split(g, 2)], 2)
            out["pyramid"] = pyr
    return out


def _exact_layout(c, seed):
    """Whole numbers: nothing to compare with but themselves."""
    return None


def exact(case, seed):
    c = dict(case)
    return {"norm": _exact_norm, "layout": _exact_layout, "attend": _exact_attend, "keep": _exact_keep}[c["op"]](c, seed)
