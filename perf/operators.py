"""Operators around the block-sparse attention: rotary positions and the 8-bit key/value cache.

A case is a dict of plain values.  Its "op" says what one pass is:

  rope    rotary positions of a layer's queries and keys, as projected ([B, N, heads, d]), into [B, heads, N, d];
          "bwd": the same for their gradients, back into the projections' order
  append  rows n_old .. N-1 of keys and values into the 8-bit cache and its mean pyramid
  attend  attention of Nq rows over their selected blocks of that cache

Cache layout: keys [B, Hkv, M, C, d] and values [B, Hkv, M, d, C] in e4m3 (bytes), a power of two per block and head as
scale, and the raw rows of the last block.
"""
import math

import torch

own = False

E4M3_MAX = 448.0
LEAST_EXP = -100
SCALINGS = ("none", "linear", "base", "parts")


def _rope(name, bwd, B, H, Hkv, N, d, rot, layout, scaling, factor, ctx, pos0, ragged, dtype="bf16"):
    c = dict(op="rope", bwd=bwd, B=B, H=H, Hkv=Hkv, N=N, d=d, rot=rot, layout=layout, scaling=scaling, factor=factor,
             ctx=ctx, pos0=pos0, ragged=ragged, dtype=dtype)
    return dict(c, name=name) if name else c


def _append(name, B, Hkv, n_old, N, cap, d, C, g, dtype="bf16"):
    c = dict(op="append", B=B, Hkv=Hkv, n_old=n_old, N=N, cap=cap, d=d, C=C, g=g, dtype=dtype)
    return dict(c, name=name) if name else c


def _attend(name, B, H, Hkv, Nq, N, cap, d, C, g, K, causal=True, empty=False, dtype="bf16"):
    c = dict(op="attend", B=B, H=H, Hkv=Hkv, Nq=Nq, N=N, cap=cap, d=d, C=C, g=g, K=K, causal=causal, empty=empty,
             dtype=dtype)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One token of each of eight sequences, at positions of their own: the latency of a generated token.
        _rope("rope-token-batch", False, 8, 16, 4, 1, 128, 128, "half", "none", 1.0, 0, 20010, True),
        # A short prompt in 32 bits, an odd length, a part of the head whose halves fit no vector.
        _rope("rope-fp32-4k", False, 1, 2, 2, 4099, 64, 50, "interleaved", "linear", 4.0, 0, 0, False, "f32"),
        # The gradients of a grouped-query layer's prompt, half of each head rotated in neighbouring pairs.
        _rope("rope-bwd-gqa-30k", True, 1, 16, 4, 30011, 128, 64, "interleaved", "base", 8.0, 0, 0, False),
        # The headline prompt, positions scaled by parts for a context longer than the original.
        _rope("rope-prompt-128k", False, 1, 8, 8, 131072, 128, 128, "half", "parts", 16.0, 8192, 0, False),
        # One generated token into a 128K-token cache.
        _append("append-token-128k", 1, 8, 131071, 131072, 132096, 128, 64, 2),
        # A chunk that ends inside a block, in 32 bits, after a cache that ended inside one.
        _append("append-chunk-fp32", 2, 2, 3001, 3777, 4096, 64, 64, 2, "f32"),
        # A whole prompt into an empty cache.
        _append("append-prompt-128k", 1, 8, 0, 131072, 131072, 128, 64, 2),
        # One token over a 128K-token cache, a head of its own per KV head.
        _attend("attend-token-128k", 1, 8, 8, 1, 131072, 132096, 128, 64, 2, 16),
        # One token for each of eight sequences, four heads per KV head; one sequence is padding and selects nothing.
        _attend("attend-batch-20k", 8, 16, 4, 1, 20011, 20480, 128, 64, 2, 16, empty=True),
        # Rows in 32 bits.
        _attend("attend-fp32-4k", 1, 2, 2, 65, 4096, 4096, 64, 64, 2, 4, dtype="f32"),
        # Drafted tokens over the longest cache: wide blocks, a wide budget.
        _attend("attend-draft-512k", 1, 8, 2, 8, 524288, 524288, 128, 128, 4, 32),
        # A prompt's chunk that attends what the cache holds of the prompt so far.
        _attend("attend-chunk-32k", 1, 16, 4, 4096, 32768, 32768, 128, 64, 2, 16),
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
    Hkv, op = rng.choice(heads), rng.choice(("rope", "append", "attend", "attend"))
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if op == "rope":
        B = rng.choice((1, 2, 8))
        N = _spread(rng, 1, min(hi, 131072 * 16 // (B * Hkv * (G + 1))) // (2 if dtype == "f32" else 1))
        rot = rng.choice((d, d, d // 2, 2 * rng.randrange(2, d // 2 + 1)))
        scaling = rng.choice(SCALINGS)
        return _rope(None, rng.random() < 0.4, B, G * Hkv, Hkv, N, d, rot, rng.choice(("half", "interleaved")), scaling,
                     1.0 if scaling == "none" else rng.choice((2.0, 4.0, 16.0)), rng.choice((4096, 8192)),
                     rng.choice((0, rng.randrange(1 << 20))), rng.random() < 0.5, dtype)
    B = rng.choice((1, 1, 2, 4))
    N = _spread(rng, 3 * C, hi // B // (2 if dtype == "f32" else 1))
    cap = N + rng.choice((0, rng.randrange(2 * C)))
    if op == "append":
        n_old = N - min(N, rng.choice((1, 1, rng.randrange(1, 4 * C), N, _spread(rng, 1, N))))
        return _append(None, B, Hkv, n_old, N, cap, d, C, g, dtype)
    Nq = min(N, rng.choice((1, 1, rng.randrange(2, 17), _spread(rng, 1, 4096 if dtype == "bf16" else 1024))))
    if Nq > 64:  # a chunk of a prompt: bounded by what the plain form holds at once
        B, N = 1, min(N, 32768)
        Hkv, cap, Nq = min(Hkv, max(1, 16 // G)), max(N, min(cap, N + C)), min(Nq, N)
    return _attend(None, B, G * Hkv, Hkv, Nq, N, cap, d, C, g, K, rng.random() < 0.85, rng.random() < 0.25, dtype)


# ---------------------------------------------------------------- geometry, frequencies ---

def _levels(n, C, g):
    """Nodes of each stored level of an n-token pyramid, leaves first."""
    sizes = [-(-n // C)]
    while sizes[-1] > 1:
        sizes.append(-(-sizes[-1] // g))
    return sizes[:-1] if len(sizes) > 1 else sizes


def _frequencies(c):
    """(radians per position of each pair, amplitude)."""
    rot, s = c["rot"], c["factor"]
    base = 10000.0 * s ** (rot / (rot - 2)) if c["scaling"] == "base" else 10000.0
    f = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    if c["scaling"] == "linear":
        return [x / s for x in f], 1.0
    if c["scaling"] == "parts":
        share = [min(1.0, max(0.0, (c["ctx"] * x / (2 * math.pi) - 1.0) / (32.0 - 1.0))) for x in f]
        return [x * (y + (1 - y) / s) for x, y in zip(f, share)], 0.1 * math.log(s) + 1.0
    return f, 1.0


# ---------------------------------------------------------------- inputs ---

def _gen(seed, what):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 16 + what)
    return gen


def _normal(shape, seed, what):
    return torch.randn(shape, generator=_gen(seed, what), device="cuda", dtype=torch.float32)


def _type(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _keys(c, n, seed, what):
    """n rows per KV head whose channels differ in size, as a trained layer's do."""
    x = _normal((c["B"], c["Hkv"], n, c["d"]), seed, what)
    return (x * torch.exp(0.5 * _normal((c["Hkv"], 1, c["d"]), seed, what + 8))).to(_type(c))


def _leaves(x, C):
    """[..., n, d] as [..., leaves, C, d] in 32 bits, zeros behind the last row."""
    n = x.shape[-2]
    M = -(-n // C)
    return torch.nn.functional.pad(x.float(), (0, 0, 0, M * C - n)).unflatten(-2, (M, C))


def _quantise(leaves):
    """e4m3 codes and the powers of two that they are multiples of, one per leaf."""
    big = leaves.abs().amax((-1, -2))
    m, e = torch.frexp(big / E4M3_MAX)  # 448 is 7 * 64: where the quotient rounds, it rounds to no power of two
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
    B, Hkv, d, C, M = c["B"], c["Hkv"], c["d"], c["C"], -(-c["cap"] // c["C"])
    new = dict(device="cuda")
    return dict(k=torch.zeros((B, Hkv, M, C, d), dtype=torch.uint8, **new),
                v=torch.zeros((B, Hkv, M, d, C), dtype=torch.uint8, **new),
                k_scale=torch.ones((B, Hkv, M), **new), v_scale=torch.ones((B, Hkv, M), **new),
                k_open=torch.zeros((B, Hkv, C, d), dtype=_type(c), **new),
                v_open=torch.zeros((B, Hkv, C, d), dtype=_type(c), **new),
                pyramid=torch.zeros((B, Hkv, sum(_levels(c["cap"], C, c["g"])), d), **new))


def _append_plain(s, c, k, v, n_old, n):
    """Rows n_old .. n-1 into the cache s (k, v: those rows)."""
    C = c["C"]
    first, last = n_old // C, (n - 1) // C
    had = n_old - first * C
    for name, new in (("k", k), ("v", v)):
        raw = torch.cat((s[name + "_open"][:, :, :had], new), 2)
        leaves = _leaves(raw, C)
        codes, scale = _quantise(leaves)
        codes = codes.transpose(-1, -2) if name == "v" else codes
        s[name].view(torch.float8_e4m3fn)[:, :, first:last + 1] = codes
        s[name + "_scale"][:, :, first:last + 1] = scale
        s[name + "_open"][:, :, :n - last * C] = raw[:, :, (last - first) * C:]
        if name == "k":
            _pyramid_update(s["pyramid"], _means(leaves, n - first * C, C), first, n, n_old, c["cap"], C, c["g"])


def _select(c, q, k, empty):
    """Blocks by block mean: the first, previous and own one where causal, then the highest; ascending, -1 behind."""
    B, H, Hkv, Nq, N, C, K = (c[x] for x in ("B", "H", "Hkv", "Nq", "N", "C", "K"))
    M = -(-N // C)
    mean = _means(_leaves(k, C), N, C)
    score = torch.matmul(q.float().view(B, Hkv, H // Hkv, Nq, -1).sum(2), mean.transpose(-1, -2).contiguous())
    if c["causal"]:
        at = (torch.arange(N - Nq, N, device="cuda") // C)[:, None]
        j = torch.arange(M, device="cuda")
        score = score.masked_fill(j > at, -math.inf).masked_fill((j == 0) | (j == at) | (j == at - 1), math.inf)
    top = score.topk(min(K, M), dim=-1)
    idx = torch.where(top.values == -math.inf, M, top.indices).sort(-1).values
    idx = torch.where(idx == M, -1, idx)
    idx = torch.nn.functional.pad(idx, (0, K - idx.shape[-1]), value=-1).to(torch.int32)
    if empty:  # the last sequence is padding; of a single one, every seventh row is
        if B > 1:
            idx[-1] = -1
        else:
            idx[:, :, ::7] = -1
    return idx.contiguous()


def prepare(case, seed):
    c = dict(case)
    s = dict(case=c, plan=None)
    if c["op"] == "rope":
        B, H, Hkv, N, d = (c[x] for x in ("B", "H", "Hkv", "N", "d"))
        wide = ((B, H, N, d), (B, Hkv, N, d))
        # as projected: rows of [H, d] one after another, seen as [B, H, N, d]; gradients come in [B, H, N, d]
        q, k = (_normal((b, n, h, d), seed, w).to(_type(c)) for w, (b, h, n, d) in enumerate(wide))
        s["q"], s["k"] = (x.transpose(1, 2).contiguous() if c["bwd"] else x.transpose(1, 2) for x in (q, k))
        s["q_out"], s["k_out"] = ((torch.empty_like(x).transpose(1, 2) for x in (q, k)) if c["bwd"] else
                                  (torch.empty(x, dtype=_type(c), device="cuda") for x in wide))
        f, amplitude = _frequencies(c)
        s["freq"], s["amplitude"] = torch.tensor(f, dtype=torch.float64, device="cuda"), amplitude
        s["positions"] = None
        if c["ragged"]:
            start = torch.randint(0, c["pos0"] + 1, (B, 1), generator=_gen(seed, 4), device="cuda")
            s["positions"] = (start + torch.arange(N, device="cuda")).to(torch.int32)
        return s
    if c["op"] == "append":
        s.update(_empty_cache(c))
        k, v = _keys(c, c["N"], seed, 0), _keys(c, c["N"], seed, 1)
        if c["n_old"]:
            _append_plain(s, c, k[:, :, :c["n_old"]], v[:, :, :c["n_old"]], 0, c["n_old"])
        s["k_new"], s["v_new"] = (x[:, :, c["n_old"]:].clone() for x in (k, v))
        s["k_was"], s["v_was"] = s["k_open"].clone(), s["v_open"].clone()
        return s
    s.update(_empty_cache(c))
    k, v = _keys(c, c["N"], seed, 0), _keys(c, c["N"], seed, 1)
    _append_plain(s, c, k, v, 0, c["N"])
    s["q"] = (0.7 * _normal((c["B"], c["H"], c["Nq"], c["d"]), seed, 2)).to(_type(c))
    s["idx"] = _select(c, s["q"], k, c["empty"])
    s["o"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty((c["B"], c["H"], c["Nq"]), dtype=torch.float32, device="cuda")
    return s


# ---------------------------------------------------------------- plain forms ---

def _rope_plain(s):
    c = s["case"]
    pos = s["positions"] if s["positions"] is not None else torch.arange(c["pos0"], c["pos0"] + c["N"], device="cuda")[None]
    angle = pos.double()[:, None, :, None] * s["freq"]
    cos, sin = (s["amplitude"] * angle.cos()).float(), (s["amplitude"] * angle.sin()).float()
    if c["bwd"]:
        sin = -sin
    return _rotate(s["q"], cos, sin, c), _rotate(s["k"], cos, sin, c)


def _rotate(x, cos, sin, c):
    rot = c["rot"]
    y, z = x[..., :rot].float(), x[..., rot:]
    if c["layout"] == "half":
        a, b = y[..., :rot // 2], y[..., rot // 2:]
        y = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    else:
        a, b = y[..., 0::2], y[..., 1::2]
        y = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    return torch.cat((y.to(x.dtype), z), -1)


def _softmax_rows(logits, values, shown):
    """Softmax over the last axis where `shown`, times values; rows that show nothing give 0 and -inf."""
    logits = logits.masked_fill(~shown, -math.inf)
    top = logits.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = torch.exp(logits - top)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, values) / torch.where(total > 0, total, torch.ones_like(total))
    return o, (top + torch.log(total)).squeeze(-1)


def _attend_plain(s):
    c = s["case"]
    B, H, Hkv, Nq, N, d, C, K = (c[x] for x in ("B", "H", "Hkv", "Nq", "N", "d", "C", "K"))
    G, M = H // Hkv, -(-N // C)
    t = torch.arange(N - Nq, N, device="cuda") if c["causal"] else torch.full((Nq,), N - 1, device="cuda")
    idx = s["idx"].long()
    q = s["q"].float().view(B, Hkv, G, Nq, d) / math.sqrt(d)
    if B * Hkv * Nq * K * C * d <= 1 << 31:  # the selected blocks of every row, side by side
        b, h = torch.arange(B, device="cuda").view(B, 1, 1, 1), torch.arange(Hkv, device="cuda").view(1, Hkv, 1, 1)
        at = idx.clamp(min=0)
        k = s["k"][b, h, at].view(torch.float8_e4m3fn).float() * s["k_scale"][b, h, at][..., None, None]
        v = s["v"][b, h, at].view(torch.float8_e4m3fn).float() * s["v_scale"][b, h, at][..., None, None]
        k, v = k.flatten(3, 4), v.transpose(-1, -2).flatten(3, 4)
        token = at[..., None] * C + torch.arange(C, device="cuda")
        shown = ((idx[..., None] >= 0) & (token <= t[:, None, None])).flatten(3)
        o, lse = _softmax_rows(torch.matmul(q.transpose(2, 3), k.transpose(-1, -2)), v, shown[..., None, :])
        o, lse = o.transpose(2, 3), lse.transpose(2, 3)
    else:  # every key, what is not selected masked
        k = (s["k"][:, :, :M].view(torch.float8_e4m3fn).float() * s["k_scale"][:, :, :M, None, None]).flatten(2, 3)
        v = s["v"][:, :, :M].view(torch.float8_e4m3fn).float() * s["v_scale"][:, :, :M, None, None]
        v = v.transpose(-1, -2).flatten(2, 3)
        kept = torch.zeros((B, Hkv, Nq, M + 1), dtype=torch.bool, device="cuda")
        kept.scatter_(-1, torch.where(idx < 0, M, idx), True)
        shown = kept[..., :M].repeat_interleave(C, -1) & (torch.arange(M * C, device="cuda") <= t[:, None])
        o, lse = _softmax_rows(torch.matmul(q, k.transpose(-1, -2)[:, :, None]), v[:, :, None], shown[:, :, None])
    return o.reshape(B, H, Nq, d).to(s["q"].dtype), lse.reshape(B, H, Nq)


# ---------------------------------------------------------------- one pass ---

def run(s):
    c = s["case"]
    if c["op"] == "rope":
        return _rope_own(s) if own else _rope_plain(s)
    if c["op"] == "attend":
        return _attend_own(s) if own else _attend_plain(s)
    if c["n_old"] % c["C"] and c["n_old"] // c["C"] != (c["N"] - 1) // c["C"]:
        # a pass that leaves its first block leaves other raw rows behind: put back what the next one starts from
        s["k_open"].copy_(s["k_was"])
        s["v_open"].copy_(s["v_was"])
    if own:
        _append_own(s)
    else:
        _append_plain(s, c, s["k_new"], s["v_new"], c["n_old"], c["N"])
    return dict(k=s["k"].view(torch.float8_e4m3fn), v=s["v"].view(torch.float8_e4m3fn), k_scale=s["k_scale"],
                v_scale=s["v_scale"], k_open=s["k_open"], v_open=s["v_open"], pyramid=s["pyramid"])


def _problem(c, Nq, H, K):
    from paper_2609_31093_amd import pisa

    return pisa.make_problem(c["B"], H, c["Hkv"], Nq, c["N"], c["d"], c["C"], c["g"], K, c.get("causal", True), c["dtype"],
                             Ncap=c["cap"])


def _cache(s):
    from paper_2609_31093_amd import pisa

    return pisa.QCache(s["k"], s["v"], s["k_scale"], s["v_scale"], s["k_open"], s["v_open"])


def _rope_own(s):
    from paper_2609_31093_amd import pisa

    c = s["case"]
    if s["plan"] is None:
        s["plan"] = pisa.make_rope(c["B"], c["H"], c["Hkv"], c["N"], c["d"], rot=c["rot"], layout=c["layout"],
                                   dtype=c["dtype"], scaling=c["scaling"], factor=c["factor"], ctx=c["ctx"], pos0=c["pos0"])
    turn = pisa.rope_bwd if c["bwd"] else pisa.rope_fwd
    return turn(s["plan"], s["q"], s["k"], s["positions"], s["q_out"], s["k_out"])


def _append_own(s):
    from paper_2609_31093_amd import pisa

    c = s["case"]
    if s["plan"] is None:
        s["plan"] = _problem(c, 1, c["Hkv"], 4), _cache(s)
    pisa.qcache_append(*s["plan"], s["k_new"], s["v_new"], c["n_old"], s["pyramid"])


def _attend_own(s):
    from paper_2609_31093_amd import pisa

    c = s["case"]
    if s["plan"] is None:
        p = _problem(c, c["Nq"], c["H"], c["K"])
        nb = pisa.pisa_qcache_attn_workspace_bytes(p)
        s["plan"] = p, _cache(s), torch.empty(max(nb, 1), dtype=torch.uint8, device="cuda"), nb
    p, cache, ws, nb = s["plan"]
    pisa.pisa_qcache_attn_fwd(p, cache, s["q"], s["idx"], s["o"], s["lse"], ws, nb)
    return s["o"], s["lse"]


# ---------------------------------------------------------------- work, exact results ---

def work(case):
    c = case
    e = 4 if c["dtype"] == "f32" else 2
    B, Hkv, N, d = c["B"], c["Hkv"], c["N"], c["d"]
    if c["op"] == "rope":
        values = B * (c["H"] + Hkv) * N
        return {"bytes": 2 * values * d * e + (4 * B * N if c["ragged"] else 0), "flops": 3 * values * c["rot"]}
    C = c["C"]
    if c["op"] == "append":
        new, first = N - c["n_old"], c["n_old"] // C
        blocks, had = (N - 1) // C + 1 - first, c["n_old"] - first * C
        nodes = sum(-(-blocks // c["g"] ** i) for i in range(len(_levels(N, C, c["g"]))))
        read = 2 * (new + had) * d * e
        write = 2 * (N - first * C) * d + 8 * blocks + 4 * nodes * d + 2 * min(new, N - (N - 1) // C * C) * d * e
        return {"bytes": B * Hkv * (read + write), "flops": 4 * B * Hkv * (new + had) * d}
    Nq, H, K = c["Nq"], c["H"], min(c["K"], -(-N // C))
    blocks = B * Hkv * min(-(-N // C), Nq * K)
    rows = B * H * Nq
    return {"bytes": 2 * rows * d * e + 4 * rows + 4 * B * Hkv * Nq * c["K"] + blocks * (2 * C * d + 8),
            "flops": 4 * rows * K * C * d}


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


def _exact_append(c, seed):
    C, g, N = c["C"], c["g"], c["N"]
    M = -(-N // C)
    s = prepare(c, seed)
    first = c["n_old"] // C
    out = {}
    for i, name in enumerate(("k", "v")):
        raw = _keys(c, N, seed, i)
        rows = raw[:, :, first * C:].double()
        n = rows.shape[2]
        rows = torch.cat((rows, rows.new_zeros((*rows.shape[:2], (M - first) * C - n, c["d"]))), 2)
        codes, scale = _exact_codes(rows.view(c["B"], c["Hkv"], M - first, C, c["d"]))
        whole = s[name].view(torch.float8_e4m3fn).double()
        whole[:, :, first:M] = codes.transpose(-1, -2) if name == "v" else codes
        out[name] = whole
        out[name + "_scale"] = s[name + "_scale"].double()
        out[name + "_scale"][:, :, first:M] = scale
        out[name + "_open"] = s[name + "_open"].double()
        out[name + "_open"][:, :, :N - (M - 1) * C] = raw[:, :, (M - 1) * C:].double()
        if name == "k":  # every level from the level below in 64 bits
            level = raw.double().split(C, 2)
            level = torch.stack([x.mean(2) for x in level], 2)
            pyr, at = s["pyramid"].double(), 0
            sizes = _levels(N, C, g)
            for size, room in zip(sizes, _levels(c["cap"], C, g)):
                pyr[:, :, at:at + size] = level
                at += room
                level = torch.stack([x.mean(2) for x in level.split(g, 2)], 2)
            out["pyramid"] = pyr
    return out


def _exact_rope(c, seed):
    s = prepare(c, seed)
    B, N, rot = c["B"], c["N"], c["rot"]
    f, amplitude = _frequencies(c)
    pos = s["positions"].double() if s["positions"] is not None else (c["pos0"] + torch.arange(N, device="cuda")).double()
    turn = torch.polar(torch.full((1,), amplitude, dtype=torch.float64, device="cuda"),
                       pos.view(-1, N, 1) * torch.tensor(f, dtype=torch.float64, device="cuda"))
    turn = (turn.conj() if c["bwd"] else turn)[:, None]
    half = c["layout"] == "half"
    out = []
    for x in (s["q"].double(), s["k"].double()):
        z = x[..., :rot].unflatten(-1, (2, rot // 2)).transpose(-1, -2) if half else x[..., :rot].unflatten(-1, (rot // 2, 2))
        z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn)
        z = z.transpose(-1, -2).flatten(-2) if half else z.flatten(-2)
        out.append(torch.cat((z, x[..., rot:]), -1))
    return tuple(out)


def _exact_attend(c, seed):
    s = prepare(c, seed)
    B, H, Hkv, Nq, N, d, C, K = (c[x] for x in ("B", "H", "Hkv", "Nq", "N", "d", "C", "K"))
    G = H // Hkv
    o = torch.zeros((B, Hkv, Nq, G, d), dtype=torch.float64, device="cuda")
    lse = torch.full((B, Hkv, Nq, G), -math.inf, dtype=torch.float64, device="cuda")
    q = s["q"].double().view(B, Hkv, G, Nq, d).transpose(2, 3)
    step = max(1, (1 << 28) // (K * C * d))
    for b in range(B):
        for h in range(Hkv):
            for r in range(0, Nq, step):
                i = s["idx"][b, h, r:r + step].long()
                at = i.clamp(min=0)
                k = s["k"][b, h][at].view(torch.float8_e4m3fn).double() * s["k_scale"][b, h][at].double()[..., None, None]
                v = s["v"][b, h][at].view(torch.float8_e4m3fn).double() * s["v_scale"][b, h][at].double()[..., None, None]
                token = (at[..., None] * C + torch.arange(C, device="cuda")).flatten(1)
                last = torch.arange(N - Nq + r, N - Nq + r + len(i), device="cuda")[:, None] if c["causal"] else N - 1
                off = (token > last) | (i < 0).repeat_interleave(C, 1)
                z = torch.bmm(q[b, h, r:r + step].contiguous(), k.flatten(1, 2).transpose(1, 2).contiguous()) / math.sqrt(d)
                z = torch.where(off[:, None], -math.inf, z)
                total = torch.logsumexp(z, -1)
                w = torch.where((total > -math.inf)[..., None], torch.exp(z - total[..., None]), 0.0)
                o[b, h, r:r + step] = torch.bmm(w, v.transpose(2, 3).flatten(1, 2).contiguous())
                lse[b, h, r:r + step] = total
    return o.transpose(2, 3).reshape(B, H, Nq, d), lse.transpose(2, 3).reshape(B, H, Nq)


def exact(case, seed):
    c = dict(case)
    return {"rope": _exact_rope, "append": _exact_append, "attend": _exact_attend}[c["op"]](c, seed)
