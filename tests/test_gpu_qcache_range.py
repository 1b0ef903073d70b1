"""Attention over the 8-bit cache with logits and values of any size that its types hold.

Large logits.  Only dimension 0 of keys and queries is not 0, so every logit is one product of a power of two and a code:
exact in 32 bits, and equal for many keys.  The rows' weights are then those of the largest logits alone, equal ones, up
to the error of what is computed from exact differences: 2^-21 of a weight (2 ulp of the exponential, the argument is 0),
2^-11 more where weights are held in fp16 (bf16 queries) and again where partials are (rows grouped by block), n 2^-24
twice for sums of n terms, 2^-8 of the result (bf16) or 2^-23.  Keys that are not the largest are at least 2^a / 16 / 12
below it (2^12 and more), so their weights are 0.  lse = (largest logit) + log(number of them): 2^-22 of it, 2^-20 of a
sum and n 2^-24.

Large and small values: the bounds of test_gpu_qcache, which scale with the values.
"""
import math

import numpy as np
import pytest
import torch

import test_gpu_qcache as base

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2609_31093_amd import pisa

FORMS = [
    # B, H, Hkv, Nq, N, d, C, g, K, causal, dtype
    (1, 8, 8, 1, 2000, 128, 64, 2, 16, 1, "bf16"),      # units over wavefronts and workgroups
    (2, 6, 2, 5, 900, 64, 96, 2, 4, 1, "bf16"),         # units of 32 keys
    (1, 16, 1, 200, 1000, 128, 256, 2, 6, 1, "bf16"),   # a wavefront takes several units
    (1, 2, 2, 65, 1000, 64, 64, 2, 4, 1, "f32"),
    (1, 4, 1, 3, 1500, 128, 128, 4, 12, 0, "f32"),
    (1, 4, 1, 3500, 9000, 128, 64, 2, 16, 1, "bf16"),   # grouped: a unit is a block
    (1, 4, 4, 2300, 2300, 64, 32, 2, 30, 1, "bf16"),
    (1, 5, 1, 2200, 4000, 128, 128, 4, 16, 1, "bf16"),  # grouped: several units to a block
    (1, 3, 1, 2500, 2500, 64, 96, 2, 24, 1, "bf16"),
]


def grouped(p):
    return p.Nq > 300 and pisa.pisa_qcache_attn_workspace_bytes(p) > p.B * p.H * p.Nq * p.K * p.d * 2


def filled(p, k, v):
    cache = pisa.make_qcache(p)
    pisa.qcache_append(p, cache, k, v, 0)
    return cache


def selection(p):
    return base.quick_selection(p, 4) if p.Nq > 300 else base.random_selection(p, 4)


@pytest.mark.parametrize("power", [20, 26, 28, 30, 45, 100])
@pytest.mark.parametrize("form", FORMS, ids=str)
def test_large_logits(form, power):
    B, H, Hkv, Nq, N, d, C, g, K, causal, dtype = form
    p = base.problem(*form)
    G, M, rng = H // Hkv, -(-N // C), np.random.default_rng(power)
    key = rng.choice([256.0, 240.0, 128.0, 2.0, -256.0, -224.0], (B, Hkv, N), p=[0.2, 0.1, 0.2, 0.2, 0.2, 0.1])
    k = torch.zeros((B, Hkv, N, d), dtype=base.TYPES[dtype], device="cuda")
    k[..., 0] = torch.from_numpy(key).to(k)
    v = base.normal((B, Hkv, N, d), 2, dtype)
    sign = rng.choice([-1.0, 1.0], (B, H, Nq))
    q = torch.zeros((B, H, Nq, d), dtype=base.TYPES[dtype], device="cuda")
    q[..., 0] = torch.from_numpy(sign * 2.0 ** (power - 8)).to(q)
    cache = filled(p, k, v)
    idx = selection(p)
    o, lse = pisa.qcache_attn_fwd(p, cache, q, idx)
    vv = (base.values(cache.v).swapaxes(-1, -2) * cache.v_scale.double().cpu().numpy()[..., None, None]).reshape(B, Hkv, M * C, d)
    assert np.array_equal((base.values(cache.k) * cache.k_scale.double().cpu().numpy()[..., None, None]).reshape(B, Hkv, M * C, d)[:, :, :N, 0], key)
    o, lse, sel = o.double().cpu().numpy(), lse.double().cpu().numpy(), idx.cpu().numpy()
    assert np.isfinite(o).all()
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -23
    weight = (2.0 ** -11 if dtype == "bf16" else 0) + (2.0 ** -11 if grouped(p) else 0)
    for b in range(B):
        for h in range(H):
            for r in base.sample(p, 5) if Nq > 97 else range(Nq):
                t = N - Nq + r if causal else N - 1
                tok = [np.arange(j * C, min((j + 1) * C, t + 1)) for j in sel[b, h // G, r] if 0 <= j < M]
                tok = np.concatenate(tok or [np.zeros(0, int)]).astype(int)
                if not len(tok):
                    assert (o[b, h, r] == 0).all() and lse[b, h, r] == -math.inf
                    continue
                z = sign[b, h, r] * key[b, h // G, tok] * 2.0 ** (power - 8)
                top = tok[z == z.max()]
                rows, n = vv[b, h // G, top], len(tok)
                want, size = rows.mean(0), abs(rows).mean(0)
                tol = (2.0 ** -20 + weight + 2 * n * 2.0 ** -24) * size + half * abs(want)
                assert (abs(o[b, h, r] - want) <= tol).all(), (b, h, r, abs(o[b, h, r] - want).max())
                want = z.max() / math.sqrt(d) + math.log(len(top))
                assert abs(lse[b, h, r] - want) <= 2.0 ** -22 * abs(want) + 2.0 ** -20 + n * 2.0 ** -24, (b, h, r)


@pytest.mark.parametrize("power", [-106, -60, 110, 125, 127])
@pytest.mark.parametrize("form", FORMS, ids=str)
def test_values_of_any_size(form, power):
    """Values of one sign near 2^power: their weighted sums, before the division by the weights' sum, would not be finite."""
    B, H, Hkv, Nq, N, d, C, g, K, causal, dtype = form
    p = base.problem(*form)
    k, q = base.normal((B, Hkv, N, d), 1, dtype, 0.5), base.normal((B, H, Nq, d), 3, dtype)
    v = torch.rand((B, Hkv, N, d), generator=torch.Generator("cuda").manual_seed(2), device="cuda") * 0.5 + 0.5
    cache = filled(p, k, (v * 2.0 ** power).to(base.TYPES[dtype]))
    idx = selection(p)
    o, lse = pisa.qcache_attn_fwd(p, cache, q, idx)
    assert torch.isfinite(o).all()
    if grouped(p):
        base.check_grouped(p, cache, q, idx, o, lse, base.sample(p, 5))
    else:
        base.check_attention(p, cache, q, idx, o, lse, base.sample(p, 5) if Nq > 97 else None)
