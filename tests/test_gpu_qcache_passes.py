"""Many rows over the 8-bit cache whose partials take several passes: over KV heads, and over the rows of one."""
import pytest
import torch

import test_gpu_qcache as base

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2609_31093_amd import pisa

# a pass holds 2^30 / (K G (2 d + 4)) rows of KV heads
PASSES = [
    ((3, 12, 3, 9000, 9000, 128, 64, 2, 16, 1, "bf16"), 9000, 9),      # 64527: 5 heads each (of 9), all rows
    ((1, 8, 2, 16500, 16500, 128, 64, 2, 64, 1, "bf16"), 8250, 2),     # 16131: half the rows of one head
    ((1, 5, 1, 19000, 19000, 64, 128, 2, 100, 0, "bf16"), 9500, 1),    # 16269: the same, blocks of several units
]


@pytest.mark.parametrize("shape,rows,heads", PASSES, ids=str)
def test_passes(shape, rows, heads):
    B, H, Hkv, Nq, N, d, C, g, K, causal, dtype = shape
    p = base.problem(*shape)
    most = 2 ** 30 // (K * (H // Hkv) * (2 * d + 4))
    assert B * Hkv == heads and (most // Nq < B * Hkv if rows == Nq else most < Nq and rows <= most)
    nb = pisa.pisa_qcache_attn_workspace_bytes(p)
    assert 2 ** 28 < nb < 2 ** 30 + 2 ** 28
    k, v = base.normal((B, Hkv, N, d), 1, dtype, 0.5), base.normal((B, Hkv, N, d), 2, dtype, 0.5)
    q = torch.randn((B, H, Nq, d), generator=torch.Generator("cuda").manual_seed(3), device="cuda").bfloat16()
    cache = pisa.make_qcache(p)
    pisa.qcache_append(p, cache, k, v, 0)
    idx = base.quick_selection(p, 4)
    o, lse = torch.full_like(q, 7.0), torch.full((B, H, Nq), 7.0, device="cuda")
    band = torch.full((nb + 8192,), 0xA5, dtype=torch.uint8, device="cuda")
    pisa.pisa_qcache_attn_fwd(p, cache, q, idx, o, lse, band[4096:], nb)
    base.check_grouped(p, cache, q, idx, o, lse, sorted({0, 97, rows - 1, rows % Nq, (rows + 1) % Nq, Nq - 1}))
    assert bool((band[:4096] == 0xA5).all()) and bool((band[-4096:] == 0xA5).all())
    assert torch.isfinite(o).all() and bool((lse != 7).all())
    # a KV head on its own
    one = base.problem(1, H // Hkv, 1, Nq, N, d, C, g, K, causal, dtype)
    cut = lambda x, n: x[B - 1:, (Hkv - 1) * n:Hkv * n].clone(memory_format=torch.contiguous_format)  # noqa: E731
    last = pisa.QCache(*(cut(x, 1) for x in (cache.k, cache.v, cache.k_scale, cache.v_scale)))
    alone = pisa.qcache_attn_fwd(one, last, cut(q, H // Hkv), cut(idx, 1))
    assert torch.equal(cut(o, H // Hkv), alone[0]) and torch.equal(cut(lse, H // Hkv), alone[1])
