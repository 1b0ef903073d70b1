"""Drafted rows that are taken back: the next append with a smaller n_old leaves the cache and the pyramid as if they had
never been there, bit for bit."""
import pytest
import torch

import test_gpu_qcache as base

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2609_31093_amd import pisa


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C,g,n0,draft,kept,more", [
    (64, 2, 300, 8, 3, 5),        # within a block
    (64, 2, 319, 9, 1, 4),        # kept up to the block's border, the draft past it
    (64, 2, 320, 5, 0, 1),        # begun on the border
    (64, 2, 310, 20, 4, 30),      # past a border and back into the block before
    (32, 2, 250, 300, 5, 90),     # past several, and the tree grew by a level
    (32, 4, 2040, 200, 8, 1),     # past a border where a level is new, back to the border itself
    (96, 3, 1, 700, 0, 300),
])
def test_taken_back(dtype, C, g, n0, draft, kept, more):
    B, Hkv, d, cap = 2, 2, 64, 2400
    p = base.problem(B, Hkv, Hkv, 1, n0 + kept + more, d, C, g, 4, 1, dtype, cap)
    k, v = base.normal((B, Hkv, p.N, d), 1, dtype, 0.7), base.normal((B, Hkv, p.N, d), 2, dtype, 0.7)
    cache, pyr = pisa.make_qcache(p), base.new_pyramid(p)
    pisa.qcache_append(base.at(p, n0), cache, k[:, :, :n0], v[:, :, :n0], 0, pyr)
    was = cache.k_open.clone(), cache.v_open.clone()
    dk, dv = base.normal((B, Hkv, draft, d), 3, dtype, 2.0), base.normal((B, Hkv, draft, d), 4, dtype, 2.0)
    dk[:, :, :kept], dv[:, :, :kept] = k[:, :, n0:n0 + kept], v[:, :, n0:n0 + kept]
    for n in range(n0, n0 + draft, 7):  # a few rows at a time
        end = min(n + 7, n0 + draft)
        pisa.qcache_append(base.at(p, end), cache, dk[:, :, n - n0:end - n0], dv[:, :, n - n0:end - n0], n, pyr)
    back = n0 + kept
    if back % C and back // C != (n0 + draft - 1) // C:
        # the rows kept of the draft belong to the block that it began in: put that back and append them again
        cache.k_open.copy_(was[0])
        cache.v_open.copy_(was[1])
        back = n0
    pisa.qcache_append(p, cache, k[:, :, back:], v[:, :, back:], back, pyr)
    base.check_cache(p, cache, k, v)
    want, tree = pisa.make_qcache(p), base.new_pyramid(p)
    pisa.qcache_append(p, want, k, v, 0, tree)
    M = -(-p.N // C)
    for x, y in ((cache.k, want.k), (cache.v, want.v), (cache.k_scale, want.k_scale), (cache.v_scale, want.v_scale)):
        assert torch.equal(x[:, :, :M], y[:, :, :M])
    used = torch.isfinite(tree)  # nodes of p's N tokens; the draft left others
    assert torch.equal(pyr[used], tree[used])
