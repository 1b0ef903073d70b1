"""Infinite values that drafted tokens' attention sees: the dimension's result is that infinity, NaN only where both signs
meet, and the other dimensions are what they are without it (tolerance of test_gpu_draft_attn.py)."""
import math

import numpy as np
import pytest
import torch

import test_gpu_draft_attn as attn
import test_gpu_qcache as base

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2609_31093_amd import pisa


@pytest.mark.parametrize("eight", [False, True], ids=["raw", "8bit"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,Hkv,T,n,d,C,K", [(1, 2, 2, 24, 1000, 128, 32, 4), (2, 8, 2, 40, 777, 64, 64, 6), (1, 8, 2, 12, 3000, 128, 64, 16),
                                               (1, 16, 1, 5, 90, 64, 32, 3), (1, 2, 2, 3, 0, 128, 64, 3)])
def test_infinite_values(eight, dtype, B, H, Hkv, T, n, d, C, K):
    p = base.problem(B, H, Hkv, T, n + T, d, C, 2, K, 1, dtype, 0)
    cache, q = attn.make(p, eight, 1, dtype), base.normal((B, H, T, d), 3, dtype)
    new, idx, mask = tuple(x.contiguous() for x in attn.drafted(p, 5, dtype)), attn.selection(p, 4), attn.trees(B, T, 6)
    finite = tuple(x.clone() for x in cache) if not eight else cache
    finite_new = tuple(x.clone() for x in new)
    # (row, dimension, sign): of the cache (codes have no infinity), and of the drafted rows
    held = [] if eight or not n else [(5, 3, 1), (n // 2, 9, -1), (n - 1, 9, 1), (7, d - 1, 1), (7, 20, -1)]
    own = [(0, 9, -1), (1, 40, 1), (T - 1, 3, 1), (2, 20, 1)]
    for j, e, sign in held:
        cache[1][:, :, j, e] = sign * math.inf
    for j, e, sign in own:
        new[1][:, :, j, e] = sign * math.inf
    o, lse = attn.attend(p, cache, q, idx, *new, mask)
    want, want_l, tol_o, tol_l = attn.reference(p, finite, q, idx, *finite_new, mask)
    got, got_l = o.double().cpu().numpy(), lse.double().cpu().numpy()

    sel, sees = idx.cpu().numpy(), attn.bits_of(mask, T)
    plus, minus = np.zeros(got.shape, bool), np.zeros(got.shape, bool)
    for b, h, r in np.ndindex(B, H, T):
        for j, e, sign in held:
            if (sel[b, h // (H // Hkv), r] == j // C).any():
                (plus if sign > 0 else minus)[b, h, r, e] = True
        for j, e, sign in own:
            if sees[b, r, j]:
                (plus if sign > 0 else minus)[b, h, r, e] = True
    assert plus.any() and minus.any()
    assert (got[plus & ~minus] == math.inf).all(), got[plus & ~minus]
    assert (got[minus & ~plus] == -math.inf).all(), got[minus & ~plus]
    assert np.isnan(got[plus & minus]).all()
    rest = ~(plus | minus)
    assert (abs(got - want)[rest] <= tol_o[rest]).all()
    empty = np.isneginf(want_l)
    assert np.array_equal(np.isneginf(got_l), empty) and (abs(got_l - want_l)[~empty] <= tol_l[~empty]).all()
