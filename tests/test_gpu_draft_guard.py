"""Sentinels around every output and workspace of the norms' and the drafted tokens' entry points: all of the output is
written, and nothing beside it."""
import numpy as np
import pytest
import torch

import test_gpu_draft_attn as attn
import test_gpu_norm_rope as norm
import test_gpu_qcache as base

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2609_31093_amd import pisa

PAD, MARK = 4096, 0xA5


class Guarded:
    def __init__(self):
        self.raws = []

    def __call__(self, shape, dtype):
        n = int(np.prod(shape)) * torch.empty((), dtype=dtype).element_size()
        raw = torch.full((n + 2 * PAD,), MARK, dtype=torch.uint8, device="cuda")
        self.raws.append((raw, n))
        return raw[PAD:PAD + n].view(dtype).reshape(shape)

    def check(self):
        torch.cuda.synchronize()
        for raw, n in self.raws:
            assert bool((raw[:PAD] == MARK).all()) and bool((raw[PAD + n:] == MARK).all())


@pytest.mark.parametrize("layout,rot", [("half", 128), ("half", 42), ("interleaved", 96)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,Hkv,N", [(1, 1, 1, 1), (3, 5, 2, 67), (1, 16, 4, 3000)])
def test_norm(layout, rot, dtype, B, H, Hkv, N):
    d, make = 128, Guarded()
    r = pisa.make_rope(B, H, Hkv, N, d, rot=rot, layout=layout, dtype=dtype)
    w = [norm.weights(d, i, dtype, 0.0) for i in (1, 2)]
    m = pisa.make_qk_norm(r, *w)
    x = [base.normal((B, h, N, d), i, dtype) for i, h in enumerate((H, Hkv, H, Hkv))]
    t = base.TYPES[dtype]
    out = [make((B, h, N, d), t) for h in (H, Hkv, H, Hkv)]
    dw = [make((d,), torch.float32) for _ in range(2)]
    nb = pisa.pisa_norm_rope_bwd_workspace_bytes(r)
    ws = make((nb,), torch.uint8)
    pisa.norm_rope_fwd(r, m, x[0], x[1], q_out=out[0], k_out=out[1])
    pisa.pisa_norm_rope_bwd(r, m, x[0], None, x[1], None, x[2], None, x[3], None, None, out[2], None, out[3], None, *dw, ws, nb)
    make.check()
    for a, b in zip((*out, *dw), (*pisa.norm_rope_fwd(r, m, *x[:2]), *pisa.norm_rope_bwd(r, m, *x))):
        assert torch.equal(a, b)


@pytest.mark.parametrize("B,T", [(1, 1), (3, 64), (2, 65), (1, 1024)])
def test_layout(B, T):
    make, parents = Guarded(), torch.randint(-2, T + 2, (B, T), dtype=torch.int32, device="cuda")
    mask, pos = make((B, T, -(-T // 64)), torch.int64), make((B, T), torch.int32)
    pisa.pisa_draft_layout(B, T, parents, 9, mask, pos)
    make.check()
    want = pisa.draft_layout(parents, 9)
    assert torch.equal(mask, want[0]) and torch.equal(pos, want[1])


@pytest.mark.parametrize("eight", [False, True], ids=["raw", "8bit"])
@pytest.mark.parametrize("shape", [(1, 1, 1, 1, 0, 64, 32, 2, 4, "bf16", 0), (2, 6, 2, 33, 450, 128, 32, 2, 6, "f32", 0),
                                   (1, 8, 8, 17, 2047, 128, 64, 2, 16, "bf16", 64), (2, 16, 1, 100, 300, 64, 64, 2, 8, "bf16", 3)], ids=str)
def test_attention(eight, shape):
    p, make = attn.problem(shape), Guarded()
    cache, q = attn.make(p, eight, 1, shape[9]), base.normal((p.B, p.H, p.Nq, p.d), 3, shape[9])
    new, idx, mask = attn.drafted(p, 5, shape[9]), attn.selection(p, 4), attn.trees(p.B, p.Nq, 6)
    nb = (pisa.pisa_qcache_draft_attn_workspace_bytes if eight else pisa.pisa_draft_attn_workspace_bytes)(p)
    o, lse, ws = make((p.B, p.H, p.Nq, p.d), q.dtype), make((p.B, p.H, p.Nq), torch.float32), make((nb,), torch.uint8)
    attn.attend(p, cache, q, idx, *new, mask, o=o, lse=lse, ws=ws)
    make.check()
    want = attn.attend(p, cache, q, idx, *new, mask)
    assert torch.equal(o, want[0]) and torch.equal(lse, want[1])


@pytest.mark.parametrize("eight", [False, True], ids=["raw", "8bit"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_old,N,C,g", [(0, 65, 64, 2), (126, 131, 64, 2), (127, 128, 32, 2), (1, 200, 128, 4), (320, 320 + 33, 32, 3)])
def test_append(eight, dtype, n_old, N, C, g):
    B, Hkv, d, make = 2, 3, 128, Guarded()
    p = base.problem(B, Hkv, Hkv, 1, N, d, C, g, 3, 1, dtype, N)
    t, M, R = base.TYPES[dtype], -(-N // C), pisa.pisa_pyramid_layout(p)[1]
    new = [base.normal((B, Hkv, 250, d), i, dtype) for i in (1, 2)]
    rows = torch.randint(0, 250, (B, N - n_old), dtype=torch.int32, device="cuda")
    pyr = make((B, Hkv, R, d), torch.float32)
    old = [base.normal((B, Hkv, max(n_old, 1), d), i, dtype) for i in (3, 4)]
    if eight:
        cache = pisa.QCache(make((B, Hkv, M, C, d), torch.uint8), make((B, Hkv, M, d, C), torch.uint8), make((B, Hkv, M), torch.float32),
                            make((B, Hkv, M), torch.float32), make((B, Hkv, C, d), t), make((B, Hkv, C, d), t))
        if n_old:
            pisa.qcache_append(base.at(p, n_old), cache, *old, 0, pyr)
        pisa.qcache_append_rows(p, cache, *new, rows, n_old, pyr)
    else:
        held = [make((B, Hkv, N, d), t) for _ in range(2)]
        if n_old:
            pisa.cache_append_rows(base.at(p, n_old), *held, *old, None, 0, pyr)
        pisa.cache_append_rows(p, *held, *new, rows, n_old, pyr)
    make.check()
