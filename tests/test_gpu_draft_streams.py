"""The wrappers of norms and drafted tokens with a stream of the caller's: what they allocate belongs to that stream, and work
that is on its way there before and after them is not disturbed."""
import pytest
import torch

import test_gpu_draft_attn as attn
import test_gpu_norm_rope as norm
import test_gpu_qcache as base

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2609_31093_amd import pisa

NAMES = ["norm_rope_fwd", "norm_rope_bwd", "draft_layout", "draft_attn_fwd", "qcache_draft_attn_fwd", "draft_attn_fwd, one launch",
         "cache_append_rows", "qcache_append_rows"]


@pytest.fixture(scope="module")
def calls():
    """name -> call(stream) -> outputs."""
    B, H, Hkv, N, d = 2, 4, 2, 500, 128
    r = pisa.make_rope(B, H, Hkv, N, d)
    m = pisa.make_qk_norm(r, norm.weights(d, 1, "bf16", 0.0), norm.weights(d, 2, "bf16", 0.0))
    x = [base.normal((B, h, N, d), i, "bf16") for i, h in enumerate((H, Hkv, H, Hkv))]
    parents = torch.randint(-1, 40, (B, 40), dtype=torch.int32, device="cuda")
    out = {
        "norm_rope_fwd": lambda s: pisa.norm_rope_fwd(r, m, *x[:2], stream=s),
        "norm_rope_bwd": lambda s: pisa.norm_rope_bwd(r, m, *x, stream=s),
        "draft_layout": lambda s: pisa.draft_layout(parents, 100, stream=s),
    }
    p = attn.problem((2, 8, 2, 10, 3000, 128, 64, 2, 16, "bf16", 64))
    few = attn.problem((2, 8, 2, 10, 100, 64, 32, 2, 3, "bf16", 64))
    assert pisa.pisa_draft_attn_workspace_bytes(p) > 0 and pisa.pisa_draft_attn_workspace_bytes(few) == 0
    args = {}
    for name, q, eight in (("raw", p, False), ("8bit", p, True), ("few", few, False)):
        args[name] = (q, attn.make(q, eight, 1, "bf16"), base.normal((2, 8, 10, q.d), 3, "bf16"), attn.selection(q, 4), *attn.drafted(q, 5, "bf16"),
                      attn.trees(2, 10, 6))
    out["draft_attn_fwd"] = lambda s: attn.attend(*args["raw"], stream=s)
    out["qcache_draft_attn_fwd"] = lambda s: attn.attend(*args["8bit"], stream=s)
    out["draft_attn_fwd, one launch"] = lambda s: attn.attend(*args["few"], stream=s)
    a = base.problem(2, 2, 2, 1, 190, 64, 64, 2, 4, 1, "bf16", 300)
    k, v = (base.normal((2, 2, 180, 64), i, "bf16") for i in (1, 2))
    new = [base.normal((2, 2, 12, 64), i, "bf16") for i in (3, 4)]
    rows = torch.tensor([[0, 1, 2, 5, 6, 7, 8, 9, 10, 11]] * 2, dtype=torch.int32, device="cuda")

    def raw(s):
        held = [torch.zeros((2, 2, 300, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        held[0][:, :, :180], held[1][:, :, :180] = k, v
        torch.cuda.synchronize()
        pisa.cache_append_rows(a, *held, *new, rows, 180, stream=s)
        return held

    def eight(s):
        cache = pisa.make_qcache(a)
        pisa.qcache_append(base.at(a, 180), cache, k, v, 0)
        torch.cuda.synchronize()
        pisa.qcache_append_rows(a, cache, *new, rows, 180, stream=s)
        return cache.k, cache.v, cache.k_open, cache.v_open
    out["cache_append_rows"], out["qcache_append_rows"] = raw, eight
    return out


@pytest.mark.parametrize("name", [n for n in NAMES if "append" not in n])
def test_allocations_are_the_streams_own(calls, monkeypatch, name):
    side, seen = torch.cuda.Stream(), []

    def watched(make):
        def call(*a, **kw):
            seen.append(torch.cuda.current_stream().cuda_stream)
            return make(*a, **kw)
        return call
    for raw in ("pisa_norm_rope_fwd", "pisa_norm_rope_bwd", "pisa_draft_layout", "pisa_draft_attn_fwd", "pisa_qcache_draft_attn_fwd"):
        monkeypatch.setattr(pisa, raw, lambda *a, **kw: 0)
    monkeypatch.setattr(torch, "empty", watched(torch.empty))
    monkeypatch.setattr(torch, "empty_like", watched(torch.empty_like))
    here = torch.cuda.current_stream().cuda_stream
    for given, want in ((side, side.cuda_stream), (side.cuda_stream, side.cuda_stream), (None, here), (here, here)):
        seen.clear()
        calls[name](given)
        assert seen and set(seen) == {want}
    assert torch.cuda.current_stream().cuda_stream == here


@pytest.mark.parametrize("name", NAMES)
def test_a_busy_stream(calls, name):
    """The stream has work before it when the wrapper returns; the current stream allocates and writes meanwhile."""
    want = [x.clone() for x in calls[name](None)]
    torch.cuda.synchronize()
    sizes = {x.numel() * x.element_size() for x in want} | {1 << i for i in range(9, 23)}
    side, a = torch.cuda.Stream(), torch.randn((4096, 4096), device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(4):
            a @ a
    got = calls[name](side)
    held = [torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") for n in sizes if n for _ in range(3)]
    torch.cuda.synchronize()
    for x, y in zip(got, want):
        assert torch.equal(x, y)
    assert len(held)


@pytest.mark.parametrize("name", [n for n in NAMES if "append" not in n])
def test_captured_on_a_forked_stream(calls, name):
    """The call's stream is a branch of a capture: its memory is the graph's, and replays give the eager result."""
    want = [x.clone() for x in calls[name](None)]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        got = calls[name](side)
        torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.full((1 << 20,), 1.0, device="cuda").sum() == 1 << 20
        for x, y in zip(got, want):
            assert torch.equal(x, y)
