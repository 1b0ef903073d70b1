"""The allocating wrappers with a stream of the caller's: what they allocate belongs to that stream.

Memory of the current stream's would go to its next allocations as soon as the wrapper returns and drops its workspace,
while the other stream still works on it."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2609_31093_amd import pisa

B, H, Hkv, N, d, C, g, K = 1, 4, 1, 3000, 128, 64, 2, 16


def problem(Nq=N):
    return pisa.make_problem(B, H, Hkv, Nq, N, d, C, g, K, 1, "bf16")


def normal(h, n, seed):
    return torch.randn((B, h, n, d), generator=torch.Generator("cuda").manual_seed(seed), device="cuda").bfloat16()


@pytest.fixture(scope="module")
def calls():
    """name -> call(stream) -> outputs, of every wrapper that allocates."""
    p, few = problem(), problem(2)
    q, k, v, d_o = normal(H, N, 1), normal(Hkv, N, 2), normal(Hkv, N, 3), normal(H, N, 4)
    pyr = pisa.build_pyramid(p, k)
    idx = pisa.select(p, q, k, pyr)
    o, lse = pisa.sparse_attn_fwd(p, q, k, v, idx)
    cache = pisa.make_qcache(p)
    pisa.qcache_append(p, cache, k, v, 0)
    rows = torch.tensor([0, 100, 2999], dtype=torch.int32, device="cuda")
    r = pisa.make_rope(B, H, Hkv, N, d)
    q2, i2 = q[:, :, -2:].contiguous(), idx[:, :, -2:].contiguous()
    return {
        "build_pyramid": lambda s: (pisa.build_pyramid(p, k, s),),
        "grow_cache": lambda s: tuple(x[:, :, :n] for x, n in zip(pisa.grow_cache(p, 4096, pyr, k, v, s)[1:], (47, N, N))),
        "select": lambda s: pisa.select(p, q, k, pyr, True, s),
        "select_flat_bsa": lambda s: (pisa.select_flat_bsa(p, q, pyr, s),),
        "sparse_attn_fwd": lambda s: pisa.sparse_attn_fwd(p, q, k, v, idx, s),
        "selection_quality": lambda s: pisa.selection_quality(p, q, k, idx, rows, s),
        "rope_fwd": lambda s: pisa.rope_fwd(r, q, k, stream=s),
        "rope_bwd": lambda s: pisa.rope_bwd(r, q, k, stream=s),
        "qcache_attn_fwd": lambda s: pisa.qcache_attn_fwd(p, cache, q, idx, s),
        "qcache_attn_fwd, few rows": lambda s: pisa.qcache_attn_fwd(few, cache, q2, i2, s),
        "sparse_attn_bwd": lambda s: pisa.sparse_attn_bwd(p, q, k, v, idx, o, lse, d_o, s),
    }


NAMES = ["build_pyramid", "grow_cache", "select", "select_flat_bsa", "sparse_attn_fwd", "selection_quality", "rope_fwd",
         "rope_bwd", "qcache_attn_fwd", "qcache_attn_fwd, few rows", "sparse_attn_bwd"]


@pytest.mark.parametrize("name", NAMES)
def test_allocations_are_the_streams_own(calls, monkeypatch, name):
    """Every allocation of the call is made while its stream is the current one; nothing is launched here."""
    side, seen = torch.cuda.Stream(), []

    def watched(make):
        def call(*a, **kw):
            seen.append(torch.cuda.current_stream().cuda_stream)
            return make(*a, **kw)
        return call
    for raw in ("pisa_build_pyramid", "pisa_cache_grow", "pisa_select", "pisa_select_flat_bsa", "pisa_sparse_attn_fwd",
                "pisa_selection_quality", "pisa_rope_fwd", "pisa_rope_bwd", "pisa_qcache_attn_fwd", "pisa_sparse_attn_bwd"):
        monkeypatch.setattr(pisa, raw, lambda *a, **kw: 0)
    monkeypatch.setattr(torch, "empty", watched(torch.empty))
    monkeypatch.setattr(torch, "empty_like", watched(torch.empty_like))
    here = torch.cuda.current_stream().cuda_stream
    for given, want in ((side, side.cuda_stream), (side.cuda_stream, side.cuda_stream), (None, here),
                        (torch.cuda.current_stream(), here), (here, here)):
        seen.clear()
        calls[name](given)
        assert seen and set(seen) == {want}
    assert torch.cuda.current_stream().cuda_stream == here


@pytest.mark.parametrize("name", NAMES)
def test_a_busy_stream(calls, name):
    """The stream has work before it when the wrapper returns; the current stream allocates and writes meanwhile.

    Results are equal, but for dk and dv: those are sums of up to n = 4 * 3000 terms that atomics add in 32 bits in an order
    of their own, so two runs differ by up to 2 n 2^-24 < 2^-9 of the terms' magnitudes, and then by a step of bf16, 2^-7.
    They are compared as a whole: 2^-6 of their norm (what the test looks for is 0xFF in them, which is NaN)."""
    want = [x.clone() for x in calls[name](None)]
    sizes = {x.numel() * x.element_size() for x in want} | {pisa.pisa_qcache_attn_workspace_bytes(problem(n)) for n in (2, N)}
    sizes |= {pisa.pisa_select_workspace_bytes(problem()), pisa.pisa_attn_workspace_bytes(problem()),
              pisa.pisa_attn_bwd_workspace_bytes(problem()), pisa.pisa_bsa_workspace_bytes(problem())}
    side, a = torch.cuda.Stream(), torch.randn((4096, 4096), device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(4):
            a @ a
    got = calls[name](side)
    held = [torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") for n in sizes if n for _ in range(3)]
    torch.cuda.synchronize()
    for i, (x, y) in enumerate(zip(got, want)):
        if name == "sparse_attn_bwd" and i > 0:
            assert (x.double() - y.double()).norm() <= 2.0 ** -6 * y.double().norm()
        else:
            assert torch.equal(x, y)
    assert len(held)


@pytest.mark.parametrize("name", ["select", "sparse_attn_fwd", "rope_fwd", "qcache_attn_fwd", "qcache_attn_fwd, few rows"])
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
        for x in got:
            x.view(torch.uint8).fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x, y)
        held = [torch.full((x.numel(),), 7.0, device="cuda") for x in want]
        del held
