"""A norm's weights are those that its parameters hold at the call: a module that is cast, or whose parameters get other
memory, is followed, and one that no longer fits is refused.  On the CPU by what reaches the C entry points, on the GPU by
the results."""
import pytest
import torch

pisa = pytest.importorskip("paper_2609_31093_amd.pisa", reason="libpisa.so not built")


class Layer(torch.nn.Module):
    def __init__(self, d, device="cpu"):
        super().__init__()
        gen = torch.Generator().manual_seed(1)
        self.q = torch.nn.Parameter((1.0 + 0.5 * torch.randn(d, generator=gen)).to(device))
        self.k = torch.nn.Parameter((1.0 + 0.5 * torch.randn(d, generator=gen)).to(device))


@pytest.fixture
def calls(monkeypatch):
    """What the entry points would be given, with CPU tensors in place of the GPU's."""
    seen = []
    monkeypatch.setattr(pisa, "_device", lambda: -1)
    monkeypatch.setattr(pisa, "_stream", lambda stream: 0)
    for name in ("pisa_norm_rope_fwd", "pisa_norm_rope_bwd"):
        monkeypatch.setattr(pisa, name, lambda r, m, *a: seen.append((m.q_weight, m.k_weight, m.weight_dtype, m.eps, m.offset)))
    return seen


def run(r, m, x):
    pisa.norm_rope_fwd(r, m, x, x)
    pisa.norm_rope_bwd(r, m, x, x, x, x)


def test_the_weights_of_the_call(calls):
    r = pisa.make_rope(1, 2, 2, 8, 64, dtype="f32")
    x, layer = torch.zeros((1, 2, 8, 64)), Layer(64)
    m = pisa.make_qk_norm(r, layer.q, layer.k, eps=1e-5, offset=0.25)

    def expect(dtype):
        run(r, m, x)
        assert calls == [(layer.q.data_ptr(), layer.k.data_ptr(), dtype, 1e-5, 0.25)] * 2
        calls.clear()

    expect(pisa.PISA_DTYPE_F32)
    was = layer.q.data, layer.k.data
    layer.to(torch.bfloat16)          # other memory, another type
    assert layer.q.data_ptr() != was[0].data_ptr()
    expect(pisa.PISA_DTYPE_BF16)
    layer.float()
    layer.k.data = torch.ones(64)     # other memory for one of them
    expect(pisa.PISA_DTYPE_F32)
    with torch.no_grad():
        layer.q.mul_(2.0)             # in place
    expect(pisa.PISA_DTYPE_F32)


def test_weights_that_no_longer_fit(calls):
    r = pisa.make_rope(1, 2, 2, 8, 64, dtype="f32")
    x = torch.zeros((1, 2, 8, 64))
    for change in (lambda l: l.half(), lambda l: setattr(l.q, "data", torch.ones(32)), lambda l: setattr(l.k, "data", torch.ones(128)[::2]),
                   lambda l: setattr(l.k, "data", l.k.data.bfloat16())):
        layer = Layer(64)
        m = pisa.make_qk_norm(r, layer.q, layer.k)
        change(layer)
        for call in (lambda: pisa.norm_rope_fwd(r, m, x, x), lambda: pisa.norm_rope_bwd(r, m, x, x, x, x)):
            with pytest.raises(ValueError):
                call()
    other = pisa.make_rope(1, 2, 2, 8, 128, dtype="f32")
    layer = Layer(64)
    m = pisa.make_qk_norm(r, layer.q, layer.k)
    with pytest.raises(ValueError):
        pisa.norm_rope_fwd(other, m, torch.zeros((1, 2, 8, 128)))
    assert not calls


def test_without_weights(calls):
    r = pisa.make_rope(1, 2, 2, 8, 64, dtype="f32")
    x = torch.zeros((1, 2, 8, 64))
    run(r, pisa.make_qk_norm(r), x)
    layer = Layer(64)
    m = pisa.make_qk_norm(r, None, layer.k)
    layer.bfloat16()
    run(r, m, x)
    assert [c[:3] for c in calls] == [(None, None, pisa.PISA_DTYPE_F32)] * 2 + [(None, layer.k.data_ptr(), pisa.PISA_DTYPE_BF16)] * 2


@pytest.mark.gpu
def test_results_follow_the_parameters():
    r = pisa.make_rope(1, 4, 2, 40, 128)
    layer = Layer(128, "cuda")
    m = pisa.make_qk_norm(r, layer.q, layer.k)
    gen = torch.Generator(device="cuda").manual_seed(2)
    q, k, gq, gk = (torch.randn((1, h, 40, 128), generator=gen, device="cuda").bfloat16() for h in (4, 2, 4, 2))
    for change in (lambda: None, lambda: layer.bfloat16(), lambda: layer.float(), lambda: setattr(layer.q, "data", layer.q.data * 3)):
        change()
        fresh = pisa.make_qk_norm(r, layer.q.detach().clone(), layer.k.detach().clone())
        # what was freed is taken again and overwritten
        junk = [torch.full((128,), float("nan"), device="cuda") for _ in range(64)]
        for a, b in zip(pisa.norm_rope_fwd(r, m, q, k), pisa.norm_rope_fwd(r, fresh, q, k)):
            assert torch.equal(a, b)
        for a, b in zip(pisa.norm_rope_bwd(r, m, q, k, gq, gk), pisa.norm_rope_bwd(r, fresh, q, k, gq, gk)):
            assert torch.equal(a, b)
        del junk
    layer.cpu()
    with pytest.raises(ValueError):
        pisa.norm_rope_fwd(r, m, q, k)
