"""The workspace that a caller gives to drafted tokens' attention: memory of the call's device that is there as a whole, or
a refusal before anything is launched."""
import pytest
import torch

pisa = pytest.importorskip("paper_2609_31093_amd.pisa", reason="libpisa.so not built")

B, H, Hkv, T, n, d, C, K = 1, 4, 2, 12, 3000, 64, 32, 60
P = pisa.make_problem(B, H, Hkv, T, n + T, d, C, 2, K, True, "bf16", Ncap=n + T)
NEED = pisa.pisa_draft_attn_workspace_bytes(P), pisa.pisa_qcache_draft_attn_workspace_bytes(P)


def inputs(device):
    new = dict(device=device, dtype=torch.bfloat16)
    q, (k, v) = torch.zeros((B, H, T, d), **new), (torch.zeros((B, Hkv, n + T, d), **new) for _ in range(2))
    k_new, v_new = (torch.zeros((B, Hkv, T, d), **new) for _ in range(2))
    idx = torch.full((B, Hkv, T, K), -1, dtype=torch.int32, device=device)
    return q, k, v, idx, k_new, v_new, torch.zeros((B, T, 1), dtype=torch.int64, device=device)


def broken(device):
    nb = max(NEED)
    return {"expanded": torch.empty(1, dtype=torch.uint8, device=device).expand(nb),
            "strided": torch.empty(2 * nb, dtype=torch.uint8, device=device)[::2],
            "turned": torch.empty((nb // 256 + 1, 256), dtype=torch.uint8, device=device).t()}


@pytest.fixture
def taken(monkeypatch):
    """The workspaces that reach the entry point, with CPU tensors in place of the GPU's."""
    seen = []
    monkeypatch.setattr(pisa, "_device", lambda: -1)
    monkeypatch.setattr(pisa, "pisa_draft_attn_fwd", lambda *a: seen.append((a[-3], a[-2])))
    return seen


def test_what_is_passed_on(taken):
    assert min(NEED) > 0
    x = inputs("cpu")
    ws = torch.empty(NEED[0] // 4, dtype=torch.float32)  # of any type
    pisa.draft_attn_fwd(P, *x, ws=ws)
    assert taken[0][0] is ws and taken[0][1] == ws.numel() * 4


@pytest.mark.parametrize("name", ["expanded", "strided", "turned"])
def test_refused_before_a_launch(taken, name):
    with pytest.raises(ValueError, match="ws"):
        pisa.draft_attn_fwd(P, *inputs("cpu"), ws=broken("cpu")[name])
    assert not taken


def test_another_device(taken, monkeypatch):
    x = inputs("cpu")

    class Elsewhere:
        """A workspace of device 1."""
        shape, device, nbytes = (NEED[0],), torch.device("cuda", 1), NEED[0]
        get_device, is_contiguous, stride = (staticmethod(lambda: 1), staticmethod(lambda: True), staticmethod(lambda: (1,)))

    with pytest.raises(ValueError, match="ws"):
        pisa.draft_attn_fwd(P, *x, ws=Elsewhere())
    assert not taken


@pytest.mark.gpu
@pytest.mark.parametrize("eight", [False, True], ids=["raw", "8bit"])
def test_refused_on_the_gpu(eight):
    q, k, v, idx, *rest = inputs("cuda")
    held = (pisa.make_qcache(P),) if eight else None

    def call(ws):
        if eight:
            return pisa.qcache_draft_attn_fwd(P, held[0], q, idx, *rest, ws=ws)
        return pisa.draft_attn_fwd(P, q, k, v, idx, *rest, ws=ws)

    for ws in (*broken("cuda").values(), torch.empty(NEED[eight], dtype=torch.uint8), torch.empty(NEED[eight], dtype=torch.uint8).pin_memory()):
        with pytest.raises(ValueError, match="ws"):
            call(ws)
    with pytest.raises(pisa.PisaError):
        call(torch.empty(NEED[eight] - 1, dtype=torch.uint8, device="cuda"))
    o, lse = call(torch.empty(NEED[eight], dtype=torch.uint8, device="cuda"))
    assert bool((o == 0).all()) and bool((lse == float("-inf")).all())
