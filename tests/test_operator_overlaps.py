"""Refusals of overlapping tensors by the rotation and the 8-bit cache, without a GPU: nothing here is launched."""
import ctypes

import pytest

pisa = pytest.importorskip("paper_2609_31093_amd.pisa", reason="libpisa.so not built")

LIB, S, INVALID = pisa.library(), pisa.Strides, pisa.PISA_ERR_INVALID_ARG
Q, K, QO, KO = ((i + 1) << 30 for i in range(4))  # where tensors are said to be; never dereferenced
B, H, HKV, N, D = 2, 4, 3, 100, 128


def rotate(name, q=Q, qs=None, k=K, ks=None, qo=QO, qos=None, ko=KO, kos=None, **kw):
    r = pisa.make_rope(**{**dict(B=B, H=H, Hkv=HKV, N=N, d=D), **kw})
    st = [None if x is None else ctypes.addressof(x) for x in (qs, ks, qos, kos)]
    return getattr(LIB, name)(ctypes.byref(r), q, st[0], k, st[1], None, qo, st[2], ko, st[3], None)


@pytest.mark.parametrize("name", ["pisa_rope_fwd", "pisa_rope_bwd"])
@pytest.mark.parametrize("b,h,n", [
    (H * N * D, D, D),                  # head 1's first row is head 0's second
    (D, H * D, H * D),
    (H * D, H * D, B * H * D),          # the batches' rows are the heads'
    (N * D, N * D, D),
    (H * N * D, N * D - 8, D),          # a head's last row ends in the next head
    (H * N * D, D, H * D - 8),          # rows that run into each other
    (H * N * D - 8, N * D, D),          # batches that do
    (98 * D, 2 * N * D, 2 * D),         # a batch between the rows of another, and on one of them
])
def test_written_rows_that_overlap(name, b, h, n):
    assert rotate(name, qos=S(b, h, n)) == INVALID
    assert "q (output)" in pisa.pisa_last_error() and "overlap" in pisa.pisa_last_error()
    if h >= D:  # the same for keys of as many heads
        assert rotate(name, kos=S(b, h, n), Hkv=H) == INVALID
        assert "k (output)" in pisa.pisa_last_error() and "overlap" in pisa.pisa_last_error()
