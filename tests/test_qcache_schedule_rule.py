"""Which form the attention over the 8-bit cache takes, seen in the workspace that it asks for; no GPU."""
import pytest

pisa = pytest.importorskip("paper_2609_31093_amd.pisa", reason="libpisa.so not built")


def workspace(B, H, Hkv, Nq, N, dtype="bf16", d=128, C=64, K=16):
    return pisa.pisa_qcache_attn_workspace_bytes(pisa.make_problem(B, H, Hkv, Nq, N, d, C, 2, K, 1, dtype))


def test_few_rows_and_many():
    """The faster of rows alone and rows grouped by block, where both were measured."""
    assert workspace(1, 16, 4, 4096, 32768) and workspace(1, 8, 8, 256, 32768)  # 373 and 203 us, 58 and 51
    assert not workspace(1, 16, 1, 16384, 32768, d=64, K=8)   # 16 heads of 64: 113 and 251
    assert not workspace(1, 32, 2, 8192, 32768, C=128)        # 16 heads: 942 and 1386
    assert not workspace(1, 16, 4, 1024, 524288)              # blocks to group: 135 and 194
    assert not workspace(1, 16, 4, 4096, 32768, dtype="f32")


def test_a_pass_takes_whole_kv_heads():
    """Rows of many KV heads go in passes of 1 GB of partials; each groups the blocks of its own KV heads, so that no block
    is grouped twice (taken by rows, every pass grouped them all: 26.5 ms instead of 7.4 in the first case)."""
    for B, Nq, N in ((32, 2048, 131072), (64, 512, 131072), (64, 512, 32768)):
        BH, G, K, d, M = B * 8, 4, 16, 128, N // 64
        most = 2 ** 30 // (K * G * (2 * d + 4)) // Nq         # KV heads of a pass
        passes = -(-BH // most)
        heads = -(-BH // passes)
        pairs = heads * Nq * K
        grouping = workspace(B, 32, 8, Nq, N) - pairs * G * (2 * d + 8) - 4 * pairs
        # three lists of the blocks, and one for every 256 rows
        want = 4 * heads * M * (3 + -(-Nq // 256))
        assert want <= grouping <= want + 4096
