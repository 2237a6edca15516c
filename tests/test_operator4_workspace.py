"""The workspaces of the 4-bit operators (no GPU, which plans for 256 compute units)."""
import ctypes

import pytest

hl = pytest.importorskip("paper_2502_00922_amd.hufflm")
A = 0x10000


def attention4(batch, queries, heads, kv_heads, dim, prefix, own, dtype=hl.HL_BF16, weights=False):
    row = hl.cache4_row_bytes(dim) // 2

    def kv(n):
        return hl.KeysValues(A, A, n, n * kv_heads * row, kv_heads * row, row, n * kv_heads * row, kv_heads * row, row)
    a = hl.AttentionShape(dtype, batch, queries, heads, kv_heads, dim, 0.1, kv(prefix), kv(own))
    return hl.lib().hl_attention4_workspace_bytes(ctypes.byref(a), int(weights))


@pytest.mark.parametrize("dtype", [hl.HL_BF16, hl.HL_F16])
@pytest.mark.parametrize("queries", [64, 256])
def test_attention_of_many_rows_holds_no_second_cache(dtype, queries):
    # blocks' parts alone: past two units a block, longer caches and prefixes add nothing
    need = attention4(16, queries, 32, 8, 128, 4096, 16384, dtype)
    assert need == attention4(16, queries, 32, 8, 128, 32768, 65536, dtype)
    # a part of 64 rows for each block and each item of 64 rows
    tiles = queries * 4 // 64
    parts = 512 + 8 * 16 * tiles + 16 * 8 * tiles
    assert need <= parts * 64 * (128 + 2) * 4 + 4096


@pytest.mark.parametrize("rows,vocab,most", [
    (1, 1, 32 << 10), (1, 32000, 256 << 10), (40000, 5, 110 << 20), (65535, 131072, 64 << 20), (4096, 32000, 110 << 20),
    (256, 131072, 32 << 20), (61, 50001, 11 << 20), (1, (1 << 20) - 1, 1 << 20), (65535, (1 << 20) - 1, 64 << 20),
    (2048, 2048, 90 << 20), (65535, 16384, 170 << 20)])
def test_sampling(rows, vocab, most):
    # rows past what fills the GPU reuse their predecessors' room, and a row has one list
    assert 0 < hl.lib().hl_sample_workspace_bytes(rows, vocab) <= most
