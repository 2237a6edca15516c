"""C ABI of the operators: sizes whose launch would have 2^32 threads or more are refused before anything is launched (no
GPU: device addresses here are made up and never read)."""
import ctypes

import pytest

hl = pytest.importorskip("paper_2502_00922_amd.hufflm")
A = 0x10000


# hidden: 8 waves a row, 16 waves a row (above 16384 columns), four rows a block of 256 threads (512 columns)
@pytest.mark.parametrize("hidden,tokens", [(4096, 1 << 23), (4096, 1 << 30), (32768, 1 << 22), (512, 1 << 26),
                                           (8, (1 << 31) - 1)])
def test_norm(hidden, tokens):
    s = hl.lib().hl_rms_norm(A, hl.HL_BF16, None, 0, A, hl.HL_BF16, tokens, hidden, 1e-5, None, A, hl.HL_BF16, 0, None,
                             None)
    assert s == hl.HL_EUNSUPPORTED


# rows that the joining kernel takes in a block: 1024 / columns (columns as 64, 128 or 256)
@pytest.mark.parametrize("dim,rows", [(64, 16), (128, 8), (80, 8), (256, 4)])
def test_attention(dim, rows):
    row = 8 * dim
    own = hl.KeysValues(A, A, 600, 600 * row, row, dim, 600 * row, row, dim)
    none = hl.KeysValues(*[0] * 9)
    for queries, fits in ((32 * rows, False), (32 * rows - 1, True)):
        # batch * queries * heads rows: 2^24 blocks of 256 threads, or somewhat fewer
        a = hl.AttentionShape(hl.HL_BF16, 1 << 15, queries, 16, 8, dim, 0.1, none, own)
        assert (hl.lib().hl_attention_workspace_bytes(ctypes.byref(a), 0) > 0) == fits
        if not fits:
            s = hl.lib().hl_prefix_attention(ctypes.byref(a), A, A, A, None, None, None, A, 1 << 60, None)
            assert s == hl.HL_EUNSUPPORTED


def test_evict():
    n = 1 << 29
    kv = ctypes.byref(hl.KeysValues(A, A, n, 0, 64, 64, 0, 64, 64))
    assert hl.lib().hl_cache_evict(kv, kv, 1, 7, 64, A, A, n, 0, A, A, A, None) == hl.HL_EUNSUPPORTED
