"""prefix_attention in a workspace of exactly the size that it asks for (MI355X): the results are those of a larger one, and
nothing is written past its end."""
import ctypes

import pytest
import torch

import paper_2502_00922_amd as hl
from paper_2502_00922_amd import hufflm
from test_gpu_prefix_attention import make

pytestmark = pytest.mark.gpu
GUARD = 1 << 16


def needed(c, weights):
    """hl_attention_workspace_bytes of these arguments."""
    def kv(k):
        if k is None:
            return hufflm.KeysValues(*[0] * 9)
        n, row = k.shape[-3], k.shape[-2] * k.shape[-1]
        return hufflm.KeysValues(1 << 16, 1 << 16, n, n * row, row, k.shape[-1], n * row, row, k.shape[-1])
    batch, queries, heads, dim = c["q"].shape
    own, prefix = c.get("k"), c.get("prefix_k")
    a = hufflm.AttentionShape(hufflm.HL_BF16, batch, queries, heads, (prefix if own is None else own).shape[-2], dim, 0.1,
                              kv(prefix), kv(own))
    return hufflm.lib().hl_attention_workspace_bytes(ctypes.byref(a), int(weights))


# batch, queries, heads, key heads, dim, prefix, own: wide prefix and narrow caches, one set alone, both wide, both narrow,
# one block a sequence and head
@pytest.mark.parametrize("shape", [(16, 1, 32, 8, 128, 2100, 300), (70, 1, 16, 4, 64, 1200, 900), (40, 1, 32, 8, 128, 0, 1500),
                                   (33, 1, 32, 8, 128, 1500, 0), (2, 64, 8, 8, 128, 0, 1300), (3, 40, 8, 2, 80, 300, 500),
                                   (2, 3, 8, 8, 256, 2000, 700), (9, 1, 8, 2, 128, 100, 120)])
@pytest.mark.parametrize("weights", [False, True])
def test_exact_workspace(shape, weights):
    c = make(torch.bfloat16, *shape)
    if weights:
        if "k" not in c:
            pytest.skip("weights are of own keys")
        c["weights"] = torch.zeros((shape[0], shape[3], shape[6]), device="cuda")
    n = needed(c, weights)
    memory = torch.full((n + GUARD,), 0xA5, dtype=torch.uint8, device="cuda")
    want = hl.prefix_attention(**c, workspace=torch.zeros(2 * n, dtype=torch.uint8, device="cuda"))
    got = hl.prefix_attention(**c, workspace=memory[:n])
    assert torch.equal(got.out, want.out) and (memory[n:] == 0xA5).all()
    assert not weights or torch.equal(got.weights, want.weights)
    with pytest.raises(hl.HLError):
        hl.prefix_attention(**c, workspace=memory[:n - 1])
