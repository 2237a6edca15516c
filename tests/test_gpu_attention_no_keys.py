"""prefix_attention of caches without room and prefixes without keys (MI355X): out = 0 and lse = minus infinity where no key
is left, and an empty set beside another changes nothing. One block a sequence and head (4 rows a key head) and parts (40)."""
import pytest
import torch

import paper_2502_00922_amd as hl

pytestmark = pytest.mark.gpu
SHAPES = [(2, 1, 8, 2), (2, 10, 8, 2)]  # batch, queries, heads, key heads


def rand(*shape):
    return torch.randn(shape, device="cuda").to(torch.bfloat16)


def none(batch, kv_heads):
    """An own cache without room and a prefix without keys."""
    own, prefix = rand(batch, 0, kv_heads, 64), rand(0, kv_heads, 64)
    return dict(k=own, v=own, lens=torch.zeros(batch, dtype=torch.int32, device="cuda")), dict(prefix_k=prefix,
                                                                                            prefix_v=prefix)


@pytest.mark.parametrize("batch,queries,heads,kv_heads", SHAPES)
@pytest.mark.parametrize("sets", ["prefix", "own", "both"])
def test_no_keys_at_all(batch, queries, heads, kv_heads, sets):
    q = rand(batch, queries, heads, 64)
    own, prefix = none(batch, kv_heads)
    given = {**(own if sets != "prefix" else {}), **(prefix if sets != "own" else {})}
    lse = torch.zeros((batch, queries, heads), device="cuda")
    out = hl.prefix_attention(q, **given, lse=lse, out=rand(*q.shape)).out
    assert (out == 0).all() and (lse == -float("inf")).all()


@pytest.mark.parametrize("batch,queries,heads,kv_heads", SHAPES)
def test_empty_set_beside_another(batch, queries, heads, kv_heads):
    q, keys = rand(batch, queries, heads, 64), rand(batch, 90, kv_heads, 64)
    own, prefix = none(batch, kv_heads)
    lens = torch.full((batch,), 90, dtype=torch.int32, device="cuda")
    want = hl.prefix_attention(q, keys, keys, lens).out
    assert torch.equal(hl.prefix_attention(q, keys, keys, lens, **prefix).out, want)
    want = hl.prefix_attention(q, prefix_k=keys[0], prefix_v=keys[0]).out
    assert torch.equal(hl.prefix_attention(q, **own, prefix_k=keys[0], prefix_v=keys[0]).out, want)


@pytest.mark.parametrize("batch,queries,heads,kv_heads", SHAPES)
def test_weights_of_no_keys(batch, queries, heads, kv_heads):
    q, keys = rand(batch, queries, heads, 64), rand(90, kv_heads, 64)
    own, _ = none(batch, kv_heads)
    w = torch.zeros((batch, kv_heads, 0), device="cuda")
    r = hl.prefix_attention(q, **own, prefix_k=keys, prefix_v=keys, weights=w)
    assert r.weights.shape == w.shape
    assert torch.equal(r.out, hl.prefix_attention(q, prefix_k=keys, prefix_v=keys).out)
