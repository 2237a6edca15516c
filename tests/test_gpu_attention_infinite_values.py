"""prefix_attention of values that are infinite or NaN and that the tokens see with a weight that float32 holds as 0 (MI355X):
the column is infinite or NaN, whichever kernels, parts and waves the keys fall to, and no other column changes."""
import pytest
import torch

import paper_2502_00922_amd as hl

pytestmark = pytest.mark.gpu
LOW = 300  # keys whose scores are 461 powers of two below the others': whole parts of up to two units of 128

# batch, queries, heads, key heads, prefix, own: a block a sequence and head; parts of items of up to 16 rows, and of more;
# the same over own caches, whose tokens see keys in order
SHAPES = {"one block": (2, 1, 4, 1, 700, 0), "narrow": (1, 1, 4, 1, 3000, 0), "wide": (20, 1, 4, 2, 3000, 0),
          "one block, own": (2, 3, 4, 1, 0, 700), "narrow, own": (2, 3, 4, 1, 0, 3000), "wide, own": (2, 30, 4, 2, 0, 3000),
          "long": (1, 1, 4, 1, 20000, 0), "both": (3, 1, 4, 2, 3000, 200)}


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("key", [5, 290])
@pytest.mark.parametrize("shape", list(SHAPES))
def test_seen_with_no_weight(shape, key, bad, dtype):
    batch, queries, heads, kv_heads, prefix, own = SHAPES[shape]
    g = torch.Generator(device="cuda").manual_seed(key)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    c = {"q": torch.ones((batch, queries, heads, 64), dtype=dtype, device="cuda")}
    sets = []
    if prefix:
        c["prefix_k"], c["prefix_v"] = (0.1 * rand(prefix, kv_heads, 64)).to(dtype), rand(prefix, kv_heads, 64).to(dtype)
        sets.append((c["prefix_k"], c["prefix_v"]))
    if own:
        c["k"], c["v"] = ((s * rand(batch, own, kv_heads, 64)).to(dtype) for s in (0.1, 1))
        c["lens"] = torch.full((batch,), own, dtype=torch.int32, device="cuda")
        sets.append((c["k"][0], c["v"][0]))
    keys, values = sets[0]
    keys[:LOW] = -40
    want = hl.prefix_attention(**c).out.clone()
    values[key, 0, 3] = bad
    got = hl.prefix_attention(**c).out
    hit = torch.zeros_like(got, dtype=torch.bool)
    hit[slice(None) if prefix else 0, :, :heads // kv_heads, 3] = True  # key head 0's heads (of sequence 0's own cache)
    assert want.isfinite().all() and not got[hit].isfinite().any()
    assert torch.equal(got[~hit], want[~hit])
