"""prefix_attention of caches whose tokens lie so far apart that offsets pass 32 bits, through the kernels of parts (MI355X):
items of up to 16 rows, and of more (whose loads go to LDS by 32-bit offsets from a step's first key). The results are those
of the same keys and values without gaps."""
import pytest
import torch

import paper_2502_00922_amd as hl
from test_gpu_prefix_attention import make

pytestmark = pytest.mark.gpu


# the greatest stride of a token that is taken, with which a step's 32 keys span 2 GiB; more keys, nearer
@pytest.mark.parametrize("queries,tokens,stride", [(20, 70, (1 << 25) - 8), (20, 1000, 1 << 23), (3, 1000, 1 << 23)])
@pytest.mark.parametrize("dim", [64, 128])
def test_far_tokens(queries, tokens, stride, dim):
    big = torch.empty(tokens * stride + dim, dtype=torch.bfloat16, device="cuda")
    far = big.as_strided((1, tokens, 1, dim), (0, stride, dim, 1))
    c = make(torch.bfloat16, 1, queries, 4, 1, dim, 0, tokens)
    k, v = c["k"], c["v"]
    for name, own in (("k", True), ("v", True), ("k", False), ("v", False)):
        far.copy_(c[name])
        got = {"k": k, "v": v, name: far}
        if own:
            a, b = (hl.prefix_attention(c["q"], x["k"], x["v"], c["lens"]).out for x in (c, got))
        else:
            a, b = (hl.prefix_attention(c["q"], prefix_k=x["k"][0], prefix_v=x["v"][0]).out for x in (c, got))
        assert torch.equal(a, b)
