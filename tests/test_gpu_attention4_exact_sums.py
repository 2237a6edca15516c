"""Scores of prefix_attention4 whose sums 24 bits hold: exact with 16 + code and the 24 taken off, and finite where q * 24 is
(MI355X).

q is 1 but for some columns L of a group, 2^18 (bf16: one of them, float16: 2^15 for eight). All sums are whole numbers,
and their parts are at most 24 and 31 times 2^18 and 127: below 2^24, exact in float32 in any order. With 128 (float16: 64) +
code they pass 2^24, and odd numbers are lost."""
import math

import pytest
import torch

import paper_2502_00922_amd as hl
from rows4 import random_rows, values

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16]


def steep(dtype, count, cols, g):
    """[count, cols] of ones, each row with its large columns in another place of one group of 32."""
    x = torch.ones((count, cols))
    for i in range(count):
        first = 32 * int(torch.randint(0, cols // 32, (1,), generator=g))
        if dtype == torch.bfloat16:
            x[i, first + 3 * i % 32] = 2.0**18
        else:
            x[i, first + (torch.arange(8) * 4 + i % 4)] = 2.0**15
    return x.to(dtype).cuda()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [32, 64, 96, 128, 160, 256])
def test_scores(dtype, dim):
    # one key: the softmax sum's logarithm is its score, a whole number times 2^-10
    g = torch.Generator(device="cuda").manual_seed(dim)
    rows = random_rows((1, 4), dim, g)
    pairs = torch.zeros((1, 4, dim // 32, 2), dtype=torch.bfloat16, device="cuda")
    pairs[..., 0] = 1
    rows[..., dim // 2:dim // 2 + dim // 8] = pairs.flatten(-2).view(torch.uint8)
    q = steep(dtype, 128, dim, torch.Generator().manual_seed(dim)).view(32, 1, 4, dim)
    lse = torch.empty((32, 1, 4), device="cuda")
    hl.prefix_attention4(q, prefix_k=rows, prefix_v=rows, scale=2.0**-10, lse=lse)
    want = (q.double().cpu()[:, 0] * values(rows, dim)[0]).sum(-1) * 2.0**-10
    # the score times log2(e) and back: that constant's rounding and those of the two products and the division
    err = (lse[:, 0].double().cpu() - want).abs()
    assert (err <= 5 * 2.0**-24 * want.abs() + 1e-7).all(), float((err / want.abs().clamp(min=1)).max())


def test_scores_of_large_q():
    # 2^121 in one column of q, keys' scales of 2^-115
    dim = 64
    g = torch.Generator(device="cuda").manual_seed(2)
    rows = random_rows((1, 2), dim, g)
    pairs = torch.zeros((1, 2, 2, 2), dtype=torch.bfloat16, device="cuda")
    pairs[..., 0] = 2.0**-115
    rows[..., 32:40] = pairs.flatten(-2).view(torch.uint8)
    q = torch.zeros((dim, 1, 2, dim), dtype=torch.bfloat16, device="cuda")
    q[torch.arange(dim), 0, :, torch.arange(dim)] = 2.0**121
    lse = torch.empty((dim, 1, 2), device="cuda")
    hl.prefix_attention4(q, prefix_k=rows, prefix_v=rows, scale=1.0, lse=lse)
    want = (q.double().cpu()[:, 0] * values(rows, dim)[0]).sum(-1)
    err = (lse[:, 0].double().cpu() - want).abs()
    assert (err <= 5 * 2.0**-24 * want.abs() + 1e-7).all() and math.isfinite(float(lse.abs().max()))
