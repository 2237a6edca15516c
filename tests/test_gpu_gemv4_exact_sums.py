"""gemv4 where 24 bits hold the sums: exact with 16 + code and the 24 taken off, and finite where x * 24 is (MI355X).

x is 1 but for some columns L of a group, 2^18 (bf16: one of them, float16: 2^15 for eight). All sums are whole numbers,
and their parts are at most 24 and 31 times 2^18 and 127: below 2^24, exact in float32 in any order. With 128 (float16: 64) +
code they pass 2^24, and odd numbers are lost."""
import pytest
import torch

import paper_2502_00922_amd as hl
from test_gpu_attention4_exact_sums import TYPES, steep

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows", [48, 8208])
def test_products(dtype, group, rows):
    g = torch.Generator().manual_seed(group)
    for first in range(0, 32, 16):
        x = steep(dtype, 32, 256, g)[first:first + 16].contiguous()
        codes = torch.randint(0, 256, (rows, 128), generator=g, dtype=torch.uint8)
        steps = torch.stack([codes & 15, codes >> 4], -1).flatten(1).double() - 8
        y = hl.gemv4(codes.cuda(), torch.ones((rows, 256 // group), dtype=dtype, device="cuda"), x)
        assert torch.equal(y.double().cpu(), x.double().cpu() @ steps.T)


def test_products_of_large_x():
    # one column at a time of 2^121: 31 times it is below 2^126
    cols = 64
    g = torch.Generator().manual_seed(1)
    codes = torch.randint(0, 256, (40, cols // 2), generator=g, dtype=torch.uint8)
    steps = torch.stack([codes & 15, codes >> 4], -1).flatten(1).double() - 8
    scales = torch.full((40, 1), 2.0**-100, dtype=torch.bfloat16)
    for first in range(0, cols, 16):
        x = torch.zeros((16, cols), dtype=torch.bfloat16)
        x[torch.arange(16), first + torch.arange(16)] = 2.0**121
        y = hl.gemv4(codes.cuda(), scales.cuda(), x.cuda())
        assert torch.equal(y.double().cpu(), x.double() @ (steps * 2.0**-100).T)
