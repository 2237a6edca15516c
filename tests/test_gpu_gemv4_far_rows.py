"""gemv4 on codes past 4 GB and on a vocabulary's height, against the product in 64 bits of some rows (MI355X)."""
import pytest
import torch

import paper_2502_00922_amd as hl
from test_gpu_gemv4 import make, reference

pytestmark = pytest.mark.gpu


def check_rows(c, y, rows):
    part = {**c, **{n: c[n][rows] for n in ("codes", "scales", "bases") if c[n] is not None}}
    want, size = reference(part)
    bound = (142 + c["scales"].shape[1]) * 2.0**-24 * size
    assert ((y[:, rows].double().cpu() - want).abs() <= bound).all()


@pytest.mark.parametrize("batch", [1, 16])
def test_vocabulary(batch):
    c = make(128256, 4096, batch, 64, bases=False)
    y = hl.gemv4(**c)
    for first in (0, 64000, 128256 - 70):
        check_rows(c, y, slice(first, first + 70))


def test_codes_past_4_gb():
    rows, cols = (1 << 20) + 5, 16384
    c = make(rows, cols, 2, 128, dtype=torch.float16)
    y = hl.gemv4(**c)
    for first in (0, (1 << 19) - 20, rows - 40):
        check_rows(c, y, slice(first, first + 40))
