"""rms_norm where the norm's factor and the weight leave float32's range together but not with the row (MI355X): a row is
normalised before the weight scales it."""
import pytest
import torch

import paper_2502_00922_amd as hl

pytestmark = pytest.mark.gpu


def test_scale_of_an_overflow():
    x = torch.ones((1, 64), device="cuda")
    x[0, 1:] = 0.5
    r = hl.rms_norm(x, torch.full((64,), 3e38, device="cuda"), eps=0.0, out_dtype=torch.float8_e4m3fn)  # the first overflows
    assert r.scale.isinf().all() and r.out[0, 0].float().isnan() and (r.out[0, 1:].float() == 0).all()


# whole loads and a row's last columns; weights times 1 / rms past the largest number, or among the subnormal ones
@pytest.mark.parametrize("hidden", [64, 77, 4099])
@pytest.mark.parametrize("size,weight", [(1e-15, 1e25), (1e15, 1e-28), (1.0, 1.0)])
def test_factors_far_apart(hidden, size, weight):
    g = torch.Generator(device="cuda").manual_seed(hidden)
    x = size * torch.randn((3, hidden), generator=g, device="cuda")
    w = weight * (1 + 0.2 * torch.randn(hidden, generator=g, device="cuda"))
    y = hl.rms_norm(x, w, eps=0.0, out_dtype=torch.float32).out.double()
    t = x.double()
    want = t / torch.sqrt((t * t).mean(-1, keepdim=True)) * w.double()
    # float32 arithmetic: 40 roundings at most (chains of 32 squares and a tree, halved by the root, and five more)
    assert ((y - want).abs() <= 40 * 2.0**-24 * want.abs()).all()
