"""rms_norm's scales of whole rows (MI355X): [..., 1], so that they multiply the 8-bit rows as they are."""
import pytest
import torch

import paper_2502_00922_amd as hl

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn


# equal counts of rows and columns, where scales without a last dimension would multiply columns, among them
@pytest.mark.parametrize("shape", [(5, 640), (1, 33), (64, 64), (2, 3, 520)])
def test_scales_multiply_rows(shape):
    g = torch.Generator(device="cuda").manual_seed(shape[-1])
    x = torch.randn(shape, generator=g, device="cuda") * torch.arange(1, shape[-2] + 1, device="cuda")[:, None]
    w = torch.linspace(0.5, 1.5, shape[-1], device="cuda")
    r = hl.rms_norm(x, w, out_dtype=E4M3)
    assert r.scale.shape == (*shape[:-1], 1) and r.scale.dtype == torch.float32
    t = x.double()
    want = t / torch.sqrt((t * t).mean(-1, keepdim=True) + 1e-5) * w.double()
    # the rounding to 8 bits: half a step of 2^-3, or of the subnormals' 2^-9
    bound = torch.maximum(want.abs() * 2.0**-4, r.scale.double() * 2.0**-10) * (1 + 2.0**-8)
    assert ((r.out.double() * r.scale.double() - want).abs() <= bound).all()


def test_given_buffer():
    x, w = torch.randn(6, 96, device="cuda"), torch.ones(96, device="cuda")
    want = hl.rms_norm(x, w, out_dtype=E4M3)
    for shape in ((6, 1), (6,)):  # with and without the last dimension
        given = torch.zeros(shape, device="cuda")
        r = hl.rms_norm(x, w, out_dtype=E4M3, scale_out=given)
        assert r.scale.shape == (6, 1) and r.scale.data_ptr() == given.data_ptr()
        assert torch.equal(r.scale, want.scale)
    for shape in ((6, 2), (1, 6), (6, 96)):
        with pytest.raises(ValueError):
            hl.rms_norm(x, w, out_dtype=E4M3, scale_out=torch.zeros(shape, device="cuda"))
    with pytest.raises(ValueError):  # groups of 32: three scales a row
        hl.rms_norm(x, w, out_dtype=E4M3, group=32, scale_out=torch.zeros(6, device="cuda"))
