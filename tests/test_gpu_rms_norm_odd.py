"""rms_norm of rows whose ends and starts fall between its loads (MI355X), against the definition in 64 bits with the
bounds of test_gpu_rms_norm."""
import pytest
import torch

import paper_2502_00922_amd as hl
import test_gpu_rms_norm as even

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("types", [(torch.float16, torch.float16), (torch.bfloat16, torch.float32),
                                   (torch.float32, None)])
@pytest.mark.parametrize("tokens,hidden", [(5, 3), (4, 9), (3, 513), (1100, 1023), (2, 4099), (3, 8191), (2, 12345),
                                           (3, 16383), (2, 32765)])
@pytest.mark.parametrize("ot", [torch.float32, torch.float16, torch.float8_e4m3fn])
def test_odd_rows(tokens, hidden, types, ot):
    x, r, w = even.make(tokens, hidden, *types, seed=hidden)
    even.check(x, w, r, hl.rms_norm(x, w, residual=r, out_dtype=ot))


@pytest.mark.parametrize("hidden", [65, 4103, 9001])
def test_in_place(hidden):
    x, r, w = even.make(7, hidden, torch.bfloat16, torch.bfloat16, seed=1)
    want = hl.rms_norm(x, w, residual=r, out_dtype=torch.bfloat16)
    got = hl.rms_norm(x, w, residual=r, out=x, sum_out=r)
    assert torch.equal(got.out, want.out) and torch.equal(got.sum, want.sum)
    assert got.out.data_ptr() == x.data_ptr() and got.sum.data_ptr() == r.data_ptr()


@pytest.mark.parametrize("offset", [1, 3])
@pytest.mark.parametrize("hidden", [64, 777, 5000])
def test_nothing_is_written_past_the_rows(hidden, offset):
    x, r, w = even.make(3, hidden, torch.float16, torch.float16, seed=2)
    want = hl.rms_norm(x, w, residual=r, out_dtype=torch.float16)
    n, places = 3 * hidden, []
    for _ in range(2):
        whole = torch.full((n + 2 * offset,), 7.0, dtype=torch.float16, device="cuda")
        places.append((whole, whole[offset:offset + n].view(3, hidden)))
    got = hl.rms_norm(x, w, residual=r, out=places[0][1], sum_out=places[1][1])
    assert torch.equal(got.out, want.out) and torch.equal(got.sum, want.sum)
    for whole, _ in places:
        assert (whole[:offset] == 7).all() and (whole[offset + n:] == 7).all()
