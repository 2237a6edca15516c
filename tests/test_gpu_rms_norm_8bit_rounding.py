"""The 8-bit norm's rounding (MI355X): each element is the float32 quotient out / scale rounded to nearest, bit for bit. Rows
of ones with eps 0 make out the weight itself, which here puts quotients next to the middle of two e4m3 neighbours."""
import numpy as np
import pytest
import torch

import paper_2502_00922_amd as hl

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn


def weights(size, columns, seed):
    """Groups of `size` columns whose largest is first and whose others are within a float32 step of a middle."""
    rng = np.random.default_rng(seed)
    top = (448 * (1 + rng.random(columns // size))).astype(np.float32)
    scale = (top / np.float32(448)).astype(np.float32)[:, None]
    middles = (rng.integers(8, 16, (columns // size, size)) + 0.5) * 2.0 ** rng.integers(-9, 5, (columns // size, size))
    w = (middles.astype(np.float32) * scale).astype(np.float32)
    w = np.where(rng.random(w.shape) < 0.3, np.nextafter(w, np.float32(1e30)), w)
    w = np.where(rng.random(w.shape) < 0.3, np.nextafter(w, np.float32(-1e30)), w).astype(np.float32)
    w *= rng.choice(np.float32([-1, 1]), w.shape)
    w[:, 0] = top
    return w.reshape(-1), scale.reshape(-1)


@pytest.mark.parametrize("hidden,group", [(8192, 32), (8192, 64), (32768, 128), (8192, 0), (771, 0), (512, 0), (20000, 0)])
@pytest.mark.parametrize("seed", range(4))
def test_quotients_next_to_the_middle(hidden, group, seed):
    w, scale = weights(group or hidden, hidden, seed)
    r = hl.rms_norm(torch.ones((3, hidden), device="cuda"), torch.from_numpy(w).cuda(), eps=0.0, out_dtype=E4M3, group=group)
    assert np.array_equal(r.scale.cpu().numpy(), np.tile(scale, (3, 1)))
    each = np.repeat(scale, group or hidden)
    want = torch.from_numpy((w / each).astype(np.float32)).to(E4M3).view(torch.uint8)
    if group:  # of many scales, some have a rounded reciprocal with which a product comes out differently
        other = torch.from_numpy(w * (np.float32(1) / each)).to(E4M3).view(torch.uint8)
        assert not torch.equal(other, want)
    assert torch.equal(r.out.view(torch.uint8).cpu(), want.expand(3, -1))


def test_scales_at_the_ends_of_the_range():
    # out / scale where 1 / scale is not a normal number, or nearly
    w = torch.zeros(64)
    w[:32] = torch.linspace(-1, 1, 32) * 3e38
    w[32:] = torch.linspace(-1, 1, 32) * 1e-35
    r = hl.rms_norm(torch.ones((1, 64), device="cuda"), w.cuda(), eps=0.0, out_dtype=E4M3, group=32)
    each = r.scale.cpu()[0].repeat_interleave(32)
    assert torch.equal(r.out.cpu()[0].view(torch.uint8), (w / each).to(E4M3).view(torch.uint8))
