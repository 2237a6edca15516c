"""gemv4 against the product in 64 bits (MI355X).

Bound: a group's sums of x (16, 64 or 128 + code) and of x are float32, of up to 128 terms (134 roundings with those of
the groups' scaling), and the groups and waves add one rounding each: (134 + groups + 8) * 2^-24 of sum |x| (279 |scale| +
|base|), which bounds every partial sum (128 + code, up to 143, less 136; 64 + code less 72; 16 + code less 24)."""
import pytest
import torch

import paper_2502_00922_amd as hl

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16]


def make(rows, cols, batch, group, dtype=torch.bfloat16, scale=torch.bfloat16, bases=True, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    shape = (rows, cols // group)
    return {"codes": torch.randint(0, 256, (rows, cols // 2), generator=g, device="cuda", dtype=torch.uint8),
            "scales": (0.01 * torch.randn(shape, generator=g, device="cuda")).to(scale),
            "bases": (0.02 * torch.randn(shape, generator=g, device="cuda")).to(scale) if bases else None,
            "x": torch.randn((batch, cols), generator=g, device="cuda").to(dtype)}


def reference(c):
    """The product and the bound's sum."""
    codes = torch.stack([c["codes"] & 15, c["codes"] >> 4], -1).flatten(1).cpu().double()
    cols = codes.shape[1]
    group = cols // c["scales"].shape[1]
    wide = lambda t: t.cpu().double().repeat_interleave(group, 1)  # noqa: E731
    scale = wide(c["scales"])
    base = wide(c["bases"]) if c["bases"] is not None else torch.zeros_like(scale)
    x = c["x"].cpu().double()
    return x @ (base + scale * (codes - 8)).T, x.abs() @ (279 * scale.abs() + base.abs()).T


def check(c, **more):
    y = hl.gemv4(**c, **more)
    want, size = reference(c)
    bound = (142 + c["scales"].shape[1]) * 2.0**-24 * size
    assert y.dtype == torch.float32 and y.shape == want.shape
    assert ((y.double().cpu() - want).abs() <= bound).all(), float(((y.double().cpu() - want).abs() / bound).max())
    return y


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", TYPES)
@pytest.mark.parametrize("bases", [True, False])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_types(dtype, scale, bases, group):
    check(make(130, 1280, 3, group, dtype, scale, bases))


@pytest.mark.parametrize("batch", list(range(1, 17)))
def test_batches(batch):
    check(make(96, 512, batch, 64))


@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 33, 1021])
@pytest.mark.parametrize("cols,group", [(32, 32), (64, 64), (128, 128), (96, 32), (4128, 32), (1088, 64), (2176, 128)])
def test_odd_sizes(rows, cols, group):
    check(make(rows, cols, 2, group))


@pytest.mark.parametrize("batch", [1, 4, 5, 16])
@pytest.mark.parametrize("rows,cols", [(4096, 4096), (1024, 8192), (16400, 512), (20000, 1056)])
def test_large(batch, rows, cols):
    check(make(rows, cols, batch, 32 if cols % 64 else 64))


def test_vector():
    c = make(48, 256, 1, 64)
    y = check(c)
    assert torch.equal(hl.gemv4(c["codes"], c["scales"], c["x"][0], c["bases"]), y)


def test_output_given():
    c = make(48, 256, 3, 64)
    y = torch.full((3, 48), 9.0, device="cuda")
    assert hl.gemv4(**c, y=y) is y
    assert torch.equal(y, hl.gemv4(**c))


def test_codes_alone():
    # x picks one column at a time: y is its weight, to one rounding of base + scale * (code - 8)
    cols = 160
    c = make(37, cols, 16, 32)
    for first in range(0, cols, 16):
        c["x"] = torch.zeros((16, cols), dtype=torch.bfloat16, device="cuda")
        c["x"][torch.arange(16), first + torch.arange(16)] = 1
        check(c)


def test_large_and_small_x():
    for size in (2.0**100, 2.0**-100):
        c = make(64, 512, 4, 64)
        c["x"] = (c["x"].float() * size).bfloat16()
        check(c)


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_infinite_scales_stay_in_their_rows(bad):
    c = make(70, 640, 3, 64)
    clean = hl.gemv4(**c)
    c["scales"][5, 3], c["bases"][33, 9] = bad, bad
    y = hl.gemv4(**c)
    rest = [r for r in range(70) if r not in (5, 33)]
    assert not y[:, [5, 33]].isfinite().any() and torch.equal(y[:, rest], clean[:, rest])


def test_infinite_x_stays_in_its_row():
    c = make(70, 640, 3, 64)
    clean = hl.gemv4(**c)
    c["x"][1, 600] = float("inf")
    y = hl.gemv4(**c)
    assert not y[1].isfinite().any() and torch.equal(y[[0, 2]], clean[[0, 2]])


def test_captured():
    c = make(300, 1024, 2, 128)
    hl.gemv4(**c)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = hl.gemv4(**c)
    for i in range(4):
        c["x"].mul_(-1.5)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held, hl.gemv4(**c))
