"""prefix_attention4 where many rows of q meet a key: the rows' values enter the sums unrounded there as well, whatever the
caches' capacity, and what they stand for may pass float16's range (MI355X).

The bounds are those of test_gpu_prefix_attention4.py for calls of few rows, without anything for a rounding of keys and
values: u of the output, r of sum p (|scale (code - 8)| + |base|), scores off by e, 96 * 2^-24 of the sums."""
import math

import pytest
import torch

import paper_2502_00922_amd as hl
from rows4 import random_rows
from test_gpu_prefix_attention4 import R, TYPES, U, make, reference

pytestmark = pytest.mark.gpu


def strict(c):
    r = hl.prefix_attention4(**c)
    out, _, _, steps, sums, most, _, _, near = reference(c)
    dtype = c["q"].dtype
    e = (39 + c["q"].shape[-1] // 32) * 2.0**-24 * most
    bound = U[dtype] * out.abs() + (1 + U[dtype]) * (R[dtype] * steps + 2 * e * near + 96 * 2.0**-24 * sums) + 2.0**-25
    got = r.out.double().cpu()
    assert got.isfinite().all()
    assert ((got - out).abs() <= bound).all(), float(((got - out).abs() / bound).max())
    return r


def set_pairs(rows, dim, scale=None, base=None):
    pairs = rows[..., dim // 2:dim // 2 + dim // 8].contiguous().view(torch.bfloat16).unflatten(-1, (dim // 32, 2))
    for i, x in enumerate((scale, base)):
        if x is not None:
            pairs[..., i] = x
    rows[..., dim // 2:dim // 2 + dim // 8] = pairs.flatten(-2).view(torch.uint8)


# batch, queries, heads, kv_heads, dim, prefix, own: 256 rows a key and more in the mean; few keys, so that a mistake in
# one score is seen
SHAPES = [(1, 64, 8, 2, 64, 9, 0), (2, 128, 4, 2, 128, 0, 130), (4, 64, 4, 1, 96, 40, 66), (1, 256, 2, 2, 256, 12, 256),
          (64, 1, 8, 2, 128, 33, 0)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_codes_far_below_a_base(dtype, shape):
    # a key's base is 512 codes' steps: 16 bits have no place for the code beside it
    c = make(dtype, *shape)
    for name in ("k", "prefix_k"):
        if name in c:
            set_pairs(c[name], shape[4], scale=0.125, base=64.0)
    strict(c)


@pytest.mark.parametrize("own", [8, 4096])
def test_capacity_is_no_matter(own):
    c = make(torch.bfloat16, 8, 8, 16, 2, 64, 64, own, lens=[8] * 8)
    for name in ("k", "prefix_k"):
        set_pairs(c[name], 64, scale=0.125, base=64.0)
    strict(c)


@pytest.mark.parametrize("shape", SHAPES)
def test_values_past_the_range_of_float16(shape):
    # every third token's values are 49152 + 7 * 2560 = 67072, the others' 49152: their mean is in the range
    c = make(torch.float16, *shape, size=0.25)
    dim = shape[4]
    for name in ("v", "prefix_v"):
        if name in c:
            set_pairs(c[name], dim, scale=2560.0, base=49152.0)
            c[name][..., :dim // 2] = 0x88
            c[name][..., ::3, :, :dim // 2] = 0xFF
    strict(c)


def test_rows_of_a_graph_share_the_smaller_workspace():
    c = make(torch.bfloat16, 4, 64, 8, 2, 128, 300, 100)
    want = strict(c).out
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = hl.prefix_attention4(**c)
    for _ in range(3):
        held.out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held.out, want)


def test_long_prefix_of_many_rows():
    # most of the time of such a call is in the wide items' steps; a tenth of the sequences is compared
    g = torch.Generator(device="cuda").manual_seed(3)
    q = (1.5 * torch.randn((70, 1, 16, 64), generator=g, device="cuda")).bfloat16()
    k, v = (random_rows((2000, 4), 64, g) for _ in range(2))
    got = hl.prefix_attention4(q, prefix_k=k, prefix_v=v)
    some = slice(0, 70, 10)
    c = {"q": q[some].contiguous(), "prefix_k": k, "prefix_v": v}
    out, _, _, steps, sums, most, _, _, near = reference(c)
    e = 41 * 2.0**-24 * most
    bound = 2.0**-8 * out.abs() + (1 + 2.0**-8) * (2.0**-8 * steps + 2 * e * near + 96 * 2.0**-24 * sums) + 2.0**-25
    assert ((got.out[some].double().cpu() - out).abs() <= bound).all()
    assert math.isfinite(float(got.out.float().abs().max()))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(1, 2048, 16, 4, 128, 0, 2048), (16, 300, 8, 2, 64, 5000, 900), (3, 700, 12, 4, 96, 1777, 1003),
                                   (2, 513, 8, 8, 256, 300, 2000), (128, 1, 32, 8, 128, 16384, 40)])
def test_large_calls_beside_16_bits(dtype, shape):
    # values (code - 8) / 16 of both types: the 16-bit attention's, on the same numbers. Either is off by u of the output and,
    # by its rounding of p, by u (r) of sum p |v|; scores and sums by some 2^-16 (|q k| below 40)
    c = make(dtype, *shape)
    dim = shape[4]
    for name in ("k", "v", "prefix_k", "prefix_v"):
        if name in c:
            set_pairs(c[name], dim, scale=0.0625, base=0.0)
    wide = {n: t if n in ("q", "lens") else hl.cache_read4(t, dim, dtype=dtype) for n, t in c.items()}
    got, want = hl.prefix_attention4(**c).out.float(), hl.prefix_attention(**wide).out.float()
    sizes = hl.prefix_attention(**{n: t.abs() if n.endswith("v") else t for n, t in wide.items()}).out.float()
    u, r = U[dtype], R[dtype]
    bound = u * (got.abs() + want.abs()) + (u + r + 2.0**-10) * sizes * (1 + 4 * u) + 2.0**-20
    assert got.isfinite().all() and ((got - want).abs() <= bound).all(), float(((got - want).abs() / bound).max())
