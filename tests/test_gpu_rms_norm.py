"""rms_norm against its formula in 64 bits (MI355X).

Bounds: one rounding to the output's type (unit roundoff u: 2^-24, 2^-8, 2^-11 for float32, bf16, float16), on top of
float32 arithmetic: the sum of squares is added in chains of at most 32 and a tree of 10 levels, its root halves the
error, and five more operations round once each, so 40 * 2^-24 relative is never passed. The sum x + residual is
rounded to float32 and then to its type. 8 bits: u = 2^-4, and 2^-10 (half the spacing of the subnormals) absolute, in
units of the scale."""
import pytest
import torch

import paper_2502_00922_amd as hl

pytestmark = pytest.mark.gpu
U = {torch.float32: 2.0**-24, torch.bfloat16: 2.0**-8, torch.float16: 2.0**-11}
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0**-25}  # half the spacing of float16's subnormals
F32 = 40 * 2.0**-24
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def reference(x, weight, residual, eps):
    t = x.double() if residual is None else x.double() + residual.double()
    return t, t / torch.sqrt((t * t).mean(-1, keepdim=True) + eps) * weight.double()


def check(x, weight, residual, r, eps=1e-5, group=0):
    t, y = reference(x, weight, residual, eps)
    if residual is not None:
        u = U[residual.dtype]
        assert ((r.sum.double() - t).abs() <= (u + 2 * 2.0**-24) * t.abs() + TINY[residual.dtype]).all()
    # an addition that cancels leaves the float32 rounding of the sum
    slack = F32 * y.abs() + 1e-37
    if r.out.dtype in U:
        assert ((r.out.double() - y).abs() <= U[r.out.dtype] * y.abs() * (1 + 2.0**-8) + slack + TINY[r.out.dtype]).all()
        return
    size = group or y.shape[-1]
    top = y.abs().unflatten(-1, (-1, size)).amax(-1)
    scale = torch.where(top > 0, top / 448, torch.ones_like(top))
    got = r.scale.double().view(scale.shape)
    assert ((got - scale).abs() <= F32 * scale).all()
    each = got.repeat_interleave(size, -1).view(y.shape)
    err = (r.out.double() * each - y).abs()
    assert (err <= each * torch.clamp(2.0**-4 * (y / each).abs(), min=2.0**-10) * (1 + 2.0**-8) + slack).all()


def make(tokens, hidden, xt, rt, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((tokens, hidden), generator=g, device="cuda").to(xt)
    r = None if rt is None else (3 * torch.randn((tokens, hidden), generator=g, device="cuda")).to(rt)
    w = (1 + 0.2 * torch.randn(hidden, generator=g, device="cuda")).to(torch.bfloat16)
    return x, r, w


@pytest.mark.parametrize("rt", [None, *TYPES])
@pytest.mark.parametrize("xt", TYPES)
@pytest.mark.parametrize("ot", [*TYPES, torch.float8_e4m3fn])
def test_types(xt, rt, ot):
    x, r, w = make(3, 1032, xt, rt)
    check(x, w, r, hl.rms_norm(x, w, residual=r, out_dtype=ot))


@pytest.mark.parametrize("ot", [torch.bfloat16, torch.float8_e4m3fn])
@pytest.mark.parametrize("tokens,hidden", [
    (1, 1), (1, 7), (2, 8), (5, 64), (9, 511), (3, 512), (7, 520), (2, 1023), (2, 2052), (3, 4096), (2, 4097), (1, 4100),
    (2, 8192), (1, 8200), (1, 11008), (1, 14336), (1, 16388), (1, 20001), (1, 28672), (2, 32768), (1, 32767),
    (1000, 24), (513, 640)])
def test_sizes(tokens, hidden, ot):
    x, r, w = make(tokens, hidden, torch.float32, torch.bfloat16, seed=hidden)
    check(x, w, r, hl.rms_norm(x, w, residual=r, out_dtype=ot))


@pytest.mark.parametrize("hidden,group", [(32, 32), (64, 64), (128, 128), (4096, 32), (4096, 64), (8192, 128), (1056, 32),
                                          (1088, 64), (1152, 128), (28672, 128), (32768, 32)])
def test_groups(hidden, group):
    x, r, w = make(5, hidden, torch.bfloat16, torch.bfloat16, seed=group)
    x[2], r[2] = 0, 0  # a row of zeros: scale 1
    y = hl.rms_norm(x, w, residual=r, out_dtype=torch.float8_e4m3fn, group=group)
    assert y.scale.shape == (5, hidden // group)
    check(x, w, r, y, group=group)
    assert (y.scale[2] == 1).all() and (y.out[2].float() == 0).all()


def test_weight_types_and_leading_dimensions():
    x, r, w = make(6, 776, torch.float16, torch.float32)
    for wt in TYPES:
        y = hl.rms_norm(x.view(2, 3, 776), w.to(wt), residual=r.view(2, 3, 776))
        assert y.out.shape == (2, 3, 776) and y.out.dtype == wt and y.sum.dtype == torch.float32
        check(x.view(2, 3, 776), w.to(wt), r.view(2, 3, 776), y)


@pytest.mark.parametrize("offset", [1, 2, 4, 8])
def test_starts_off_16_bytes(offset):
    x, r, w = make(4, 520, torch.bfloat16, torch.bfloat16)
    places = [torch.empty(4 * 520 + offset, dtype=torch.bfloat16, device="cuda")[offset:].view(4, 520) for _ in range(4)]
    places[0].copy_(x), places[1].copy_(r)
    y = hl.rms_norm(places[0], w, residual=places[1], out=places[2], sum_out=places[3])
    want = hl.rms_norm(x, w, residual=r)
    check(x, w, r, y)
    assert torch.equal(y.sum, want.sum)


def test_in_place():
    x, r, w = make(5, 4096, torch.bfloat16, torch.bfloat16)
    want = hl.rms_norm(x, w, residual=r)
    x2, r2 = x.clone(), r.clone()
    y = hl.rms_norm(x2, w, residual=r2, sum_out=r2, out=x2)
    assert torch.equal(y.out, want.out) and torch.equal(y.sum, want.sum)
    assert y.out is x2 and y.sum is r2


def test_extremes():
    x, _, w = make(6, 256, torch.float32, None)
    x[0] = 0                    # nothing but eps
    x[1] *= 1e-30               # squares below the normal range
    x[2, 5] = float("nan")
    x[3, 7] = float("inf")
    x[4] *= 1e15
    y = hl.rms_norm(x, w, out_dtype=torch.float32).out
    assert (y[0] == 0).all()
    assert y[2].isnan().all()
    assert y[3, 7].isnan() and (y[3, :7] == 0).all()
    _, want = reference(x, w, None, 1e-5)
    for i in (1, 4, 5):
        assert ((y[i].double() - want[i]).abs() <= 2 * F32 * want[i].abs() + 1e-37).all()
    q = hl.rms_norm(x, w, out_dtype=torch.float8_e4m3fn)
    assert q.out[2].float().isnan().all()


def test_stream_and_repeat():
    x, r, w = make(64, 8192, torch.float32, torch.bfloat16)
    want = hl.rms_norm(x, w, residual=r)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        a = hl.rms_norm(x, w, residual=r)
    b = hl.rms_norm(x, w, residual=r, out=torch.empty_like(want.out), sum_out=torch.empty_like(r), stream=s)
    s.synchronize()
    assert torch.equal(a.out, want.out) and torch.equal(b.out, want.out) and torch.equal(b.sum, want.sum)


def test_refusals():
    x, r, w = make(2, 64, torch.bfloat16, torch.bfloat16)
    bad = [dict(x=x.cpu()), dict(weight=w.cpu()), dict(x=x.double()), dict(weight=w[:32]), dict(residual=r[:1]),
           dict(residual=r.int()), dict(x=x[:, ::2], weight=w[:32].clone()), dict(out_dtype=torch.int8), dict(group=32),
           dict(out_dtype=torch.float8_e4m3fn, group=48), dict(out_dtype=torch.float8_e4m3fn, group=128),
           dict(sum_out=torch.empty_like(x)), dict(out=torch.empty(2, 32, dtype=torch.bfloat16, device="cuda")),
           dict(x=x[:0]), dict(scale_out=torch.empty(2, device="cuda")),
           dict(residual=r, sum_out=torch.empty(2, 64, device="cuda"))]
    for b in bad:
        with pytest.raises(ValueError):
            hl.rms_norm(**{"x": x, "weight": w, **b})
    big = torch.zeros((1, 32769), device="cuda")
    with pytest.raises(hl.HLError):
        hl.rms_norm(big, big[0])
    with pytest.raises(hl.HLError):
        hl.rms_norm(x, w, eps=-1.0)
