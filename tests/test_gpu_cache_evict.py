"""cache_evict against a plain selection on the host (MI355X): all outputs are exact."""
import numpy as np
import pytest
import torch

import paper_2502_00922_amd as hl

pytestmark = pytest.mark.gpu


def kept_slots(w, n, keep, recent):
    """Kept slots of one head, ascending: w as float64, NaN below every number, ties to the lowest slot."""
    if n <= keep:
        return np.arange(n)
    old = n - recent
    rank = np.where(np.isnan(w[:old]), -np.inf, w[:old])
    low = np.isnan(w[:old])
    order = np.lexsort((np.arange(old), low, -rank))
    return np.concatenate([np.sort(order[:keep - recent]), np.arange(old, n)])


def check(k, v, w, lens, keep, recent, **more):
    r = hl.cache_evict(k, v, w, lens, keep=keep, recent=recent, **more)
    batch, cap, heads, dim = k.shape
    slots, w64, got = r.slots.cpu().numpy(), w.double().cpu().numpy(), r.weights.cpu().numpy()
    bits = lambda t: t.contiguous().view(torch.int16).cpu().numpy()  # noqa: E731
    kb, vb, ko, vo = (bits(t) for t in (k, v, r.k, r.v))
    w32 = w.cpu().numpy()
    for b in range(batch):
        n = min(max(int(lens[b]), 0), cap)
        assert int(r.lens[b]) == min(n, keep)
        for h in range(heads):
            at = kept_slots(w64[b, h], n, keep, recent)
            m = len(at)
            assert np.array_equal(slots[b, h, :m], at) and (slots[b, h, m:] == -1).all()
            assert np.array_equal(got[b, h, :m], w32[b, h, at], equal_nan=True) and (got[b, h, m:] == 0).all()
            for src, dst in ((kb, ko), (vb, vo)):
                assert np.array_equal(dst[b, :m, h], src[b, at, h]) and (dst[b, m:keep, h] == 0).all()
    return r


def make(batch, cap, heads, dim, dtype=torch.bfloat16, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    k, v = (torch.randn((batch, cap, heads, dim), generator=g, device="cuda").to(dtype) for _ in range(2))
    return k, v, torch.rand((batch, heads, cap), generator=g, device="cuda").pow_(8)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.int16])
@pytest.mark.parametrize("batch,cap,heads,dim,keep,recent", [
    (1, 1, 1, 8, 1, 0), (1, 2, 1, 8, 1, 0), (1, 2, 1, 8, 1, 1), (2, 100, 3, 64, 17, 5), (3, 257, 8, 128, 256, 0),
    (2, 1000, 2, 80, 999, 999), (2, 1500, 2, 96, 700, 100), (1, 8191, 2, 16, 64, 8), (1, 8193, 2, 16, 8000, 1),
    (2, 20001, 1, 8, 3000, 333), (1, 40000, 2, 8, 39999, 12), (17, 64, 5, 256, 30, 10)])
def test_sizes(dtype, batch, cap, heads, dim, keep, recent):
    k, v, w = make(batch, cap, heads, dim, dtype if dtype != torch.int16 else torch.bfloat16, seed=cap)
    if dtype == torch.int16:
        k, v = k.view(torch.int16), v.view(torch.int16)
    lens = torch.tensor([cap - (cap * i) // (batch + 1) for i in range(batch)], dtype=torch.int32, device="cuda")
    check(k, v, w, lens, keep, recent)


@pytest.mark.parametrize("recent", [0, 3, 20])
def test_lengths(recent):
    k, v, w = make(8, 90, 2, 32)
    lens = torch.tensor([0, 1, 19, 20, 21, 90, -4, 1000], dtype=torch.int32, device="cuda")
    check(k, v, w, lens, 20, recent)


@pytest.mark.parametrize("kind", ["equal", "few values", "zeros", "special", "negative", "subnormal", "near"])
@pytest.mark.parametrize("cap", [300, 9000])
def test_ties_and_special_weights(kind, cap):
    k, v, w = make(2, cap, 2, 8, seed=3)
    g = torch.Generator(device="cuda").manual_seed(4)
    pick = lambda values: torch.tensor(values, device="cuda")[  # noqa: E731
        torch.randint(len(values), w.shape, generator=g, device="cuda")]
    if kind == "equal":
        w[...] = 0.25
    elif kind == "few values":
        w = pick([0.5, 0.25, 0.25, 1.0])
    elif kind == "zeros":
        w = pick([0.0, -0.0, 0.0])
    elif kind == "special":
        w = pick([float("nan"), float("inf"), -float("inf"), 1.0, -0.0, 0.0, -1e-40])
    elif kind == "negative":
        w = -w
    elif kind == "subnormal":
        w = w * 1e-38 * 1e-3
    else:  # differ in the last bits alone
        w = (torch.randint(0, 1000, w.shape, generator=g, device="cuda").int() + 0x3F800000).view(torch.float32)
    lens = torch.tensor([cap, cap - 77], dtype=torch.int32, device="cuda")
    for keep, recent in ((cap // 2, 0), (100, 30), (cap - 78, 1)):
        check(k, v, w.contiguous(), lens, keep, recent)


def test_strides_and_larger_target():
    k, v, w = make(3, 200, 4, 64)
    kt = k.transpose(1, 2).contiguous().transpose(1, 2)
    lens = torch.tensor([200, 150, 20], dtype=torch.int32, device="cuda")
    k_out = torch.full((3, 4, 100, 64), 7.0, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    v_out = torch.full((3, 100, 4, 80), 7.0, dtype=torch.bfloat16, device="cuda")[..., 8:72]
    r = check(kt, v, w, lens, 60, 10, k_out=k_out, v_out=v_out)
    assert r.k is k_out and (k_out[:, 60:] == 7).all() and (v_out[:, 60:] == 7).all()


def test_offsets_past_32_bits():
    rows, stride = 70, 1 << 26
    k, v, w = make(1, rows, 1, 64)
    big = torch.empty(rows * stride, dtype=torch.bfloat16, device="cuda").as_strided((1, rows, 1, 64), (0, stride, 64, 1))
    big.copy_(k)
    lens = torch.tensor([rows], dtype=torch.int32, device="cuda")
    r = check(big, v, w, lens, 40, 5)
    k_out = big.clone()  # keeps the strides' order, not their size: rows in a row
    far = torch.empty(rows * stride, dtype=torch.bfloat16, device="cuda").as_strided((1, rows, 1, 64), (0, stride, 64, 1))
    s = hl.cache_evict(k_out, v, w, lens, keep=40, recent=5, k_out=far, v_out=torch.empty_like(v))
    assert torch.equal(s.k[:, :40], r.k)


def test_repeat_and_stream():
    k, v, w = make(4, 5000, 8, 128)
    lens = torch.full((4,), 5000, dtype=torch.int32, device="cuda")
    want = hl.cache_evict(k, v, w, lens, keep=2000, recent=100)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = hl.cache_evict(k, v, w, lens, keep=2000, recent=100)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_refusals():
    k, v, w = make(2, 50, 2, 64)
    lens = torch.tensor([50, 40], dtype=torch.int32, device="cuda")
    good = dict(k=k, v=v, weights=w, lens=lens, keep=20, recent=4)
    small = torch.empty((2, 19, 2, 64), dtype=torch.bfloat16, device="cuda")
    for bad in (dict(keep=0), dict(recent=21), dict(recent=-1), dict(weights=w.double()), dict(weights=w[:, :, :49]),
                dict(lens=lens.long()), dict(lens=lens.cpu()), dict(k=k.float(), v=v.float()), dict(v=v.half()),
                dict(k=k.cpu(), v=v.cpu()), dict(k_out=small, v_out=small), dict(k_out=torch.empty_like(k)), dict(k=k[0])):
        with pytest.raises(ValueError):
            hl.cache_evict(**{**good, **bad})
    off = torch.zeros(2 * 50 * 2 * 60, dtype=torch.bfloat16, device="cuda").view(2, 50, 2, 60)
    with pytest.raises(hl.HLError):
        hl.cache_evict(**{**good, "k": off, "v": off})
