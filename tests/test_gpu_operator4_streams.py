"""The 4-bit operators and sampling on a stream that the caller names (MI355X): what a call allocates there is not given to
the current stream's work while the named one may still use it."""
import pytest
import torch

import paper_2502_00922_amd as hl
import test_gpu_gemv4 as products
import test_gpu_prefix_attention4 as attention
import test_gpu_sample as sampling

pytestmark = pytest.mark.gpu


def read(stream=None):
    c = attention.make(torch.bfloat16, 5, 1, 8, 4, 128, 0, 900)
    return (c["k"],), lambda k: (hl.cache_read4(k, 128, stream=stream),)


def write(stream=None):
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn((3, 500, 4, 128), generator=g, device="cuda").half()
    caches = [torch.zeros((3, 500, 4, 80), dtype=torch.uint8, device="cuda") for _ in range(2)]

    def run(x, k, v):
        hl.cache_write4(x, x, k, v, stream=stream)
        return k, v
    return (x, *caches), run


def attend(stream=None, queries=2):
    c = attention.make(torch.bfloat16, 5, queries, 16, 4, 128, 1500, 700)
    w = torch.zeros((5, 4, 700), device="cuda")
    return (*c.values(), w), lambda q, k, v, n, pk, pv, w: hl.prefix_attention4(q, k, v, n, prefix_k=pk, prefix_v=pv, weights=w,
                                                                                stream=stream)


def attend_many(stream=None):
    return attend(stream, 128)  # its keys and values get room in 16 bits


def product(stream=None):
    c = products.make(5000, 1024, 7, 64)
    return (c["codes"], c["scales"], c["x"], c["bases"]), lambda *a: (hl.gemv4(*a, stream=stream),)


def draw(stream=None):
    return sampling.make(9, 50000), lambda x, u: hl.sample(x, u, temperature=0.7, top_p=0.9, stream=stream)


CALLS = [read, write, attend, attend_many, product, draw]


@pytest.mark.parametrize("make", CALLS)
def test_named_stream_owns_what_the_call_allocates(make):
    args, run = make()
    want = [t if t is None else t.clone() for t in run(*args)]
    s = torch.cuda.Stream()
    args, run = make(s)
    busy = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(20):
            other = busy @ busy  # the operator waits behind these
    got = run(*args)
    # the current stream's work goes on meanwhile, with the memory that it can get
    poison = [torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") for n in (1 << 10, 1 << 16, 1 << 20) for _ in range(8)]
    poison += [torch.full((n << 20,), 0xFF, dtype=torch.uint8, device="cuda") for n in (2, 4, 8, 16, 32, 64)]
    torch.cuda.synchronize()
    assert all((t == 0xFF).all() for t in poison)
    del other, poison
    for a, b in zip(got, want):
        assert (a is None) == (b is None) and (a is None or torch.equal(a.view(torch.uint8), b.view(torch.uint8)))


@pytest.mark.parametrize("make", CALLS)
def test_two_calls_at_once(make):
    streams = [torch.cuda.Stream() for _ in range(2)]
    made = [make(s) for s in streams]
    torch.cuda.synchronize()
    want = [t if t is None else t.clone() for t in make()[1](*make()[0])]
    torch.cuda.synchronize()
    for _ in range(5):
        got = [run(*args) for args, run in made]
        torch.cuda.synchronize()
        for outputs in got:
            for a, b in zip(outputs, want):
                assert (a is None) == (b is None) and (a is None or torch.equal(a.view(torch.uint8), b.view(torch.uint8)))


@pytest.mark.parametrize("make", CALLS)
def test_stream_of_another_gpu(make):
    class Elsewhere:
        device_index, cuda_stream = 1, 0
    args, run = make(Elsewhere())
    with pytest.raises(ValueError):
        run(*args)
