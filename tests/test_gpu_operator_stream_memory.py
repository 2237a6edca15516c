"""The operators on a stream that the caller names (MI355X): work of the current stream that is pending or comes later has
its memory to itself, and so has the call."""
import pytest
import torch

import test_gpu_operator_streams as calls
from test_gpu_attention_workspace import needed

pytestmark = pytest.mark.gpu


def busy():
    """Some 20 ms of work on the current stream."""
    a = torch.full((4096, 4096), 1e-3, device="cuda")
    b = torch.empty_like(a)
    for _ in range(20):
        torch.matmul(a, a, out=b)
    return a, b


def workspace(args):
    q, k, _, _, prefix, _, _ = args
    return needed({"q": q, "k": k, "prefix_k": prefix}, True)


def sizes(make, args, outputs):
    """Bytes of what the call allocates."""
    return [t.nbytes for t in outputs if t is not None] + ([workspace(args)] if make is calls.attention else [])


def start(make):
    """The call's inputs and outputs, and the call on a stream of its own, with nothing left in torch's cache."""
    args, run = make()
    want = run(*args)
    s = torch.cuda.Stream()
    run = make(s)[1]
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    return args, want, s, run


def check(got, want):
    for a, b in zip(got, want):
        assert (a is None) == (b is None) and (a is None or torch.equal(a.view(torch.uint8), b.view(torch.uint8)))


@pytest.mark.parametrize("make", [calls.norm, calls.attention, calls.evict])
def test_later_work_of_the_current_stream(make):
    args, want, s, run = start(make)
    with torch.cuda.stream(s):
        waits = busy()  # the call waits behind this
    got = run(*args)
    later = [torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") for n in sizes(make, args, want) for _ in range(4)]
    torch.cuda.synchronize()
    assert all((t == 0xFF).all() for t in later)
    check(got, want)
    del waits


@pytest.mark.parametrize("make", [calls.norm, calls.attention, calls.evict])
def test_pending_work_of_the_current_stream(make):
    args, want, s, run = start(make)
    waits = busy()
    # written behind that, and given back for what this stream does later
    pending = [torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") for n in sizes(make, args, want) for _ in range(2)]
    copies = [t.clone() for t in pending]
    del pending
    got = run(*args)
    torch.cuda.synchronize()
    check(got, want)
    assert all((t == 0xFF).all() for t in copies)
    del waits
