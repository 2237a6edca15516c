"""The operators on a stream that the caller names (no GPU: tensors that say they are on GPU 1, and a library that notes what
is current): all that a call allocates, and its launch, happen while that stream is the current one, so that torch gives
the memory to no other stream's work meanwhile."""
import contextlib

import pytest
import torch

hl = pytest.importorskip("paper_2502_00922_amd.hufflm")


class Stream:
    device_index, cuda_stream = 1, 77


class World:
    """What the calls did, in order, each with the stream that was current then (None: the caller's own)."""

    def __init__(self):
        self.stream, self.done = None, []

    @contextlib.contextmanager
    def on(self, stream):
        before, self.stream = self.stream, stream
        try:
            yield
        finally:
            self.stream = before

    def noted(self, what, f):
        def call(*args, **more):
            self.done.append((what, self.stream))
            return f(*args, **more)
        return call

    def __getattr__(self, name):  # the library
        return self.noted(name, lambda *args: 64 if name == "hl_attention_workspace_bytes" else 0)


world = World()


class OnGpu1(torch.Tensor):
    """A host tensor that says it is on GPU 1."""
    is_cuda = True

    def get_device(self):
        return 1

    def new_empty(self, shape):
        return world.noted("allocate", torch.empty)(shape, dtype=self.dtype).as_subclass(OnGpu1)


def ones(*shape, dtype=torch.float32):
    return torch.ones(shape, dtype=dtype).as_subclass(OnGpu1)


@pytest.fixture(autouse=True)
def gpu(monkeypatch):
    global world
    world = World()
    T = hl._Torch()
    T.lib, T.current_device, T.raw_stream = world, lambda: 1, world.noted("stream", lambda index: 0)
    T.empty = lambda *a, **k: world.noted("allocate", torch.empty)(*a, **k).as_subclass(OnGpu1)
    T.empty_like = lambda *a, **k: world.noted("allocate", torch.empty_like)(*a, **k)
    monkeypatch.setattr(hl, "_torch", T)
    monkeypatch.setattr(torch.cuda, "stream", world.on)


def norm(stream):
    x = ones(4, 64)
    hl.rms_norm(x, ones(64), residual=x, out_dtype=torch.float8_e4m3fn, stream=stream)
    return "hl_rms_norm", 3  # out, sum and scale


def attention(stream):
    k = ones(2, 10, 2, 64, dtype=torch.bfloat16)
    hl.prefix_attention(ones(2, 1, 4, 64, dtype=torch.bfloat16), k, k, ones(2, dtype=torch.int32), weights=ones(2, 2, 10),
                        stream=stream)
    return "hl_prefix_attention", 3  # out, weights and workspace


def evict(stream):
    k = ones(2, 10, 2, 64, dtype=torch.bfloat16)
    hl.cache_evict(k, k, ones(2, 2, 10), ones(2, dtype=torch.int32), keep=4, recent=1, stream=stream)
    return "hl_cache_evict", 5  # keys, values, weights, slots and lengths


@pytest.mark.parametrize("run", [norm, attention, evict])
@pytest.mark.parametrize("stream", [Stream(), None])
def test_memory_and_launch_are_the_streams(run, stream):
    function, allocations = run(stream)
    what = [w for w, _ in world.done]
    assert what.count("allocate") == allocations and what.count("stream") == 1 and function in what
    assert all(then is stream for _, then in world.done), world.done
    assert world.stream is None
