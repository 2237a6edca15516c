"""The operators on tensors of a GPU that is not the current one (no GPU: tensors that say they are on GPU 1, and a library
that notes which GPU is current when it is called). A kernel runs on the current GPU, so each call has to make the
tensors' GPU that one, and leave the caller's as it was."""
import contextlib

import pytest
import torch

hl = pytest.importorskip("paper_2502_00922_amd.hufflm")


class OnGpu1(torch.Tensor):
    """A host tensor that says it is on GPU 1."""

    def get_device(self):
        return 1

    is_cuda = True


def on1(t):
    return t.as_subclass(OnGpu1)


class Library:
    """Notes the current GPU at each call and launches nothing."""

    def __init__(self, current):
        self.current, self.calls = current, []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, self.current[0]))
            return 64 if name == "hl_attention_workspace_bytes" else 0
        return call


@pytest.fixture
def gpus(monkeypatch):
    """The library, with GPU 0 as the current one and a GPU 1 beside it."""
    current = [0]

    @contextlib.contextmanager
    def device(index):
        before, current[0] = current[0], index
        try:
            yield
        finally:
            current[0] = before

    T = hl._Torch()
    T.lib = Library(current)
    T.raw_stream, T.current_device = lambda index: 0, lambda: current[0]
    T.empty = lambda *a, **k: on1(torch.empty(*a, **k))
    monkeypatch.setattr(hl, "_torch", T)
    monkeypatch.setattr(torch.cuda, "device", device)
    return T.lib, current


def norm():
    x = on1(torch.ones(4, 64))
    return hl.rms_norm(x, on1(torch.ones(64)), residual=x, out_dtype=torch.float8_e4m3fn)


def attention():
    k = on1(torch.ones(2, 10, 2, 64, dtype=torch.bfloat16))
    return hl.prefix_attention(on1(torch.ones(2, 1, 4, 64, dtype=torch.bfloat16)), k, k,
                               on1(torch.ones(2, dtype=torch.int32)), prefix_k=k[0], prefix_v=k[0],
                               weights=on1(torch.zeros(2, 2, 10)))


def evict():
    k = on1(torch.ones(2, 10, 2, 64, dtype=torch.bfloat16))
    return hl.cache_evict(k, k, on1(torch.zeros(2, 2, 10)), on1(torch.ones(2, dtype=torch.int32)), keep=4, recent=1)


@pytest.mark.parametrize("run,calls", [(norm, ["hl_rms_norm"]), (evict, ["hl_cache_evict"]),
                                       (attention, ["hl_attention_workspace_bytes", "hl_prefix_attention"])])
def test_library_is_called_on_the_tensors_gpu(gpus, run, calls):
    library, current = gpus
    run()
    assert library.calls == [(name, 1) for name in calls]
    assert current == [0]


@pytest.mark.parametrize("run", [norm, attention, evict])
def test_current_gpu_is_left_after_an_error(gpus, run, monkeypatch):
    library, current = gpus
    monkeypatch.setattr(hl._torch, "raw_stream", lambda index: 1 / 0)
    with pytest.raises(ZeroDivisionError):
        run()
    assert current == [0]


def test_host_tensors_are_still_refused(gpus):
    x = torch.ones(4, 64)
    with pytest.raises(ValueError):
        hl.rms_norm(x, torch.ones(64))
    with pytest.raises(ValueError):
        hl.prefix_attention(x.bfloat16().view(4, 1, 1, 64))
    with pytest.raises(ValueError):
        hl.cache_evict(*(x.bfloat16().view(1, 4, 1, 64),) * 2, torch.zeros(1, 1, 4), torch.ones(1, dtype=torch.int32), 2)
    assert gpus[0].calls == []
