"""The 4-bit operators and sampling: bad arguments come back as status codes before any device work, or as ValueError from
the binding before the library is called (no GPU: device addresses here are made up and never read, and tensors that say
they are on a GPU meet a library that notes its calls)."""
import contextlib
import ctypes
import math

import pytest
import torch

hl = pytest.importorskip("paper_2502_00922_amd.hufflm")
A = 0x10000


@pytest.fixture(scope="module")
def L():
    return hl.lib()


def kv(tokens=10, row=40, heads=2):
    t = heads * row
    return hl.KeysValues(A, A, tokens, tokens * t, t, row, tokens * t, t, row)


@pytest.mark.parametrize("dim,n", [(32, 32), (64, 48), (96, 64), (128, 80), (160, 112), (192, 128), (224, 144), (256, 160),
                                   (0, 0), (16, 0), (100, 0), (288, 0), (1 << 31, 0)])
def test_row_bytes(L, dim, n):
    assert L.hl_cache4_row_bytes(dim) == n
    if n:
        assert hl.cache4_row_bytes(dim) == n
    else:
        with pytest.raises(ValueError):
            hl.cache4_row_bytes(dim)


@pytest.mark.parametrize("bad,status", [
    (dict(src=None), hl.HL_EINVAL), (dict(dst=None), hl.HL_EINVAL), (dict(dtype=hl.HL_F32), hl.HL_EINVAL),
    (dict(batch=0), hl.HL_EINVAL), (dict(heads=0), hl.HL_EINVAL), (dict(dim=0), hl.HL_EINVAL), (dict(dim=48), hl.HL_EINVAL),
    (dict(lens=A + 2), hl.HL_EINVAL), (dict(dim=288), hl.HL_EUNSUPPORTED), (dict(batch=70000), hl.HL_EUNSUPPORTED),
    (dict(heads=70000), hl.HL_EUNSUPPORTED)])
def test_write(L, bad, status):
    good = dict(src=ctypes.byref(kv(3, 128)), dtype=hl.HL_BF16, dst=ctypes.byref(kv()), batch=2, heads=2, dim=128, lens=A)
    assert L.hl_cache_write4(*{**good, **bad}.values(), None) == status


@pytest.mark.parametrize("field,value,status", [
    ("k_dev", None, hl.HL_EINVAL), ("v_dev", A + 8, hl.HL_EINVAL), ("tokens", 0, hl.HL_EINVAL), ("k_token", 36, hl.HL_EINVAL),
    ("v_seq", 1 << 41, hl.HL_EUNSUPPORTED), ("tokens", 1 << 30, hl.HL_EUNSUPPORTED)])
def test_write_strides(L, field, value, status):
    for side in (0, 1):
        sets = [kv(3, 128), kv()]
        setattr(sets[side], field, value)
        assert L.hl_cache_write4(ctypes.byref(sets[0]), hl.HL_F16, ctypes.byref(sets[1]), 2, 2, 128, A, None) == status


@pytest.mark.parametrize("bad,status", [
    (dict(rows=None), hl.HL_EINVAL), (dict(rows=A + 8), hl.HL_EINVAL), (dict(out=None), hl.HL_EINVAL),
    (dict(out=A + 4), hl.HL_EINVAL), (dict(dtype=hl.HL_E4M3), hl.HL_EINVAL), (dict(token=88), hl.HL_EINVAL),
    (dict(batch=0), hl.HL_EINVAL), (dict(tokens=0), hl.HL_EINVAL), (dict(heads=0), hl.HL_EINVAL), (dict(dim=40), hl.HL_EINVAL),
    (dict(dim=512), hl.HL_EUNSUPPORTED), (dict(tokens=1 << 30), hl.HL_EUNSUPPORTED), (dict(seq=1 << 41), hl.HL_EUNSUPPORTED),
    (dict(batch=60000, tokens=1 << 24), hl.HL_EUNSUPPORTED)])
def test_read(L, bad, status):
    good = dict(rows=A, seq=1600, token=160, head=80, batch=2, tokens=10, heads=2, dim=128, out=A, dtype=hl.HL_BF16)
    assert L.hl_cache_read4(*{**good, **bad}.values(), None) == status


def attention(**bad):
    a = hl.AttentionShape(hl.HL_BF16, 2, 1, 8, 2, 128, 0.1, kv(100), kv(100))
    for name, value in bad.items():
        where, _, field = name.rpartition("__")
        setattr(getattr(a, where) if where else a, field, value)
    return a


@pytest.mark.parametrize("bad,status", [
    (dict(dtype=hl.HL_F32), hl.HL_EINVAL), (dict(batch=0), hl.HL_EINVAL), (dict(queries=0), hl.HL_EINVAL),
    (dict(heads=0), hl.HL_EINVAL), (dict(kv_heads=3), hl.HL_EINVAL), (dict(dim=0), hl.HL_EINVAL), (dict(dim=80), hl.HL_EINVAL),
    (dict(dim=8), hl.HL_EINVAL), (dict(scale=float("nan")), hl.HL_EINVAL), (dict(dim=288), hl.HL_EUNSUPPORTED),
    (dict(own__k_dev=None), hl.HL_EINVAL), (dict(prefix__v_dev=A + 8), hl.HL_EINVAL), (dict(own__k_token=44), hl.HL_EINVAL),
    (dict(prefix__k_token=1 << 25), hl.HL_EUNSUPPORTED), (dict(prefix__tokens=1 << 30), hl.HL_EUNSUPPORTED),
    (dict(batch=70000), hl.HL_EUNSUPPORTED)])
def test_attention_shape(L, bad, status):
    a = attention(**bad)
    args = (ctypes.byref(a), A, A, A, None, None, None, A, 1 << 40, None)
    assert L.hl_prefix_attention4(*args) == status
    assert L.hl_attention4_workspace_bytes(ctypes.byref(a), 0) == 0


def test_attention_buffers(L):
    a = attention(own__tokens=3000)
    need = L.hl_attention4_workspace_bytes(ctypes.byref(a), 0)
    assert 0 < need < L.hl_attention4_workspace_bytes(ctypes.byref(a), 1)
    good = dict(q=A, lens=A, out=A, lse=A, w_in=A, w_out=A, ws=A, n=1 << 40)
    for bad in (dict(q=None), dict(q=A + 8), dict(lens=None), dict(lens=A + 2), dict(out=None), dict(out=A + 2),
                dict(lse=A + 1), dict(w_out=None), dict(w_out=A + 2), dict(ws=None), dict(ws=A + 4), dict(n=need)):
        assert L.hl_prefix_attention4(ctypes.byref(a), *{**good, **bad}.values(), None) == hl.HL_EINVAL, bad
    assert L.hl_prefix_attention4(None, *good.values(), None) == hl.HL_EINVAL
    assert L.hl_attention4_workspace_bytes(None, 0) == 0


@pytest.mark.parametrize("bad,status", [
    (dict(codes=None), hl.HL_EINVAL), (dict(codes=A + 8), hl.HL_EINVAL), (dict(scales=None), hl.HL_EINVAL),
    (dict(scales=A + 2), hl.HL_EINVAL), (dict(bases=A + 2), hl.HL_EINVAL), (dict(st=hl.HL_F32), hl.HL_EINVAL),
    (dict(rows=0), hl.HL_EINVAL), (dict(cols=0), hl.HL_EINVAL), (dict(cols=320), hl.HL_EINVAL), (dict(group=16), hl.HL_EINVAL),
    (dict(group=0), hl.HL_EINVAL), (dict(group=256, cols=512), hl.HL_EINVAL), (dict(x=None), hl.HL_EINVAL),
    (dict(x=A + 2), hl.HL_EINVAL), (dict(xt=hl.HL_F32), hl.HL_EINVAL), (dict(batch=0), hl.HL_EINVAL),
    (dict(batch=17), hl.HL_EINVAL), (dict(y=None), hl.HL_EINVAL), (dict(y=A + 2), hl.HL_EINVAL),
    (dict(rows=1 << 31), hl.HL_EUNSUPPORTED), (dict(cols=1 << 24), hl.HL_EUNSUPPORTED)])
def test_gemv(L, bad, status):
    good = dict(codes=A, scales=A, bases=A, st=hl.HL_BF16, rows=64, cols=384, group=128, x=A, xt=hl.HL_F16, batch=2, y=A)
    assert L.hl_gemv4(*{**good, **bad}.values(), None) == status


@pytest.mark.parametrize("bad,status", [
    (dict(settings=None), hl.HL_EINVAL), (dict(logits=None), hl.HL_EINVAL), (dict(logits=A + 2), hl.HL_EINVAL),
    (dict(dtype=hl.HL_E4M3), hl.HL_EINVAL), (dict(stride=99), hl.HL_EINVAL), (dict(rows=0), hl.HL_EINVAL),
    (dict(vocab=0), hl.HL_EINVAL), (dict(u=None), hl.HL_EINVAL), (dict(u=A + 2), hl.HL_EINVAL), (dict(tokens=None), hl.HL_EINVAL),
    (dict(tokens=A + 1), hl.HL_EINVAL), (dict(logprobs=None), hl.HL_EINVAL), (dict(logprobs=A + 1), hl.HL_EINVAL),
    (dict(vocab=1 << 20, stride=1 << 20), hl.HL_EUNSUPPORTED), (dict(stride=1 << 40), hl.HL_EUNSUPPORTED),
    (dict(rows=65536), hl.HL_EUNSUPPORTED), (dict(ws=None), hl.HL_EINVAL), (dict(ws=A + 8), hl.HL_EINVAL),
    (dict(n=100), hl.HL_EINVAL)])
def test_sample(L, bad, status):
    settings = hl.Sampling(None, None, None, None, 1.0, 0, 1.0, 0.0)
    good = dict(settings=ctypes.byref(settings), logits=A, dtype=hl.HL_F32, stride=100, rows=2, vocab=100, u=A, tokens=A,
                logprobs=A, ws=A, n=1 << 40)
    assert L.hl_sample(*{**good, **bad}.values(), None) == status


@pytest.mark.parametrize("field", ["temperature_dev", "top_k_dev", "top_p_dev", "min_p_dev"])
def test_sample_settings_misaligned(L, field):
    settings = hl.Sampling(A, A, A, A, 1.0, 0, 1.0, 0.0)
    setattr(settings, field, A + 2)
    assert L.hl_sample(ctypes.byref(settings), A, hl.HL_F32, 100, 2, 100, A, A, A, A, 1 << 40, None) == hl.HL_EINVAL


def test_sample_workspace(L):
    assert 0 < L.hl_sample_workspace_bytes(1, 1) < L.hl_sample_workspace_bytes(1, 100000) < L.hl_sample_workspace_bytes(9, 100000)
    assert L.hl_sample_workspace_bytes(0, 9) == L.hl_sample_workspace_bytes(9, 0) == L.hl_sample_workspace_bytes(1, 1 << 20) == 0


def test_packed_settings():
    assert hl._SAMPLING.pack(1, 2, 3, 4, 0.5, -6, 0.25, 8.0) == bytes(hl.Sampling(1, 2, 3, 4, 0.5, -6, 0.25, 8.0))


# ---- the binding, with tensors that say they are on GPU 1 and a library that notes its calls

class OnGpu1(torch.Tensor):
    is_cuda = True

    def get_device(self):
        return 1


class Library:
    def __init__(self, current):
        self.current, self.calls = current, []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, self.current[0]))
            return 64 if name.endswith("workspace_bytes") else 0
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
    T.empty = lambda *a, **k: torch.empty(*a, **k).as_subclass(OnGpu1)
    monkeypatch.setattr(hl, "_torch", T)
    monkeypatch.setattr(torch.cuda, "device", device)
    return T.lib, current


def ones(*shape, dtype=torch.float32):
    return torch.ones(shape, dtype=dtype).as_subclass(OnGpu1)


BF16, U8, I32 = torch.bfloat16, torch.uint8, torch.int32


def write_args():
    return dict(k=ones(2, 3, 2, 128, dtype=BF16), v=ones(2, 3, 2, 128, dtype=BF16), cache_k=ones(2, 9, 2, 80, dtype=U8),
                cache_v=ones(2, 9, 2, 80, dtype=U8), lens=ones(2, dtype=I32))


def attention_args():
    return dict(q=ones(2, 1, 4, 128, dtype=BF16), k=ones(2, 9, 2, 80, dtype=U8), v=ones(2, 9, 2, 80, dtype=U8),
                lens=ones(2, dtype=I32), prefix_k=ones(5, 2, 80, dtype=U8), prefix_v=ones(5, 2, 80, dtype=U8),
                weights=ones(2, 2, 9))


def gemv_args():
    return dict(codes=ones(6, 64, dtype=U8), scales=ones(6, 2, dtype=BF16), x=ones(3, 128, dtype=BF16),
                bases=ones(6, 2, dtype=BF16), y=ones(3, 6))


def sample_args():
    return dict(logits=ones(3, 50), uniforms=ones(3), temperature=ones(3), top_k=ones(3, dtype=I32), top_p=0.9, min_p=0.0)


RUNS = [(lambda **m: hl.cache_write4(**{**write_args(), **m}), ["hl_cache_write4"]),
        (lambda **m: hl.cache_read4(**{**dict(cache=ones(2, 9, 2, 80, dtype=U8), dim=128), **m}), ["hl_cache_read4"]),
        (lambda **m: hl.prefix_attention4(**{**attention_args(), **m}),
         ["hl_attention4_workspace_bytes", "hl_prefix_attention4"]),
        (lambda **m: hl.gemv4(**{**gemv_args(), **m}), ["hl_gemv4"]),
        (lambda **m: hl.sample(**{**sample_args(), **m}), ["hl_sample_workspace_bytes", "hl_sample"])]
WRITE, READ, ATTENTION, GEMV, SAMPLE = range(5)


@pytest.mark.parametrize("run,calls", RUNS)
def test_library_is_called_on_the_tensors_gpu(gpus, run, calls):
    library, current = gpus
    run()
    assert library.calls == [(name, 1) for name in calls]
    assert current == [0]


def host(*shape, dtype=torch.float32):
    return torch.ones(shape, dtype=dtype)


@pytest.mark.parametrize("which,bad", [
    (WRITE, dict(k=ones(2, 3, 2, 128))), (WRITE, dict(k=ones(2, 3, 256, dtype=BF16))), (WRITE, dict(v=ones(2, 3, 2, 128))),
    (WRITE, dict(v=ones(2, 2, 2, 128, dtype=BF16))), (WRITE, dict(cache_k=ones(2, 9, 2, 64, dtype=U8))),
    (WRITE, dict(cache_k=ones(2, 9, 2, 40, dtype=BF16))), (WRITE, dict(cache_v=ones(2, 8, 2, 80, dtype=U8))),
    (WRITE, dict(cache_k=ones(3, 9, 2, 80, dtype=U8), cache_v=ones(3, 9, 2, 80, dtype=U8))),
    (WRITE, dict(cache_k=ones(2, 9, 1, 80, dtype=U8), cache_v=ones(2, 9, 1, 80, dtype=U8))),
    (WRITE, dict(lens=ones(2))), (WRITE, dict(lens=ones(3, dtype=I32))), (WRITE, dict(lens=host(2, dtype=I32))),
    (WRITE, dict(cache_k=host(2, 9, 2, 80, dtype=U8))), (WRITE, dict(v=host(2, 3, 2, 128, dtype=BF16))),
    (WRITE, dict(cache_k=ones(1, 9, 2, 80, dtype=U8).expand(2, 9, 2, 80))),
    (WRITE, dict(k=ones(2, 3, 2, 48, dtype=BF16), v=ones(2, 3, 2, 48, dtype=BF16))),
    (WRITE, dict(cache_k=ones(2, 9, 2, 88, dtype=U8)[..., :80])),
    (WRITE, dict(k=ones(2, 3, 128, 2, dtype=BF16).transpose(2, 3))),
    (READ, dict(cache=ones(9, 80, dtype=U8))), (READ, dict(cache=ones(2, 9, 2, 80))), (READ, dict(dim=64)), (READ, dict(dim=100)),
    (READ, dict(dtype=torch.int32)), (READ, dict(out=ones(2, 9, 2, 128), dtype=BF16)), (READ, dict(out=ones(9, 2, 128))),
    (READ, dict(out=host(2, 9, 2, 128))), (READ, dict(cache=host(2, 9, 2, 80, dtype=U8))),
    (READ, dict(cache=ones(0, 2, 80, dtype=U8))), (READ, dict(cache=ones(2, 9, 2, 160, dtype=U8)[..., ::2])),
    (ATTENTION, dict(q=ones(2, 1, 4, 128))), (ATTENTION, dict(q=ones(2, 1, 4, 120, dtype=BF16))),
    (ATTENTION, dict(q=ones(2, 1, 4, 320, dtype=BF16))), (ATTENTION, dict(q=ones(2, 1, 5, 128, dtype=BF16))),
    (ATTENTION, dict(k=ones(2, 9, 2, 128, dtype=BF16))), (ATTENTION, dict(v=None)),
    (ATTENTION, dict(k=ones(2, 9, 2, 64, dtype=U8), v=ones(2, 9, 2, 64, dtype=U8))),
    (ATTENTION, dict(prefix_k=ones(5, 2, 96, dtype=U8), prefix_v=ones(5, 2, 96, dtype=U8))),
    (ATTENTION, dict(prefix_k=ones(5, 4, 80, dtype=U8), prefix_v=ones(5, 4, 80, dtype=U8))), (ATTENTION, dict(lens=None)),
    (ATTENTION, dict(k=ones(2, 9, 2, 88, dtype=U8)[..., :80])), (ATTENTION, dict(weights=ones(2, 2, 8))),
    (ATTENTION, dict(prefix_k=host(5, 2, 80, dtype=U8))),
    (GEMV, dict(codes=ones(6, 64))), (GEMV, dict(codes=ones(384, dtype=U8))), (GEMV, dict(codes=ones(6, 50, dtype=U8))),
    (GEMV, dict(scales=ones(6, 2))), (GEMV, dict(scales=ones(5, 2, dtype=BF16))), (GEMV, dict(scales=ones(6, 8, dtype=BF16))),
    (GEMV, dict(scales=ones(6, 3, dtype=BF16))), (GEMV, dict(x=ones(3, 128))), (GEMV, dict(x=ones(17, 128, dtype=BF16))),
    (GEMV, dict(x=ones(3, 64, dtype=BF16))), (GEMV, dict(bases=ones(6, 2, dtype=torch.float16))),
    (GEMV, dict(bases=ones(6, 4, dtype=BF16))), (GEMV, dict(y=ones(3, 7))), (GEMV, dict(y=ones(6))),
    (GEMV, dict(x=host(3, 128, dtype=BF16))), (GEMV, dict(scales=host(6, 2, dtype=BF16))),
    (GEMV, dict(bases=host(6, 2, dtype=BF16))), (GEMV, dict(codes=ones(64, 6, dtype=U8).t())),
    (GEMV, dict(x=ones(128, 3, dtype=BF16).t())),
    (SAMPLE, dict(logits=ones(3, 50, dtype=I32))), (SAMPLE, dict(logits=ones(3, 5, 10))), (SAMPLE, dict(logits=ones(50, 3).t())),
    (SAMPLE, dict(logits=ones(1, 50).expand(3, 50))), (SAMPLE, dict(logits=host(3, 50))), (SAMPLE, dict(uniforms=ones(2))),
    (SAMPLE, dict(uniforms=host(3))), (SAMPLE, dict(temperature=-1.0)), (SAMPLE, dict(temperature=math.nan)),
    (SAMPLE, dict(top_k=-1)), (SAMPLE, dict(top_p=-0.1)), (SAMPLE, dict(top_p=math.nan)), (SAMPLE, dict(min_p=1.5)),
    (SAMPLE, dict(top_k=ones(3))), (SAMPLE, dict(temperature=ones(3).double())), (SAMPLE, dict(top_p=ones(4))),
    (SAMPLE, dict(min_p=host(3))), (SAMPLE, dict(tokens=ones(3))), (SAMPLE, dict(logprobs=ones(2))),
    (SAMPLE, dict(logits=ones(3, 0))), (SAMPLE, dict(logits=ones(0, 50), uniforms=ones(0)))])
def test_refusals(gpus, which, bad):
    library, current = gpus
    with pytest.raises(ValueError):
        RUNS[which][0](**bad)
    assert library.calls == [] and current == [0]


@pytest.mark.parametrize("run", [r for r, _ in RUNS])
def test_stream_of_another_gpu(gpus, run):
    class Elsewhere:
        device_index, cuda_stream = 0, 0
    with pytest.raises(ValueError):
        run(stream=Elsewhere())
    assert gpus[0].calls == []


@pytest.mark.parametrize("run,calls", RUNS)
def test_named_stream_is_current_during_the_call(gpus, run, calls, monkeypatch):
    now, seen = [None], []

    class Stream:
        device_index, cuda_stream = 1, 77

    @contextlib.contextmanager
    def on(stream):
        before, now[0] = now[0], stream
        try:
            yield
        finally:
            now[0] = before

    monkeypatch.setattr(torch.cuda, "stream", on)
    for name in ("empty", "raw_stream"):
        f = getattr(hl._torch, name)
        monkeypatch.setattr(hl._torch, name, lambda *a, f=f, **k: (seen.append(now[0]), f(*a, **k))[1])
    s = Stream()
    run(stream=s)
    assert seen and all(x is s for x in seen) and now == [None]
