"""C ABI of the operators between the products: bad arguments come back as status codes before any device work (no GPU:
device addresses here are made up and never read), and the built kernels keep their registers out of memory."""
import ctypes
import os
import re
import subprocess

import pytest

hl = pytest.importorskip("paper_2502_00922_amd.hufflm")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2502_00922_amd", "libhufflm.so")
LLVM = "/opt/rocm/llvm/bin"
A = 0x10000


@pytest.fixture(scope="module")
def L():
    return hl.lib()


NORM = dict(x=A, xt=hl.HL_F32, r=A, rt=hl.HL_BF16, w=A, wt=hl.HL_BF16, tokens=2, hidden=64, eps=1e-5, sum=A, out=A,
            ot=hl.HL_BF16, group=0, scale=A)


@pytest.mark.parametrize("bad,status", [
    (dict(x=None), hl.HL_EINVAL), (dict(w=None), hl.HL_EINVAL), (dict(out=None), hl.HL_EINVAL),
    (dict(sum=None), hl.HL_EINVAL), (dict(tokens=0), hl.HL_EINVAL), (dict(hidden=0), hl.HL_EINVAL),
    (dict(eps=-1.0), hl.HL_EINVAL), (dict(eps=float("nan")), hl.HL_EINVAL), (dict(xt=hl.HL_E4M3), hl.HL_EINVAL),
    (dict(rt=7), hl.HL_EINVAL), (dict(wt=hl.HL_E4M3), hl.HL_EINVAL), (dict(ot=4), hl.HL_EINVAL),
    (dict(group=32), hl.HL_EINVAL), (dict(ot=hl.HL_E4M3, scale=None), hl.HL_EINVAL),
    (dict(ot=hl.HL_E4M3, group=16), hl.HL_EINVAL), (dict(ot=hl.HL_E4M3, group=128), hl.HL_EINVAL),
    (dict(ot=hl.HL_E4M3, group=32, r=A + 2), hl.HL_EINVAL), (dict(x=A + 2), hl.HL_EINVAL), (dict(out=A + 1), hl.HL_EINVAL),
    (dict(hidden=32769), hl.HL_EUNSUPPORTED), (dict(tokens=1 << 31), hl.HL_EUNSUPPORTED)])
def test_norm(L, bad, status):
    assert L.hl_rms_norm(*{**NORM, **bad}.values(), None) == status


def attention(**bad):
    kv = hl.KeysValues(A, A, 100, 100 * 256, 256, 128, 100 * 256, 256, 128)
    a = hl.AttentionShape(hl.HL_BF16, 2, 1, 8, 2, 128, 0.1, kv, hl.KeysValues.from_buffer_copy(kv))
    for name, value in bad.items():
        where, _, field = name.rpartition("__")
        setattr(getattr(a, where) if where else a, field, value)
    return a


@pytest.mark.parametrize("bad,status", [
    (dict(dtype=hl.HL_F32), hl.HL_EINVAL), (dict(batch=0), hl.HL_EINVAL), (dict(queries=0), hl.HL_EINVAL),
    (dict(heads=0), hl.HL_EINVAL), (dict(kv_heads=0), hl.HL_EINVAL), (dict(kv_heads=3), hl.HL_EINVAL),
    (dict(dim=0), hl.HL_EINVAL), (dict(dim=100), hl.HL_EINVAL), (dict(scale=float("nan")), hl.HL_EINVAL),
    (dict(dim=264), hl.HL_EUNSUPPORTED), (dict(own__k_dev=None), hl.HL_EINVAL), (dict(prefix__v_dev=A + 8), hl.HL_EINVAL),
    (dict(own__k_token=132), hl.HL_EINVAL), (dict(own__v_seq=4), hl.HL_EINVAL),
    (dict(prefix__k_token=1 << 25), hl.HL_EUNSUPPORTED), (dict(prefix__tokens=1 << 30), hl.HL_EUNSUPPORTED),
    (dict(batch=70000), hl.HL_EUNSUPPORTED), (dict(queries=1 << 25), hl.HL_EUNSUPPORTED)])
def test_attention_shape(L, bad, status):
    a = attention(**bad)
    args = (ctypes.byref(a), A, A, A, None, None, None, A, 1 << 40, None)
    assert L.hl_prefix_attention(*args) == status
    assert L.hl_attention_workspace_bytes(ctypes.byref(a), 0) == 0


def test_attention_buffers(L):
    a = attention()
    need = L.hl_attention_workspace_bytes(ctypes.byref(a), 0)
    assert 0 < need < L.hl_attention_workspace_bytes(ctypes.byref(a), 1)
    good = dict(q=A, lens=A, out=A, lse=A, w_in=A, w_out=A, ws=A, n=1 << 40)
    for bad in (dict(q=None), dict(q=A + 8), dict(lens=None), dict(lens=A + 2), dict(out=None), dict(out=A + 2),
                dict(lse=A + 1), dict(w_out=None), dict(w_out=A + 2), dict(ws=None), dict(ws=A + 4), dict(n=need)):
        assert L.hl_prefix_attention(ctypes.byref(a), *{**good, **bad}.values(), None) == hl.HL_EINVAL, bad
    assert L.hl_prefix_attention(None, *good.values(), None) == hl.HL_EINVAL
    a = attention(own__tokens=0)
    assert L.hl_prefix_attention(ctypes.byref(a), *good.values(), None) == hl.HL_EINVAL  # weights of no keys
    assert L.hl_attention_workspace_bytes(None, 0) == 0


@pytest.mark.parametrize("bad,status", [
    (dict(batch=0), hl.HL_EINVAL), (dict(heads=0), hl.HL_EINVAL), (dict(dim=0), hl.HL_EINVAL), (dict(dim=12), hl.HL_EINVAL),
    (dict(w=None), hl.HL_EINVAL), (dict(lens=None), hl.HL_EINVAL), (dict(keep=0), hl.HL_EINVAL),
    (dict(recent=21), hl.HL_EINVAL), (dict(keep=101), hl.HL_EINVAL), (dict(w_out=None), hl.HL_EINVAL),
    (dict(slots=A + 2), hl.HL_EINVAL), (dict(lens_out=None), hl.HL_EINVAL), (dict(batch=65536), hl.HL_EUNSUPPORTED)])
def test_evict(L, bad, status):
    kv = hl.KeysValues(A, A, 100, 100 * 256, 256, 128, 100 * 256, 256, 128)
    good = dict(src=ctypes.byref(kv), dst=ctypes.byref(kv), batch=2, heads=2, dim=128, w=A, lens=A, keep=20, recent=4, w_out=A,
                slots=A, lens_out=A)
    assert L.hl_cache_evict(*{**good, **bad}.values(), None) == status
    for field, value in (("k_dev", None), ("v_dev", A + 8), ("tokens", 0), ("k_token", 4), ("v_seq", 1 << 41)):
        other = hl.KeysValues.from_buffer_copy(kv)
        setattr(other, field, value)
        for side in ("src", "dst"):
            got = L.hl_cache_evict(*{**good, side: ctypes.byref(other)}.values(), None)
            assert got == (hl.HL_EUNSUPPORTED if field == "v_seq" else hl.HL_EINVAL)
        assert L.hl_cache_evict(*{**good, "src": None}.values(), None) == hl.HL_EINVAL


def test_packed_structures():
    # the bytes that the binding packs are the structures' own
    kv = hl.KeysValues(*range(1, 10))
    assert hl._KV.pack(*range(1, 10)) == bytes(kv)
    a = hl.AttentionShape(hl.HL_F16, 2, 3, 4, 5, 6, 0.25, kv, hl.KeysValues(*range(11, 20)))
    assert hl._ATTENTION.pack(hl.HL_F16, 2, 3, 4, 5, 6, 0.25, *range(1, 10), *range(11, 20)) == bytes(a)


def test_registers(tmp_path):
    # every code object of the library, not the first alone
    fat = str(tmp_path / "fat")
    subprocess.run([f"{LLVM}/llvm-objcopy", f"--dump-section=.hip_fatbin={fat}", LIB, str(tmp_path / "copy")], check=True)
    data, seen = open(fat, "rb").read(), {}
    starts = [m.start() for m in re.finditer(b"__CLANG_OFFLOAD_BUNDLE__", data)]
    for i, at in enumerate(starts):
        part, obj = str(tmp_path / f"part{i}"), str(tmp_path / f"obj{i}")
        with open(part, "wb") as f:
            f.write(data[at:starts[i + 1] if i + 1 < len(starts) else len(data)])
        subprocess.run([f"{LLVM}/clang-offload-bundler", "--unbundle", "--type=o", f"--input={part}", f"--output={obj}",
                        "--targets=hipv4-amdgcn-amd-amdhsa--gfx950"], check=True)
        notes = subprocess.run([f"{LLVM}/llvm-readelf", "--notes", obj], check=True, capture_output=True, text=True).stdout
        for m in re.finditer(r"\.name:\s+(\S+)(.*?)\.vgpr_spill_count:\s+(\d+)", notes, re.S):
            private = int(re.search(r"\.private_segment_fixed_size:\s+(\d+)", m.group(2)).group(1))
            seen[m.group(1)] = (int(m.group(3)), private)
    for kernel in ("norm_kernel", "parts_kernel", "join_kernel", "weights_kernel", "select_kernel", "move_kernel"):
        mine = {n: s for n, s in seen.items() if kernel in n and "hl" in n}
        assert mine, kernel
        assert all(s == (0, 0) for s in mine.values()), mine
