"""ctypes binding of libhufflm.so (argument marshalling only).

Every step of the codec runs in the library: the host encoder in C++, decoding,
the fused decode-GEMV and the operators between the products (norm, attention,
cache eviction) in gfx950 kernels. PyTorch only provides device
memory and the current HIP stream. There is no fallback: if the library is
missing, loading raises.
"""
from __future__ import annotations

import ctypes
import math
import os
import struct
from typing import NamedTuple, Optional

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libhufflm.so")

HL_OK, HL_EINVAL, HL_ENOMEM, HL_ECORRUPT, HL_EUNSUPPORTED, HL_EHIP = range(6)
HL_F32, HL_BF16, HL_F16, HL_E4M3 = 0, 1, 2, 3
HL_FORMAT_SPLIT, HL_FORMAT_WHOLE_EXPONENT, HL_FORMAT_FP16 = 0, 1, 2
HEADER_BYTES = 128
LUT_BYTES = 49440
MAX_BATCH = 16


class HLError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_str(status)} ({status})")


class FieldCode(ctypes.Structure):
    _fields_ = [("nsym", ctypes.c_uint8), ("single", ctypes.c_uint8), ("len", ctypes.c_uint8 * 16)]

    @property
    def lengths(self):
        return list(self.len)


class Codebook(ctypes.Structure):
    _fields_ = [("lmax", ctypes.c_uint32), ("eh", FieldCode), ("el", FieldCode)]


class Codebook8(ctypes.Structure):
    _fields_ = [("lmax", ctypes.c_uint32), ("nsym", ctypes.c_uint16), ("single", ctypes.c_uint8),
                ("reserved", ctypes.c_uint8), ("len", ctypes.c_uint8 * 256)]

    @property
    def lengths(self):
        return list(self.len)


class FieldCode5(ctypes.Structure):
    _fields_ = [("nsym", ctypes.c_uint8), ("single", ctypes.c_uint8), ("len", ctypes.c_uint8 * 32)]

    @property
    def lengths(self):
        return list(self.len)


class Codebook16(ctypes.Structure):
    _fields_ = [("lmax", ctypes.c_uint32), ("e", FieldCode5), ("mh", FieldCode5), ("ml", FieldCode5)]


class TensorView(ctypes.Structure):
    _fields_ = [("blob_dev", ctypes.c_void_p), ("lut_dev", ctypes.c_void_p),
                ("rows", ctypes.c_uint64), ("cols", ctypes.c_uint64), ("n_seg", ctypes.c_uint64),
                ("n_grp", ctypes.c_uint64), ("total_bytes", ctypes.c_uint64),
                ("off_seg_bits", ctypes.c_uint64), ("off_grp_off", ctypes.c_uint64),
                ("off_stream", ctypes.c_uint64), ("off_raw", ctypes.c_uint64),
                ("seg_len", ctypes.c_uint32), ("grp_rows", ctypes.c_uint32), ("lmax", ctypes.c_uint32),
                ("max_grp_units", ctypes.c_uint32), ("max_seg_bits", ctypes.c_uint32),
                ("format", ctypes.c_uint32),
                ("cb", Codebook), ("cb8", Codebook8), ("cb16", Codebook16)]


class KeysValues(ctypes.Structure):
    """hl_kv: keys and values by strides."""
    _fields_ = [("k_dev", ctypes.c_void_p), ("v_dev", ctypes.c_void_p), ("tokens", ctypes.c_uint64),
                ("k_seq", ctypes.c_uint64), ("k_token", ctypes.c_uint64), ("k_head", ctypes.c_uint64),
                ("v_seq", ctypes.c_uint64), ("v_token", ctypes.c_uint64), ("v_head", ctypes.c_uint64)]


class AttentionShape(ctypes.Structure):
    """hl_attention."""
    _fields_ = [("dtype", ctypes.c_int), ("batch", ctypes.c_uint32), ("queries", ctypes.c_uint32),
                ("heads", ctypes.c_uint32), ("kv_heads", ctypes.c_uint32), ("dim", ctypes.c_uint32),
                ("scale", ctypes.c_float), ("prefix", KeysValues), ("own", KeysValues)]


_lib = None

EXPORTS = ["hl_status_str", "hl_default_seg_len", "hl_default_grp_rows", "hl_build_codebook", "hl_encode",
           "hl_build_codebook8", "hl_encode8", "hl_build_codebook16", "hl_encode16", "hl_validate",
           "hl_tensor_view", "hl_tensor_prepare", "hl_decode", "hl_gemv_workspace_bytes",
           "hl_decode_gemv", "hl_decode_gemv_noalloc", "hl_decode_gemv_multi", "hl_gemm_workspace_bytes",
           "hl_decode_gemm",
           "hl_gemv_bf16", "hl_rms_norm", "hl_attention_workspace_bytes", "hl_prefix_attention", "hl_cache_evict"]


def lib() -> ctypes.CDLL:
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with paper_2502_00922_amd/build.py")
    L = ctypes.CDLL(LIB_PATH)
    c = ctypes
    L.hl_status_str.restype = c.c_char_p
    L.hl_status_str.argtypes = [c.c_int]
    L.hl_default_seg_len.restype = c.c_uint32
    L.hl_default_seg_len.argtypes = [c.c_uint64]
    L.hl_default_grp_rows.restype = c.c_uint32
    L.hl_default_grp_rows.argtypes = [c.c_uint64, c.c_uint32]
    L.hl_build_codebook.restype = c.c_int
    L.hl_build_codebook.argtypes = [c.c_void_p, c.c_size_t, c.c_uint32, c.c_uint32, c.POINTER(Codebook)]
    L.hl_encode.restype = c.c_int
    L.hl_encode.argtypes = [c.c_void_p, c.c_uint64, c.c_uint64, c.POINTER(Codebook), c.c_uint32,
                            c.c_uint32, c.c_uint32, c.c_void_p, c.POINTER(c.c_size_t)]
    L.hl_build_codebook8.restype = c.c_int
    L.hl_build_codebook8.argtypes = [c.c_void_p, c.c_size_t, c.c_uint32, c.POINTER(Codebook8)]
    L.hl_encode8.restype = c.c_int
    L.hl_encode8.argtypes = [c.c_void_p, c.c_uint64, c.c_uint64, c.POINTER(Codebook8), c.c_uint32,
                             c.c_uint32, c.c_uint32, c.c_void_p, c.POINTER(c.c_size_t)]
    L.hl_build_codebook16.restype = c.c_int
    L.hl_build_codebook16.argtypes = [c.c_void_p, c.c_size_t, c.c_uint32, c.POINTER(Codebook16)]
    L.hl_encode16.restype = c.c_int
    L.hl_encode16.argtypes = [c.c_void_p, c.c_uint64, c.c_uint64, c.POINTER(Codebook16), c.c_uint32,
                              c.c_uint32, c.c_uint32, c.c_void_p, c.POINTER(c.c_size_t)]
    L.hl_validate.restype = c.c_int
    L.hl_validate.argtypes = [c.c_void_p, c.c_size_t]
    L.hl_tensor_view.restype = c.c_int
    L.hl_tensor_view.argtypes = [c.c_void_p, c.c_void_p, c.c_size_t, c.c_void_p, c.POINTER(TensorView)]
    L.hl_tensor_prepare.restype = c.c_int
    L.hl_tensor_prepare.argtypes = [c.POINTER(TensorView), c.c_void_p]
    L.hl_decode.restype = c.c_int
    L.hl_decode.argtypes = [c.POINTER(TensorView), c.c_void_p, c.c_void_p]
    L.hl_gemv_workspace_bytes.restype = c.c_size_t
    L.hl_gemv_workspace_bytes.argtypes = [c.POINTER(TensorView), c.c_uint32]
    L.hl_decode_gemv.restype = c.c_int
    L.hl_decode_gemv.argtypes = [c.POINTER(TensorView), c.c_void_p, c.c_int, c.c_uint32, c.c_void_p,
                                 c.c_void_p, c.c_size_t, c.c_void_p]
    L.hl_decode_gemv_noalloc.restype = c.c_int
    L.hl_decode_gemv_noalloc.argtypes = [c.POINTER(TensorView), c.c_void_p, c.c_int, c.c_uint32, c.c_void_p,
                                         c.c_void_p]
    L.hl_decode_gemv_multi.restype = c.c_int
    L.hl_decode_gemv_multi.argtypes = [c.c_void_p, c.c_uint32, c.c_void_p, c.c_int, c.c_uint32, c.c_void_p,
                                       c.c_void_p, c.c_size_t, c.c_void_p]
    L.hl_gemm_workspace_bytes.restype = c.c_size_t
    L.hl_gemm_workspace_bytes.argtypes = [c.POINTER(TensorView), c.c_uint32]
    L.hl_decode_gemm.restype = c.c_int
    L.hl_decode_gemm.argtypes = [c.POINTER(TensorView), c.c_void_p, c.c_int, c.c_uint32, c.c_void_p,
                                 c.c_void_p, c.c_size_t, c.c_void_p]
    L.hl_gemv_bf16.restype = c.c_int
    L.hl_gemv_bf16.argtypes = [c.c_void_p, c.c_uint64, c.c_uint64, c.c_void_p, c.c_int, c.c_uint32,
                               c.c_void_p, c.c_void_p]
    L.hl_rms_norm.restype = c.c_int
    L.hl_rms_norm.argtypes = [c.c_void_p, c.c_int, c.c_void_p, c.c_int, c.c_void_p, c.c_int, c.c_uint64, c.c_uint64,
                              c.c_float, c.c_void_p, c.c_void_p, c.c_int, c.c_uint32, c.c_void_p, c.c_void_p]
    L.hl_attention_workspace_bytes.restype = c.c_size_t
    L.hl_attention_workspace_bytes.argtypes = [c.c_void_p, c.c_int]
    L.hl_prefix_attention.restype = c.c_int
    L.hl_prefix_attention.argtypes = [c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p,
                                      c.c_void_p, c.c_void_p, c.c_void_p, c.c_size_t, c.c_void_p]
    L.hl_cache_evict.restype = c.c_int
    L.hl_cache_evict.argtypes = [c.c_void_p, c.c_void_p, c.c_uint32, c.c_uint32, c.c_uint32,
                                 c.c_void_p, c.c_void_p, c.c_uint64, c.c_uint64, c.c_void_p, c.c_void_p, c.c_void_p,
                                 c.c_void_p]
    _lib = L
    return L


def status_str(s: int) -> str:
    return lib().hl_status_str(s).decode()


def _check(s: int, where: str) -> None:
    if s != HL_OK:
        raise HLError(s, where)


def default_seg_len(cols: int) -> int:
    return int(lib().hl_default_seg_len(cols))


PAIR_MAX = 11  # default joint limit of a weight's two exponent codes (the fused kernel's table window)


def build_codebook(w: np.ndarray, lmax: int = 12, pair_max: int = PAIR_MAX) -> Codebook:
    """Codes of the two exponent fields: each at most lmax bits, the pair at
    most pair_max bits (0: no joint limit)."""
    w = np.ascontiguousarray(w, dtype=np.uint16)
    cb = Codebook()
    _check(lib().hl_build_codebook(w.ctypes.data, w.size, lmax, pair_max, ctypes.byref(cb)), "hl_build_codebook")
    return cb


def build_codebook8(w: np.ndarray, lmax: int = 12) -> Codebook8:
    """Whole-exponent code: one 256-symbol code over the exponent bytes."""
    w = np.ascontiguousarray(w, dtype=np.uint16)
    cb = Codebook8()
    _check(lib().hl_build_codebook8(w.ctypes.data, w.size, lmax, ctypes.byref(cb)), "hl_build_codebook8")
    return cb


def build_codebook16(w: np.ndarray, lmax: int = 12) -> Codebook16:
    """Float16 codes: one 32-symbol code per 5-bit field (exponent, mantissa halves)."""
    w = np.ascontiguousarray(w, dtype=np.uint16)
    cb = Codebook16()
    _check(lib().hl_build_codebook16(w.ctypes.data, w.size, lmax, ctypes.byref(cb)), "hl_build_codebook16")
    return cb


def default_grp_rows(cols: int, seg_len: int = 0) -> int:
    return int(lib().hl_default_grp_rows(cols, seg_len))


def encode(w: np.ndarray, seg_len: int = 0, lmax: int = 12, codebook=None,
           nthreads: int = 0, grp_rows: int = 0, whole_exponent: bool = False, fp16: bool = False,
           pair_max: int = PAIR_MAX) -> np.ndarray:
    """HLF1 container (uint8 array) of a bf16 matrix given as uint16 bits [rows, cols].

    whole_exponent selects the format with one 256-symbol exponent code
    (``codebook`` then is a Codebook8); fp16 takes float16 bits and selects the
    {1,5,5,5} format (``codebook``: a Codebook16). pair_max (split format):
    joint limit of a weight's two exponent codes, 0 for none."""
    w = np.ascontiguousarray(w, dtype=np.uint16)
    if w.ndim != 2:
        raise ValueError("expected a 2-D matrix")
    L = lib()
    if fp16:
        cb = codebook if codebook is not None else build_codebook16(w, lmax)
        fn, name = L.hl_encode16, "hl_encode16"
    elif whole_exponent:
        cb = codebook if codebook is not None else build_codebook8(w, lmax)
        fn, name = L.hl_encode8, "hl_encode8"
    else:
        cb = codebook if codebook is not None else build_codebook(w, lmax, pair_max)
        fn, name = L.hl_encode, "hl_encode"
    n = ctypes.c_size_t(0)
    _check(fn(w.ctypes.data, w.shape[0], w.shape[1], ctypes.byref(cb), seg_len, grp_rows, nthreads,
              None, ctypes.byref(n)), name + "(size)")
    out = np.empty(n.value, dtype=np.uint8)
    _check(fn(w.ctypes.data, w.shape[0], w.shape[1], ctypes.byref(cb), seg_len, grp_rows, nthreads,
              out.ctypes.data, ctypes.byref(n)), name)
    return out


def validate(blob) -> int:
    b = np.frombuffer(blob, dtype=np.uint8) if not isinstance(blob, np.ndarray) else blob
    b = np.ascontiguousarray(b)
    return int(lib().hl_validate(b.ctypes.data, b.size))


def _stream_ptr(stream=None):
    """hipStream_t of `stream`, or of the current device's current stream (its
    raw handle: building torch's stream object for it takes 3 us a call)."""
    import torch
    if stream is not None:
        return stream.cuda_stream
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _dev_arg(t, name: str, dtypes=None, shape=None, numel: int = 0):
    """Checks a device buffer's dtype, shape (or at least `numel` elements)
    and contiguity before it reaches a kernel. The C ABI takes no sizes for
    these buffers, so a wrong one would be read or written out of bounds on
    the device; raises ValueError instead."""
    import torch
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name} must be a torch tensor")
    if dtypes is not None and t.dtype not in dtypes:
        raise ValueError(f"{name}: dtype {t.dtype} not in {tuple(dtypes)}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.numel() < numel:
        raise ValueError(f"{name}: {t.numel()} elements, at least {numel} needed")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def _on_device(device, **bufs):
    """Every given buffer lives on `device`, a GPU (else ValueError): a host
    pointer would reach the kernel as a device address."""
    for name, t in bufs.items():
        if t is None or t is False:
            continue
        if not t.is_cuda or (device is not None and t.device != device):
            raise ValueError(f"{name} must be on {device if device is not None else 'the GPU'}, not {t.device}")


def _x_dtype(x):
    import torch
    dt = {torch.float32: HL_F32, torch.bfloat16: HL_BF16, torch.float16: HL_F16}.get(x.dtype)
    if dt is None:
        raise ValueError("x must be float32, bfloat16 or float16")
    return dt


def _check_x(x, K: int):
    """x as a [batch, K] tensor of a supported dtype, batch in 1..16."""
    import torch
    if x.dim() == 1:
        x = x.unsqueeze(0)
    if x.dim() != 2 or x.shape[1] != K or not 1 <= x.shape[0] <= MAX_BATCH:
        raise ValueError(f"x must be [batch <= {MAX_BATCH}, {K}], got {tuple(x.shape)}")
    _dev_arg(x, "x", (torch.float32, torch.bfloat16, torch.float16))
    return x


def _check_ws(ws):
    if ws is False or ws is None:
        return ws
    return _dev_arg(ws, "workspace")


class DeviceTensor:
    """A container resident in device memory plus its decode table."""

    def __init__(self, blob: np.ndarray, device="cuda", stream=None):
        import torch
        blob = np.ascontiguousarray(blob, dtype=np.uint8)
        self.blob = torch.from_numpy(blob).to(device)
        self.lut = torch.empty(LUT_BYTES // 4, dtype=torch.int32, device=device)
        self.view = TensorView()
        _check(lib().hl_tensor_view(self.blob.data_ptr(), blob.ctypes.data, blob.size,
                                    self.lut.data_ptr(), ctypes.byref(self.view)),
               "hl_tensor_view")
        _check(lib().hl_tensor_prepare(ctypes.byref(self.view), _stream_ptr(stream)), "hl_tensor_prepare")

    def copy(self):
        """Another resident copy of the same container and table (device to
        device; the host-side validation of the container is not repeated)."""
        t = DeviceTensor.__new__(DeviceTensor)
        t.blob = self.blob.clone()
        t.lut = self.lut.clone()
        t.view = TensorView.from_buffer_copy(self.view)
        t.view.blob_dev = t.blob.data_ptr()
        t.view.lut_dev = t.lut.data_ptr()
        return t

    @property
    def shape(self):
        return int(self.view.rows), int(self.view.cols)

    @property
    def nbytes(self) -> int:
        return int(self.view.total_bytes)

    def decode(self, out=None, stream=None):
        """Weight bit patterns (bf16, or float16 for the float16 format) as a torch.int16 tensor [rows, cols] on the device."""
        import torch
        R, K = self.shape
        if out is None:
            out = torch.empty((R, K), dtype=torch.int16, device=self.blob.device)
        _dev_arg(out, "out", (torch.int16, torch.bfloat16, torch.float16), numel=R * K)
        _on_device(self.blob.device, out=out)
        _check(lib().hl_decode(ctypes.byref(self.view), out.data_ptr(), _stream_ptr(stream)),
               "hl_decode")
        return out

    def workspace(self, batch: int = MAX_BATCH):
        """Zeroed device workspace for gemv at up to ``batch`` rows (cached)."""
        import torch
        ws = getattr(self, "_ws", None)
        if ws is not None and batch <= getattr(self, "_ws_batch", 0):
            return ws
        need = int(lib().hl_gemv_workspace_bytes(ctypes.byref(self.view), batch))
        if ws is None or ws.numel() < need:
            ws = torch.zeros(max(need, 4), dtype=torch.uint8, device=self.blob.device)
            self._ws = ws
        if 1 <= batch <= MAX_BATCH:  # other batches have no size (0); between these it grows with the batch
            self._ws_batch = batch
        return ws

    def gemv(self, x, y=None, stream=None, workspace=None):
        """y[b, r] = sum_k W[r, k] x[b, k]; x: [batch, cols] float32 or bfloat16 (device).

        ``workspace`` defaults to a cached zeroed buffer owned by this tensor;
        pass False to run without one."""
        import torch
        R, K = self.shape
        dev = self.blob.device
        x = _check_x(x, K)
        dt = _x_dtype(x)
        if y is None:
            y = torch.empty((x.shape[0], R), dtype=torch.float32, device=x.device)
        _dev_arg(y, "y", (torch.float32,), numel=x.shape[0] * R)
        _check_ws(workspace)
        _on_device(dev, x=x, y=y, workspace=workspace)
        if workspace is None:
            workspace = self.workspace()
        ws_ptr, ws_n = ((None, 0) if workspace is False
                        else (workspace.data_ptr(), workspace.numel() * workspace.element_size()))
        _check(lib().hl_decode_gemv(ctypes.byref(self.view), x.data_ptr(), dt, x.shape[0],
                                    y.data_ptr(), ws_ptr, ws_n, _stream_ptr(stream)),
               "hl_decode_gemv")
        return y

    def gemv_noalloc(self, x, y, stream=None):
        """The product of gemv without a workspace (hl_decode_gemv_noalloc):
        the library's per-GPU scratch holds the partial sums. y must be given."""
        import torch
        R, K = self.shape
        x = _check_x(x, K)
        _dev_arg(y, "y", (torch.float32,), numel=x.shape[0] * R)
        _on_device(self.blob.device, x=x, y=y)
        _check(lib().hl_decode_gemv_noalloc(ctypes.byref(self.view), x.data_ptr(), _x_dtype(x),
                                            x.shape[0], y.data_ptr(), _stream_ptr(stream)),
               "hl_decode_gemv_noalloc")
        return y

    def gemm(self, x, y=None, stream=None):
        """Y[n, r] = sum_k W[r, k] X[n, k]; X: [tokens, cols] bfloat16 (device).
        Uses a cached zeroed workspace owned by the tensor, grown as needed."""
        import torch
        R, K = self.shape
        dev = self.blob.device
        if x.dim() != 2 or x.shape[1] != K or x.shape[0] < 1:
            raise ValueError(f"x must be [tokens, {K}], got {tuple(x.shape)}")
        _dev_arg(x, "x", (torch.bfloat16,))
        T = x.shape[0]
        if y is None:
            y = torch.empty((T, R), dtype=torch.float32, device=x.device)
        _dev_arg(y, "y", (torch.float32,), numel=T * R)
        _on_device(dev, x=x, y=y)
        need = int(lib().hl_gemm_workspace_bytes(ctypes.byref(self.view), T))
        ws = getattr(self, "_gemm_ws", None)
        if ws is None or ws.numel() < need:
            ws = torch.zeros(max(need, 4), dtype=torch.uint8, device=self.blob.device)
            self._gemm_ws = ws
        _check(lib().hl_decode_gemm(ctypes.byref(self.view), x.data_ptr(), HL_BF16, T,
                                    y.data_ptr(), ws.data_ptr(), ws.numel(),
                                    _stream_ptr(stream)), "hl_decode_gemm")
        return y


def gemv_multi(tensors, x, ys=None, stream=None, workspace=None):
    """ys[m][b, r] = sum_k W_m[r, k] x[b, k] for up to 4 DeviceTensors with the
    same columns that share x (one grouped launch where the library can).

    ``workspace`` defaults to the largest of the tensors' cached workspaces;
    pass False to run without one."""
    import torch
    if not 1 <= len(tensors) <= 4:
        raise ValueError("one to four tensors")
    K = tensors[0].shape[1]
    dev = tensors[0].blob.device
    if any(t.shape[1] != K or t.blob.device != dev for t in tensors):
        raise ValueError("the tensors must have the same columns and device")
    x = _check_x(x, K)
    dt = _x_dtype(x)
    if ys is None:
        ys = [torch.empty((x.shape[0], t.shape[0]), dtype=torch.float32, device=x.device) for t in tensors]
    if len(ys) != len(tensors):
        raise ValueError("one output per tensor")
    for m, (t, y) in enumerate(zip(tensors, ys)):
        _dev_arg(y, f"ys[{m}]", (torch.float32,), numel=x.shape[0] * t.shape[0])
    _check_ws(workspace)
    _on_device(dev, x=x, workspace=workspace, **{f"ys[{m}]": y for m, y in enumerate(ys)})
    if workspace is None:
        workspace = max((t.workspace() for t in tensors), key=lambda w: w.numel())
    ws_ptr, ws_n = ((None, 0) if workspace is False
                    else (workspace.data_ptr(), workspace.numel() * workspace.element_size()))
    views = (ctypes.c_void_p * len(tensors))(*[ctypes.addressof(t.view) for t in tensors])
    outs = (ctypes.c_void_p * len(tensors))(*[y.data_ptr() for y in ys])
    _check(lib().hl_decode_gemv_multi(views, len(tensors), x.data_ptr(), dt, x.shape[0], outs, ws_ptr, ws_n,
                                      _stream_ptr(stream)), "hl_decode_gemv_multi")
    return ys


def gemv_bf16(w, x, y=None, stream=None):
    """Uncompressed comparator: w [rows, cols] bf16 (or int16 bits) on the device."""
    import torch
    if w.dim() != 2:
        raise ValueError("w must be [rows, cols]")
    R, K = w.shape
    _dev_arg(w, "w", (torch.bfloat16, torch.int16))
    x = _check_x(x, K)
    if x.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("x must be float32 or bfloat16")
    dt = _x_dtype(x)
    if y is None:
        y = torch.empty((x.shape[0], R), dtype=torch.float32, device=x.device)
    _dev_arg(y, "y", (torch.float32,), numel=x.shape[0] * R)
    _on_device(w.device if w.is_cuda else None, w=w, x=x, y=y)
    _check(lib().hl_gemv_bf16(w.data_ptr(), R, K, x.data_ptr(), dt,
                              x.shape[0], y.data_ptr(), _stream_ptr(stream)), "hl_gemv_bf16")
    return y


class NormResult(NamedTuple):
    out: object              # the normalised rows
    sum: Optional[object]    # x + residual, in residual's type (None without one)
    scale: Optional[object]  # of an 8-bit out: [..., hidden / group], or [..., 1] for whole rows


class AttentionResult(NamedTuple):
    out: object
    weights: Optional[object]
    lse: Optional[object]


class EvictResult(NamedTuple):
    k: object
    v: object
    weights: object
    lens: object
    slots: object


class _Torch:
    """What a call of the operators needs of torch and of the library, looked up once: an import statement and the
    attributes' chains cost a small call a tenth of its time."""

    def __init__(self):
        import torch
        self.codes = {torch.float32: HL_F32, torch.bfloat16: HL_BF16, torch.float16: HL_F16,
                      torch.float8_e4m3fn: HL_E4M3}
        self.float32, self.int32, self.uint8 = torch.float32, torch.int32, torch.uint8
        self.half = {torch.bfloat16: HL_BF16, torch.float16: HL_F16}
        self.two_bytes = (torch.bfloat16, torch.float16, torch.int16)
        self.empty, self.empty_like, self.Tensor = torch.empty, torch.empty_like, torch.Tensor
        self.raw_stream = torch._C._cuda_getCurrentRawStream
        self.current_device = torch._C._cuda_getDevice
        self.lib = lib()


_torch = None


def _lookups() -> _Torch:
    global _torch
    if _torch is None:
        _torch = _Torch()
    return _torch


def _plain(device: int, bufs) -> None:
    """Every given buffer is contiguous and on this GPU (get_device's number), else ValueError. A call's checks go
    through here only to say what is wrong: the call itself asks the same in one expression."""
    for name, t in bufs.items():
        if t is None:
            continue
        if t.get_device() != device or not t.is_cuda:
            raise ValueError(f"{name} must be on GPU {device}, not {t.device}")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")


def _on_stream(stream, device: int, f, *args):
    """f(*args) with `stream` as the current one, so that what the call allocates belongs to it as well: memory that
    another stream's work may still use, or get again before this stream has used it, is not touched."""
    if stream.device_index != device:
        raise ValueError(f"stream is on GPU {stream.device_index}, the tensors on {device}")
    import torch
    with torch.cuda.stream(stream):
        return f(*args)


def _on_gpu(device: int, f, *args):
    """f(*args) with this GPU as the current one: a kernel runs on the current GPU, also where its stream is another's
    default stream (whose handle is 0 on each), and a launch is planned for that GPU."""
    import torch
    with torch.cuda.device(device):
        return f(*args)


def rms_norm(x, weight, residual=None, eps: float = 1e-5, out_dtype=None, group: int = 0, out=None, sum_out=None,
             scale_out=None, stream=None) -> NormResult:
    """t = x + residual; out = t / sqrt(mean(t^2) + eps) * weight over the last dimension.

    x and residual: [..., hidden] float32, bfloat16 or float16, contiguous; weight: [hidden]. The sum is kept in
    residual's type (``sum_out`` may be ``residual`` itself). ``out_dtype`` defaults to weight's type;
    torch.float8_e4m3fn gives 8 bits and float32 scales [..., hidden / group], one for each ``group`` columns (32, 64
    or 128), or, with 0, [..., 1], one for each row: ``out.float() * scale`` are the row's values. (``scale_out`` may
    leave that last 1 out; the result's ``scale`` has it.) Outputs that are not given are allocated (on ``stream``,
    where one is given)."""
    if stream is not None:
        return _on_stream(stream, x.get_device(), rms_norm, x, weight, residual, eps, out_dtype, group, out, sum_out,
                          scale_out)
    T = _torch or _lookups()
    types = T.codes
    shape, dev = x.shape, x.get_device()
    if dev >= 0 and dev != T.current_device():
        return _on_gpu(dev, rms_norm, x, weight, residual, eps, out_dtype, group, out, sum_out, scale_out)
    if weight.dim() != 1 or not shape or shape[-1] != weight.shape[0] or x.numel() == 0:
        raise ValueError(f"x must be [..., hidden] and weight [hidden], got {tuple(shape)} and {tuple(weight.shape)}")
    hidden = shape[-1]
    ot = out_dtype if out_dtype is not None else weight.dtype if out is None else out.dtype
    xt, wt, oc = types.get(x.dtype), types.get(weight.dtype), types.get(ot)
    if xt is None or wt is None or oc is None or xt == HL_E4M3 or wt == HL_E4M3:
        raise ValueError("x and weight must be float32, bfloat16 or float16; out these or float8_e4m3fn")
    if out is None:
        out = T.empty_like(x, dtype=ot)
    elif out.dtype != ot or out.shape != shape:
        raise ValueError(f"out must be {tuple(shape)} of {ot}")
    good = dev >= 0 and x.is_contiguous() and weight.is_contiguous() and weight.get_device() == dev \
        and out.is_contiguous() and out.get_device() == dev
    rt, r_ptr, s_ptr, scale_ptr = HL_F32, None, None, None
    if residual is not None:
        rt = types.get(residual.dtype)
        if rt is None or rt == HL_E4M3 or residual.shape != shape:
            raise ValueError(f"residual must have x's shape {tuple(shape)} and be float32, bfloat16 or float16")
        if sum_out is None:
            sum_out = T.empty_like(residual)
        elif sum_out.dtype != residual.dtype or sum_out.shape != shape:
            raise ValueError("sum_out must have residual's shape and type")
        good = good and residual.is_contiguous() and residual.get_device() == dev and sum_out.is_contiguous() \
            and sum_out.get_device() == dev
        r_ptr, s_ptr = residual.data_ptr(), sum_out.data_ptr()
    elif sum_out is not None:
        raise ValueError("sum_out needs a residual")
    if oc == HL_E4M3:
        if group not in (0, 32, 64, 128) or (group and hidden % group):
            raise ValueError("group must be 0, or 32, 64 or 128 and divide hidden")
        need = (*shape[:-1], hidden // group if group else 1)
        if scale_out is None:
            scale_out = T.empty(need, dtype=T.float32, device=x.device)
        elif scale_out.dtype == T.float32 and not group and scale_out.shape == shape[:-1]:
            scale_out = scale_out.unsqueeze(-1)
        elif scale_out.dtype != T.float32 or tuple(scale_out.shape) != need:
            raise ValueError(f"scale_out must be float32 {need}")
        good = good and scale_out.is_contiguous() and scale_out.get_device() == dev
        scale_ptr = scale_out.data_ptr()
    elif group or scale_out is not None:
        raise ValueError("group and scale_out need an 8-bit out")
    if not good:
        _plain(dev, {"x": x, "weight": weight, "out": out, "residual": residual, "sum_out": sum_out,
                     "scale_out": scale_out})
    s = T.lib.hl_rms_norm(x.data_ptr(), xt, r_ptr, rt, weight.data_ptr(), wt, x.numel() // hidden, hidden, eps, s_ptr,
                          out.data_ptr(), oc, group, scale_ptr, T.raw_stream(dev))
    if s:
        _check(s, "hl_rms_norm")
    return NormResult(out, sum_out, scale_out)


def _keys_values(k, v, name: str, dims: int, dtype, device: int):
    """The fields of hl_kv for keys and values [(sequence,) token, key head, column] with any strides but columns in a
    row."""
    if k is None or v is None or k.dim() != dims or v.shape != k.shape:
        raise ValueError(f"{name}: keys and values of one shape, {dims} dimensions")
    if k.dtype != dtype or v.dtype != dtype:
        raise ValueError(f"{name}: dtype {k.dtype} and {v.dtype}, expected {dtype}")
    if k.get_device() != device or v.get_device() != device or device < 0:
        raise ValueError(f"{name} must be on GPU {device}, not {k.device} and {v.device}")
    ks, vs = k.stride(), v.stride()
    if (ks[-1] != 1 or vs[-1] != 1) and k.shape[-1] > 1:
        raise ValueError(f"{name}: the columns of a head must lie next to each other")
    if dims == 3:
        return (k.data_ptr(), v.data_ptr(), k.shape[0], 0, ks[0], ks[1], 0, vs[0], vs[1])
    return (k.data_ptr(), v.data_ptr(), k.shape[1], *ks[:3], *vs[:3])


def _small(t, name: str, dtype, shape, device: int):
    """A contiguous buffer of this type, shape and device (else ValueError)."""
    if not (isinstance(t, _torch.Tensor) and t.dtype == dtype and t.shape == shape and t.is_contiguous()
            and t.get_device() == device):
        _dev_arg(t, name, (dtype,), shape)
        raise ValueError(f"{name} must be on GPU {device}, not {t.device}")
    return t


_NO_KV = (0,) * 9
# hl_attention and hl_kv as bytes: filling them field by field takes longer than a small call's kernels
_ATTENTION = struct.Struct("=i5If4x18Q")
_KV = struct.Struct("=9Q")


def prefix_attention(q, k=None, v=None, lens=None, prefix_k=None, prefix_v=None, scale: Optional[float] = None,
                     weights=None, out=None, weights_out=None, lse=None, stream=None,
                     workspace=None) -> AttentionResult:
    """Attention of new tokens over a prefix shared by the batch and over each sequence's own cache.

    q: [batch, queries, heads, dim] bfloat16 or float16, contiguous. k, v: the own caches
    [batch, capacity, kv_heads, dim] (any strides with columns in a row), of which sequence b's first ``lens[b]``
    (int32) tokens are there, the new ones at their end. prefix_k, prefix_v: [length, kv_heads, dim]. Either set may
    be left out. Token i sees the whole prefix and the own keys before lens[b] - (queries - 1 - i). ``scale`` defaults
    to 1/sqrt(dim).

    ``weights`` (float32 [batch, kv_heads, capacity]) or ``weights_out``: also gives the weights plus what each own
    key was given by this call (``weights_out`` may be ``weights``; without ``weights``, plus zeros). ``lse``: a
    float32 [batch, queries, heads] buffer for the logarithms of the softmax sums. ``workspace``: a device buffer of
    hl_attention_workspace_bytes. Buffers that are not given are allocated (on ``stream``, where one is given)."""
    if stream is not None:
        return _on_stream(stream, q.get_device(), prefix_attention, q, k, v, lens, prefix_k, prefix_v, scale, weights,
                          out, weights_out, lse, None, workspace)
    T = _torch or _lookups()
    dtype = q.dtype
    code = T.half.get(dtype)
    if code is None or q.dim() != 4:
        raise ValueError("q must be [batch, queries, heads, dim] bfloat16 or float16")
    batch, queries, heads, dim = q.shape
    dev = q.get_device()
    if dev < 0 or not q.is_contiguous():
        raise ValueError("q must be contiguous and on the GPU")
    if dev != T.current_device():
        return _on_gpu(dev, prefix_attention, q, k, v, lens, prefix_k, prefix_v, scale, weights, out, weights_out, lse,
                       None, workspace)
    own = prefix = _NO_KV
    kv_heads = lens_ptr = w_ptr = w_out_ptr = lse_ptr = None
    if k is not None or v is not None:
        own = _keys_values(k, v, "k, v", 4, dtype, dev)
        kv_heads = k.shape[2]
        if k.shape[0] != batch or k.shape[3] != dim:
            raise ValueError(f"k, v must be [{batch}, capacity, kv_heads, {dim}], got {tuple(k.shape)}")
        lens_ptr = _small(lens, "lens", T.int32, (batch,), dev).data_ptr()
    if prefix_k is not None or prefix_v is not None:
        prefix = _keys_values(prefix_k, prefix_v, "prefix_k, prefix_v", 3, dtype, dev)
        if prefix_k.shape[2] != dim or (kv_heads is not None and kv_heads != prefix_k.shape[1]):
            raise ValueError(f"prefix_k, prefix_v must be [length, kv_heads, {dim}] with the own caches' kv_heads, "
                             f"got {tuple(prefix_k.shape)}")
        kv_heads = prefix_k.shape[1]
    if not kv_heads or heads % kv_heads:
        raise ValueError("a prefix or own caches are needed, with kv_heads that divide heads")
    if out is None:
        out = T.empty_like(q)
    else:
        _small(out, "out", dtype, q.shape, dev)
    if weights is not None or weights_out is not None:
        if k is None:
            raise ValueError("weights are of the own caches' keys")
        need = (batch, kv_heads, k.shape[1])
        if weights is not None:
            w_ptr = _small(weights, "weights", T.float32, need, dev).data_ptr()
        if weights_out is None:
            weights_out = T.empty(need, dtype=T.float32, device=q.device)
        else:
            _small(weights_out, "weights_out", T.float32, need, dev)
        w_out_ptr = weights_out.data_ptr() if k.shape[1] else None
    if lse is not None:
        lse_ptr = _small(lse, "lse", T.float32, (batch, queries, heads), dev).data_ptr()
    a = _ATTENTION.pack(code, batch, queries, heads, kv_heads, dim,
                        1.0 / math.sqrt(dim) if scale is None else scale, *prefix, *own)
    L = T.lib
    if workspace is None:
        workspace = T.empty(L.hl_attention_workspace_bytes(a, w_out_ptr is not None), dtype=T.uint8, device=q.device)
    else:
        _dev_arg(workspace, "workspace")
        _on_device(q.device, workspace=workspace)
    s = L.hl_prefix_attention(a, q.data_ptr(), lens_ptr, out.data_ptr(), lse_ptr, w_ptr, w_out_ptr,
                              workspace.data_ptr(), workspace.nbytes, T.raw_stream(dev))
    if s:
        _check(s, "hl_prefix_attention")
    return AttentionResult(out, weights_out, lse)


def cache_evict(k, v, weights, lens, keep: int, recent: int = 0, k_out=None, v_out=None, stream=None) -> EvictResult:
    """At most ``keep`` tokens of every sequence and key head, moved in their order to the first slots of another cache:
    the newest ``recent`` and, of the others, those of greatest accumulated weight (ties: the lowest slot).

    k, v: [batch, capacity, kv_heads, dim], 16-bit, any strides with columns in a row; weights: float32
    [batch, kv_heads, capacity]; lens: int32 [batch]. k_out, v_out (default: new ones of capacity ``keep``): caches of
    at least ``keep`` tokens that do not overlap k and v. Gives these, the kept tokens' weights (float32) and slots
    (int32) [batch, kv_heads, keep] - 0 and -1 past the kept ones, whose rows are zeros - and the new lengths, allocated
    (on ``stream``, where one is given)."""
    if stream is not None:
        return _on_stream(stream, k.get_device(), cache_evict, k, v, weights, lens, keep, recent, k_out, v_out)
    T = _torch or _lookups()
    if k.dim() != 4 or k.dtype not in T.two_bytes:
        raise ValueError("k must be [batch, capacity, kv_heads, dim] bfloat16, float16 or int16")
    batch, capacity, heads, dim = k.shape
    dev = k.get_device()
    if dev >= 0 and dev != T.current_device():
        return _on_gpu(dev, cache_evict, k, v, weights, lens, keep, recent, k_out, v_out)
    src = _keys_values(k, v, "k, v", 4, k.dtype, dev)
    if keep < 1 or not 0 <= recent <= keep:
        raise ValueError("keep must be at least 1 and recent between 0 and keep")
    _small(weights, "weights", T.float32, (batch, heads, capacity), dev)
    _small(lens, "lens", T.int32, (batch,), dev)
    if k_out is None and v_out is None:
        k_out = k.new_empty((batch, keep, heads, dim))
        v_out = T.empty_like(k_out)
    dst = _keys_values(k_out, v_out, "k_out, v_out", 4, k.dtype, dev)
    if k_out.shape[0] != batch or k_out.shape[2] != heads or k_out.shape[3] != dim or k_out.shape[1] < keep:
        raise ValueError(f"k_out must be [{batch}, at least {keep}, {heads}, {dim}], got {tuple(k_out.shape)}")
    w_out = weights.new_empty((batch, heads, keep))
    slots = lens.new_empty((batch, heads, keep))
    lens_out = T.empty_like(lens)
    s = T.lib.hl_cache_evict(_KV.pack(*src), _KV.pack(*dst), batch, heads, dim, weights.data_ptr(), lens.data_ptr(),
                             keep, recent, w_out.data_ptr(), slots.data_ptr(), lens_out.data_ptr(), T.raw_stream(dev))
    if s:
        _check(s, "hl_cache_evict")
    return EvictResult(k_out, v_out, w_out, lens_out, slots)
