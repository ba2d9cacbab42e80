"""ctypes binding of libgsrq.so (the C ABI in include/gsrq.h).

Argument marshalling only: every step of the GSRQ path runs in the HIP
kernels of the library.  torch supplies device memory and the stream; a torch
tensor is passed as its data pointer.  If the library is not built, importing
functions from here raises instead of falling back to anything else.
"""
from __future__ import annotations

import ctypes
import math
import os
import struct
from dataclasses import dataclass
from typing import Optional

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgsrq.so")

GSRQ_OK, GSRQ_E_ARG, GSRQ_E_UNSUPPORTED, GSRQ_E_WORKSPACE, GSRQ_E_HIP = range(5)
GSRQ_F32, GSRQ_F16, GSRQ_BF16, GSRQ_E4M3 = 0, 1, 2, 3
GSRQ_RESUME, GSRQ_ASSIGN_IN, GSRQ_NO_EARLY_STOP, GSRQ_KMEANS, GSRQ_CHECK_INPUTS = 1, 2, 4, 8, 16


class GsrqError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


class Shape(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int64), ("D", ctypes.c_int32), ("d", ctypes.c_int32),
                ("K", ctypes.c_int32), ("M", ctypes.c_int32)]


class AttnShape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("cap", ctypes.c_int32), ("Hq", ctypes.c_int32),
                ("Hkv", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("rope_base", ctypes.c_float), ("scale", ctypes.c_float),
                ("flags", ctypes.c_uint32)]


class Pages(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_stride", ctypes.c_int64 * 3),
                ("v_stride", ctypes.c_int64 * 3), ("table", ctypes.c_void_p),
                ("ldt", ctypes.c_int64), ("pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("per", ctypes.c_int32), ("B", ctypes.c_int32), ("Hkv", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int)]


class Heads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64)]


class PageExps(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_stride", ctypes.c_int64 * 2),
                ("v_stride", ctypes.c_int64 * 2)]


class PagedBatch(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int64), ("ldt", ctypes.c_int64), ("B", ctypes.c_int32),
                ("per", ctypes.c_int32), ("page_size", ctypes.c_int32), ("F", ctypes.c_int32)]


class PagedAttn(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int64), ("Hq", ctypes.c_int32), ("window", ctypes.c_int32),
                ("scale", ctypes.c_float), ("flags", ctypes.c_uint32)]


_lib = None
_vp = ctypes.c_void_p


def load_library(path: str = LIB_PATH):
    """Load libgsrq.so once; raise if it is missing (no fallback exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is not built; run `python -c 'import __graft_entry__ as g; g.build()'`")
    # torch first: the library then binds to the HIP runtime torch ships and
    # uses, instead of loading a second runtime that cannot see torch's
    # device memory
    _torch()
    lib = ctypes.CDLL(path)
    SP = ctypes.POINTER(Shape)
    lib.gsrq_status_string.restype = ctypes.c_char_p
    lib.gsrq_status_string.argtypes = [ctypes.c_int]
    lib.gsrq_code_words.restype = ctypes.c_size_t
    lib.gsrq_code_words.argtypes = [SP]
    lib.gsrq_bits_per_element.restype = ctypes.c_double
    lib.gsrq_bits_per_element.argtypes = [SP]
    lib.gsrq_train_workspace_bytes.restype = ctypes.c_int
    lib.gsrq_train_workspace_bytes.argtypes = [SP, ctypes.POINTER(ctypes.c_size_t)]
    lib.gsrq_encode_workspace_bytes.restype = ctypes.c_int
    lib.gsrq_encode_workspace_bytes.argtypes = [SP, ctypes.POINTER(ctypes.c_size_t)]
    lib.gsrq_train_stage.restype = ctypes.c_int
    lib.gsrq_train_stage.argtypes = [SP, _vp, ctypes.c_int, ctypes.c_int64, _vp, ctypes.c_int32,
                                     _vp, ctypes.c_uint32, _vp, _vp, _vp, _vp, _vp, _vp,
                                     _vp, ctypes.c_size_t, _vp]
    lib.gsrq_encode.restype = ctypes.c_int
    lib.gsrq_encode.argtypes = [SP, _vp, ctypes.c_int, ctypes.c_int64, _vp, _vp, _vp, _vp,
                                _vp, ctypes.c_size_t, _vp]
    lib.gsrq_prepared_bytes.restype = ctypes.c_int
    lib.gsrq_prepared_bytes.argtypes = [SP, ctypes.POINTER(ctypes.c_size_t)]
    lib.gsrq_encode_prepare.restype = ctypes.c_int
    lib.gsrq_encode_prepare.argtypes = [SP, _vp, _vp, _vp, ctypes.c_size_t, _vp]
    lib.gsrq_encode_prepared.restype = ctypes.c_int
    lib.gsrq_encode_prepared.argtypes = [SP, _vp, ctypes.c_int, ctypes.c_int64, _vp, _vp, _vp,
                                         _vp]
    lib.gsrq_decode.restype = ctypes.c_int
    lib.gsrq_decode.argtypes = [SP, _vp, ctypes.c_int32, _vp, _vp, _vp, ctypes.c_int,
                                ctypes.c_int64, _vp]
    lib.gsrq_row_weights.restype = ctypes.c_int
    lib.gsrq_row_weights.argtypes = [_vp, ctypes.c_int, ctypes.c_int64, ctypes.c_int32,
                                     ctypes.c_int64, ctypes.c_float, _vp, _vp, _vp, _vp]
    AP = ctypes.POINTER(AttnShape)
    lib.gsrq_attn_workspace_bytes.restype = ctypes.c_int
    lib.gsrq_attn_workspace_bytes.argtypes = [AP, ctypes.POINTER(ctypes.c_size_t)]
    lib.gsrq_attn_workspace_bytes_kv.restype = ctypes.c_int
    lib.gsrq_attn_workspace_bytes_kv.argtypes = [AP, SP, ctypes.POINTER(ctypes.c_size_t)]
    lib.gsrq_attn_decode.restype = ctypes.c_int
    lib.gsrq_attn_decode.argtypes = [AP, SP, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                     ctypes.c_int, _vp, _vp, ctypes.c_size_t, _vp]
    lib.gsrq_attn_decode_noalloc.restype = ctypes.c_int
    lib.gsrq_attn_decode_noalloc.argtypes = [AP, SP, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                             ctypes.c_int, _vp, _vp]
    PP = HP = XP = _vp               # packed structures, or byref() of Pages, Heads, PagedAttn
    lib.gsrq_paged_append.restype = ctypes.c_int
    lib.gsrq_paged_append.argtypes = [PP, ctypes.c_int64, _vp, _vp, HP, HP, HP, ctypes.c_int32,
                                      ctypes.c_int, _vp, _vp, _vp, ctypes.c_float, _vp, _vp]
    lib.gsrq_paged_restore.restype = ctypes.c_int
    lib.gsrq_paged_restore.argtypes = [PP, SP, ctypes.c_int32, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                       _vp, _vp]
    lib.gsrq_paged_append8.restype = ctypes.c_int
    lib.gsrq_paged_append8.argtypes = [PP, _vp, ctypes.c_int64, _vp, _vp, HP, HP, HP,
                                       ctypes.c_int32, ctypes.c_int, _vp, _vp, _vp, ctypes.c_float,
                                       _vp, ctypes.c_int, _vp]
    lib.gsrq_attn_paged8_workspace_bytes.restype = ctypes.c_int
    lib.gsrq_attn_paged8_workspace_bytes.argtypes = [XP, PP, ctypes.POINTER(ctypes.c_size_t)]
    lib.gsrq_attn_paged8.restype = ctypes.c_int
    lib.gsrq_attn_paged8.argtypes = [XP, PP, _vp, _vp, _vp, HP, ctypes.c_int, _vp, _vp, _vp,
                                     ctypes.c_size_t, _vp]
    lib.gsrq_paged_plan.restype = ctypes.c_int
    lib.gsrq_paged_plan.argtypes = [_vp] * 10
    lib.gsrq_verify_drafts_workspace_bytes.restype = ctypes.c_int
    lib.gsrq_verify_drafts_workspace_bytes.argtypes = [ctypes.c_int64, ctypes.c_int64,
                                                       ctypes.c_int32,
                                                       ctypes.POINTER(ctypes.c_size_t)]
    lib.gsrq_verify_drafts.restype = ctypes.c_int
    lib.gsrq_verify_drafts.argtypes = [ctypes.c_int64, ctypes.c_int64, ctypes.c_int32, _vp, _vp,
                                       ctypes.c_int64, _vp, ctypes.c_int64, ctypes.c_int, _vp,
                                       _vp, _vp, _vp, _vp, _vp, ctypes.c_size_t, _vp]
    lib.gsrq_attn_paged_workspace_bytes.restype = ctypes.c_int
    lib.gsrq_attn_paged_workspace_bytes.argtypes = [XP, PP, ctypes.POINTER(ctypes.c_size_t)]
    lib.gsrq_attn_paged.restype = ctypes.c_int
    lib.gsrq_attn_paged.argtypes = [XP, PP, _vp, _vp, HP, _vp, _vp, _vp, ctypes.c_size_t, _vp]
    lib.gsrq_timing_enable.restype = ctypes.c_int
    lib.gsrq_timing_enable.argtypes = [ctypes.c_int]
    lib.gsrq_timing_enable_kinds.restype = ctypes.c_int
    lib.gsrq_timing_enable_kinds.argtypes = [ctypes.c_uint32]
    lib.gsrq_timing_read.restype = ctypes.c_int
    lib.gsrq_timing_read.argtypes = [ctypes.POINTER(ctypes.c_double),
                                     ctypes.POINTER(ctypes.c_int64), ctypes.c_int]
    _lib = lib
    return lib


KERNEL_KINDS = ("assign", "finalize", "encode", "decode", "transpose", "accumulate",
                "fragments", "exact", "attention", "append", "serving")


def timing_enable(on: bool = True, kinds=None):
    """Bracket kernel launches with HIP events on their stream (measurement):
    every kind, or only the named ones (names from KERNEL_KINDS)."""
    if kinds is None:
        _check(load_library().gsrq_timing_enable(1 if on else 0), "gsrq_timing_enable")
        return
    mask = 0
    for k in kinds:
        mask |= 1 << KERNEL_KINDS.index(k)
    _check(load_library().gsrq_timing_enable_kinds(ctypes.c_uint32(mask if on else 0)),
           "gsrq_timing_enable_kinds")


def timing_read():
    """{kind: (total_ms, launches)} for the launches recorded since enabling."""
    n = len(KERNEL_KINDS)
    ms = (ctypes.c_double * n)()
    cnt = (ctypes.c_int64 * n)()
    _check(load_library().gsrq_timing_read(ms, cnt, n), "gsrq_timing_read")
    return {k: (float(ms[i]), int(cnt[i])) for i, k in enumerate(KERNEL_KINDS)}


def status_string(status: int) -> str:
    return load_library().gsrq_status_string(int(status)).decode()


def _check(status: int, where: str):
    if status != GSRQ_OK:
        raise GsrqError(status, where)


def make_shape(N, D, d, K, M=1) -> Shape:
    return Shape(int(N), int(D), int(d), int(K), int(M))


def code_words(N, D, d, K, M) -> int:
    return int(load_library().gsrq_code_words(ctypes.byref(make_shape(N, D, d, K, M))))


def bits_per_element(d, K, M, D=None) -> float:
    D = d if D is None else D
    return float(load_library().gsrq_bits_per_element(ctypes.byref(make_shape(1, D, d, K, M))))


def train_workspace_bytes(N, D, d, K) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().gsrq_train_workspace_bytes(ctypes.byref(make_shape(N, D, d, K, 1)),
                                                      ctypes.byref(n)), "train_workspace_bytes")
    return int(n.value)


def encode_workspace_bytes(N, D, d, K, M) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().gsrq_encode_workspace_bytes(ctypes.byref(make_shape(N, D, d, K, M)),
                                                       ctypes.byref(n)), "encode_workspace_bytes")
    return int(n.value)


# ------------------------------------------------------------ torch plumbing

_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _ptr(t) -> Optional[int]:
    return None if t is None else int(t.data_ptr())


def _stream_handle(stream) -> Optional[int]:
    s = _torch().cuda.current_stream() if stream is None else stream
    return int(s.cuda_stream) or None


def _append_stream_handle(stream) -> Optional[int]:
    """_stream_handle for the call of every decoding step: the handle of the
    current stream without a Stream object (a microsecond of a call's seven),
    where this torch has the calls that give it."""
    C = _torch()._C
    raw, device = getattr(C, "_cuda_getCurrentRawStream", None), getattr(C, "_cuda_getDevice", None)
    if stream is not None or raw is None or device is None:
        return _stream_handle(stream)
    return raw(device()) or None


def _dtype_code(t) -> int:
    torch = _torch()
    dtype = t.dtype
    if dtype == torch.float16:
        return GSRQ_F16
    if dtype == torch.float32:
        return GSRQ_F32
    raise TypeError(f"unsupported dtype {dtype}; float16 or float32 expected")


def _rows(X):
    stride = X.stride()
    if len(stride) != 2 or stride[1] != 1:
        raise ValueError("X must be a 2-D tensor with unit column stride")
    N, D = X.shape
    return N, D, stride[0]


def _need(t, name, dtypes, device, shape=None):
    """Check a tensor argument passed as a dense pointer: dtype, device,
    contiguity and (optionally) shape; None passes."""
    if t is None:
        return
    if t.dtype not in dtypes:
        raise TypeError(f"{name} must be {' or '.join(str(d) for d in dtypes)}, not {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if shape is not None and t.numel() != math.prod(shape):
        raise ValueError(f"{name} has {t.numel()} elements, expected {tuple(shape)}")


def _workspace(nbytes, device, workspace):
    torch = _torch()
    if workspace is not None:
        if workspace.numel() * workspace.element_size() < nbytes:
            raise ValueError("workspace too small")
        return workspace
    # torch's caching allocator returns 512-byte aligned blocks
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)


@dataclass
class TrainResult:
    gain: object          # [G, K] float32
    shape: object         # [G, K, d] float32
    assign: object        # [G, N] int16 holding uint16 codes
    iters: object         # [G] int32
    trace: object         # [G, T] float64 or None
    residual: object      # [N, D] float32 or None
    seed_rows: object = None  # host table kept alive with the results


def train_stage(X, d, K, T, seed_rows=None, w=None, *, gain=None, shape=None, assign=None,
                resume=False, assign_in=False, no_early_stop=False, residual=False,
                trace=True, kmeans=False, check_inputs=False, workspace=None,
                stream=None) -> TrainResult:
    """One stage of weighted GSKM on device tensor X [N, D] (see gsrq_train_stage).

    residual: True for a new R_next tensor, or an [N, D] float32 tensor to
    write it into.  kmeans: the K-means baseline (GSRQ_KMEANS) instead of
    GSKM; its centroids are gain[:, :, None] * shape.  check_inputs: the
    device check of GSRQ_CHECK_INPUTS (weights, finite X, nonzero seeds;
    the call then waits for the stream)."""
    torch = _torch()
    lib = load_library()
    N, D, ldx = _rows(X)
    G = D // d if d > 0 and D % d == 0 else 0
    dev = X.device
    _need(w, "w", (torch.float32,), dev, (N,))
    _need(gain, "gain", (torch.float32,), dev, (G, K))
    _need(shape, "shape", (torch.float32,), dev, (G, K, d))
    _need(assign, "assign", (torch.int16, torch.uint16), dev, (G, N))
    if residual is not True and residual is not False and residual is not None:
        _need(residual, "residual", (torch.float32,), dev, (N, D))
    if gain is None:
        gain = torch.empty((max(G, 1), K), dtype=torch.float32, device=dev)
    if shape is None:
        shape = torch.empty((max(G, 1), K, d), dtype=torch.float32, device=dev)
    if assign is None:
        assign = torch.empty((max(G, 1), N), dtype=torch.int16, device=dev)
    iters = torch.empty(max(G, 1), dtype=torch.int32, device=dev)
    tr = torch.empty((max(G, 1), max(T, 1)), dtype=torch.float64, device=dev) if trace and T > 0 else None
    if residual is True:
        res = torch.empty((N, D), dtype=torch.float32, device=dev)
    else:   # False / None, or an [N, D] float32 output tensor
        res = residual if residual is not False else None
    seeds = None
    if seed_rows is not None:
        seeds = np.ascontiguousarray(np.asarray(seed_rows), dtype=np.int32)
    flags = ((GSRQ_RESUME if resume else 0) | (GSRQ_ASSIGN_IN if assign_in else 0)
             | (GSRQ_NO_EARLY_STOP if no_early_stop else 0) | (GSRQ_KMEANS if kmeans else 0)
             | (GSRQ_CHECK_INPUTS if check_inputs else 0))
    sh = make_shape(N, D, d, K, 1)
    n = ctypes.c_size_t(0)
    st = lib.gsrq_train_workspace_bytes(ctypes.byref(sh), ctypes.byref(n))
    _check(st, "gsrq_train_workspace_bytes")
    ws = _workspace(n.value, dev, workspace)
    st = lib.gsrq_train_stage(
        ctypes.byref(sh), _ptr(X), _dtype_code(X), ldx, _ptr(w), int(T),
        None if seeds is None else seeds.ctypes.data, flags, _ptr(gain), _ptr(shape),
        _ptr(res), _ptr(assign), _ptr(iters), _ptr(tr), _ptr(ws),
        ws.numel() * ws.element_size(), _stream_handle(stream))
    _check(st, "gsrq_train_stage")
    return TrainResult(gain, shape, assign, iters, tr, res, seeds)


def encode(X, gain, shape, *, codes=None, residual=False, workspace=None, stream=None):
    """Stage-fused encode of device tensor X [N, D] with codebooks
    gain [M, G, K], shape [M, G, K, d].  Returns (codes [N, W] int32 words
    holding uint32 bit fields, residual [N, D] float32 or None)."""
    torch = _torch()
    lib = load_library()
    N, D, ldx = _rows(X)
    M, G, K = gain.shape
    d = shape.shape[-1]
    _need(gain, "gain", (torch.float32,), X.device)
    _need(shape, "shape", (torch.float32,), X.device, (M, G, K, d))
    sh = make_shape(N, D, d, K, M)
    W = int(lib.gsrq_code_words(ctypes.byref(sh)))
    _need(codes, "codes", (torch.int32, torch.uint32), X.device, (N, max(W, 1)))
    if codes is None:
        codes = torch.empty((N, max(W, 1)), dtype=torch.int32, device=X.device)
    res = torch.empty((N, D), dtype=torch.float32, device=X.device) if residual else None
    n = ctypes.c_size_t(0)
    _check(lib.gsrq_encode_workspace_bytes(ctypes.byref(sh), ctypes.byref(n)),
           "gsrq_encode_workspace_bytes")
    ws = _workspace(n.value, X.device, workspace)
    st = lib.gsrq_encode(ctypes.byref(sh), _ptr(X), _dtype_code(X), ldx, _ptr(gain),
                         _ptr(shape), _ptr(codes), _ptr(res), _ptr(ws),
                         ws.numel() * ws.element_size(), _stream_handle(stream))
    _check(st, "gsrq_encode")
    return codes, res


@dataclass
class Prepared:
    """A prepared codebook (gsrq_encode_prepare): the device buffer and the
    shape it was built for."""
    buf: object
    D: int
    d: int
    K: int
    M: int


def prepare_codebook(gain, shape, *, stream=None) -> Prepared:
    """Prepared codebook of gain [M, G, K], shape [M, G, K, d] (narrow
    family, d <= 8, K <= 256) for encode_prepared."""
    torch = _torch()
    lib = load_library()
    M, G, K = gain.shape
    d = shape.shape[-1]
    _need(gain, "gain", (torch.float32,), gain.device)
    _need(shape, "shape", (torch.float32,), gain.device, (M, G, K, d))
    sh = make_shape(1, G * d, d, K, M)
    n = ctypes.c_size_t(0)
    _check(lib.gsrq_prepared_bytes(ctypes.byref(sh), ctypes.byref(n)), "gsrq_prepared_bytes")
    buf = torch.empty(n.value, dtype=torch.uint8, device=gain.device)
    _check(lib.gsrq_encode_prepare(ctypes.byref(sh), _ptr(gain), _ptr(shape), _ptr(buf), n.value,
                                   _stream_handle(stream)), "gsrq_encode_prepare")
    return Prepared(buf, G * d, d, K, M)


def encode_prepared(X, prep: Prepared, *, codes=None, residual=False, stream=None):
    """encode() with a prepared codebook (no operand-table build per call).

    The call of every decoding step: a few microseconds of kernel, so its
    Python work is kept short (the code words per row come from integer
    arithmetic, and a codes tensor made here needs no checks)."""
    torch = _torch()
    lib = _lib or load_library()
    N, D, ldx = _rows(X)
    if D != prep.D:
        raise ValueError("X does not match the prepared codebook's vector length")
    dtype = _dtype_code(X)
    d, K, M = int(prep.d), int(prep.K), int(prep.M)
    sh = Shape(N, D, d, K, M)
    # gsrq_code_words: ceil(M G log2(K) / 32) (invalid shapes: the call's error)
    W = max(-(-M * (D // d) * (K.bit_length() - 1) // 32), 1) if d > 0 else 1
    if codes is None:
        codes = torch.empty((N, W), dtype=torch.int32, device=X.device)
    else:
        _need(codes, "codes", (torch.int32, torch.uint32), X.device, (N, W))
    res = torch.empty((N, D), dtype=torch.float32, device=X.device) if residual else None
    st = lib.gsrq_encode_prepared(ctypes.byref(sh), X.data_ptr(), dtype, ldx, prep.buf.data_ptr(),
                                  codes.data_ptr(), _ptr(res), _append_stream_handle(stream))
    if st != GSRQ_OK:
        _check(st, "gsrq_encode_prepared")
    return codes, res


def decode(codes, gain, shape, D, M_use=None, *, out_dtype=None, out=None, stream=None):
    """Gather-sum decode of packed codes [N, W] with codebooks gain [M, G, K],
    shape [M, G, K, d] into [N, D] (float16 by default)."""
    torch = _torch()
    lib = load_library()
    M, G, K = gain.shape
    d = shape.shape[-1]
    N = codes.shape[0]
    M_use = M if M_use is None else int(M_use)
    dev = codes.device
    _need(codes, "codes", (torch.int32, torch.uint32), dev)
    _need(gain, "gain", (torch.float32,), dev)
    _need(shape, "shape", (torch.float32,), dev, (M, G, K, d))
    if out is None:
        out = torch.empty((N, D), dtype=out_dtype or torch.float16, device=dev)
    elif out.dim() != 2 or out.stride(1) != 1 or out.device != dev or tuple(out.shape) != (N, D):
        raise ValueError("out must be an [N, D] tensor with unit column stride on the codes' device")
    sh = make_shape(N, D, d, K, M)
    st = lib.gsrq_decode(ctypes.byref(sh), _ptr(codes), M_use, _ptr(gain), _ptr(shape),
                         _ptr(out), _dtype_code(out), out.stride(0), _stream_handle(stream))
    _check(st, "gsrq_decode")
    return out


def row_weights(grad=None, *, norms=None, tau=1.0, stream=None):
    """Per-token weights of Sec. 5.3 / Appendix B (see gsrq_row_weights):
    from gradient rows grad [N, D] (float16/float32), or from precomputed
    norms [N] float32 when grad is None.  Returns (w [N], norms [N],
    stats [2] float64 = (median, lambda))."""
    torch = _torch()
    lib = load_library()
    if grad is not None:
        N, D, ldg = _rows(grad)
        dev = grad.device
        if norms is None:
            norms = torch.empty(N, dtype=torch.float32, device=dev)
        dt = _dtype_code(grad)
    else:
        if norms is None:
            raise ValueError("either grad or norms is needed")
        N, D, ldg, dev, dt = norms.shape[0], 0, 0, norms.device, GSRQ_F32
    w = torch.empty(N, dtype=torch.float32, device=dev)
    stats = torch.empty(2, dtype=torch.float64, device=dev)
    st = lib.gsrq_row_weights(_ptr(grad), dt, N, D, ldg, float(tau), _ptr(norms), _ptr(w),
                              _ptr(stats), _stream_handle(stream))
    _check(st, "gsrq_row_weights")
    return w, norms, stats


GSRQ_ATTN_TABLES_READY = 1


def make_attn_shape(B, cap, Hq, Hkv, head_dim=128, rope_base=500000.0, scale=None,
                    flags=0) -> AttnShape:
    scale = 1.0 / math.sqrt(head_dim) if scale is None else float(scale)
    return AttnShape(int(B), int(cap), int(Hq), int(Hkv), int(head_dim), float(rope_base), scale,
                     int(flags))


def attn_workspace_bytes(B, cap, Hq, Hkv, head_dim=128, *, d=8, M=1) -> int:
    """Workspace of gsrq_attn_decode for codes of subvector length d and M
    stages (d = 8, M = 1: the 1-bit layout; d = head_dim: residual-coded)."""
    n = ctypes.c_size_t()
    sh = make_attn_shape(B, cap, Hq, Hkv, head_dim)
    kv = make_shape(B * cap, Hkv * head_dim, d, 256, M)
    _check(load_library().gsrq_attn_workspace_bytes_kv(ctypes.byref(sh), ctypes.byref(kv),
                                                       ctypes.byref(n)),
           "gsrq_attn_workspace_bytes_kv")
    return int(n.value)


ATTN_NOALLOC_BYTES = 16 << 20


def attn_decode(k_codes, v_codes, seq_len, k_gain, k_shape, v_gain, v_shape, q, *,
                rope_base=500000.0, scale=None, out=None, workspace=None, stream=None,
                tables_ready=False, noalloc=False):
    """One decoding step of attention over coded caches (see gsrq_attn_decode).
    k_codes, v_codes [B, cap, W] packed codes; seq_len [B] int32; codebooks
    [M, G, 256] / [M, G, 256, d] (the 1-bit layout d = 8, M = 1, or the
    residual-coded one d = 128, M <= 16); q [B, Hq, 128] (float16/float32).  Returns
    out [B, Hq, 128] float32.  tables_ready: the given workspace holds the
    tables of these codebooks from an earlier call (GSRQ_ATTN_TABLES_READY).
    noalloc: gsrq_attn_decode_noalloc (the library's per-GPU scratch instead
    of a workspace; workspace must then be None)."""
    torch = _torch()
    lib = load_library()
    B, cap, W = k_codes.shape
    Hq, hd = q.shape[1], q.shape[2]
    M, G, K = k_gain.shape
    d = k_shape.shape[-1]
    D = G * d
    Hkv = D // hd
    for t in (k_codes, v_codes, seq_len, k_gain, k_shape, v_gain, v_shape, q):
        if not t.is_contiguous():
            raise ValueError("attn_decode expects contiguous tensors")
    if tuple(v_codes.shape) != (B, cap, W) or q.shape[0] != B or seq_len.numel() != B:
        raise ValueError("inconsistent shapes")
    if seq_len.dtype != torch.int32:
        raise TypeError("seq_len must be int32")
    ash = make_attn_shape(B, cap, Hq, Hkv, hd, rope_base, scale,
                          GSRQ_ATTN_TABLES_READY if tables_ready else 0)
    sh = make_shape(B * cap, D, d, K, M)
    if out is None:
        out = torch.empty((B, Hq, hd), dtype=torch.float32, device=q.device)
    if noalloc:
        if workspace is not None:
            raise ValueError("noalloc takes no workspace")
        st = lib.gsrq_attn_decode_noalloc(
            ctypes.byref(ash), ctypes.byref(sh), _ptr(k_codes), _ptr(v_codes), _ptr(seq_len),
            _ptr(k_gain), _ptr(k_shape), _ptr(v_gain), _ptr(v_shape), _ptr(q), _dtype_code(q),
            _ptr(out), _stream_handle(stream))
        _check(st, "gsrq_attn_decode_noalloc")
        return out
    n = ctypes.c_size_t()
    _check(lib.gsrq_attn_workspace_bytes_kv(ctypes.byref(ash), ctypes.byref(sh), ctypes.byref(n)),
           "gsrq_attn_workspace_bytes_kv")
    ws = _workspace(n.value, q.device, workspace)
    st = lib.gsrq_attn_decode(ctypes.byref(ash), ctypes.byref(sh), _ptr(k_codes), _ptr(v_codes),
                              _ptr(seq_len), _ptr(k_gain), _ptr(k_shape), _ptr(v_gain),
                              _ptr(v_shape), _ptr(q), _dtype_code(q), _ptr(out), _ptr(ws),
                              ws.numel() * ws.element_size(), _stream_handle(stream))
    _check(st, "gsrq_attn_decode")
    return out


# ------------------------------------------------------------- paged cache

# The structures of the calls of every decoding step are packed, not built
# field by field (a few microseconds of a call); layouts as Pages, Heads,
# PagedAttn, PageExps and PagedBatch above.
_PAGES = struct.Struct("@PP3q3qPq7i0q")
_HEADS = struct.Struct("@Pqq")
_PAGED_ATTN = struct.Struct("@qiifI0q")
_PAGE_EXPS = struct.Struct("@PPqqqq")
_PAGED_BATCH = struct.Struct("@qqiiii")


def _paged_types():
    torch = _torch()
    return {torch.float16: GSRQ_F16, torch.bfloat16: GSRQ_BF16, torch.float32: GSRQ_F32}


def _paged_dtype(t, name) -> int:
    code = _paged_types().get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float16, bfloat16 or float32, not {t.dtype}")
    return code


def _paged_device(device, stream):
    """Context of a paged call, or None where the device is current and the
    stream its current one: the stream's device is made current and new
    tensors come from the stream's memory, so that a workspace freed when the
    call returns is not handed to another stream while it is in use."""
    torch = _torch()
    if device.type != "cuda":
        raise ValueError(f"the tensors are on {device}, expected a GPU")
    if stream is None:
        current = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
        return None if device.index == current() else torch.cuda.device(device)
    if stream.device != device:
        raise ValueError(f"the stream is on {stream.device}, the tensors on {device}")
    return torch.cuda.stream(stream)


def _dense(t, name, dtype, like, n) -> int:
    """Address of a contiguous tensor of n elements on `like`'s device."""
    if (t.dtype is dtype and t.numel() == n and t.get_device() == like.get_device()
            and t.is_contiguous()):
        return t.data_ptr()
    _need(t, name, (dtype,), like.device, (n,))
    raise ValueError(f"{name} must be a dense tensor of {n} elements")


def _pages(k_pages, v_pages, table, eight=False) -> bytes:
    """gsrq_pages of two pools [pages, page_size, Hkv, head_dim] and their table."""
    torch = _torch()
    shape, dtype, index = k_pages.shape, k_pages.dtype, k_pages.get_device()
    if len(shape) != 4 or v_pages.shape != shape:
        raise ValueError("k_pages and v_pages must be [pages, page_size, Hkv, head_dim], both alike")
    if eight:
        if dtype is not torch.float8_e4m3fn or v_pages.dtype is not dtype:
            raise TypeError("pages with exponents must be float8_e4m3fn")
    elif dtype is not torch.float16 and dtype is not torch.bfloat16 or v_pages.dtype is not dtype:
        raise TypeError("pages must be float16 or bfloat16, both alike (float8_e4m3fn with exponents)")
    if table.dim() != 2 or table.dtype is not torch.int32:
        raise TypeError("table must be a 2-D int32 tensor")
    if v_pages.get_device() != index or table.get_device() != index:
        raise ValueError(f"v_pages and table must be on {k_pages.device}")
    k0, k1, k2, k3 = k_pages.stride()
    v0, v1, v2, v3 = v_pages.stride()
    t0, t1 = table.stride()
    B, per = table.shape
    if k3 != 1 or v3 != 1 or (t1 != 1 and per > 1):
        raise ValueError("elements of a head and entries of a table row must be adjacent")
    n, size, Hkv, hd = shape
    try:
        return _PAGES.pack(k_pages.data_ptr(), v_pages.data_ptr(), k0, k1, k2, v0, v1, v2,
                           table.data_ptr(), t0 if B > 1 else per, n, size, per, B, Hkv, hd,
                           GSRQ_E4M3 if eight else GSRQ_F16 if dtype is torch.float16
                           else GSRQ_BF16)
    except struct.error:
        raise ValueError("a dimension of the pages or the table does not fit 32 bits") from None


def _exps(k_exp, v_exp, k_pages):
    """gsrq_page_exps of two tensors [pages, Hkv] of exponents."""
    if k_exp is None or v_exp is None:
        raise ValueError("k_exp and v_exp come together")
    int8, shape, index = _torch().int8, k_pages.shape, k_pages.get_device()
    shape = (shape[0], shape[2]) if len(shape) == 4 else ()
    for name, t in (("k_exp", k_exp), ("v_exp", v_exp)):
        if t.dtype is not int8:
            raise TypeError(f"{name} must be int8, not {t.dtype}")
        if t.shape != shape:
            raise ValueError(f"{name} must be [pages, Hkv] of the pages, not {tuple(t.shape)}")
        if t.get_device() != index:
            raise ValueError(f"{name} is on {t.device}, expected {k_pages.device}")
    k0, k1 = k_exp.stride()
    v0, v1 = v_exp.stride()
    return _PAGE_EXPS.pack(k_exp.data_ptr(), v_exp.data_ptr(), k0, k1, v0, v1)


def _heads(x, name, heads, head_dim, rows, dtype, like) -> bytes:
    """gsrq_heads of rows [rows, heads, head_dim]."""
    if x.shape != (rows, heads, head_dim):
        raise ValueError(f"{name} must be [{rows}, {heads}, {head_dim}], not {tuple(x.shape)}")
    if x.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, not {x.dtype}")
    if x.get_device() != like.get_device():
        raise ValueError(f"{name} is on {x.device}, expected {like.device}")
    s0, s1, s2 = x.stride()
    if s2 != 1:
        raise ValueError(f"{name}: elements of a head must be adjacent")
    return _HEADS.pack(x.data_ptr(), s0, s1)


def _empty(like, shape, dtype):
    """A dense tensor of this shape and type on `like`'s device."""
    torch = _torch()
    if like.dtype is dtype and like.shape == shape and like.is_contiguous():
        return torch.empty_like(like)
    return torch.empty(shape, dtype=dtype, device=like.device)


def paged_append(k, v, k_pages, v_pages, table, q_start, seq_len, *, q=None, theta=None,
                 k_norm=None, q_norm=None, eps=1e-6, q_out=None, k_exp=None, v_exp=None,
                 stream=None):
    """Put new tokens' keys and values into their pages (see gsrq_paged_append,
    and gsrq_paged_append8 for 8-bit pages).

    k, v [T, Hkv, head_dim] and q [T, Hq, head_dim] (float32, float16 or
    bfloat16, any strides); k_pages, v_pages [pages, page_size, Hkv, head_dim]
    (float16 or bfloat16); table [B, per] int32; q_start [B + 1] and
    seq_len [B] int32 (seq_len with the new tokens).  theta [head_dim / 2]
    float64: angle per position, e.g. base ** (-2 * arange(hd / 2) / hd); keys
    and queries are turned by it.  k_norm, q_norm [head_dim] float32.
    Returns the queries [T, Hq, head_dim] in the pages' type (q_out, or a new
    tensor in which rows of no sequence hold anything), or None without q.
    Keys that are also coded (encode, float16 or float32 rows) are coded after
    their norm, which the caller applies for it, and before the rotation:
    paged_restore turns them and norms nothing.
    8-bit pages: k_pages, v_pages float8_e4m3fn with the exponents of their
    scales, k_exp, v_exp [pages, Hkv] int8 (any strides), which the call updates;
    the queries come in q_out's type, or else q's, of float32 rows bfloat16."""
    torch = _torch()
    lib = _lib or load_library()
    exps = None if k_exp is None is v_exp else _exps(k_exp, v_exp, k_pages)
    pages = _pages(k_pages, v_pages, table, exps is not None)
    B = table.shape[0]
    _, _, Hkv, hd = k_pages.shape
    T, dtype, held = k.shape[0], k.dtype, k_pages.dtype
    dt = _paged_dtype(k, "k")
    if exps is not None:
        held = (q_out.dtype if q_out is not None else
                torch.bfloat16 if dtype is torch.float32 else dtype)
        if held is not torch.float16 and held is not torch.bfloat16:
            raise TypeError(f"q_out must be float16 or bfloat16, not {held}")
    kh = _heads(k, "k", Hkv, hd, T, dtype, k_pages)
    vh = _heads(v, "v", Hkv, hd, T, dtype, k_pages)
    Hq, qh = 0, None
    if q is not None:
        Hq = q.shape[1] if q.dim() == 3 else 0
        qh = _heads(q, "q", Hq, hd, T, dtype, k_pages)
    elif q_norm is not None or q_out is not None:
        raise ValueError("q_norm and q_out need q")
    start = _dense(q_start, "q_start", torch.int32, k_pages, B + 1)
    lens = _dense(seq_len, "seq_len", torch.int32, k_pages, B)
    angles = None if theta is None else _dense(theta, "theta", torch.float64, k_pages, hd // 2)
    kn = None if k_norm is None else _dense(k_norm, "k_norm", torch.float32, k_pages, hd)
    qn = None if q_norm is None else _dense(q_norm, "q_norm", torch.float32, k_pages, hd)
    if q_out is not None:
        _dense(q_out, "q_out", held, k_pages, T * Hq * hd)

    def call():
        out = q_out
        if q is not None and out is None:
            out = _empty(q, (T, Hq, hd), held)
        if T > 0 and exps is not None:
            st = lib.gsrq_paged_append8(pages, exps, T, start, lens, kh, vh, qh, Hq, dt, angles,
                                        kn, qn, eps, _ptr(out),
                                        GSRQ_F16 if held is torch.float16 else GSRQ_BF16,
                                        _append_stream_handle(stream))
            if st != GSRQ_OK:
                _check(st, "gsrq_paged_append8")
        elif T > 0:
            st = lib.gsrq_paged_append(pages, T, start, lens, kh, vh, qh, Hq, dt, angles, kn, qn,
                                       eps, _ptr(out), _append_stream_handle(stream))
            if st != GSRQ_OK:
                _check(st, "gsrq_paged_append")
        return out

    context = _paged_device(k_pages.device, stream)
    if context is None:
        return call()
    with context:
        return call()


def attn_paged_workspace_bytes(T, Hq, k_pages, v_pages, table, *, window=0) -> int:
    """Workspace of attn_paged for T rows of Hq query heads over these pages, of
    16 or 8 bits."""
    n = ctypes.c_size_t()
    lib, eight = load_library(), k_pages.dtype is _torch().float8_e4m3fn
    call = lib.gsrq_attn_paged8_workspace_bytes if eight else lib.gsrq_attn_paged_workspace_bytes
    _check(call(_PAGED_ATTN.pack(int(T), int(Hq), int(window), 1.0, 0),
                _pages(k_pages, v_pages, table, eight), ctypes.byref(n)),
           "gsrq_attn_paged_workspace_bytes")
    return int(n.value)


def attn_paged(q, k_pages, v_pages, table, q_start, seq_len, *, scale=None, window=0, lse=False,
               out=None, workspace=None, k_exp=None, v_exp=None, stream=None):
    """Causal attention of new tokens over their sequences' pages (see
    gsrq_attn_paged), after paged_append of the same rows.  q [T, Hq, head_dim]
    of the pages' type, any strides.  Returns out [T, Hq, head_dim] of the
    same type (apart from q; rows of no sequence are left as they are, in a
    new tensor anything), with lse=True also the rows' log-sum-exp [T, Hq]
    float32.  workspace: a uint8 tensor of attn_paged_workspace_bytes, or None (one is
    made for the call).  8-bit pages (gsrq_attn_paged8): float8_e4m3fn with
    k_exp, v_exp [pages, Hkv] int8 as paged_append keeps them, q float16 or
    bfloat16."""
    torch = _torch()
    lib = _lib or load_library()
    exps = None if k_exp is None is v_exp else _exps(k_exp, v_exp, k_pages)
    pages = _pages(k_pages, v_pages, table, exps is not None)
    if q.dim() != 3:
        raise ValueError("q must be [T, Hq, head_dim]")
    T, Hq, hd = q.shape
    B, dtype = table.shape[0], k_pages.dtype if exps is None else q.dtype
    if exps is not None and dtype is not torch.float16 and dtype is not torch.bfloat16:
        raise TypeError(f"q must be float16 or bfloat16, not {dtype}")
    qh = _heads(q, "q", Hq, k_pages.shape[3], T, dtype, k_pages)
    start = _dense(q_start, "q_start", torch.int32, k_pages, B + 1)
    lens = _dense(seq_len, "seq_len", torch.int32, k_pages, B)
    if out is not None:
        _dense(out, "out", dtype, k_pages, T * Hq * hd)
    if workspace is not None and (workspace.device != k_pages.device
                                  or not workspace.is_contiguous()):
        raise ValueError(f"workspace must be contiguous, on {k_pages.device}")
    try:
        s = _PAGED_ATTN.pack(T, Hq, window, hd ** -0.5 if scale is None else scale, 0)
    except (struct.error, ZeroDivisionError):        # (heads of no elements)
        raise ValueError("window must be a number of tokens, or 0, and scale a number") from None

    def call():
        res = _empty(q, (T, Hq, hd), dtype) if out is None else out
        total = (torch.empty((T, Hq), dtype=torch.float32, device=q.device) if lse else None)
        if T > 0:
            n = ctypes.c_size_t()
            st = (lib.gsrq_attn_paged_workspace_bytes(s, pages, ctypes.byref(n)) if exps is None
                  else lib.gsrq_attn_paged8_workspace_bytes(s, pages, ctypes.byref(n)))
            if st != GSRQ_OK:
                _check(st, "gsrq_attn_paged_workspace_bytes")
            ws, size = None, n.value
            if size:
                ws = _workspace(size, q.device, workspace)
                size = ws.numel() * ws.element_size()
            if exps is None:
                st = lib.gsrq_attn_paged(s, pages, start, lens, qh, res.data_ptr(), _ptr(total),
                                         _ptr(ws), size, _append_stream_handle(stream))
            else:
                st = lib.gsrq_attn_paged8(s, pages, exps, start, lens, qh,
                                          GSRQ_F16 if dtype is torch.float16 else GSRQ_BF16,
                                          res.data_ptr(), _ptr(total), _ptr(ws), size,
                                          _append_stream_handle(stream))
            if st != GSRQ_OK:
                _check(st, "gsrq_attn_paged" if exps is None else "gsrq_attn_paged8")
        return (res, total) if lse else res

    context = _paged_device(k_pages.device, stream)
    if context is None:
        return call()
    with context:
        return call()


def paged_restore(k_codes, v_codes, seq_len, k_gain, k_shape, v_gain, v_shape, k_pages, v_pages,
                  table, *, theta=None, stream=None):
    """Decode coded contexts into pages (see gsrq_paged_restore): k_codes,
    v_codes [B, cap, W] packed codes, seq_len [B] int32, codebooks [M, G, K]
    and [M, G, K, d]; the pages, the table and theta as paged_append takes
    them.  Keys: as they were before the rotation, normed if the model norms
    its keys."""
    torch = _torch()
    lib = load_library()
    pages = _pages(k_pages, v_pages, table)
    dev, hd = k_pages.device, k_pages.shape[3]
    if k_codes.dim() != 3 or k_shape.dim() != 4:
        raise ValueError("codes must be [B, cap, W] and codebook shapes [M, G, K, d]")
    B, cap, W = k_codes.shape
    M, G, K, d = k_shape.shape
    if B != table.shape[0]:
        raise ValueError(f"codes of {B} sequences, a table of {table.shape[0]}")
    sh = make_shape(max(B * cap, 1), G * d, d, K, M)
    words = int(lib.gsrq_code_words(ctypes.byref(sh)))
    if W != words:
        raise ValueError(f"codes have {W} words a row, expected {words}")
    for name, t in (("k_codes", k_codes), ("v_codes", v_codes)):
        _need(t, name, (torch.int32, torch.uint32), dev, (B, cap, W))
    _need(seq_len, "seq_len", (torch.int32,), dev, (B,))
    for name, t, size in (("k_gain", k_gain, (M, G, K)), ("k_shape", k_shape, (M, G, K, d)),
                          ("v_gain", v_gain, (M, G, K)), ("v_shape", v_shape, (M, G, K, d))):
        _need(t, name, (torch.float32,), dev, size)
    _need(theta, "theta", (torch.float64,), dev, (hd // 2,))
    if B == 0 or cap == 0:
        return

    def call():
        st = lib.gsrq_paged_restore(
            pages, ctypes.byref(sh), cap, _ptr(k_codes), _ptr(v_codes), _ptr(seq_len),
            _ptr(k_gain), _ptr(k_shape), _ptr(v_gain), _ptr(v_shape), _ptr(theta),
            _append_stream_handle(stream))
        _check(st, "gsrq_paged_restore")

    context = _paged_device(dev, stream)
    if context is None:
        return call()
    with context:
        call()


def paged_plan(table, free_pages, n_free, seq_len, change, *, page_size, rows, q_start=None,
               slots=None, positions=None, stream=None):
    """Pages, rows and slots of a batch whose requests' lengths change (see
    gsrq_paged_plan): change [B] int32 counts the tokens that every sequence
    brings or, below zero, gives back.  In place: table [B, per] int32,
    free_pages [F] int32 with its count n_free [1] int32, seq_len [B] int32.
    Returns (q_start [B + 1] int32, slots [rows] int64, positions [rows] int32),
    new tensors or those given; q_start and seq_len are as paged_append and
    attn_paged take them.  A sequence that grows but has no rows in q_start was
    not served: the list, the rows or its table row did not suffice."""
    torch = _torch()
    lib = _lib or load_library()
    if table.dim() != 2 or table.dtype is not torch.int32:
        raise TypeError("table must be a 2-D int32 tensor")
    B, per = table.shape
    t0, t1 = table.stride()
    if t1 != 1 and per > 1:
        raise ValueError("entries of a table row must be adjacent")
    rows = int(rows)
    if rows < 0:
        raise ValueError("rows must not be negative")
    F = free_pages.numel()
    pool = _dense(free_pages, "free_pages", torch.int32, table, F)
    count = _dense(n_free, "n_free", torch.int32, table, 1)
    lens = _dense(seq_len, "seq_len", torch.int32, table, B)
    moves = _dense(change, "change", torch.int32, table, B)
    for name, t, dtype, n in (("q_start", q_start, torch.int32, B + 1),
                              ("slots", slots, torch.int64, rows),
                              ("positions", positions, torch.int32, rows)):
        if t is not None:
            _dense(t, name, dtype, table, n)
    try:
        s = _PAGED_BATCH.pack(rows, t0 if B > 1 else per, B, per, page_size, F)
    except struct.error:
        raise ValueError("a size does not fit 32 bits, or page_size is no number of tokens") from None

    def call():
        out = (table.new_empty(B + 1) if q_start is None else q_start,
               table.new_empty(rows, dtype=torch.int64) if slots is None else slots,
               table.new_empty(rows) if positions is None else positions)
        st = lib.gsrq_paged_plan(s, table.data_ptr(), pool, count, lens, moves, out[0].data_ptr(),
                                 out[1].data_ptr() or None, out[2].data_ptr() or None,
                                 _append_stream_handle(stream))
        if st != GSRQ_OK:
            _check(st, "gsrq_paged_plan")
        return out

    context = _paged_device(table.device, stream)
    if context is None:
        return call()
    with context:
        return call()


def verify_drafts_workspace_bytes(T, V, B) -> int:
    """Workspace of verify_drafts for T rows of V probabilities, B sequences."""
    n = ctypes.c_size_t()
    _check(load_library().gsrq_verify_drafts_workspace_bytes(int(T), int(V), int(B),
                                                             ctypes.byref(n)),
           "gsrq_verify_drafts_workspace_bytes")
    return int(n.value)


def verify_drafts(tokens, target, draft, uniform, draw, q_start, *, accepted=None, next_token=None,
                  workspace=None, stream=None):
    """How many of every sequence's drafts stand, and the token after them (see
    gsrq_verify_drafts).  Rows as attn_paged takes them: a sequence's last token
    and its drafts, tokens [T] int32; target [T, V] and draft [T, V] (or None:
    drafts chosen without chance) probabilities of the token that follows each
    row, float32, float16 or bfloat16, rows at any stride; uniform [T] and
    draw [B] float32 numbers of [0, 1); q_start [B + 1] int32.  Returns
    (accepted [B], next token [B]) int32, new tensors or those given.  With n
    rows of a sequence (as q_start has them, not as it asked for), paged_plan
    takes its n - 1 - accepted other drafts back; none where n is 0."""
    torch = _torch()
    lib = _lib or load_library()
    if target.dim() != 2:
        raise ValueError("target must be [T, V]")
    T, V = target.shape
    B = q_start.numel() - 1
    if B < 1:
        raise ValueError("q_start must be [B + 1], of one sequence or more")
    dt, ld = _paged_dtype(target, "target"), [V, V]
    for i, (name, t) in enumerate((("target", target), ("draft", draft))):
        if t is None:
            continue
        if t.shape != target.shape or t.dtype is not target.dtype:
            raise ValueError(f"{name} must be like target")
        if t.get_device() != target.get_device():
            raise ValueError(f"{name} is on {t.device}, expected {target.device}")
        s0, s1 = t.stride()
        if (s1 != 1 and V > 1) or (T > 1 and s0 < V):
            raise ValueError(f"{name}: a row's probabilities must be adjacent, rows apart")
        ld[i] = s0 if T > 1 else V
    ids = _dense(tokens, "tokens", torch.int32, target, T)
    u = _dense(uniform, "uniform", torch.float32, target, T)
    d = _dense(draw, "draw", torch.float32, target, B)
    start = _dense(q_start, "q_start", torch.int32, target, B + 1)
    for name, t in (("accepted", accepted), ("next_token", next_token)):
        if t is not None:
            _dense(t, name, torch.int32, target, B)
    if workspace is not None and (workspace.device != target.device
                                  or not workspace.is_contiguous()):
        raise ValueError(f"workspace must be contiguous, on {target.device}")

    def call():
        out = (q_start.new_empty(B) if accepted is None else accepted,
               q_start.new_empty(B) if next_token is None else next_token)
        n = ctypes.c_size_t()
        st = lib.gsrq_verify_drafts_workspace_bytes(T, V, B, ctypes.byref(n))
        if st != GSRQ_OK:
            _check(st, "gsrq_verify_drafts_workspace_bytes")
        ws, size = None, n.value
        if size:
            ws = _workspace(size, target.device, workspace)
            size = ws.numel() * ws.element_size()
        st = lib.gsrq_verify_drafts(T, V, B, ids or None, target.data_ptr() or None, ld[0],
                                    _ptr(draft), ld[1], dt, u or None, d, start,
                                    out[0].data_ptr(), out[1].data_ptr(), _ptr(ws), size,
                                    _append_stream_handle(stream))
        if st != GSRQ_OK:
            _check(st, "gsrq_verify_drafts")
        return out

    context = _paged_device(target.device, stream)
    if context is None:
        return call()
    with context:
        return call()
