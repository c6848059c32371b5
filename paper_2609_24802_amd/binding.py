"""Python binding of the gfx950 fused message-passing library (ctypes).

Argument marshalling only: every function below checks tensor shapes, dtypes
and devices, allocates outputs and the workspace with torch (device memory and
the current stream are the only things torch provides here), and calls the
C entry point of the same name.  All computation happens in the HIP kernels of
``libtiga_mp.so``; if that library is missing or cannot be loaded, every call
raises instead of falling back to anything else.
"""
from __future__ import annotations

import ctypes as C
import os
import threading

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtiga_mp.so")

TIGA_OK, TIGA_EINVAL, TIGA_EGRAPH, TIGA_EUNSUPPORTED, TIGA_EWORKSPACE, TIGA_EDEVICE = 0, -1, -2, -3, -4, -5
REDUCE_SUM, REDUCE_MAX = 0, 1
MSG_SRC, MSG_EDGE_SCALED_SRC = 0, 1
DT_F16, DT_BF16, DT_F32 = 0, 1, 2
REL_TRIANGULAR, REL_DENSE = 0, 1
PAIRS_HALF, PAIRS_ADJACENT = 0, 1
ROTARY_PLAIN, ROTARY_LINEAR, ROTARY_BASE, ROTARY_BANDS = 0, 1, 2, 3
_STATUS = {0: "TIGA_OK", -1: "TIGA_EINVAL", -2: "TIGA_EGRAPH", -3: "TIGA_EUNSUPPORTED",
           -4: "TIGA_EWORKSPACE", -5: "TIGA_EDEVICE"}


class TigaError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"{_STATUS.get(code, code)}: {message}")
        self.code = code


class _Csr(C.Structure):
    _fields_ = [("num_dst", C.c_int64), ("num_src", C.c_int64), ("num_edges", C.c_int64),
                ("row_ptr", C.c_void_p), ("col_idx", C.c_void_p)]


class _CsrT(C.Structure):
    _fields_ = [("src_ptr", C.c_void_p), ("edge_id", C.c_void_p)]


class _View(C.Structure):
    _fields_ = [("data", C.c_void_p), ("batch", C.c_int64), ("head", C.c_int64), ("row", C.c_int64)]


class _Cross(C.Structure):
    _fields_ = [("num_dst", C.c_int64), ("num_src", C.c_int64), ("batch", C.c_int32), ("heads", C.c_int32),
                ("kv_heads", C.c_int32), ("width", C.c_int32), ("dtype", C.c_int32), ("src_len", C.c_void_p)]


class _Packed(C.Structure):
    _fields_ = [("num_rows", C.c_int64), ("batch", C.c_int32), ("heads", C.c_int32), ("kv_heads", C.c_int32),
                ("width", C.c_int32), ("dtype", C.c_int32), ("ptr", C.c_void_p)]


class _Rotary(C.Structure):
    _fields_ = [("freq", C.c_void_p), ("rot", C.c_int32), ("pairs", C.c_int32), ("amplitude", C.c_float)]


class _Cache(C.Structure):
    _fields_ = [("num_pages", C.c_int64), ("page_size", C.c_int32), ("kv_heads", C.c_int32), ("width", C.c_int32),
                ("dtype", C.c_int32), ("batch", C.c_int32), ("table_width", C.c_int32), ("k", _View), ("v", _View),
                ("table", C.c_void_p), ("length", C.c_void_p)]


class _Prefix(C.Structure):
    _fields_ = [("groups", C.c_int32), ("ptr", C.c_void_p), ("len", C.c_void_p)]


_lib = None
_lock = threading.Lock()

_SIGS = {
    "tiga_last_error": (C.c_char_p, []),
    "tiga_mp_abi_version": (C.c_int, []),
    "tiga_mp_csr_fwd_workspace": (C.c_size_t, [C.c_void_p, C.c_int32, C.c_int]),
    "tiga_mp_csr_fwd": (C.c_int, [C.c_void_p, C.c_int32, C.c_void_p, C.c_int, C.c_void_p, C.c_int, C.c_void_p,
                                  C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "tiga_mp_csr_fwd_noalloc_limit": (C.c_size_t, []),
    "tiga_mp_csr_fwd_noalloc": (C.c_int, [C.c_void_p, C.c_int32, C.c_void_p, C.c_int, C.c_void_p, C.c_int,
                                          C.c_void_p, C.c_void_p, C.c_void_p]),
    "tiga_mp_csr_bwd_workspace": (C.c_size_t, [C.c_void_p, C.c_int32, C.c_int]),
    "tiga_mp_csr_bwd": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_int, C.c_void_p, C.c_int,
                                  C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t,
                                  C.c_void_p]),
    "tiga_csr_transpose_workspace": (C.c_size_t, [C.c_void_p]),
    "tiga_csr_transpose": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "tiga_csr_validate": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p]),
    "tiga_mp_radius_workspace": (C.c_size_t, [C.c_int64, C.c_int32]),
    "tiga_mp_radius_fwd": (C.c_int, [C.c_int64, C.c_int32, C.c_void_p, C.c_void_p, C.c_float, C.c_float, C.c_int,
                                     C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "tiga_mp_radius_bwd": (C.c_int, [C.c_int64, C.c_int32, C.c_void_p, C.c_void_p, C.c_float, C.c_float,
                                     C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "tiga_radius_neighbors": (C.c_int, [C.c_int64, C.c_void_p, C.c_float, C.c_void_p, C.c_void_p, C.c_void_p,
                                        C.c_size_t, C.c_void_p]),
    "tiga_mp_dense_workspace": (C.c_size_t, [C.c_int64]),
    "tiga_mp_dense_fwd": (C.c_int, [C.c_int64, C.c_void_p, C.c_void_p, C.c_float, C.c_int, C.c_void_p,
                                    C.c_void_p, C.c_size_t, C.c_void_p]),
    "tiga_mp_csr_fwd_paged_workspace": (C.c_size_t, [C.c_int32, C.c_int, C.c_int64]),
    "tiga_mp_csr_fwd_paged": (C.c_int, [C.c_void_p, C.c_int32, C.c_void_p, C.c_int, C.c_void_p, C.c_int, C.c_void_p,
                                        C.c_void_p, C.c_int64, C.c_void_p, C.c_size_t, C.c_void_p]),
    "tiga_mp_edgenn_workspace": (C.c_size_t, [C.c_int64, C.c_int32, C.c_int32, C.c_int32]),
    "tiga_mp_edgenn_fwd": (C.c_int, [C.c_int64, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_float,
                                     C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                     C.c_size_t, C.c_void_p]),
    "tiga_mp_edgenn_bwd": (C.c_int, [C.c_int64, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_float,
                                     C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                     C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                     C.c_size_t, C.c_void_p]),
    "tiga_mp_knn_workspace": (C.c_size_t, [C.c_int64]),
    "tiga_mp_knn_fwd": (C.c_int, [C.c_int64, C.c_int32, C.c_void_p, C.c_void_p, C.c_int32, C.c_int, C.c_void_p,
                                  C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "tiga_mp_attention_fwd": (C.c_int, [C.c_int64, C.c_int32, C.c_int32, C.c_int, C.c_void_p, C.c_void_p,
                                        C.c_void_p, C.c_float, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p]),
    "tiga_mp_attention_cross_fwd_workspace": (C.c_size_t, [C.c_void_p]),
    "tiga_mp_attention_cross_fwd": (C.c_int, [C.c_void_p] * 4 + [C.c_float] + [C.c_void_p] * 3 +
                                    [C.c_size_t, C.c_void_p]),
    "tiga_mp_attention_cross_bwd_workspace": (C.c_size_t, [C.c_void_p]),
    "tiga_mp_attention_cross_bwd": (C.c_int, [C.c_void_p] * 7 + [C.c_float] + [C.c_void_p] * 4 +
                                    [C.c_size_t, C.c_void_p]),
    "tiga_mp_attention_packed_fwd_workspace": (C.c_size_t, [C.c_void_p]),
    "tiga_mp_attention_packed_fwd": (C.c_int, [C.c_void_p] * 4 + [C.c_float] + [C.c_void_p] * 3 +
                                     [C.c_size_t, C.c_void_p]),
    "tiga_mp_attention_packed_bwd_workspace": (C.c_size_t, [C.c_void_p]),
    "tiga_mp_attention_packed_bwd": (C.c_int, [C.c_void_p] * 7 + [C.c_float] + [C.c_void_p] * 4 +
                                     [C.c_size_t, C.c_void_p]),
    "tiga_rotary_frequencies": (C.c_int, [C.c_int32, C.c_double, C.c_int, C.c_double, C.c_double, C.c_double,
                                          C.c_double, C.c_void_p]),
    "tiga_mp_rotary_fwd": (C.c_int, [C.c_int32, C.c_int32, C.c_int64, C.c_int32, C.c_int, C.c_void_p, C.c_void_p,
                                     C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p]),
    "tiga_mp_rotary_bwd": (C.c_int, [C.c_int32, C.c_int32, C.c_int64, C.c_int32, C.c_int, C.c_void_p, C.c_void_p,
                                     C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p]),
    "tiga_cache_validate": (C.c_int, [C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]),
    "tiga_mp_cache_append": (C.c_int, [C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                       C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]),
    "tiga_mp_attention_paged_fwd_workspace": (C.c_size_t, [C.c_void_p, C.c_int64, C.c_int32]),
    "tiga_mp_attention_paged_fwd": (C.c_int, [C.c_void_p, C.c_int64, C.c_void_p, C.c_int32, C.c_void_p, C.c_float,
                                              C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "tiga_prefix_validate": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]),
    "tiga_mp_attention_prefix_fwd_workspace": (C.c_size_t, [C.c_void_p, C.c_void_p, C.c_int64, C.c_int32]),
    "tiga_mp_attention_prefix_fwd": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int32, C.c_void_p,
                                               C.c_float, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "tiga_retention_validate": (C.c_int, [C.c_void_p, C.c_void_p]),
    "tiga_mp_cache_weights_workspace": (C.c_size_t, [C.c_void_p, C.c_int64, C.c_int32]),
    "tiga_mp_cache_weights": (C.c_int, [C.c_void_p, C.c_int64, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_float,
                                        C.c_float, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "tiga_mp_cache_evict_workspace": (C.c_size_t, [C.c_void_p, C.c_void_p, C.c_int32]),
    "tiga_mp_cache_evict": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                      C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "tiga_mp_set_kernel_events": (C.c_int, [C.c_void_p, C.c_void_p]),
}


def load(path: str = LIB_PATH):
    """Load the HIP library (torch's HIP runtime is loaded first and shared)."""
    global _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(path):
                raise RuntimeError(f"HIP library not built: {path} is missing (run __graft_entry__.build())")
            lib = C.CDLL(path)
            for name, (res, args) in _SIGS.items():
                fn = getattr(lib, name)
                fn.restype = res
                fn.argtypes = args
            _lib = lib
    return _lib


def _check(rc: int):
    if rc != TIGA_OK:
        raise TigaError(rc, load().tiga_last_error().decode())


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream():
    """The current HIP stream of the current device, as a void pointer.  torch's raw-stream
    accessor avoids building a Stream object (about 3 us per call); the public call is the
    fallback."""
    if _raw_stream is not None:
        return C.c_void_p(_raw_stream(torch.cuda.current_device()))
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _dev(t, dtype, name, shape=None):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    return t


def _workspace(nbytes: int, device):
    ws = torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)
    assert ws.data_ptr() % 256 == 0
    return ws


class Csr:
    """A destination-major CSR relation on the device (row_ptr int64, col_idx int32)."""

    def __init__(self, row_ptr: torch.Tensor, col_idx: torch.Tensor, num_src: int):
        self.row_ptr = _dev(row_ptr, torch.int64, "row_ptr")
        self.col_idx = _dev(col_idx, torch.int32, "col_idx")
        self.num_dst = row_ptr.numel() - 1
        self.num_src = int(num_src)
        self.num_edges = col_idx.numel()
        self._c = _Csr(self.num_dst, self.num_src, self.num_edges, self.row_ptr.data_ptr(),
                       self.col_idx.data_ptr() if self.num_edges else None)

    @property
    def ref(self):
        return C.byref(self._c)


class CsrT:
    """Reverse incidence built by :func:`tiga_csr_transpose`."""

    def __init__(self, src_ptr, edge_id):
        self.src_ptr, self.edge_id = src_ptr, edge_id
        self._c = _CsrT(src_ptr.data_ptr(), edge_id.data_ptr() if edge_id.numel() else None)

    @property
    def ref(self):
        return C.byref(self._c)


def tiga_mp_abi_version() -> int:
    return int(load().tiga_mp_abi_version())


def tiga_mp_set_kernel_events(start=None, stop=None):
    """Arm hipEvents (torch.cuda.Event, already recorded once) around the next dominant kernel."""
    lib = load()
    s = C.c_void_p(start.cuda_event) if start is not None else None
    e = C.c_void_p(stop.cuda_event) if stop is not None else None
    _check(lib.tiga_mp_set_kernel_events(s, e))


def tiga_mp_csr_fwd(rel: Csr, x: torch.Tensor, w: torch.Tensor | None = None, reducer: int = REDUCE_SUM,
                    y: torch.Tensor | None = None, argmax: torch.Tensor | None = None, ws=None):
    """Fused forward over a stored CSR relation; returns (y, argmax or None)."""
    lib = load()
    feat = x.shape[1]
    _dev(x, torch.float32, "x", (rel.num_src, feat))
    msg = MSG_SRC
    if w is not None:
        _dev(w, torch.float32, "w", (rel.num_edges,))
        msg = MSG_EDGE_SCALED_SRC
    if y is None:
        y = torch.empty(rel.num_dst, feat, dtype=torch.float32, device=x.device)
    if reducer == REDUCE_MAX and argmax is None:
        argmax = torch.empty(rel.num_dst, feat, dtype=torch.int32, device=x.device)
    need = lib.tiga_mp_csr_fwd_workspace(rel.ref, feat, reducer)
    if ws is None:
        ws = _workspace(need, x.device)
    _check(lib.tiga_mp_csr_fwd(rel.ref, feat, _ptr(x), msg, _ptr(w), reducer, _ptr(y), _ptr(argmax),
                               _ptr(ws), ws.numel(), _stream()))
    return y, argmax


def tiga_mp_csr_fwd_noalloc(rel: Csr, x: torch.Tensor, w: torch.Tensor | None = None, reducer: int = REDUCE_SUM,
                            y: torch.Tensor | None = None, argmax: torch.Tensor | None = None):
    """tiga_mp_csr_fwd without a workspace (the library's fixed per-device array); pass y (and argmax)
    to make the whole call allocation-free.  Returns (y, argmax or None)."""
    lib = load()
    feat = x.shape[1]
    _dev(x, torch.float32, "x", (rel.num_src, feat))
    msg = MSG_SRC
    if w is not None:
        _dev(w, torch.float32, "w", (rel.num_edges,))
        msg = MSG_EDGE_SCALED_SRC
    if y is None:
        y = torch.empty(rel.num_dst, feat, dtype=torch.float32, device=x.device)
    if reducer == REDUCE_MAX and argmax is None:
        argmax = torch.empty(rel.num_dst, feat, dtype=torch.int32, device=x.device)
    _check(lib.tiga_mp_csr_fwd_noalloc(rel.ref, feat, _ptr(x), msg, _ptr(w), reducer, _ptr(y), _ptr(argmax),
                                       _stream()))
    return y, argmax


def _host(t, dtype, name, n=None):
    if not isinstance(t, torch.Tensor) or t.is_cuda:
        raise TypeError(f"{name} must be a host (CPU) tensor")
    if t.dtype != dtype or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous {dtype} host tensor")
    if n is not None and t.numel() != n:
        raise ValueError(f"{name} has {t.numel()} entries, expected {n}")
    return t


class HostCsr:
    """A destination-major CSR relation kept in host memory (pin it for asynchronous copies)."""

    def __init__(self, row_ptr: torch.Tensor, col_idx: torch.Tensor, num_src: int):
        self.row_ptr = _host(row_ptr, torch.int64, "row_ptr")
        self.col_idx = _host(col_idx, torch.int32, "col_idx")
        self.num_dst = row_ptr.numel() - 1
        self.num_src = int(num_src)
        self.num_edges = col_idx.numel()
        self._c = _Csr(self.num_dst, self.num_src, self.num_edges, self.row_ptr.data_ptr(),
                       self.col_idx.data_ptr() if self.num_edges else None)

    @property
    def ref(self):
        return C.byref(self._c)


def tiga_mp_csr_fwd_paged(rel: HostCsr, x: torch.Tensor, w: torch.Tensor | None = None, reducer: int = REDUCE_SUM,
                          page_edges: int = 1 << 24, ws=None):
    """tiga_mp_csr_fwd with the relation (and w) in host memory, staged in pages of whole rows with at most
    page_edges edges; x and the outputs on the device.  Returns (y, argmax or None)."""
    lib = load()
    feat = x.shape[1]
    _dev(x, torch.float32, "x", (rel.num_src, feat))
    msg = MSG_SRC
    if w is not None:
        _host(w, torch.float32, "w", rel.num_edges)
        msg = MSG_EDGE_SCALED_SRC
    y = torch.empty(rel.num_dst, feat, dtype=torch.float32, device=x.device)
    argmax = torch.empty(rel.num_dst, feat, dtype=torch.int32, device=x.device) if reducer == REDUCE_MAX else None
    if ws is None:
        ws = _workspace(lib.tiga_mp_csr_fwd_paged_workspace(feat, reducer, int(page_edges)), x.device)
    _check(lib.tiga_mp_csr_fwd_paged(rel.ref, feat, _ptr(x), msg, _ptr(w), reducer, _ptr(y), _ptr(argmax),
                                     int(page_edges), _ptr(ws), ws.numel(), _stream()))
    return y, argmax


def tiga_mp_csr_bwd(rel: Csr, dy: torch.Tensor, x: torch.Tensor | None = None, w: torch.Tensor | None = None,
                    reducer: int = REDUCE_SUM, argmax: torch.Tensor | None = None, rev: CsrT | None = None,
                    want_dx: bool = True, want_dw: bool = True, ws=None):
    """VJP of tiga_mp_csr_fwd; returns (dx or None, dw or None)."""
    lib = load()
    feat = dy.shape[1]
    _dev(dy, torch.float32, "dy", (rel.num_dst, feat))
    msg = MSG_EDGE_SCALED_SRC if w is not None else MSG_SRC
    want_dw = want_dw and w is not None
    dx = torch.empty(rel.num_src, feat, dtype=torch.float32, device=dy.device) if want_dx else None
    dw = torch.empty(rel.num_edges, dtype=torch.float32, device=dy.device) if want_dw else None
    need = lib.tiga_mp_csr_bwd_workspace(rel.ref, feat, reducer)
    if ws is None:
        ws = _workspace(need, dy.device)
    _check(lib.tiga_mp_csr_bwd(rel.ref, rev.ref if rev is not None else None, feat, _ptr(x), msg, _ptr(w),
                               reducer, _ptr(argmax), _ptr(dy), _ptr(dx), _ptr(dw), _ptr(ws), ws.numel(),
                               _stream()))
    return dx, dw


def tiga_csr_transpose(rel: Csr) -> CsrT:
    lib = load()
    dev = rel.row_ptr.device
    src_ptr = torch.empty(rel.num_src + 1, dtype=torch.int64, device=dev)
    edge_id = torch.empty(rel.num_edges, dtype=torch.int32, device=dev)
    ws = _workspace(lib.tiga_csr_transpose_workspace(rel.ref), dev)
    _check(lib.tiga_csr_transpose(rel.ref, _ptr(src_ptr), _ptr(edge_id) if rel.num_edges else None, _ptr(ws),
                                  ws.numel(), _stream()))
    return CsrT(src_ptr, edge_id)


def tiga_csr_validate(rel: Csr, level: int = 2):
    """Raise TigaError (TIGA_EGRAPH) on an invalid relation."""
    _check(load().tiga_csr_validate(rel.ref, level, _stream()))


def tiga_mp_radius_fwd(pos: torch.Tensor, x: torch.Tensor, radius: float, sigma: float, want_count: bool = True,
                       y=None, count=None, ws=None):
    lib = load()
    n, feat = x.shape
    _dev(pos, torch.float32, "pos", (n, 3))
    _dev(x, torch.float32, "x", (n, feat))
    if y is None:
        y = torch.empty(n, feat, dtype=torch.float32, device=x.device)
    if want_count and count is None:
        count = torch.empty(n, dtype=torch.int32, device=x.device)
    if ws is None:
        ws = _workspace(lib.tiga_mp_radius_workspace(n, feat), x.device)
    _check(lib.tiga_mp_radius_fwd(n, feat, _ptr(pos), _ptr(x), float(radius), float(sigma), REDUCE_SUM, _ptr(y),
                                  _ptr(count), _ptr(ws), ws.numel(), _stream()))
    return y, count


def tiga_mp_radius_bwd(pos, x, dy, radius: float, sigma: float, want_dx: bool = True, want_dpos: bool = True,
                       ws=None):
    lib = load()
    n, feat = dy.shape
    _dev(pos, torch.float32, "pos", (n, 3))
    _dev(dy, torch.float32, "dy", (n, feat))
    if want_dpos:
        _dev(x, torch.float32, "x", (n, feat))
    dx = torch.empty(n, feat, dtype=torch.float32, device=dy.device) if want_dx else None
    dpos = torch.empty(n, 3, dtype=torch.float32, device=dy.device) if want_dpos else None
    if ws is None:
        ws = _workspace(lib.tiga_mp_radius_workspace(n, feat), dy.device)
    _check(lib.tiga_mp_radius_bwd(n, feat, _ptr(pos), _ptr(x) if want_dpos else None, float(radius), float(sigma),
                                  _ptr(dy), _ptr(dx), _ptr(dpos), _ptr(ws), ws.numel(), _stream()))
    return dx, dpos


def tiga_radius_neighbors(pos: torch.Tensor, radius: float, count: torch.Tensor | None = None):
    """Accepted neighbour lists; returns (count int32, ptr int64 [n+1], idx int32).  Synchronizes.

    The two phases of the C call: the counts come from the forward with no features (or are
    passed in), their exclusive prefix sum is the caller's nbr_ptr, then the lists are filled."""
    lib = load()
    n = pos.shape[0]
    _dev(pos, torch.float32, "pos", (n, 3))
    ws = _workspace(lib.tiga_mp_radius_workspace(n, 0), pos.device)
    if count is None:
        count = torch.empty(n, dtype=torch.int32, device=pos.device)
        _check(lib.tiga_mp_radius_fwd(n, 0, _ptr(pos), None, float(radius), 1.0, REDUCE_SUM, None, _ptr(count),
                                      _ptr(ws), ws.numel(), _stream()))
    else:
        _dev(count, torch.int32, "count", (n,))
    ptr = torch.zeros(n + 1, dtype=torch.int64, device=pos.device)
    torch.cumsum(count, 0, out=ptr[1:])
    total = int(ptr[-1].item())
    idx = torch.empty(max(total, 1), dtype=torch.int32, device=pos.device)
    _check(lib.tiga_radius_neighbors(n, _ptr(pos), float(radius), _ptr(ptr), _ptr(idx), _ptr(ws), ws.numel(),
                                     _stream()))
    return count, ptr, idx[:total]


def tiga_mp_dense_fwd(pos: torch.Tensor, q: torch.Tensor, eps: float, y=None, ws=None):
    lib = load()
    n = pos.shape[0]
    _dev(pos, torch.float32, "pos", (n, 3))
    _dev(q, torch.float32, "q", (n,))
    if y is None:
        y = torch.empty(n, 3, dtype=torch.float32, device=pos.device)
    if ws is None:
        ws = _workspace(lib.tiga_mp_dense_workspace(n), pos.device)
    _check(lib.tiga_mp_dense_fwd(n, _ptr(pos), _ptr(q), float(eps), REDUCE_SUM, _ptr(y), _ptr(ws), ws.numel(),
                                 _stream()))
    return y


def _edgenn_args(pos, x, W1, b1, W2, b2):
    n = pos.shape[0]
    _dev(pos, torch.float32, "pos", (n, 3))
    H, D = W1.shape
    F = D - 3
    O = W2.shape[0]
    _dev(W1, torch.float32, "W1", (H, D))
    _dev(b1, torch.float32, "b1", (H,))
    _dev(W2, torch.float32, "W2", (O, H))
    _dev(b2, torch.float32, "b2", (O,))
    if F > 0:
        _dev(x, torch.float32, "x", (n, F))
    return n, F, H, O


def tiga_mp_edgenn_fwd(pos, x, radius, W1, b1, W2, b2, ws=None):
    """y_i = sum over the radius relation of W2 relu(W1 [p_j - p_i; x_j] + b1) + b2; returns y fp32 [n, out]."""
    lib = load()
    n, F, H, O = _edgenn_args(pos, x, W1, b1, W2, b2)
    y = torch.empty(n, O, dtype=torch.float32, device=pos.device)
    if ws is None:
        ws = _workspace(lib.tiga_mp_edgenn_workspace(n, F, H, O), pos.device)
    _check(lib.tiga_mp_edgenn_fwd(n, F, H, O, _ptr(pos), _ptr(x) if F else None, float(radius), _ptr(W1), _ptr(b1),
                                  _ptr(W2), _ptr(b2), _ptr(y), _ptr(ws), ws.numel(), _stream()))
    return y


def tiga_mp_edgenn_bwd(pos, x, radius, W1, b1, W2, b2, dy, want=("dx", "dpos", "dW1", "db1", "dW2", "db2"), ws=None):
    """The VJP of tiga_mp_edgenn_fwd for the cotangent dy [n, out]; returns a dict of the wanted gradients."""
    lib = load()
    n, F, H, O = _edgenn_args(pos, x, W1, b1, W2, b2)
    _dev(dy, torch.float32, "dy", (n, O))
    shapes = dict(dx=(n, F), dpos=(n, 3), dW1=(H, 3 + F), db1=(H,), dW2=(O, H), db2=(O,))
    out = {k: torch.empty(*shapes[k], dtype=torch.float32, device=pos.device) for k in want if shapes[k][-1] > 0}
    if ws is None:
        ws = _workspace(lib.tiga_mp_edgenn_workspace(n, F, H, O), pos.device)
    g = lambda k: _ptr(out.get(k))
    _check(lib.tiga_mp_edgenn_bwd(n, F, H, O, _ptr(pos), _ptr(x) if F else None, float(radius), _ptr(W1), _ptr(b1),
                                  _ptr(W2), _ptr(b2), _ptr(dy), g("dx"), g("dpos"), g("dW1"), g("db1"), g("dW2"),
                                  g("db2"), _ptr(ws), ws.numel(), _stream()))
    return out


def tiga_mp_knn_fwd(pos: torch.Tensor, x: torch.Tensor | None, k: int, want_nbr: bool = False, ws=None):
    """Exact kNN relation (self excluded, key (fp32 d2, index)) with the neighbour sum y_i = sum x_j.

    pos fp32 [n, 3]; x fp32 [n, F] or None.  Returns y fp32 [n, F] (None without x), and the selected
    indices int32 [n, k] in key order when want_nbr."""
    lib = load()
    n = pos.shape[0]
    _dev(pos, torch.float32, "pos", (n, 3))
    F = 0
    if x is not None:
        _dev(x, torch.float32, "x")
        if x.dim() != 2 or x.shape[0] != n:
            raise ValueError(f"x must be [n, F] with n = {n}")
        F = x.shape[1]
    y = torch.empty(n, F, dtype=torch.float32, device=pos.device) if x is not None else None
    nbr = torch.empty(n, k, dtype=torch.int32, device=pos.device) if want_nbr else None
    if ws is None:
        ws = _workspace(lib.tiga_mp_knn_workspace(n), pos.device)
    _check(lib.tiga_mp_knn_fwd(n, F, _ptr(pos), _ptr(x) if F else None, int(k), REDUCE_SUM, _ptr(y) if F else None,
                               _ptr(nbr), _ptr(ws), ws.numel(), _stream()))
    return (y, nbr) if want_nbr else y


def _head_major(t, name, layout, shape=None):
    """The [heads, n, width] storage of t: t itself ("hnd": contiguous [heads, n, width]) or, for "nhd",
    the (n, heads, width) view of a contiguous (heads, n, width) allocation permuted back."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if t.dtype not in (torch.float16, torch.bfloat16):
        raise TypeError(f"{name} must be float16 or bfloat16, got {t.dtype}")
    if t.dim() != 3:
        raise ValueError(f"{name} must have 3 dimensions")
    if layout == "nhd":
        t = t.permute(1, 0, 2)
    elif layout != "hnd":
        raise ValueError(f"unknown layout {layout!r}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be head-major storage (layout {layout!r})")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has head-major shape {tuple(t.shape)}, expected {tuple(shape)}")
    return t


def tiga_mp_attention_fwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, scale: float | None = None,
                          relation: str = "triangular", want_lse: bool = False, layout: str = "hnd"):
    """Online-softmax attention over the triangular (causal, diagonal included) or dense relation.

    q, k, v: float16 or bfloat16, head-major [heads, n, width] (layout "hnd") or the (n, heads, width)
    view of head-major storage (layout "nhd").  scale defaults to width ** -0.5.  Returns y in the
    layout of q (and lse fp32 [heads, n] when want_lse)."""
    lib = load()
    qh = _head_major(q, "q", layout)
    H, n, D = qh.shape
    kh = _head_major(k, "k", layout, (H, n, D))
    vh = _head_major(v, "v", layout, (H, n, D))
    if kh.dtype != qh.dtype or vh.dtype != qh.dtype:
        raise TypeError("q, k and v must share one dtype")
    dt = DT_F16 if qh.dtype == torch.float16 else DT_BF16
    rel = {"triangular": REL_TRIANGULAR, "dense": REL_DENSE}[relation]
    if scale is None:
        scale = D ** -0.5
    yh = torch.empty(H, n, D, dtype=qh.dtype, device=qh.device)
    lse = torch.empty(H, n, dtype=torch.float32, device=qh.device) if want_lse else None
    _check(lib.tiga_mp_attention_fwd(n, H, D, dt, _ptr(qh), _ptr(kh), _ptr(vh), float(scale), rel, _ptr(yh),
                                     _ptr(lse), _stream()))
    y = yh.permute(1, 0, 2) if layout == "nhd" else yh
    return (y, lse) if want_lse else y


# ------------------------------------------- rectangular relations: cross attention, paged cache, rotary positions

_HALF_TYPES = {torch.float16: DT_F16, torch.bfloat16: DT_BF16}
_ROTARY_TYPES = {torch.float16: DT_F16, torch.bfloat16: DT_BF16, torch.float32: DT_F32}


# positions of the axes batch, heads, rows, width in a tensor of each layout (-1: no batch axis)
_AXES = {"bhnd": (0, 1, 2, 3), "bnhd": (0, 2, 1, 3), "hnd": (-1, 0, 1, 2), "nhd": (-1, 1, 0, 2)}


def _axes(layout, dims):
    if layout not in _AXES or len(layout) not in dims:
        raise ValueError(f"unknown layout {layout!r}")
    return _AXES[layout]


def _same_device(device: int, **tensors):
    """The call's tensors lie on one device, and that is the current one (whose stream the work goes to)."""
    for name, t in tensors.items():
        if t is not None and t.get_device() != device:
            raise ValueError(f"{name} is on {t.device}, expected cuda:{device}")
    if device != torch.cuda.current_device():
        raise ValueError(f"the tensors are on cuda:{device}, the current device is {torch.cuda.current_device()}")


def _rows(t, name, axes, dtype=None, shape=None):
    """(batch, heads, rows, width) of t and its view: any strides, the width contiguous."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if dtype is not None and t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    s, st = t.shape, t.stride()
    b, h, n, d = axes
    if len(s) != d + 1:
        raise ValueError(f"{name} must have {d + 1} dimensions")
    got = (s[b] if b >= 0 else 1, s[h], s[n], s[d])
    if shape is not None and got != shape:
        raise ValueError(f"{name} has (batch, heads, rows, width) {got}, expected {tuple(shape)}")
    if got[3] > 1 and st[d] != 1 and t.numel():
        raise ValueError(f"{name}: the width must be contiguous")
    # the stride of an axis with one entry is never used; torch leaves anything there
    return got, _View(t.data_ptr() or None, st[b] if got[0] > 1 else 0, st[h] if got[1] > 1 else 0,
                      st[n] if got[2] > 1 else 0)


def _given_or_new(ws, query, *args, device):
    """The workspace of a call on `device`: the caller's, or one of the size that query(*args) tells."""
    if ws is None:
        return _workspace(query(*args), device)
    if not isinstance(ws, torch.Tensor) or not ws.is_cuda:
        raise TypeError("ws must be a CUDA (HIP) tensor")
    if ws.device != device:
        raise ValueError(f"ws is on {ws.device}, expected {device}")
    if not ws.is_contiguous():
        raise ValueError("ws must be contiguous")
    return ws


def _like(t, axes):
    """A new contiguous tensor of t's shape, and its view."""
    y = t.new_empty(t.shape)
    return y, _rows(y, "output", axes)[1]


def _cross(q, k, v, src_len, layout):
    axes = _axes(layout, (4,))
    (B, H, N, D), qv = _rows(q, "q", axes)
    dt = _HALF_TYPES.get(q.dtype)
    if dt is None:
        raise TypeError("q must be a float16 or bfloat16 tensor")
    (Bk, Hk, S, Dk), kv = _rows(k, "k", axes, q.dtype)
    if Bk != B or Dk != D:
        raise ValueError(f"k has batch {Bk} and width {Dk}, q has {B} and {D}")
    _, vv = _rows(v, "v", axes, q.dtype, (B, Hk, S, D))
    _same_device(q.get_device(), k=k, v=v, src_len=src_len)
    if src_len is not None:
        _dev(src_len, torch.int32, "src_len", (B,))
    return _Cross(N, S, B, H, Hk, D, dt, src_len.data_ptr() if src_len is not None else None), qv, kv, vv, axes


def tiga_mp_attention_cross_fwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                                src_len: torch.Tensor | None = None, scale: float | None = None,
                                want_lse: bool = False, layout: str = "bhnd", ws=None):
    """Online-softmax attention of num_dst destinations over num_src sources a sequence (an encoder's states).

    q: float16 or bfloat16 [batch, heads, num_dst, width] (layout "bhnd"; "bnhd" has rows before heads);
    k, v: [batch, kv_heads, num_src, width], heads a multiple of kv_heads.  Any strides that are multiples
    of 8 elements, the width contiguous.  src_len: int32 [batch] on the device, the sources of each sequence
    (None: all).  A sequence without sources gives y = 0, lse = -inf.  scale defaults to width ** -0.5.
    Returns y in q's shape (and lse fp32 [batch, heads, num_dst] when want_lse)."""
    lib = load()
    rel, qv, kv, vv, axes = _cross(q, k, v, src_len, layout)
    y, yv = _like(q, axes)
    lse = q.new_empty((rel.batch, rel.heads, rel.num_dst), dtype=torch.float32) if want_lse else None
    ref = C.byref
    ws = _given_or_new(ws, lib.tiga_mp_attention_cross_fwd_workspace, ref(rel), device=q.device)
    _check(lib.tiga_mp_attention_cross_fwd(ref(rel), ref(qv), ref(kv), ref(vv),
                                           rel.width ** -0.5 if scale is None else float(scale), ref(yv), _ptr(lse),
                                           _ptr(ws), ws.nbytes, _stream()))
    return (y, lse) if want_lse else y


def tiga_mp_attention_cross_bwd(q, k, v, y, lse, dy, src_len: torch.Tensor | None = None,
                                scale: float | None = None, want=("dq", "dk", "dv"), layout: str = "bhnd", ws=None):
    """The VJP of tiga_mp_attention_cross_fwd for the cotangent dy, from the forward's y and lse; returns a
    dict of the wanted gradients in the inputs' shapes.  Gradients of sources past src_len are 0."""
    lib = load()
    rel, qv, kv, vv, axes = _cross(q, k, v, src_len, layout)
    shape = (rel.batch, rel.heads, rel.num_dst, rel.width)
    _, yv = _rows(y, "y", axes, q.dtype, shape)
    _, dyv = _rows(dy, "dy", axes, q.dtype, shape)
    _dev(lse, torch.float32, "lse", shape[:3])
    _same_device(q.get_device(), y=y, dy=dy, lse=lse)
    ref = C.byref
    out, refs = {}, [None, None, None]
    for i, (name, t) in enumerate((("dq", q), ("dk", k), ("dv", v))):
        if name in want:
            out[name], view = _like(t, axes)
            refs[i] = ref(view)
    ws = _given_or_new(ws, lib.tiga_mp_attention_cross_bwd_workspace, ref(rel), device=q.device)
    _check(lib.tiga_mp_attention_cross_bwd(ref(rel), ref(qv), ref(kv), ref(vv), ref(yv), _ptr(lse), ref(dyv),
                                           rel.width ** -0.5 if scale is None else float(scale), *refs, _ptr(ws),
                                           ws.nbytes, _stream()))
    return out


def _packed(q, k, v, ptr, layout):
    axes = _axes(layout, (3,))
    (_, H, N, D), qv = _rows(q, "q", axes)
    dt = _HALF_TYPES.get(q.dtype)
    if dt is None:
        raise TypeError("q must be a float16 or bfloat16 tensor")
    (_, Hk, Nk, Dk), kv = _rows(k, "k", axes, q.dtype)
    if Nk != N or Dk != D:
        raise ValueError(f"k has {Nk} rows of width {Dk}, q has {N} of {D}")
    _, vv = _rows(v, "v", axes, q.dtype, (1, Hk, N, D))
    _dev(ptr, torch.int32, "ptr")
    if ptr.dim() != 1 or ptr.numel() < 1:
        raise ValueError("ptr must be [batch + 1]")
    _same_device(q.get_device(), k=k, v=v, ptr=ptr)
    return _Packed(N, ptr.numel() - 1, H, Hk, D, dt, ptr.data_ptr()), qv, kv, vv, axes


def tiga_mp_attention_packed_fwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, ptr: torch.Tensor,
                                 scale: float | None = None, want_lse: bool = False, layout: str = "hnd", ws=None):
    """Causal attention within packed sequences: whole prompts of different lengths, or training documents.

    q: float16 or bfloat16 [heads, rows, width] (layout "hnd"; "nhd" has rows first); k, v: [kv_heads, rows, width],
    heads a multiple of kv_heads.  Any strides that are multiples of 8 elements, the width contiguous.  ptr: int32
    [batch + 1] on the device, sequence b is rows ptr[b] to ptr[b + 1], and a row reads its sequence's rows up to
    itself.  Rows of no sequence give y = 0, lse = -inf.  scale defaults to width ** -0.5.
    Returns y in q's shape (and lse fp32 [heads, rows] when want_lse)."""
    lib = load()
    rel, qv, kv, vv, axes = _packed(q, k, v, ptr, layout)
    y, yv = _like(q, axes)
    lse = q.new_empty((rel.heads, rel.num_rows), dtype=torch.float32) if want_lse else None
    ref = C.byref
    ws = _given_or_new(ws, lib.tiga_mp_attention_packed_fwd_workspace, ref(rel), device=q.device)
    _check(lib.tiga_mp_attention_packed_fwd(ref(rel), ref(qv), ref(kv), ref(vv),
                                            rel.width ** -0.5 if scale is None else float(scale), ref(yv), _ptr(lse),
                                            _ptr(ws), ws.nbytes, _stream()))
    return (y, lse) if want_lse else y


def tiga_mp_attention_packed_bwd(q, k, v, y, lse, dy, ptr: torch.Tensor, scale: float | None = None,
                                 want=("dq", "dk", "dv"), layout: str = "hnd", ws=None):
    """The VJP of tiga_mp_attention_packed_fwd for the cotangent dy, from the forward's y and lse; returns a dict of
    the wanted gradients in the inputs' shapes.  Gradients of rows of no sequence are 0."""
    lib = load()
    rel, qv, kv, vv, axes = _packed(q, k, v, ptr, layout)
    shape = (1, rel.heads, rel.num_rows, rel.width)
    _, yv = _rows(y, "y", axes, q.dtype, shape)
    _, dyv = _rows(dy, "dy", axes, q.dtype, shape)
    _dev(lse, torch.float32, "lse", shape[1:3])
    _same_device(q.get_device(), y=y, dy=dy, lse=lse)
    ref = C.byref
    out, refs = {}, [None, None, None]
    for i, (name, t) in enumerate((("dq", q), ("dk", k), ("dv", v))):
        if name in want:
            out[name], view = _like(t, axes)
            refs[i] = ref(view)
    ws = _given_or_new(ws, lib.tiga_mp_attention_packed_bwd_workspace, ref(rel), device=q.device)
    _check(lib.tiga_mp_attention_packed_bwd(ref(rel), ref(qv), ref(kv), ref(vv), ref(yv), _ptr(lse), ref(dyv),
                                            rel.width ** -0.5 if scale is None else float(scale), *refs, _ptr(ws),
                                            ws.nbytes, _stream()))
    return out


def tiga_rotary_frequencies(rot: int, base: float = 10000.0, scaling: str = "plain", factor: float = 1.0,
                            trained: float = 0.0, low: float = 1.0, high: float = 4.0) -> torch.Tensor:
    """Radians a position of each of the rot / 2 pairs: float64 on the host.

    scaling stretches them for contexts `factor` times the trained length: "linear" (all by the factor),
    "base" (a larger base) or "bands" (pairs of at most `low` turns over the trained length by the factor,
    of at least `high` turns not at all)."""
    kinds = dict(plain=ROTARY_PLAIN, linear=ROTARY_LINEAR, base=ROTARY_BASE, bands=ROTARY_BANDS)
    if scaling not in kinds:
        raise ValueError(f"unknown scaling {scaling!r}")
    freq = torch.empty(max(int(rot), 2) // 2, dtype=torch.float64)
    _check(load().tiga_rotary_frequencies(int(rot), float(base), kinds[scaling], float(factor), float(trained),
                                          float(low), float(high), _ptr(freq)))
    return freq


def _bound(name):
    """A tensor whose address a handle holds: written into freely, but not replaced (the handle would keep reading the
    old one, freed or not).  `handle.name += 1` writes in place and is fine."""

    def get(self):
        return self.__dict__[name]

    def put(self, value):
        if value is not self.__dict__.setdefault(name, value):
            raise AttributeError(f"{name} of a {type(self).__name__} cannot be replaced: write into it, or make another")

    return property(get, put)


class Rotary:
    """A rotation by positions: freq float64 [rot / 2] on the device (radians a position), the pairs (i, i + rot / 2)
    or (interleaved) (2 i, 2 i + 1), and an amplitude that multiplies the rotated elements.  freq's contents may
    change; another tensor in its place needs another Rotary."""

    freq = _bound("freq")

    def __init__(self, freq: torch.Tensor, interleaved: bool = False, amplitude: float = 1.0):
        self.freq = _dev(freq, torch.float64, "freq")
        if freq.dim() != 1:
            raise ValueError("freq must have one dimension")
        self._c = _Rotary(freq.data_ptr() if freq.numel() else None, 2 * freq.numel(),
                          PAIRS_ADJACENT if interleaved else PAIRS_HALF, float(amplitude))

    @property
    def ref(self):
        return C.byref(self._c)


def _rotary_call(name, x, pos, rot, layout, out):
    axes = _axes(layout, (3, 4))
    (B, H, N, D), xv = _rows(x, "x", axes)
    dt = _ROTARY_TYPES.get(x.dtype)
    if dt is None:
        raise TypeError("x must be a float16, bfloat16 or float32 tensor")
    pos_batch = 0
    if pos is not None:
        if pos.dim() == 2:
            _dev(pos, torch.int32, "pos", (B, N))
            pos_batch = N
        else:
            _dev(pos, torch.int32, "pos", (N,))
    if out is None:
        out, ov = _like(x, axes)
    else:
        _, ov = _rows(out, "out", axes, x.dtype, (B, H, N, D))
    _same_device(x.get_device(), pos=pos, freq=rot.freq, out=out)
    _check(getattr(load(), name)(B, H, N, D, dt, C.byref(xv), _ptr(pos), pos_batch, rot.ref, C.byref(ov), _stream()))
    return out


def tiga_mp_rotary_fwd(x: torch.Tensor, pos: torch.Tensor | None, rot: Rotary, layout: str = "bhnd", out=None):
    """Every row of x rotated by its position: pair (a, b) -> amplitude (a cos t - b sin t, a sin t + b cos t)
    with t = position * freq; elements past the rotated part are copied.

    x: float16, bfloat16 or float32, layout "bhnd", "bnhd", "hnd" or "nhd", any strides with a contiguous
    width.  pos: int32 [batch, rows] or [rows], None for the row's index.  out may be x (in place)."""
    return _rotary_call("tiga_mp_rotary_fwd", x, pos, rot, layout, out)


def tiga_mp_rotary_bwd(dy: torch.Tensor, pos: torch.Tensor | None, rot: Rotary, layout: str = "bhnd", out=None):
    """The VJP of tiga_mp_rotary_fwd: dy turned back by the same angles."""
    return _rotary_call("tiga_mp_rotary_bwd", dy, pos, rot, layout, out)


class KvCache:
    """A paged cache on the device.

    k_pages, v_pages: float16 or bfloat16 [num_pages, kv_heads, page_size, width], any strides that are
    multiples of 8 elements with a contiguous width (pages stored rows first are passed permuted);
    table: int32 [batch, table_width], position p of sequence b is row p % page_size of page
    table[b, p // page_size]; length: int32 [batch], positions of each sequence with the new ones of a
    call.  The tensors are the caller's; their contents may change between calls, other tensors in their
    places need another KvCache."""

    k_pages, v_pages, table, length = _bound("k_pages"), _bound("v_pages"), _bound("table"), _bound("length")

    def __init__(self, k_pages: torch.Tensor, v_pages: torch.Tensor, table: torch.Tensor, length: torch.Tensor):
        shape, kv = _rows(k_pages, "k_pages", _AXES["bhnd"])
        if k_pages.dtype not in _HALF_TYPES:
            raise TypeError("k_pages must be a float16 or bfloat16 tensor")
        _, vv = _rows(v_pages, "v_pages", _AXES["bhnd"], k_pages.dtype, shape)
        self.table = _dev(table, torch.int32, "table")
        if table.dim() != 2:
            raise ValueError("table must be [batch, table_width]")
        self.length = _dev(length, torch.int32, "length", (table.shape[0],))
        for name, t in (("v_pages", v_pages), ("table", table), ("length", length)):
            if t.device != k_pages.device:
                raise ValueError(f"{name} is on {t.device}, expected {k_pages.device}")
        self.k_pages, self.v_pages = k_pages, v_pages
        P, H, R, D = shape
        self.kv_heads, self.width, self.batch = H, D, table.shape[0]
        self._c = _Cache(P, R, H, D, _HALF_TYPES[k_pages.dtype], table.shape[0], table.shape[1], kv, vv,
                         table.data_ptr() if table.numel() else None, length.data_ptr() if length.numel() else None)

    @property
    def ref(self):
        return C.byref(self._c)


def _new_rows(cache, t, name, axes, heads=None, rows=None):
    """heads, rows and the view of a packed tensor of new tokens in the cache's type and width."""
    got, view = _rows(t, name, axes, cache.k_pages.dtype)
    if got[3] != cache.width or heads not in (None, got[1]) or rows not in (None, got[2]):
        raise ValueError(f"{name} has (heads, rows, width) {got[1:]}, expected "
                         f"({'heads' if heads is None else heads}, {'rows' if rows is None else rows}, {cache.width})")
    return got[1], got[2], view


def tiga_cache_validate(cache: KvCache, num_dst: int, dst_ptr: torch.Tensor):
    """Raise TigaError (TIGA_EGRAPH) if dst_ptr, the lengths or the pages they need are inconsistent.  Synchronizes."""
    _dev(dst_ptr, torch.int32, "dst_ptr", (cache.batch + 1,))
    _same_device(cache.k_pages.get_device(), dst_ptr=dst_ptr)
    _check(load().tiga_cache_validate(cache.ref, int(num_dst), _ptr(dst_ptr), _stream()))


def tiga_mp_cache_append(cache: KvCache, k: torch.Tensor, v: torch.Tensor, dst_ptr: torch.Tensor,
                         rot: Rotary | None = None, q: torch.Tensor | None = None, layout: str = "hnd", q_out=None):
    """Store new tokens' keys (rotated by their positions with rot) and values in the cache's pages.

    k, v: [kv_heads, rows, width] (layout "hnd"; "nhd" has rows first) of the cache's type, the new tokens
    of all sequences packed: sequence b owns rows dst_ptr[b] to dst_ptr[b + 1] (int32 [batch + 1]), its last
    row at position length[b] - 1.  With q [heads, rows, width] the queries are rotated by the same
    positions in the same launch and returned (q_out may be q).  Rows before dst_ptr[0] are returned
    unrotated; rows behind dst_ptr[batch] are left as q_out has them (uninitialized without q_out)."""
    axes = _axes(layout, (3,))
    _, rows, kv = _new_rows(cache, k, "k", axes, cache.kv_heads)
    _, _, vv = _new_rows(cache, v, "v", axes, cache.kv_heads, rows)
    _dev(dst_ptr, torch.int32, "dst_ptr", (cache.batch + 1,))
    ref = C.byref
    heads, qv, ov = 0, None, None
    if q is not None:
        if rot is None:
            raise ValueError("q is only taken to be rotated: rot is missing")
        heads, _, qv = _new_rows(cache, q, "q", axes, None, rows)
        if q_out is None:
            q_out, ov = _like(q, axes)
        else:
            _, _, ov = _new_rows(cache, q_out, "q_out", axes, heads, rows)
    elif q_out is not None:
        raise ValueError("q_out without q")
    _same_device(cache.k_pages.get_device(), k=k, v=v, dst_ptr=dst_ptr, q=q, q_out=q_out,
                 freq=rot.freq if rot is not None else None)
    _check(load().tiga_mp_cache_append(cache.ref, rows, _ptr(dst_ptr), ref(kv), ref(vv),
                                       rot.ref if rot is not None else None, heads, ref(qv) if qv is not None else None,
                                       ref(ov) if ov is not None else None, _stream()))
    return q_out


def tiga_mp_attention_paged_fwd(cache: KvCache, q: torch.Tensor, dst_ptr: torch.Tensor, scale: float | None = None,
                                want_lse: bool = False, layout: str = "hnd", y=None, ws=None):
    """Causal attention of new tokens over a paged cache that already holds their own keys and values.

    q: [heads, rows, width] (layout "hnd"; "nhd" has rows first) packed as in tiga_mp_cache_append, heads a
    multiple of the cache's; the row at position p reads positions 0 to p of its sequence.  Rows before
    dst_ptr[0] and behind dst_ptr[batch] are left as y has them (uninitialized without y, and in lse).  Returns y in q's shape (and lse fp32 [heads, rows])."""
    lib = load()
    axes = _axes(layout, (3,))
    heads, rows, qv = _new_rows(cache, q, "q", axes)
    _dev(dst_ptr, torch.int32, "dst_ptr", (cache.batch + 1,))
    if y is None:
        y, yv = _like(q, axes)
    else:
        _, _, yv = _new_rows(cache, y, "y", axes, heads, rows)
    _same_device(cache.k_pages.get_device(), q=q, y=y, dst_ptr=dst_ptr)
    lse = q.new_empty((heads, rows), dtype=torch.float32) if want_lse else None
    ref = C.byref
    ws = _given_or_new(ws, lib.tiga_mp_attention_paged_fwd_workspace, cache.ref, rows, heads, device=q.device)
    _check(lib.tiga_mp_attention_paged_fwd(cache.ref, rows, _ptr(dst_ptr), heads, ref(qv),
                                           cache.width ** -0.5 if scale is None else float(scale), ref(yv), _ptr(lse),
                                           _ptr(ws), ws.nbytes, _stream()))
    return (y, lse) if want_lse else y


def _prefix(cache, group_ptr, group_len):
    _dev(group_ptr, torch.int32, "group_ptr")
    if group_ptr.dim() != 1 or group_ptr.numel() < 1:
        raise ValueError("group_ptr must be [groups + 1]")
    _dev(group_len, torch.int32, "group_len", (group_ptr.numel() - 1,))
    _same_device(cache.k_pages.get_device(), group_ptr=group_ptr, group_len=group_len)
    return _Prefix(group_ptr.numel() - 1, group_ptr.data_ptr(), group_len.data_ptr() if group_len.numel() else None)


def tiga_prefix_validate(cache: KvCache, num_dst: int, dst_ptr: torch.Tensor, group_ptr: torch.Tensor,
                         group_len: torch.Tensor):
    """tiga_cache_validate, and raise TigaError (TIGA_EGRAPH) if the groups are inconsistent or a sequence's first new
    token lies below its group's length, whether or not so much would be read once.  Synchronizes."""
    _dev(dst_ptr, torch.int32, "dst_ptr", (cache.batch + 1,))
    _same_device(cache.k_pages.get_device(), dst_ptr=dst_ptr)
    _check(load().tiga_prefix_validate(cache.ref, C.byref(_prefix(cache, group_ptr, group_len)), int(num_dst),
                                       _ptr(dst_ptr), _stream()))


def tiga_mp_attention_prefix_fwd(cache: KvCache, q: torch.Tensor, dst_ptr: torch.Tensor, group_ptr: torch.Tensor,
                                 group_len: torch.Tensor, scale: float | None = None, want_lse: bool = False,
                                 layout: str = "hnd", y=None, ws=None):
    """tiga_mp_attention_paged_fwd for sequences of which groups share their first positions (a system prompt, a document):
    their keys and values are read once a group, for all of its rows.

    Group g is sequences group_ptr[g] to group_ptr[g + 1] (int32 [groups + 1] on the device), whose positions below
    group_len[g] (int32 [groups]) hold the same, in the same pages or in copies.  New tokens lie behind them (NaN for a
    sequence of whose own tokens some would be read once).  Other arguments and results as tiga_mp_attention_paged_fwd."""
    lib = load()
    axes = _axes(layout, (3,))
    heads, rows, qv = _new_rows(cache, q, "q", axes)
    _dev(dst_ptr, torch.int32, "dst_ptr", (cache.batch + 1,))
    if y is None:
        y, yv = _like(q, axes)
    else:
        _, _, yv = _new_rows(cache, y, "y", axes, heads, rows)
    prefix = _prefix(cache, group_ptr, group_len)
    _same_device(cache.k_pages.get_device(), q=q, y=y, dst_ptr=dst_ptr)
    lse = q.new_empty((heads, rows), dtype=torch.float32) if want_lse else None
    ref = C.byref
    ws = _given_or_new(ws, lib.tiga_mp_attention_prefix_fwd_workspace, cache.ref, ref(prefix), rows, heads, device=q.device)
    _check(lib.tiga_mp_attention_prefix_fwd(cache.ref, ref(prefix), rows, _ptr(dst_ptr), heads, ref(qv),
                                            cache.width ** -0.5 if scale is None else float(scale), ref(yv), _ptr(lse),
                                            _ptr(ws), ws.nbytes, _stream()))
    return (y, lse) if want_lse else y


def tiga_retention_validate(cache: KvCache):
    """Raise TigaError (TIGA_EGRAPH) if two sequences' positions lie in one page, or one's twice: tiga_mp_cache_weights and the
    cache that tiga_mp_cache_evict moves to need pages of each sequence's own.  Synchronizes."""
    _check(load().tiga_retention_validate(cache.ref, _stream()))


def _cells(cache, t, name):
    P, H, R = cache.k_pages.shape[:3]
    return _dev(t, torch.float32, name, (P, H, R))


def tiga_mp_cache_weights(cache: KvCache, q: torch.Tensor, lse: torch.Tensor, dst_ptr: torch.Tensor,
                          weights: torch.Tensor, out: torch.Tensor | None = None, decay: float = 1.0,
                          scale: float | None = None, layout: str = "hnd", ws=None):
    """Add the attention weights that new tokens give to the cached positions: decay * weights + sum exp(s - lse).

    q, dst_ptr, scale as for tiga_mp_attention_paged_fwd, lse fp32 [heads, rows] from it.  weights: fp32
    [num_pages, kv_heads, page_size], one for each row of the cache's pages, summed over the heads that share it; the
    new tokens' own count as 0 before.  out: where the sums go (None: weights, in place).  No page may be two sequences'
    (tiga_retention_validate): a prefix that several share lies in copies here.  Returns out."""
    lib = load()
    axes = _axes(layout, (3,))
    heads, rows, qv = _new_rows(cache, q, "q", axes)
    _dev(dst_ptr, torch.int32, "dst_ptr", (cache.batch + 1,))
    _dev(lse, torch.float32, "lse", (heads, rows))
    _cells(cache, weights, "weights")
    out = weights if out is None else _cells(cache, out, "out")
    _same_device(cache.k_pages.get_device(), q=q, lse=lse, dst_ptr=dst_ptr, weights=weights, out=out)
    ws = _given_or_new(ws, lib.tiga_mp_cache_weights_workspace, cache.ref, rows, heads, device=q.device)
    _check(lib.tiga_mp_cache_weights(cache.ref, rows, _ptr(dst_ptr), heads, C.byref(qv), _ptr(lse),
                                     cache.width ** -0.5 if scale is None else float(scale), float(decay), _ptr(weights),
                                     _ptr(out), _ptr(ws), ws.nbytes, _stream()))
    return out


def tiga_mp_cache_evict(cache: KvCache, weights: torch.Tensor, to: KvCache | None = None,
                        to_weights: torch.Tensor | None = None, *, keep: int, recent: int = 0, kept=None, ws=None):
    """Keep `keep` positions of each sequence and source head: the last `recent`, and those of the largest weights.

    weights: fp32 [num_pages, kv_heads, page_size].  They move in order to the first positions of `to` (keys, values, and
    weights to to_weights if given), whose pages are none of the cache's sequences' own; to.length is set to
    min(length, keep).  Without `to` the cache is evicted from in place, weights and length too.  No page that rows move to
    may be two sequences' (tiga_retention_validate), in place none of the cache.  Keys keep the rotation of their old
    positions: rotate later tokens by their true positions (tiga_mp_rotary_fwd) and append them unrotated.
    Returns kept: int32 [batch, kv_heads, keep], the positions that stayed, -1 past them."""
    lib = load()
    if max(abs(int(keep)), abs(int(recent))) >= 1 << 31:  # the C arguments have 32 bits
        raise ValueError("keep and recent must be below 2^31")
    _cells(cache, weights, "weights")
    if to is None:
        to, to_weights = cache, weights if to_weights is None else to_weights
    if to_weights is not None:
        _cells(to, to_weights, "to_weights")
    shape = (cache.batch, cache.kv_heads, int(keep))
    if int(keep) < 1:
        raise ValueError("keep must be at least 1")
    kept = weights.new_empty(shape, dtype=torch.int32) if kept is None else _dev(kept, torch.int32, "kept", shape)
    _same_device(cache.k_pages.get_device(), weights=weights, to=to.k_pages, to_weights=to_weights, kept=kept)
    ref = cache.ref, to.ref
    ws = _given_or_new(ws, lib.tiga_mp_cache_evict_workspace, *ref, int(keep), device=weights.device)
    _check(lib.tiga_mp_cache_evict(ref[0], _ptr(weights), int(keep), int(recent), ref[1], _ptr(to_weights), _ptr(to.length),
                                   _ptr(kept), _ptr(ws), ws.nbytes, _stream()))
    return kept


# ------------------------------------------------------------ autograd wrappers
#
# The paper's Torch interop (the fused operator as a differentiable function):
# the forward calls the fused entry point, the backward its vector-Jacobian
# product.  The sum saves x and w (dx needs w, dw needs x); max also saves the
# forward's argmax, which routes its gradients.  The relation is a topology
# snapshot: it is not differentiated.


class CsrAggregate(torch.autograd.Function):
    """y = reduce_{e in row i} w[e] * x[col[e]] over a stored CSR relation."""

    @staticmethod
    def forward(ctx, x, w, rel, reducer, rev):
        y, arg = tiga_mp_csr_fwd(rel, x, w, reducer=reducer)
        ctx.rel, ctx.reducer, ctx.rev = rel, reducer, rev
        ctx.save_for_backward(x, w, arg)
        if arg is not None:
            ctx.mark_non_differentiable(arg)
        return y, arg

    @staticmethod
    def backward(ctx, gy, _garg):
        x, w, arg = ctx.saved_tensors
        want_dx = ctx.needs_input_grad[0]
        want_dw = w is not None and ctx.needs_input_grad[1]
        if not (want_dx or want_dw):
            return None, None, None, None, None
        dx, dw = tiga_mp_csr_bwd(ctx.rel, gy.contiguous(), x, w, reducer=ctx.reducer, argmax=arg, rev=ctx.rev,
                                 want_dx=want_dx, want_dw=want_dw)
        return dx, dw, None, None, None


def csr_aggregate(rel: Csr, x: torch.Tensor, w: torch.Tensor | None = None, reducer: int = REDUCE_SUM,
                  rev: CsrT | None = None):
    """Differentiable fused aggregation; returns (y, argmax or None).  With `rev` (the reverse incidence)
    the backward is the deterministic single traversal, without it dx accumulates by atomics."""
    return CsrAggregate.apply(x, w, rel, reducer, rev)


class RadiusAggregate(torch.autograd.Function):
    """y_i = sum_{j != i, |p_j - p_i| < r} exp(-|p_j - p_i|^2 / sigma^2) x_j (membership not differentiated)."""

    @staticmethod
    def forward(ctx, pos, x, radius, sigma):
        y, _ = tiga_mp_radius_fwd(pos, x, radius, sigma, want_count=False)
        ctx.radius, ctx.sigma = radius, sigma
        ctx.save_for_backward(pos, x)
        return y

    @staticmethod
    def backward(ctx, gy):
        pos, x = ctx.saved_tensors
        want_dpos, want_dx = ctx.needs_input_grad[0], ctx.needs_input_grad[1]
        if not (want_dpos or want_dx):
            return None, None, None, None
        dx, dpos = tiga_mp_radius_bwd(pos, x, gy.contiguous(), ctx.radius, ctx.sigma, want_dx=want_dx,
                                      want_dpos=want_dpos)
        return dpos, dx, None, None


def radius_aggregate(pos: torch.Tensor, x: torch.Tensor, radius: float, sigma: float) -> torch.Tensor:
    """Differentiable fused aggregation over the generated radius relation."""
    return RadiusAggregate.apply(pos, x, radius, sigma)


class EdgeMLP(torch.autograd.Function):
    """y = sum over the radius relation of W2 relu(W1 [p_j - p_i; x_j] + b1) + b2 (membership fixed)."""

    @staticmethod
    def forward(ctx, pos, x, W1, b1, W2, b2, radius):
        ctx.radius = radius
        ctx.save_for_backward(pos, x, W1, b1, W2, b2)
        return tiga_mp_edgenn_fwd(pos, x, radius, W1, b1, W2, b2)

    @staticmethod
    def backward(ctx, dy):
        pos, x, W1, b1, W2, b2 = ctx.saved_tensors
        g = tiga_mp_edgenn_bwd(pos, x, ctx.radius, W1, b1, W2, b2, dy.contiguous())
        return g["dpos"], g.get("dx"), g["dW1"], g["db1"], g["dW2"], g["db2"], None


def edge_mlp(pos, x, W1, b1, W2, b2, radius):
    return EdgeMLP.apply(pos, x, W1, b1, W2, b2, radius)


class CrossAttention(torch.autograd.Function):
    """y_i = sum_j softmax_j(scale <q_i, k_j>) v_j over the sources of a padded batch (lengths not differentiated)."""

    @staticmethod
    def forward(ctx, q, k, v, src_len, scale, layout):
        y, lse = tiga_mp_attention_cross_fwd(q, k, v, src_len, scale, want_lse=True, layout=layout)
        ctx.scale, ctx.layout = scale, layout
        ctx.save_for_backward(q, k, v, src_len, y, lse)
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        q, k, v, src_len, y, lse = ctx.saved_tensors
        want = [n for n, need in zip(("dq", "dk", "dv"), ctx.needs_input_grad) if need]
        if not want:
            return None, None, None, None, None, None
        if _unreadable(dy):
            dy = dy.clone(memory_format=torch.contiguous_format)
        g = tiga_mp_attention_cross_bwd(q, k, v, y, lse, dy, src_len, ctx.scale, want=want, layout=ctx.layout)
        return g.get("dq"), g.get("dk"), g.get("dv"), None, None, None


def _unreadable(t):
    """Whether a cotangent's strides or alignment are none the kernels take (autograd may hand over any)."""
    return t.stride(-1) != 1 or t.data_ptr() % 16 != 0 or any(s % 8 for s in t.stride()[:-1])


def cross_attention(q, k, v, src_len: torch.Tensor | None = None, scale: float | None = None, layout: str = "bhnd"):
    """Differentiable cross attention; see tiga_mp_attention_cross_fwd.  Gradients once, not of gradients.

    Forward and backward can be captured in a graph.  As with every differentiable function of torch, a backward
    pass that accumulates into leaves (loss.backward()) must not be captured while an eager graph of the same leaves
    is alive; torch.autograd.grad inside the capture has no such condition."""
    return CrossAttention.apply(q, k, v, src_len, scale, layout)


class PackedAttention(torch.autograd.Function):
    """y_i = sum_{j <= i} softmax_j(scale <q_i, k_j>) v_j within packed sequences (their bounds not differentiated)."""

    @staticmethod
    def forward(ctx, q, k, v, ptr, scale, layout):
        y, lse = tiga_mp_attention_packed_fwd(q, k, v, ptr, scale, want_lse=True, layout=layout)
        ctx.scale, ctx.layout = scale, layout
        ctx.save_for_backward(q, k, v, ptr, y, lse)
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        q, k, v, ptr, y, lse = ctx.saved_tensors
        want = [n for n, need in zip(("dq", "dk", "dv"), ctx.needs_input_grad) if need]
        if not want:
            return None, None, None, None, None, None
        if _unreadable(dy):
            dy = dy.clone(memory_format=torch.contiguous_format)
        g = tiga_mp_attention_packed_bwd(q, k, v, y, lse, dy, ptr, ctx.scale, want=want, layout=ctx.layout)
        return g.get("dq"), g.get("dk"), g.get("dv"), None, None, None


def packed_attention(q, k, v, ptr: torch.Tensor, scale: float | None = None, layout: str = "hnd"):
    """Differentiable causal attention of packed sequences; see tiga_mp_attention_packed_fwd.  Gradients once, not of
    gradients.  What cross_attention says of graphs holds here too."""
    return PackedAttention.apply(q, k, v, ptr, scale, layout)


class RotaryPositions(torch.autograd.Function):
    """Rows rotated by their positions (positions and frequencies not differentiated)."""

    @staticmethod
    def forward(ctx, x, pos, rot, layout):
        ctx.rot, ctx.layout = rot, layout
        ctx.save_for_backward(pos, rot.freq)  # freq too: torch then refuses a backward after a change in place
        return tiga_mp_rotary_fwd(x, pos, rot, layout)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        pos, _ = ctx.saved_tensors
        if dy.stride(-1) != 1:
            dy = dy.contiguous()
        return tiga_mp_rotary_bwd(dy, pos, ctx.rot, ctx.layout), None, None, None


def rotary(x: torch.Tensor, pos: torch.Tensor | None, rot: Rotary, layout: str = "bhnd") -> torch.Tensor:
    """Differentiable rotary positions; see tiga_mp_rotary_fwd.  Gradients once, not of gradients.  What cross_attention says
    of graphs holds here too."""
    return RotaryPositions.apply(x, pos, rot, layout)
