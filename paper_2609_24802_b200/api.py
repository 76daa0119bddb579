"""ctypes binding of libtiga.so -- argument marshalling only.

Every function has the name of the C entry point it calls (see ``include/tiga.h``) and takes
torch CUDA tensors for the device arrays.  Nothing is computed here; when the library is
missing the import fails, there is no fallback of any kind.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
import struct

import torch

__all__ = [
    "TigaError", "load_library", "EXPORTS", "SUM", "MAX", "MAX64", "F32", "F16",
    "MSG_COPY", "MSG_WEIGHTED", "MSG_GAUSS", "MSG_DIST", "MSG_LJ",
    "CsrRelation", "tiga_status_string", "tiga_csr_workspace_bytes", "tiga_validate_csr",
    "tiga_apply_csr", "tiga_apply_csr_builtin_ws", "tiga_apply_csr_backward", "tiga_csr_degree_histogram",
    "CsrPlan", "tiga_csr_plan_build", "tiga_csr_planned_workspace_bytes", "tiga_apply_csr_planned",
    "tiga_radius_grid", "tiga_validate_points", "tiga_radius_workspace_bytes", "tiga_radius_bin",
    "tiga_apply_radius", "tiga_apply_radius_backward", "tiga_apply_radius_mlp",
    "tiga_apply_radius_mlp_backward", "tiga_knn_workspace_bytes", "tiga_apply_knn",
    "tiga_csr_attention_workspace_bytes", "tiga_apply_csr_attention", "launch_count",
    "BF16", "DenseRelation", "tiga_dense_attention_workspace_bytes", "tiga_apply_dense_attention",
    "tiga_apply_dense_attention_backward", "TriangularRelation", "tiga_triangular_attention_workspace_bytes",
    "tiga_apply_triangular_attention", "tiga_apply_triangular_attention_backward", "PagedCache", "tiga_paged_attention_workspace_bytes", "tiga_apply_paged_attention",
    "SharedPrefixes", "tiga_shared_attention_workspace_bytes", "tiga_apply_shared_attention",
    "tiga_paged_weights_workspace_bytes", "tiga_paged_attention_weights", "tiga_paged_evict",
    "tiga_paged_append", "ROT_PLAIN", "ROT_LINEAR", "ROT_BASE", "ROT_BANDS", "tiga_rotary_frequencies", "Rotary", "tiga_apply_rotary",
]

SUM, MAX, MAX64 = 0, 1, 2      # MAX64: max reducer whose argmax holds 64-bit edge positions (int64)
F32, F16, BF16 = 0, 1, 2
I32, I64 = 0, 1
MSG_COPY, MSG_WEIGHTED, MSG_GAUSS, MSG_DIST, MSG_LJ = 0, 1, 2, 3, 4
ROT_HALVES, ROT_PAIRS = 0, 1
ROT_PLAIN, ROT_LINEAR, ROT_BASE, ROT_BANDS = 0, 1, 2, 3

EXPORTS = [
    "tiga_status_string", "tiga_kernel_launches", "tiga_checked_status", "tiga_is_checked_build", "tiga_csr_workspace_bytes", "tiga_validate_csr", "tiga_apply_csr",
    "tiga_apply_csr_builtin_ws", "tiga_apply_csr_backward", "tiga_csr_degree_histogram", "tiga_radius_grid",
    "tiga_csr_plan_bytes", "tiga_csr_plan_workspace_bytes", "tiga_csr_plan_build", "tiga_csr_planned_workspace_bytes",
    "tiga_apply_csr_planned",
    "tiga_validate_points", "tiga_radius_workspace_bytes", "tiga_radius_bin", "tiga_apply_radius",
    "tiga_apply_radius_backward", "tiga_apply_radius_mlp", "tiga_apply_radius_mlp_backward",
    "tiga_knn_workspace_bytes", "tiga_apply_knn", "tiga_csr_attention_workspace_bytes", "tiga_apply_csr_attention",
    "tiga_dense_attention_workspace_bytes", "tiga_apply_dense_attention", "tiga_apply_dense_attention_backward",
    "tiga_triangular_attention_workspace_bytes", "tiga_apply_triangular_attention", "tiga_apply_triangular_attention_backward",
    "tiga_paged_attention_workspace_bytes", "tiga_apply_paged_attention", "tiga_paged_append", "tiga_rotary_frequencies", "tiga_apply_rotary",
    "tiga_shared_attention_workspace_bytes", "tiga_apply_shared_attention",
    "tiga_paged_weights_workspace_bytes", "tiga_paged_attention_weights", "tiga_paged_evict",
]

_HERE = os.path.dirname(os.path.abspath(__file__))
# TIGA_CHECKED=1 in the environment selects the checked build (range-checked indices, status word)
CHECKED = os.environ.get("TIGA_CHECKED", "0") not in ("", "0")
LIB_PATH = os.path.join(_HERE, "libtiga_checked.so" if CHECKED else "libtiga.so")


class TigaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {tiga_status_string(status)} (status {status})")


class _Msg(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("p0", ctypes.c_float), ("p1", ctypes.c_float)]


class _Csr(ctypes.Structure):
    _fields_ = [("rowptr", ctypes.c_void_p), ("rowptr_type", ctypes.c_int32), ("col", ctypes.c_void_p),
                ("n_dst", ctypes.c_int64), ("n_src", ctypes.c_int64), ("n_edges", ctypes.c_int64)]


class _Box(ctypes.Structure):
    _fields_ = [("len", ctypes.c_float * 3), ("periodic", ctypes.c_int32 * 3)]


class _EdgeMlp(ctypes.Structure):
    _fields_ = [("f_in", ctypes.c_int32), ("hidden", ctypes.c_int32), ("f_out", ctypes.c_int32),
                ("W1", ctypes.c_void_p), ("b1", ctypes.c_void_p), ("W2", ctypes.c_void_p), ("b2", ctypes.c_void_p)]


class _Plan(ctypes.Structure):
    _fields_ = [("n_dst", ctypes.c_int64), ("n_src", ctypes.c_int64), ("n_edges", ctypes.c_int64), ("n_hot", ctypes.c_int64),
                ("min_hot_degree", ctypes.c_int64), ("hot_edges", ctypes.c_int64), ("off_col", ctypes.c_int64),
                ("off_hot_id", ctypes.c_int64), ("used_bytes", ctypes.c_int64)]


class _Stride(ctypes.Structure):
    _fields_ = [("row", ctypes.c_int64), ("head", ctypes.c_int64)]


class _Heads(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("D", ctypes.c_int32),
                ("scale", ctypes.c_float), ("q", _Stride), ("key", _Stride), ("value", _Stride), ("grad_out", _Stride)]


class _Dense(ctypes.Structure):
    _fields_ = [("q_start", ctypes.c_void_p), ("kv_start", ctypes.c_void_p), ("kv_mask", ctypes.c_void_p),
                ("n_seg", ctypes.c_int64), ("n_q", ctypes.c_int64), ("n_kv", ctypes.c_int64)]


class _Pages(ctypes.Structure):
    _fields_ = [("key", ctypes.c_void_p), ("value", ctypes.c_void_p), ("table", ctypes.c_void_p), ("kv_len", ctypes.c_void_p),
                ("n_seg", ctypes.c_int64), ("n_pages", ctypes.c_int64), ("page_size", ctypes.c_int64), ("table_stride", ctypes.c_int64),
                ("max_pages", ctypes.c_int64), ("page_stride", ctypes.c_int64), ("slot_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class _Prefixes(ctypes.Structure):
    _fields_ = [("group_start", ctypes.c_void_p), ("shared", ctypes.c_void_p), ("n_groups", ctypes.c_int64)]


class _Weights(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("seg", ctypes.c_int64), ("head", ctypes.c_int64), ("length", ctypes.c_int64)]


class _Rotary(ctypes.Structure):
    _fields_ = [("freq", ctypes.c_void_p), ("turned", ctypes.c_int32), ("layout", ctypes.c_int32), ("magnitude", ctypes.c_float)]


_lib = None


def load_library() -> ctypes.CDLL:
    """Load libtiga.so; raises ImportError when it has not been built (no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with "
                          "`python -m paper_2609_24802_b200.build` (nvcc, sm_100a)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, sz, f = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float
    lib.tiga_status_string.restype = ctypes.c_char_p
    lib.tiga_status_string.argtypes = [ctypes.c_int]
    lib.tiga_kernel_launches.restype = i64
    lib.tiga_kernel_launches.argtypes = []
    lib.tiga_checked_status.restype = ctypes.c_uint32
    lib.tiga_checked_status.argtypes = [ctypes.c_int]
    lib.tiga_is_checked_build.restype = ctypes.c_int
    lib.tiga_is_checked_build.argtypes = []
    lib.tiga_csr_workspace_bytes.restype = sz
    lib.tiga_csr_workspace_bytes.argtypes = [ctypes.POINTER(_Csr), i32, ctypes.c_int, ctypes.c_int, ctypes.c_int]
    lib.tiga_validate_csr.restype = ctypes.c_int
    lib.tiga_validate_csr.argtypes = [ctypes.POINTER(_Csr), ctypes.c_int, vp, sz, vp]
    lib.tiga_apply_csr.restype = ctypes.c_int
    lib.tiga_apply_csr.argtypes = [ctypes.POINTER(_Csr), vp, ctypes.c_int, i32, vp, ctypes.POINTER(_Msg), ctypes.c_int,
                                   vp, vp, vp, sz, vp]
    lib.tiga_apply_csr_builtin_ws.restype = ctypes.c_int
    lib.tiga_apply_csr_builtin_ws.argtypes = [ctypes.POINTER(_Csr), vp, ctypes.c_int, i32, vp, ctypes.POINTER(_Msg),
                                              ctypes.c_int, vp, vp, vp]
    lib.tiga_apply_csr_backward.restype = ctypes.c_int
    lib.tiga_apply_csr_backward.argtypes = [ctypes.POINTER(_Csr), vp, ctypes.c_int, i32, vp, ctypes.POINTER(_Msg), ctypes.c_int,
                                            vp, vp, vp, vp, vp, sz, vp]
    lib.tiga_csr_plan_bytes.restype = sz
    lib.tiga_csr_plan_bytes.argtypes = [ctypes.POINTER(_Csr), i64]
    lib.tiga_csr_plan_workspace_bytes.restype = sz
    lib.tiga_csr_plan_workspace_bytes.argtypes = [ctypes.POINTER(_Csr)]
    lib.tiga_csr_plan_build.restype = ctypes.c_int
    lib.tiga_csr_plan_build.argtypes = [ctypes.POINTER(_Csr), i64, vp, sz, vp, sz, ctypes.POINTER(_Plan), vp]
    lib.tiga_csr_planned_workspace_bytes.restype = sz
    lib.tiga_csr_planned_workspace_bytes.argtypes = [ctypes.POINTER(_Csr), ctypes.POINTER(_Plan), i32, ctypes.c_int, ctypes.c_int]
    lib.tiga_apply_csr_planned.restype = ctypes.c_int
    lib.tiga_apply_csr_planned.argtypes = [ctypes.POINTER(_Csr), ctypes.POINTER(_Plan), vp, vp, ctypes.c_int, i32, vp,
                                           ctypes.POINTER(_Msg), ctypes.c_int, vp, vp, vp, sz, vp]
    lib.tiga_csr_degree_histogram.restype = ctypes.c_int
    lib.tiga_csr_degree_histogram.argtypes = [ctypes.POINTER(_Csr), vp, i64, vp, vp]
    lib.tiga_radius_grid.restype = ctypes.c_int
    lib.tiga_radius_grid.argtypes = [i64, f, ctypes.POINTER(_Box), ctypes.POINTER(i32), ctypes.POINTER(f)]
    lib.tiga_validate_points.restype = ctypes.c_int
    lib.tiga_validate_points.argtypes = [vp, i64, ctypes.POINTER(_Box), ctypes.c_int, vp, sz, vp]
    lib.tiga_radius_workspace_bytes.restype = sz
    lib.tiga_radius_workspace_bytes.argtypes = [i64, i32, f, ctypes.POINTER(_Box), ctypes.c_int]
    lib.tiga_radius_bin.restype = ctypes.c_int
    lib.tiga_radius_bin.argtypes = [vp, i64, f, ctypes.POINTER(_Box), vp, vp, vp, vp, sz, vp]
    lib.tiga_apply_radius.restype = ctypes.c_int
    lib.tiga_apply_radius.argtypes = [vp, vp, i64, i32, f, ctypes.POINTER(_Box), ctypes.POINTER(_Msg), vp, vp, vp, sz, vp]
    lib.tiga_apply_radius_backward.restype = ctypes.c_int
    lib.tiga_apply_radius_backward.argtypes = [vp, vp, i64, i32, f, ctypes.POINTER(_Box), ctypes.POINTER(_Msg), vp, vp, vp,
                                               vp, sz, ctypes.c_int, vp]
    lib.tiga_apply_radius_mlp.restype = ctypes.c_int
    lib.tiga_apply_radius_mlp.argtypes = [vp, vp, i64, f, ctypes.POINTER(_Box), ctypes.POINTER(_EdgeMlp), vp, vp, vp, sz, vp]
    lib.tiga_apply_radius_mlp_backward.restype = ctypes.c_int
    lib.tiga_apply_radius_mlp_backward.argtypes = [vp, vp, i64, f, ctypes.POINTER(_Box), ctypes.POINTER(_EdgeMlp), vp,
                                                   vp, vp, vp, vp, vp, vp, vp, sz, ctypes.c_int, vp]
    lib.tiga_csr_attention_workspace_bytes.restype = sz
    lib.tiga_csr_attention_workspace_bytes.argtypes = [ctypes.POINTER(_Csr), i32]
    lib.tiga_apply_csr_attention.restype = ctypes.c_int
    lib.tiga_apply_csr_attention.argtypes = [ctypes.POINTER(_Csr), vp, vp, vp, i32, f, vp, vp, vp, sz, vp]
    d, ref = ctypes.c_double, ctypes.POINTER
    lib.tiga_dense_attention_workspace_bytes.restype = sz
    lib.tiga_dense_attention_workspace_bytes.argtypes = [ref(_Dense), ref(_Heads), ctypes.c_int]
    lib.tiga_apply_dense_attention.restype = ctypes.c_int
    lib.tiga_apply_dense_attention.argtypes = [ref(_Dense), ref(_Heads), vp, vp, vp, vp, vp, vp, sz, vp]
    lib.tiga_apply_dense_attention_backward.restype = ctypes.c_int
    lib.tiga_apply_dense_attention_backward.argtypes = [ref(_Dense), ref(_Heads), vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.tiga_triangular_attention_workspace_bytes.restype = sz
    lib.tiga_triangular_attention_workspace_bytes.argtypes = lib.tiga_dense_attention_workspace_bytes.argtypes
    lib.tiga_apply_triangular_attention.restype = ctypes.c_int
    lib.tiga_apply_triangular_attention.argtypes = lib.tiga_apply_dense_attention.argtypes
    lib.tiga_apply_triangular_attention_backward.restype = ctypes.c_int
    lib.tiga_apply_triangular_attention_backward.argtypes = lib.tiga_apply_dense_attention_backward.argtypes
    lib.tiga_paged_attention_workspace_bytes.restype = sz
    lib.tiga_paged_attention_workspace_bytes.argtypes = [ref(_Pages), ref(_Heads), i64]
    lib.tiga_apply_paged_attention.restype = ctypes.c_int
    lib.tiga_apply_paged_attention.argtypes = [ref(_Pages), ref(_Heads), vp, vp, i64, ctypes.c_int, vp, vp, vp, sz, vp]
    lib.tiga_shared_attention_workspace_bytes.restype = sz
    lib.tiga_shared_attention_workspace_bytes.argtypes = [ref(_Pages), ref(_Heads), ref(_Prefixes), i64]
    lib.tiga_apply_shared_attention.restype = ctypes.c_int
    lib.tiga_apply_shared_attention.argtypes = [ref(_Pages), ref(_Heads), ref(_Prefixes), vp, vp, i64, ctypes.c_int, vp, vp, vp, sz, vp]
    lib.tiga_paged_weights_workspace_bytes.restype = sz
    lib.tiga_paged_weights_workspace_bytes.argtypes = [ref(_Pages), ref(_Heads), i64]
    lib.tiga_paged_attention_weights.restype = ctypes.c_int
    lib.tiga_paged_attention_weights.argtypes = [ref(_Pages), ref(_Heads), vp, vp, i64, vp, ctypes.c_int, ref(_Weights), ref(_Weights), vp, sz, vp]
    lib.tiga_paged_evict.restype = ctypes.c_int
    lib.tiga_paged_evict.argtypes = [ref(_Pages), ref(_Pages), ref(_Heads), ref(_Weights), i64, i64, ref(_Weights), vp, vp, vp]
    lib.tiga_paged_append.restype = ctypes.c_int
    lib.tiga_paged_append.argtypes = [ref(_Pages), ref(_Heads), vp, vp, vp, i64, ref(_Rotary), vp]
    lib.tiga_rotary_frequencies.restype = ctypes.c_int
    lib.tiga_rotary_frequencies.argtypes = [i32, d, i32, d, d, d, d, ref(d), ref(f)]
    lib.tiga_apply_rotary.restype = ctypes.c_int
    lib.tiga_apply_rotary.argtypes = [ref(_Rotary), vp, ref(_Stride), vp, ref(_Stride), ctypes.c_int, i64, i32, i32, vp, i32, ctypes.c_int, vp]
    lib.tiga_knn_workspace_bytes.restype = sz
    lib.tiga_knn_workspace_bytes.argtypes = [i64, i32, ctypes.POINTER(_Box)]
    lib.tiga_apply_knn.restype = ctypes.c_int
    lib.tiga_apply_knn.argtypes = [vp, vp, i64, i32, i32, ctypes.POINTER(_Box), vp, vp, vp, vp, sz, vp]
    _lib = lib
    return lib


_L = load_library()      # fail at import time, loudly, when the CUDA library is not there

# A call on a small relation is bound by its marshalling, so the calls below avoid what costs a microsecond each:
# the message structs of the stored relation are built once, a stream is looked up by its handle (no Stream object),
# pointers are passed as plain integers, outputs are allocated with new_empty.
# (The two look-ups are torch's own shortcuts, not its documented interface: where a build of torch lacks them, a stream
# object is asked.)
_current_device = getattr(torch._C, "_cuda_getDevice", None)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def checked_status(reset: bool = True) -> int:
    """Bits of the checked build's status word (0 in the normal build): 1 source index, 2 edge position,
    4 point id, 8 slot.  Synchronises the device."""
    return int(_L.tiga_checked_status(int(reset)))


def is_checked_build() -> bool:
    return bool(_L.tiga_is_checked_build())


def launch_count() -> int:
    """Kernels launched by the library so far in this process (counted inside the library)."""
    return int(_L.tiga_kernel_launches())


def _ptr(t):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device arrays must be contiguous CUDA tensors"
    return t.data_ptr()


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    return _raw_stream(_current_device()) if _raw_stream and _current_device else torch.cuda.current_stream().cuda_stream


def _ok(st, where):
    if st != 0:
        raise TigaError(st, where)


def _ws(nbytes, like):
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=like.device)


def _new(like, shape, dtype=torch.float32):
    """Uninitialised fp32 (or `dtype`) array on the device of `like`."""
    return like.new_empty(shape) if like.dtype is dtype else like.new_empty(shape, dtype=dtype)


_ARG_DTYPE = {MAX: torch.int32, MAX64: torch.int64}


def _dt(t):
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.float16:
        return F16
    raise TypeError("features must be float32 or float16")


def tiga_status_string(status: int) -> str:
    return _L.tiga_status_string(int(status)).decode()


class CsrRelation:
    """Host-side descriptor (the C struct ``tiga_csr``) of device CSR arrays."""

    def __init__(self, rowptr: torch.Tensor, col: torch.Tensor, n_src: int):
        assert rowptr.dtype in (torch.int32, torch.int64) and col.dtype == torch.int32
        self.rowptr, self.col = rowptr, col
        self.n_dst = rowptr.numel() - 1
        self.n_src = int(n_src)
        self.n_edges = col.numel()
        self.c = _Csr(rowptr.data_ptr(), I32 if rowptr.dtype == torch.int32 else I64,
                      col.data_ptr() if col.numel() else 0, self.n_dst, self.n_src, self.n_edges)

        self.ref = ctypes.byref(self.c)


_MSG_REF = {False: ctypes.byref(_Msg(MSG_COPY, 0.0, 0.0)), True: ctypes.byref(_Msg(MSG_WEIGHTED, 0.0, 0.0))}     # by "has weights"


def tiga_csr_workspace_bytes(g: CsrRelation, F: int, x_dtype: int = F32, reducer: int = SUM,
                             backward: bool = False) -> int:
    return int(_L.tiga_csr_workspace_bytes(g.ref, F, x_dtype, reducer, int(backward)))


def tiga_validate_csr(g: CsrRelation, level: int = 1, stream=None) -> None:
    ws = _ws(256, g.rowptr)
    _ok(_L.tiga_validate_csr(g.ref, level, _ptr(ws), ws.numel(), _stream(stream)), "tiga_validate_csr")


def tiga_apply_csr(g: CsrRelation, x, w=None, reducer: int = SUM, out=None, argmax=None, ws=None, stream=None):
    """out[i,:] = reduce over the row's edges of w[e] * x[col[e],:].  Returns (out, argmax)."""
    F = x.shape[1]
    if out is None:
        out = _new(x, (g.n_dst, F))
    if reducer in _ARG_DTYPE and argmax is None:
        argmax = _new(x, (g.n_dst, F), _ARG_DTYPE[reducer])
    if ws is None:
        ws = _ws(tiga_csr_workspace_bytes(g, F, _dt(x), reducer, False), x)
    _ok(_L.tiga_apply_csr(g.ref, _ptr(x), _dt(x), F, _ptr(w), _MSG_REF[w is not None], reducer, _ptr(out),
                                      _ptr(argmax), _ptr(ws), ws.numel(), _stream(stream)), "tiga_apply_csr")
    return out, argmax


BUILTIN_WS_BYTES = 8 << 20


def tiga_apply_csr_builtin_ws(g: CsrRelation, x, w=None, reducer: int = SUM, out=None, argmax=None, stream=None):
    """tiga_apply_csr without a workspace argument: the library's fixed 8 MiB device array is the
    scratch, for callers that may not allocate device memory.  Raises TigaError (status 6) when the
    relation needs more than that.  Calls that overlap on the GPU race on the shared array.
    `out` (and `argmax` for MAX) should be passed in by such callers; they are created here only
    as a convenience when omitted.  Returns (out, argmax)."""
    F = x.shape[1]
    if out is None:
        out = _new(x, (g.n_dst, F))
    if reducer in _ARG_DTYPE and argmax is None:
        argmax = _new(x, (g.n_dst, F), _ARG_DTYPE[reducer])
    _ok(_L.tiga_apply_csr_builtin_ws(g.ref, _ptr(x), _dt(x), F, _ptr(w), _MSG_REF[w is not None], reducer,
                                                 _ptr(out), _ptr(argmax), _stream(stream)), "tiga_apply_csr_builtin_ws")
    return out, argmax


def tiga_apply_csr_backward(g: CsrRelation, x, w, grad_out, reducer: int = SUM, argmax=None,
                            grad_x=None, grad_w=None, want_x=True, want_w=True, ws=None, stream=None):
    """Returns (grad_x, grad_w); either is None when not requested."""
    F = x.shape[1]
    if want_x and grad_x is None:
        grad_x = _new(x, (g.n_src, F))
    if want_w and grad_w is None:
        grad_w = _new(x, (g.n_edges,))
    if ws is None:
        ws = _ws(tiga_csr_workspace_bytes(g, F, _dt(x), reducer, True), x)
    _ok(_L.tiga_apply_csr_backward(g.ref, _ptr(x), _dt(x), F, _ptr(w), _MSG_REF[w is not None], reducer, _ptr(grad_out),
                                               _ptr(argmax), _ptr(grad_x), _ptr(grad_w), _ptr(ws), ws.numel(),
                                               _stream(stream)), "tiga_apply_csr_backward")
    return grad_x, grad_w


class CsrPlan:
    """A built hot-source plan: the host struct ``tiga_csr_plan``, the device buffer it describes and
    the relation it was built for."""

    def __init__(self, g, c, buf, scratch_bytes):
        self.g, self.c, self.buf, self.scratch_bytes = g, c, buf, int(scratch_bytes)

    n_hot = property(lambda self: int(self.c.n_hot))
    hot_edges = property(lambda self: int(self.c.hot_edges))
    min_hot_degree = property(lambda self: int(self.c.min_hot_degree))
    nbytes = property(lambda self: int(self.c.used_bytes))

    def array(self, name):
        """View of one of the plan's device arrays: 'col' or 'hot_id'."""
        off, n = {"col": (self.c.off_col, self.c.n_edges), "hot_id": (self.c.off_hot_id, self.c.n_hot)}[name]
        return self.buf[off:off + 4 * n].view(torch.int32)


def tiga_csr_plan_build(g: CsrRelation, max_hot_rows: int = None, row_bytes: int = 16, hot_bytes: int = 48 << 20,
                        stream=None) -> CsrPlan:
    """Builds the hot-source plan of a relation (one-time, synchronises).  ``max_hot_rows`` defaults to
    as many rows as fit ``hot_bytes`` of compact feature table."""
    lib = _L
    if max_hot_rows is None:
        max_hot_rows = max(1, hot_bytes // row_bytes)
    max_hot_rows = int(min(max_hot_rows, g.n_src))
    nbytes = int(lib.tiga_csr_plan_bytes(g.ref, max_hot_rows))
    wbytes = int(lib.tiga_csr_plan_workspace_bytes(g.ref))
    if nbytes == 0:
        raise TigaError(2, "tiga_csr_plan_bytes")
    buf = torch.empty(nbytes, dtype=torch.uint8, device=g.col.device)
    ws = torch.empty(wbytes, dtype=torch.uint8, device=g.col.device)
    c = _Plan()
    _ok(lib.tiga_csr_plan_build(g.ref, max_hot_rows, _ptr(buf), nbytes, _ptr(ws), wbytes, ctypes.byref(c), _stream(stream)),
        "tiga_csr_plan_build")
    return CsrPlan(g, c, buf, wbytes)


def tiga_csr_planned_workspace_bytes(plan: CsrPlan, F: int, x_dtype: int = F32, reducer: int = SUM) -> int:
    return int(_L.tiga_csr_planned_workspace_bytes(plan.g.ref, ctypes.byref(plan.c), F, x_dtype, reducer))


def tiga_apply_csr_planned(plan: CsrPlan, x, w=None, reducer: int = SUM, out=None, argmax=None, ws=None, stream=None):
    """tiga_apply_csr through a hot-source plan.  Returns (out, argmax)."""
    F = x.shape[1]
    g = plan.g
    if out is None:
        out = _new(x, (g.n_dst, F))
    if reducer in _ARG_DTYPE and argmax is None:
        argmax = _new(x, (g.n_dst, F), _ARG_DTYPE[reducer])
    if ws is None:
        ws = _ws(tiga_csr_planned_workspace_bytes(plan, F, _dt(x), reducer), x)
    _ok(_L.tiga_apply_csr_planned(g.ref, ctypes.byref(plan.c), _ptr(plan.buf), _ptr(x), _dt(x), F, _ptr(w),
                                              _MSG_REF[w is not None], reducer, _ptr(out), _ptr(argmax), _ptr(ws), ws.numel(),
                                              _stream(stream)), "tiga_apply_csr_planned")
    return out, argmax


def tiga_csr_degree_histogram(g: CsrRelation, nbins: int = 4096, stream=None):
    """Returns (hist int64[nbins], max_degree int64[1]) as device tensors."""
    hist, mx = _new(g.rowptr, (nbins,), torch.int64), _new(g.rowptr, (1,), torch.int64)
    _ok(_L.tiga_csr_degree_histogram(g.ref, _ptr(hist), nbins, _ptr(mx), _stream(stream)),
        "tiga_csr_degree_histogram")
    return hist, mx


_BOX_BYTES = struct.Struct("=3f3i")
_BOX_OF = _Box.from_buffer_copy


def _box(box, periodic):
    try:
        return _BOX_OF(_BOX_BYTES.pack(box[0], box[1], box[2], int(periodic[0]), int(periodic[1]), int(periodic[2])))
    except (struct.error, OverflowError, TypeError):      # a number that fp32 or int32 does not hold, a text: as ctypes converts them
        b = _Box()
        for d in range(3):
            b.len[d], b.periodic[d] = float(box[d]), int(periodic[d])
        return b


def tiga_radius_grid(n: int, r: float, box, periodic):
    """Returns (ncell list[3], invh list[3]) -- host only."""
    b = _box(box, periodic)
    nc = (ctypes.c_int32 * 3)()
    ih = (ctypes.c_float * 3)()
    _ok(_L.tiga_radius_grid(n, float(r), ctypes.byref(b), nc, ih), "tiga_radius_grid")
    return list(nc), list(ih)


def tiga_validate_points(pos, box, periodic=(0, 0, 0), level: int = 1, stream=None) -> None:
    """Raises TigaError (status 7) when a coordinate is not finite or lies outside [0, len]."""
    b = _box(box, periodic)
    ws = _ws(256, pos)
    _ok(_L.tiga_validate_points(_ptr(pos), pos.shape[0], ctypes.byref(b), level, _ptr(ws), ws.numel(),
                                            _stream(stream)), "tiga_validate_points")


def tiga_radius_workspace_bytes(n: int, F: int, r: float, box, periodic, backward: bool = False) -> int:
    b = _box(box, periodic)
    return int(_L.tiga_radius_workspace_bytes(n, F, float(r), ctypes.byref(b), int(backward)))


def tiga_radius_bin(pos, r: float, box, periodic, ws=None, stream=None):
    """Returns dict(cell, cell_start, order, ncell, ws)."""
    n = pos.shape[0]
    b = _box(box, periodic)
    ncell, _ = tiga_radius_grid(n, r, box, periodic)
    nc = ncell[0] * ncell[1] * ncell[2]
    cell = torch.empty(n, dtype=torch.int32, device=pos.device)
    start = torch.empty(nc + 1, dtype=torch.int32, device=pos.device)
    order = torch.empty(n, dtype=torch.int32, device=pos.device)
    if ws is None:
        ws = _ws(tiga_radius_workspace_bytes(n, 0, r, box, periodic), pos)
    _ok(_L.tiga_radius_bin(_ptr(pos), n, float(r), ctypes.byref(b), _ptr(cell), _ptr(start),
                                       _ptr(order), _ptr(ws), ws.numel(), _stream(stream)), "tiga_radius_bin")
    return dict(cell=cell, cell_start=start, order=order, ncell=ncell, ws=ws)


def tiga_apply_radius(pos, feat, r: float, box, periodic, kind: int = MSG_GAUSS, p0: float = 1.0,
                      p1: float = 1.0, out=None, count=None, want_count=False, ws=None, stream=None):
    """Fused bin + traverse + message + sum.  Returns (out, count, ws)."""
    n = pos.shape[0]
    F = 4 if kind == MSG_LJ else feat.shape[1]
    b = _box(box, periodic)
    if out is None:
        out = _new(pos, (n, F))
    if want_count and count is None:
        count = _new(pos, (n,), torch.int32)
    if ws is None:
        ws = _ws(tiga_radius_workspace_bytes(n, F, r, box, periodic), pos)
    _ok(_L.tiga_apply_radius(_ptr(pos), _ptr(feat), n, F, float(r), ctypes.byref(b),
                                         ctypes.byref(_Msg(kind, float(p0), float(p1))), _ptr(out), _ptr(count), _ptr(ws),
                                         ws.numel(), _stream(stream)), "tiga_apply_radius")
    return out, count, ws


def tiga_apply_radius_backward(pos, feat, grad_out, r: float, box, periodic, sigma: float, ws=None,
                               reuse_plan=False, grad_feat=None, grad_pos=None, want_feat=True, want_pos=True,
                               stream=None):
    """Reverse mode of the Gaussian message.  Returns (grad_feat, grad_pos)."""
    n, F = feat.shape
    b = _box(box, periodic)
    if want_feat and grad_feat is None:
        grad_feat = _new(pos, (n, F))
    if want_pos and grad_pos is None:
        grad_pos = _new(pos, (n, 3))
    if ws is None:
        assert not reuse_plan
        ws = _ws(tiga_radius_workspace_bytes(n, F, r, box, periodic, True), pos)
    _ok(_L.tiga_apply_radius_backward(_ptr(pos), _ptr(feat), n, F, float(r), ctypes.byref(b),
                                                  ctypes.byref(_Msg(MSG_GAUSS, float(sigma), 0.0)), _ptr(grad_out),
                                                  _ptr(grad_feat), _ptr(grad_pos), _ptr(ws), ws.numel(),
                                                  int(bool(reuse_plan)), _stream(stream)),
        "tiga_apply_radius_backward")
    return grad_feat, grad_pos


def _edge_mlp(W1, b1, W2, b2):
    for t in (W1, b1, W2, b2):
        assert t.is_cuda and t.is_contiguous() and t.dtype == torch.float32
    H, K = W1.shape
    return _EdgeMlp(K - 3, H, W2.shape[0], W1.data_ptr(), b1.data_ptr(), W2.data_ptr(), b2.data_ptr())


def tiga_apply_radius_mlp(pos, feat, r: float, box, periodic, W1, b1, W2, b2, out=None, count=None,
                          want_count=False, ws=None, stream=None):
    """out[i] = sum_{j in N(i)} [W2 relu(W1 [p_j - p_i; x_j] + b1) + b2].  Returns (out, count, ws)."""
    n = pos.shape[0]
    m = _edge_mlp(W1, b1, W2, b2)
    bx = _box(box, periodic)
    if out is None:
        out = _new(pos, (n, m.f_out))
    if want_count and count is None:
        count = _new(pos, (n,), torch.int32)
    if ws is None:
        ws = _ws(tiga_radius_workspace_bytes(n, m.f_in, r, box, periodic), pos)
    _ok(_L.tiga_apply_radius_mlp(_ptr(pos), _ptr(feat), n, float(r), ctypes.byref(bx), ctypes.byref(m),
                                             _ptr(out), _ptr(count), _ptr(ws), ws.numel(), _stream(stream)),
        "tiga_apply_radius_mlp")
    return out, count, ws


def tiga_apply_radius_mlp_backward(pos, feat, grad_out, r: float, box, periodic, W1, b1, W2, b2, ws=None,
                                   reuse_plan=False, stream=None):
    """Returns dict(grad_feat, grad_pos, grad_W1, grad_b1, grad_W2, grad_b2)."""
    n = pos.shape[0]
    m = _edge_mlp(W1, b1, W2, b2)
    bx = _box(box, periodic)
    g = dict(grad_feat=_new(pos, (n, m.f_in)), grad_pos=_new(pos, (n, 3)), grad_W1=torch.empty_like(W1),
             grad_b1=torch.empty_like(b1), grad_W2=torch.empty_like(W2), grad_b2=torch.empty_like(b2))
    if ws is None:
        assert not reuse_plan
        ws = _ws(tiga_radius_workspace_bytes(n, m.f_in, r, box, periodic, True), pos)
    _ok(_L.tiga_apply_radius_mlp_backward(_ptr(pos), _ptr(feat), n, float(r), ctypes.byref(bx), ctypes.byref(m),
                                                      _ptr(grad_out), _ptr(g["grad_feat"]), _ptr(g["grad_pos"]),
                                                      _ptr(g["grad_W1"]), _ptr(g["grad_b1"]), _ptr(g["grad_W2"]),
                                                      _ptr(g["grad_b2"]), _ptr(ws), ws.numel(), int(bool(reuse_plan)),
                                                      _stream(stream)), "tiga_apply_radius_mlp_backward")
    return g


def tiga_knn_workspace_bytes(n: int, k: int, box) -> int:
    b = _box(box, (0, 0, 0))
    return int(_L.tiga_knn_workspace_bytes(n, k, ctypes.byref(b)))


def tiga_apply_knn(pos, feat, k: int, box, periodic=(0, 0, 0), out=None, nbr=None, nbr_d2=None,
                   want_nbr=True, ws=None, stream=None):
    """out[i] = sum of feat[j] over the k nearest j != i by the key (fp32 squared distance, index).
    Returns (out, nbr int32 [n,k] or None, nbr_d2 fp32 [n,k] or None, ws)."""
    n, F = feat.shape
    b = _box(box, periodic)
    if out is None:
        out = _new(pos, (n, F))
    if want_nbr and nbr is None:
        nbr = _new(pos, (n, k), torch.int32)
    if want_nbr and nbr_d2 is None:
        nbr_d2 = _new(pos, (n, k))
    if ws is None:
        ws = _ws(tiga_knn_workspace_bytes(n, k, box), pos)
    _ok(_L.tiga_apply_knn(_ptr(pos), _ptr(feat), n, F, int(k), ctypes.byref(b), _ptr(out), _ptr(nbr),
                                      _ptr(nbr_d2), _ptr(ws), ws.numel(), _stream(stream)), "tiga_apply_knn")
    return out, nbr, nbr_d2, ws


def tiga_csr_attention_workspace_bytes(g: CsrRelation, D: int) -> int:
    return int(_L.tiga_csr_attention_workspace_bytes(g.ref, int(D)))


def tiga_apply_csr_attention(g: CsrRelation, q, key, value, scale: float, out=None, lse=None, want_lse=True,
                             ws=None, stream=None):
    """out[i] = sum_e softmax_e(scale * <q[i], key[col[e]]>) value[col[e]] over the edges of row i
    (online-softmax reducer).  Returns (out, lse, ws)."""
    D = q.shape[1]
    if out is None:
        out = _new(q, (g.n_dst, D))
    if want_lse and lse is None:
        lse = _new(q, (g.n_dst,))
    if ws is None:
        ws = _ws(tiga_csr_attention_workspace_bytes(g, D), q)
    _ok(_L.tiga_apply_csr_attention(g.ref, _ptr(q), _ptr(key), _ptr(value), D, float(scale), _ptr(out),
                                                _ptr(lse), _ptr(ws), ws.numel(), _stream(stream)), "tiga_apply_csr_attention")
    return out, lse, ws


# ------------------------------------------------------------------------------------ dense and paged relations, rotary positions

_HALF = {torch.float16: F16, torch.bfloat16: BF16}
_REAL = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}
_NO_CONTEXT = contextlib.nullcontext()


def _on(like, stream):
    """The device and stream that a call allocates and launches on: `stream`, or the current stream of the device of `like`."""
    if not like.is_cuda:
        raise ValueError("device arrays must be CUDA tensors")
    if stream is not None:
        if stream.device != like.device:
            raise ValueError("the stream belongs to another device than the arrays")
        return torch.cuda.stream(stream)
    current = _current_device() if _current_device else torch.cuda.current_device()
    return _NO_CONTEXT if like.get_device() == current else torch.cuda.device(like.device)


def _same(like, *arrays):
    device = like.get_device()         # (-1: on the host)
    for t in arrays:
        if t is not None and t.get_device() != device:
            raise ValueError("all arrays of a call must lie on one device")


def _like(t):
    """An array of the shape and type of t whose rows follow one another."""
    return torch.empty_like(t) if t.is_contiguous() else t.new_empty(t.shape)


def _scratch(nbytes, like):
    return like.new_empty(nbytes if nbytes > 256 else 256, dtype=torch.uint8)


def _ints(t, n, name):
    if t.dtype != torch.int32 or t.dim() != 1 or not t.is_contiguous() or (n is not None and t.numel() != n):
        raise ValueError(f"{name} must be a contiguous int32 array" + ("" if n is None else f" of {n} entries"))
    return t.data_ptr()


def _step(t, d):
    return t.stride(d) if t.shape[d] > 1 else 0       # the stride of a single entry means nothing


def _stride_of(t, shape, dtype, name):
    """(row, head) strides of an array [rows, heads, D] whose features are contiguous."""
    if t.dtype is not dtype or t.shape != shape:
        raise ValueError(f"{name} must be {dtype} {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")
    row, head, one = t.stride()
    if one != 1 and shape[2] > 1:
        raise ValueError(f"the features of {name} must be contiguous")
    return (row if shape[0] > 1 else 0), (head if shape[1] > 1 else 0)


def _dense_out(t, shape, dtype, name):
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} array {tuple(shape)}")
    return t.data_ptr()


# the descriptors' fields packed at once: a ctypes structure filled field by field costs several times as much
_HEADS_BYTES, _HEADS_OF, _NO_STRIDE = struct.Struct("=4if4x8q"), _Heads.from_buffer_copy, (0, 0)
_DENSE_BYTES, _DENSE_OF = struct.Struct("=6q"), _Dense.from_buffer_copy
_STRIDE_BYTES, _STRIDE_OF = struct.Struct("=2q"), _Stride.from_buffer_copy
_PAGES_BYTES, _PAGES_OF = struct.Struct("=12q"), _Pages.from_buffer_copy
_WEIGHTS_BYTES, _WEIGHTS_OF = struct.Struct("=4q"), _Weights.from_buffer_copy
assert _PAGES_BYTES.size == ctypes.sizeof(_Pages)
assert _HEADS_BYTES.size == ctypes.sizeof(_Heads) and _DENSE_BYTES.size == ctypes.sizeof(_Dense)


def _heads_of(dt, heads, kv_heads, D, scale, q, key=_NO_STRIDE, value=_NO_STRIDE, grad_out=_NO_STRIDE):
    try:
        return _HEADS_OF(_HEADS_BYTES.pack(dt, heads, kv_heads, D, scale, *q, *key, *value, *grad_out))
    except (struct.error, OverflowError):          # a number that int32 or fp32 does not hold, another kind of number: as ctypes converts them
        return _Heads(dt, heads, kv_heads, D, float(scale), _Stride(*q), _Stride(*key), _Stride(*value), _Stride(*grad_out))


def _type_of(t, types):
    if t.dtype not in types:
        raise TypeError(f"storage must be one of {[str(k) for k in types]}, got {t.dtype}")
    if t.dim() != 3:
        raise ValueError("arrays with heads have three dimensions: [rows, heads, D]")
    return types[t.dtype]


class _Held:
    """A descriptor holds the addresses of the arrays that it was made of.  They may be written into; another array in the place of one
    would leave the old address behind, so it takes a new descriptor."""
    _held = ()

    def __setattr__(self, name, value):
        if name in self._held and value is not self.__dict__.get(name):
            raise AttributeError(f"{type(self).__name__}.{name} is what the descriptor was made of: write into it, or make another {type(self).__name__}")
        self.__dict__[name] = value


class _Segments(_Held):
    _held = ("q_start", "kv_start", "mask")

    def __init__(self, q_start, kv_start, mask=None):
        _ints(q_start, None, "q_start")
        _ints(kv_start, q_start.numel(), "kv_start")
        if q_start.numel() < 1:
            raise ValueError("q_start has one entry more than there are segments")
        if mask is not None and (mask.dtype not in (torch.bool, torch.uint8) or mask.dim() != 1 or not mask.is_contiguous()):
            raise ValueError("mask must be a contiguous bool or uint8 array")
        _same(q_start, kv_start, mask)
        self.__dict__.update(q_start=q_start, kv_start=kv_start, mask=mask, q_ptr=q_start.data_ptr(), kv_ptr=kv_start.data_ptr(),
                             mask_ptr=0 if mask is None else mask.data_ptr(), n_seg=q_start.numel() - 1)


class DenseRelation(_Segments):
    """Block-diagonal dense relation: the rows [q_start[s], q_start[s+1]) read the keys [kv_start[s], kv_start[s+1]) of their
    segment, those that `mask` (bool or uint8 [n_kv], optional) leaves."""


class TriangularRelation(_Segments):
    """Block-diagonal triangular relation (causal attention of packed sequences): row t of the n rows [q_start[s], q_start[s+1]) reads, of
    the m keys [kv_start[s], kv_start[s+1]), those up to m - n + t that `mask` leaves.  Without kv_start rows and keys have the same
    segments."""

    def __init__(self, q_start, kv_start=None, mask=None):
        super().__init__(q_start, q_start if kv_start is None else kv_start, mask)


def _dense_args(g, q, key, value, scale, grad_out=None, kind=DenseRelation):
    if type(g) is not kind and not isinstance(g, kind):
        raise TypeError(f"the relation must be a {kind.__name__}")
    dt, dtype, shape = _type_of(q, _HALF), q.dtype, q.shape
    n_q, heads, D = shape
    if key.dim() != 3:
        raise ValueError("arrays with heads have three dimensions: [rows, heads, D]")
    n_kv, kv_heads, _ = key.shape
    _same(q, key, value, grad_out, g.q_start)
    if g.mask is not None and g.mask.numel() != n_kv:
        raise ValueError("the mask has one entry per key")
    keys = (n_kv, kv_heads, D)
    h = _heads_of(dt, heads, kv_heads, D, scale, _stride_of(q, shape, dtype, "q"), _stride_of(key, keys, dtype, "key"),
                  _stride_of(value, keys, dtype, "value"), _NO_STRIDE if grad_out is None else _stride_of(grad_out, shape, dtype, "grad_out"))
    return _DENSE_OF(_DENSE_BYTES.pack(g.q_ptr, g.kv_ptr, g.mask_ptr, g.n_seg, n_q, n_kv)), h


def _segments_forward(name, size, call, kind, g, q, key, value, scale, out, lse, want_lse, ws, stream):
    with _on(q, stream):
        c, h = _dense_args(g, q, key, value, scale, None, kind)
        if out is None:
            out = _like(q)
        if want_lse and lse is None:
            lse = q.new_empty(q.shape[:2], dtype=torch.float32)
        _same(q, out, lse, ws)
        if ws is None:
            ws = _scratch(size(ctypes.byref(c), ctypes.byref(h), 0), q)
        _ok(call(ctypes.byref(c), ctypes.byref(h), q.data_ptr(), key.data_ptr(), value.data_ptr(), _dense_out(out, q.shape, q.dtype, "out"),
                 None if lse is None else _dense_out(lse, q.shape[:2], torch.float32, "lse"), _ptr(ws), ws.numel(), _stream(stream)), name)
    return out, lse, ws


def _segments_backward(name, size, call, kind, g, q, key, value, out, lse, grad_out, scale, grad_q, grad_key, grad_value, want_q, want_kv, ws, stream):
    with _on(q, stream):
        c, h = _dense_args(g, q, key, value, scale, grad_out, kind)
        if want_q and grad_q is None:
            grad_q = _like(q)
        if want_kv and grad_key is None:
            grad_key = _like(key)
        if want_kv and grad_value is None:
            grad_value = _like(key)
        _same(q, out, lse, grad_q, grad_key, grad_value, ws)
        if ws is None:
            ws = _scratch(size(ctypes.byref(c), ctypes.byref(h), 1), q)
        grads = [None if t is None else _dense_out(t, like.shape, q.dtype, what)
                 for t, like, what in ((grad_q, q, "grad_q"), (grad_key, key, "grad_key"), (grad_value, key, "grad_value"))]
        _ok(call(ctypes.byref(c), ctypes.byref(h), q.data_ptr(), key.data_ptr(), value.data_ptr(), _dense_out(out, q.shape, q.dtype, "out"),
                 _dense_out(lse, q.shape[:2], torch.float32, "lse"), grad_out.data_ptr(), *grads, _ptr(ws), ws.numel(), _stream(stream)), name)
    return grad_q, grad_key, grad_value, ws


def tiga_dense_attention_workspace_bytes(g: DenseRelation, q, key, value, backward: bool = False) -> int:
    c, h = _dense_args(g, q, key, value, 1.0)
    return int(_L.tiga_dense_attention_workspace_bytes(ctypes.byref(c), ctypes.byref(h), int(backward)))


def tiga_apply_dense_attention(g: DenseRelation, q, key, value, scale: float, out=None, lse=None, want_lse=True, ws=None, stream=None):
    """out[i,h] = sum_j softmax_j(scale <q[i,h], key[j,h']>) value[j,h'] over the keys of the row's segment, h' the head of h's
    group.  q [n_q, heads, D], key and value [n_kv, kv_heads, D], fp16 or bf16, rows and heads strided.  Returns (out, lse, ws)."""
    return _segments_forward("tiga_apply_dense_attention", _L.tiga_dense_attention_workspace_bytes, _L.tiga_apply_dense_attention, DenseRelation,
                             g, q, key, value, scale, out, lse, want_lse, ws, stream)


def tiga_apply_dense_attention_backward(g: DenseRelation, q, key, value, out, lse, grad_out, scale: float, grad_q=None, grad_key=None,
                                        grad_value=None, want_q=True, want_kv=True, ws=None, stream=None):
    """Reverse mode of tiga_apply_dense_attention; out and lse are its outputs.  Returns (grad_q, grad_key, grad_value, ws); a
    gradient is None where it is not wanted."""
    return _segments_backward("tiga_apply_dense_attention_backward", _L.tiga_dense_attention_workspace_bytes, _L.tiga_apply_dense_attention_backward,
                              DenseRelation, g, q, key, value, out, lse, grad_out, scale, grad_q, grad_key, grad_value, want_q, want_kv, ws, stream)


def tiga_triangular_attention_workspace_bytes(g: TriangularRelation, q, key, value, backward: bool = False) -> int:
    c, h = _dense_args(g, q, key, value, 1.0, None, TriangularRelation)
    return int(_L.tiga_triangular_attention_workspace_bytes(ctypes.byref(c), ctypes.byref(h), int(backward)))


def tiga_apply_triangular_attention(g: TriangularRelation, q, key, value, scale: float, out=None, lse=None, want_lse=True, ws=None, stream=None):
    """tiga_apply_dense_attention over a triangular relation (causal attention of packed sequences).  Returns (out, lse, ws)."""
    return _segments_forward("tiga_apply_triangular_attention", _L.tiga_triangular_attention_workspace_bytes, _L.tiga_apply_triangular_attention,
                             TriangularRelation, g, q, key, value, scale, out, lse, want_lse, ws, stream)


def tiga_apply_triangular_attention_backward(g: TriangularRelation, q, key, value, out, lse, grad_out, scale: float, grad_q=None, grad_key=None,
                                             grad_value=None, want_q=True, want_kv=True, ws=None, stream=None):
    """Reverse mode of tiga_apply_triangular_attention; out and lse are its outputs.  Returns (grad_q, grad_key, grad_value, ws); a
    gradient is None where it is not wanted."""
    return _segments_backward("tiga_apply_triangular_attention_backward", _L.tiga_triangular_attention_workspace_bytes,
                              _L.tiga_apply_triangular_attention_backward, TriangularRelation, g, q, key, value, out, lse, grad_out, scale,
                              grad_q, grad_key, grad_value, want_q, want_kv, ws, stream)


class PagedCache(_Held):
    """Keys and values in pages: key and value [n_pages, page_size, kv_heads, D] with equal strides, table int32 [n_seg, max_pages]
    (entries outside [0, n_pages) name no page), kv_len int32 [n_seg]: tokens in the cache, the current chunk's included."""
    _held = ("key", "value", "table", "kv_len")

    def __init__(self, key, value, table, kv_len):
        shape, steps = key.shape, key.stride()
        if len(shape) != 4 or shape != value.shape or key.dtype is not value.dtype or key.dtype not in _HALF:
            raise ValueError("key and value must be fp16 or bf16 arrays [n_pages, page_size, kv_heads, D] of one shape")
        n_pages, page_size, kv_heads, D = shape

        def used(s):            # (the stride of a single entry means nothing)
            return s[0] if n_pages > 1 else 0, s[1] if page_size > 1 else 0, s[2] if kv_heads > 1 else 0, s[3] if D > 1 else 1
        step, of_value = used(steps), value.stride()
        if (steps != of_value and step != used(of_value)) or step[3] != 1:
            raise ValueError("key and value must have the same strides and contiguous features")
        if table.dtype is not torch.int32 or table.dim() != 2 or (table.shape[1] > 1 and table.stride(1) != 1):
            raise ValueError("table must be an int32 array [n_seg, max_pages] with contiguous rows")
        n_seg, max_pages = table.shape
        _ints(kv_len, n_seg, "kv_len")
        _same(key, value, table, kv_len)
        c = _PAGES_OF(_PAGES_BYTES.pack(key.data_ptr(), value.data_ptr(), table.data_ptr(), kv_len.data_ptr(), n_seg, n_pages, page_size,
                                        table.stride(0) if n_seg > 1 else 0, max_pages, step[0], step[1], step[2]))
        self.__dict__.update(key=key, value=value, table=table, kv_len=kv_len, n_seg=n_seg, kv_heads=kv_heads, c=c, ref=ctypes.byref(c))


def _paged_heads(cache, q, scale):
    if _type_of(q, _HALF) != _HALF[cache.key.dtype] or q.shape[2] != cache.key.shape[3]:
        raise ValueError("queries and cache must have one storage type and width")
    _same(q, cache.key)
    return _heads_of(_HALF[q.dtype], q.shape[1], cache.key.shape[2], q.shape[2], scale, _stride_of(q, q.shape, q.dtype, "q"))


def tiga_paged_attention_workspace_bytes(cache: PagedCache, q) -> int:
    return int(_L.tiga_paged_attention_workspace_bytes(cache.ref, ctypes.byref(_paged_heads(cache, q, 1.0)), q.shape[0]))


def tiga_apply_paged_attention(cache: PagedCache, q, q_start, scale: float, causal=True, out=None, lse=None, want_lse=True, ws=None, stream=None):
    """Attention of a chunk of new tokens over a paged cache: the rows [q_start[s], q_start[s+1]) of q [n_q, heads, D] are the last
    tokens of sequence s, and read its cache up to themselves (causal) or all of it.  Returns (out, lse, ws)."""
    with _on(q, stream):
        h = _paged_heads(cache, q, scale)
        _same(q, q_start, out, lse, ws)
        start = _ints(q_start, cache.n_seg + 1, "q_start")
        if out is None:
            out = _like(q)
        if want_lse and lse is None:
            lse = q.new_empty(q.shape[:2], dtype=torch.float32)
        if ws is None:
            ws = _scratch(_L.tiga_paged_attention_workspace_bytes(cache.ref, ctypes.byref(h), q.shape[0]), q)
        _ok(_L.tiga_apply_paged_attention(cache.ref, ctypes.byref(h), q.data_ptr(), start, q.shape[0], int(bool(causal)),
                                          _dense_out(out, q.shape, q.dtype, "out"),
                                          None if lse is None else _dense_out(lse, q.shape[:2], torch.float32, "lse"),
                                          _ptr(ws), ws.numel(), _stream(stream)), "tiga_apply_paged_attention")
    return out, lse, ws


class SharedPrefixes(_Held):
    """Sequences whose caches begin with the same pages: those of group g, [group_start[g], group_start[g+1]), that have new tokens share
    their positions [0, shared[g]); group_start int32 [n_groups + 1], shared int32 [n_groups], both on the device."""
    _held = ("group_start", "shared")

    def __init__(self, group_start, shared):
        _ints(shared, None, "shared")
        _ints(group_start, shared.numel() + 1, "group_start")
        _same(group_start, shared)
        self.c = _Prefixes(group_start.data_ptr(), shared.data_ptr(), shared.numel())
        self.__dict__.update(group_start=group_start, shared=shared, ref=ctypes.byref(self.c))


def tiga_shared_attention_workspace_bytes(cache: PagedCache, prefixes: SharedPrefixes, q) -> int:
    return int(_L.tiga_shared_attention_workspace_bytes(cache.ref, ctypes.byref(_paged_heads(cache, q, 1.0)), prefixes.ref, q.shape[0]))


def tiga_apply_shared_attention(cache: PagedCache, prefixes: SharedPrefixes, q, q_start, scale: float, causal=True, out=None, lse=None, want_lse=True,
                                ws=None, stream=None):
    """tiga_apply_paged_attention for sequences that share prefixes: what a group shares is read once for all of its rows (a few users of
    a short prompt are served sooner by that call).  Returns (out, lse, ws)."""
    with _on(q, stream):
        h = _paged_heads(cache, q, scale)
        _same(q, q_start, prefixes.shared, out, lse, ws)
        start = _ints(q_start, cache.n_seg + 1, "q_start")
        if out is None:
            out = _like(q)
        if want_lse and lse is None:
            lse = q.new_empty(q.shape[:2], dtype=torch.float32)
        if ws is None:
            ws = _scratch(_L.tiga_shared_attention_workspace_bytes(cache.ref, ctypes.byref(h), prefixes.ref, q.shape[0]), q)
        _ok(_L.tiga_apply_shared_attention(cache.ref, ctypes.byref(h), prefixes.ref, q.data_ptr(), start, q.shape[0], int(bool(causal)),
                                           _dense_out(out, q.shape, q.dtype, "out"),
                                           None if lse is None else _dense_out(lse, q.shape[:2], torch.float32, "lse"),
                                           _ptr(ws), ws.numel(), _stream(stream)), "tiga_apply_shared_attention")
    return out, lse, ws


def _weights_of(t, cache, name):
    shape = t.shape
    if t.dtype is not torch.float32 or len(shape) != 3 or shape[0] != cache.n_seg or shape[1] != cache.kv_heads:
        raise ValueError(f"{name} must be an fp32 array [n_seg, kv_heads, positions]")
    seg, head, one = t.stride()
    if one != 1 and shape[2] > 1:
        raise ValueError(f"the positions of {name} must be contiguous")
    if t.get_device() != cache.key.get_device():
        raise ValueError("all arrays of a call must lie on one device")
    return ctypes.byref(_WEIGHTS_OF(_WEIGHTS_BYTES.pack(t.data_ptr(), seg if shape[0] > 1 else 0, head if shape[1] > 1 else 0, shape[2])))


def tiga_paged_weights_workspace_bytes(cache: PagedCache, q) -> int:
    return int(_L.tiga_paged_weights_workspace_bytes(cache.ref, ctypes.byref(_paged_heads(cache, q, 1.0)), q.shape[0]))


def tiga_paged_attention_weights(cache: PagedCache, q, q_start, lse, scale: float, causal=True, before=None, weights=None, ws=None, stream=None):
    """weights[s,h',j] = before[s,h',j] + the softmax weights that position j of sequence s receives from the chunk's rows and the heads of
    group h'; q, q_start, scale, causal and lse as in, and from, tiga_apply_paged_attention.  weights and before fp32 [n_seg, kv_heads,
    positions]; weights may be before (the sums are kept in place).  Positions without a page receive nothing.  Entries behind a sequence's
    end are left alone (zeros where weights is allocated here).  Returns (weights, ws)."""
    with _on(q, stream):
        h = _paged_heads(cache, q, scale)
        start = _ints(q_start, cache.n_seg + 1, "q_start")
        if weights is None:
            like = (cache.n_seg, cache.kv_heads, cache.table.shape[1] * cache.key.shape[1] if before is None else before.shape[2])
            weights = q.new_zeros(like, dtype=torch.float32)
        b, o = None if before is None else _weights_of(before, cache, "before"), _weights_of(weights, cache, "weights")
        _same(q, q_start, lse, ws)
        if ws is None:
            ws = _scratch(_L.tiga_paged_weights_workspace_bytes(cache.ref, ctypes.byref(h), q.shape[0]), q)
        _ok(_L.tiga_paged_attention_weights(cache.ref, ctypes.byref(h), q.data_ptr(), start, q.shape[0], _dense_out(lse, q.shape[:2], torch.float32, "lse"),
                                            int(bool(causal)), b, o, _ptr(ws), ws.numel(), _stream(stream)), "tiga_paged_attention_weights")
    return weights, ws


def tiga_paged_evict(cache: PagedCache, to: PagedCache, weights, keep: int, recent: int = 0, to_weights=None, want_weights=True, kept=None, stream=None):
    """Every kv head of a sequence keeps its last `recent` positions and those with the largest weights [n_seg, kv_heads, positions], `keep`
    in all; their keys and values move in order to the first places of `to` (pages apart from those that `cache` names), to.kv_len is
    written.  Returns (kept int32 [n_seg, kv_heads, keep]: their positions, -1 behind them; to_weights [n_seg, kv_heads, positions of
    `to`]: their weights, zeros behind them, or None)."""
    with _on(cache.key, stream):
        _, _, kv_heads, D = cache.key.shape
        if to.key.dtype is not cache.key.dtype or to.kv_heads != kv_heads or to.key.shape[3] != D or to.n_seg != cache.n_seg:
            raise ValueError("both caches must have one storage type, number of sequences and heads, and width")
        _same(cache.key, to.key, kept)
        if kept is None:
            kept = cache.table.new_empty((cache.n_seg, kv_heads, max(int(keep), 0)))
        if want_weights and to_weights is None:
            to_weights = weights.new_empty((cache.n_seg, kv_heads, to.table.shape[1] * to.key.shape[1]))
        h = _heads_of(_HALF[cache.key.dtype], kv_heads, kv_heads, D, 1.0, _NO_STRIDE)
        _ok(_L.tiga_paged_evict(cache.ref, to.ref, ctypes.byref(h), _weights_of(weights, cache, "weights"), int(keep), int(recent),
                                None if to_weights is None else _weights_of(to_weights, cache, "to_weights"), to.kv_len.data_ptr(),
                                _dense_out(kept, (cache.n_seg, kv_heads, int(keep)), torch.int32, "kept"), _stream(stream)), "tiga_paged_evict")
    return kept, to_weights


def tiga_rotary_frequencies(turned: int, base: float = 10000.0, scaling: int = ROT_PLAIN, factor: float = 1.0, length: float = 0.0,
                            slow: float = 1.0, fast: float = 32.0):
    """Radians per position of every pair, on the host in 64 bits.  Returns (freq float64 [turned / 2] on the CPU, magnitude)."""
    freq = torch.empty(max(int(turned), 0) // 2, dtype=torch.float64)
    m = ctypes.c_float()
    _ok(_L.tiga_rotary_frequencies(int(turned), float(base), int(scaling), float(factor), float(length), float(slow), float(fast),
                                   ctypes.cast(freq.data_ptr(), ctypes.POINTER(ctypes.c_double)), ctypes.byref(m)), "tiga_rotary_frequencies")
    return freq, m.value


class Rotary(_Held):
    """Descriptor of rotary positions: freq float64 [turned / 2] on the device, the layout of the pairs (halves, or interleaved with
    pairs=True) and the magnitude."""
    _held = ("freq",)

    def __init__(self, freq, pairs=False, magnitude=1.0):
        if freq.dtype != torch.float64 or freq.dim() != 1 or not freq.is_cuda or not freq.is_contiguous():
            raise ValueError("freq must be a contiguous float64 CUDA array")
        self.__dict__["freq"] = freq
        self.c = _Rotary(freq.data_ptr(), 2 * freq.numel(), ROT_PAIRS if pairs else ROT_HALVES, magnitude)
        self.ref = ctypes.byref(self.c)


def tiga_apply_rotary(rotary: Rotary, x, positions, out=None, inverse=False, stream=None):
    """x [n, heads, D] with its first 2 * len(freq) features turned by positions (int32 or int64 [n]); inverse: the gradient of that.
    out may be x (in place).  Returns out."""
    with _on(x, stream):
        dt = _type_of(x, _REAL)
        if positions.dtype not in (torch.int32, torch.int64) or positions.shape != x.shape[:1] or not positions.is_contiguous():
            raise ValueError("positions must be a contiguous int32 or int64 array with one entry per row")
        shape, dtype = x.shape, x.dtype
        if out is None:
            out = x.new_empty(shape)
        _same(x, positions, out, rotary.freq)
        xs = _STRIDE_OF(_STRIDE_BYTES.pack(*_stride_of(x, shape, dtype, "x")))
        ys = _STRIDE_OF(_STRIDE_BYTES.pack(*_stride_of(out, shape, dtype, "out")))
        _ok(_L.tiga_apply_rotary(rotary.ref, x.data_ptr(), ctypes.byref(xs), out.data_ptr(), ctypes.byref(ys), dt, *shape, positions.data_ptr(),
                                 I32 if positions.dtype is torch.int32 else I64, 1 if inverse else 0, _stream(stream)), "tiga_apply_rotary")
    return out


def tiga_paged_append(cache: PagedCache, key, value, start, rotary: Rotary = None, stream=None) -> None:
    """Writes key (rotated to its position) and value [n_new, kv_heads, D] of the rows [start[s], start[s+1]) to the last positions of
    sequence s in the cache.  Pages that are written must belong to one sequence alone."""
    with _on(key, stream):
        dt = _type_of(key, _HALF)
        if key.dtype != cache.key.dtype or key.shape[1:] != cache.key.shape[2:]:
            raise ValueError("the rows must have the cache's storage type, heads and width")
        _same(key, value, start, cache.key, None if rotary is None else rotary.freq)
        n, heads, D = key.shape
        h = _heads_of(dt, heads, heads, D, 1.0, _NO_STRIDE, _stride_of(key, key.shape, key.dtype, "key"), _stride_of(value, key.shape, key.dtype, "value"))
        _ok(_L.tiga_paged_append(cache.ref, ctypes.byref(h), key.data_ptr(), value.data_ptr(), _ints(start, cache.n_seg + 1, "start"), n,
                                 None if rotary is None else rotary.ref, _stream(stream)), "tiga_paged_append")
