"""Thin ctypes binding of libf3m.so (include/f3m.h): argument marshalling only.

Tensors are torch CUDA(HIP) tensors used purely as device memory; every step of
the path runs inside the library's kernels.  There is no fallback: if the
library is missing, importing a symbol from it raises.
"""
import ctypes
import os
import warnings

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libf3m.so")

MAX_DIM = 7
MAX_LEVELS = 20

STATUS = {0: "F3M_OK", 1: "F3M_ERR_INVALID_ARG", 2: "F3M_ERR_NONFINITE", 3: "F3M_ERR_UNSUPPORTED",
          4: "F3M_ERR_OOM", 5: "F3M_ERR_HIP", 6: "F3M_ERR_BREAKDOWN"}


class F3MError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__("%s: %s" % (STATUS.get(status, status), msg))
        self.status = status


class Options(ctypes.Structure):
    _fields_ = [("leaf_max", ctypes.c_int32), ("max_depth", ctypes.c_int32),
                ("force_all_near", ctypes.c_int32), ("overlap", ctypes.c_int32),
                ("eta_smooth", ctypes.c_float), ("adaptive_far", ctypes.c_int32), ("small_field", ctypes.c_int32),
                ("route_min_points", ctypes.c_int32)]


class Info(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int64), ("D", ctypes.c_int32), ("interp_nodes", ctypes.c_int32),
                ("nodes_per_box", ctypes.c_int32), ("depth", ctypes.c_int32), ("quant_depth", ctypes.c_int32),
                ("far_threshold", ctypes.c_int32), ("edge", ctypes.c_float), ("scale", ctypes.c_float),
                ("alpha", ctypes.c_float * MAX_DIM),
                ("nboxes", ctypes.c_int64 * (MAX_LEVELS + 1)), ("max_box", ctypes.c_int64 * (MAX_LEVELS + 1)),
                ("near_pairs", ctypes.c_int64 * (MAX_LEVELS + 1)), ("far_pairs", ctypes.c_int64 * (MAX_LEVELS + 1)),
                ("far_point_pairs", ctypes.c_int64 * (MAX_LEVELS + 1)),
                ("near_point_pairs", ctypes.c_int64), ("device_bytes", ctypes.c_int64),
                ("smooth_depth", ctypes.c_int32), ("level_nodes", ctypes.c_int32 * (MAX_LEVELS + 1)),
                ("small_pairs", ctypes.c_int64 * (MAX_LEVELS + 1)),
                ("small_point_pairs", ctypes.c_int64 * (MAX_LEVELS + 1))]


class SourceInfo(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int64), ("two_sets", ctypes.c_int32), ("alpha", ctypes.c_float * MAX_DIM),
                ("nboxes", ctypes.c_int64 * (MAX_LEVELS + 1)), ("max_box", ctypes.c_int64 * (MAX_LEVELS + 1))]


class ProductInfo(ctypes.Structure):
    _fields_ = [("near_depth", ctypes.c_int32), ("far_points", ctypes.c_int32 * (MAX_LEVELS + 1))]


class Times(ctypes.Structure):
    _fields_ = [(k, ctypes.c_float) for k in
                ("bbox_keys", "sort", "gather", "boxes", "lists", "tables", "plan_total",
                 "permute_in", "p2p", "p2m", "m2l", "l2p", "permute_out", "kmvm_total")]

    def as_dict(self):
        return {k: float(getattr(self, k)) for k, _ in self._fields_}


class Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("row", ctypes.c_int64), ("head", ctypes.c_int64)]


class AttentionArgs(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("batch", ctypes.c_int32), ("heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("causal", ctypes.c_int32), ("window", ctypes.c_int32), ("sinks", ctypes.c_int32),
                ("scale", ctypes.c_float), ("max_q", ctypes.c_int32), ("max_k", ctypes.c_int32), ("total_q", ctypes.c_int64),
                ("total_k", ctypes.c_int64), ("q_offsets", ctypes.c_void_p), ("k_offsets", ctypes.c_void_p),
                ("q", Rows), ("k", Rows), ("v", Rows)]


class CacheInfo(ctypes.Structure):
    _fields_ = [("held", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("pages", ctypes.c_int64), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_exp", ctypes.c_void_p),
                ("v_exp", ctypes.c_void_p)]


DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float8_e4m3fn: 2}

_lib = None


def lib():
    """The loaded C-ABI library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libf3m.so is missing (%s): build it with "
                               "`python -m paper_2202_01085_amd.build`; there is no fallback path" % LIB_PATH)
        L = ctypes.CDLL(LIB_PATH)
        vp, i64, ci, cf = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float
        L.f3m_plan.argtypes = [vp, i64, ci, cf, ci, cf, vp, ctypes.POINTER(vp)]
        L.f3m_plan_ex.argtypes = [vp, i64, ci, cf, ci, cf, ctypes.POINTER(Options), vp, ctypes.POINTER(vp)]
        L.f3m_plan_xy.argtypes = [vp, i64, vp, i64, ci, cf, ci, cf, ctypes.POINTER(Options), vp, ctypes.POINTER(vp)]
        L.f3m_kmvm.argtypes = [vp, vp, vp, vp]
        L.f3m_kmvm_multi.argtypes = [vp, vp, i64, vp, i64, ci, vp]
        L.f3m_kmvm_multi.restype = ci
        L.f3m_cg_solve.argtypes = [vp, cf, vp, vp, ci, cf, ctypes.POINTER(ci), vp, vp]
        L.f3m_cg_solve.restype = ci
        L.direct_kmvm_xy.argtypes = [vp, i64, vp, i64, ci, cf, vp, vp, vp]
        L.direct_kmvm_xy_rows_f64.argtypes = [vp, i64, vp, i64, ci, cf, vp, vp, i64, vp, vp]
        L.f3m_plan_source_info.argtypes = [vp, ctypes.POINTER(SourceInfo)]
        L.f3m_plan_get_source_perm.argtypes = [vp, vp]
        L.f3m_plan_get_source_boxes.argtypes = [vp, ci, vp, vp]
        L.direct_kmvm.argtypes = [vp, i64, ci, cf, vp, vp, vp]
        L.direct_kmvm_rows_f64.argtypes = [vp, i64, ci, cf, vp, vp, i64, vp, vp]
        L.direct_kmvm_rows_f64_static.argtypes = [vp, i64, ci, cf, vp, vp, i64, vp, vp]
        L.f3m_destroy.argtypes = [vp]
        L.f3m_destroy.restype = None
        L.f3m_trim_memory.argtypes = []
        L.f3m_trim_memory.restype = ctypes.c_int64
        L.f3m_last_error.restype = ctypes.c_char_p
        L.f3m_plan_info.argtypes = [vp, ctypes.POINTER(Info)]
        L.f3m_plan_product_info.argtypes = [vp, ctypes.POINTER(ProductInfo)]
        L.f3m_plan_near_weighted.argtypes = [vp]
        L.f3m_plan_get_perm.argtypes = [vp, vp]
        L.f3m_plan_get_point_keys.argtypes = [vp, vp]
        L.f3m_plan_get_boxes.argtypes = [vp, ci, vp, vp]
        L.f3m_plan_get_list.argtypes = [vp, ci, ci, vp, vp]
        L.f3m_stage_times.argtypes = [vp, ctypes.POINTER(Times)]
        L.f3m_level_times.argtypes = [vp, ci, vp]
        args, rows, cache = ctypes.POINTER(AttentionArgs), ctypes.POINTER(Rows), ctypes.POINTER(CacheInfo)
        L.f3m_attention_workspace.argtypes = [args]
        L.f3m_attention_grad_workspace.argtypes = [args]
        L.f3m_attention_workspace.restype = L.f3m_attention_grad_workspace.restype = i64
        L.f3m_attention.argtypes = [args, rows, vp, vp, i64, vp]
        L.f3m_attention_grad.argtypes = [args, rows, rows, vp, rows, rows, rows, vp, i64, vp]
        L.f3m_cache_write.argtypes = L.f3m_cache_read.argtypes = [cache, ci, rows, rows, vp, i64, vp]
        L.f3m_cache_attention.argtypes = [cache, args, vp, i64, ctypes.c_int32, vp, rows, vp, vp, i64, vp]
        for name in ("f3m_attention", "f3m_attention_grad", "f3m_cache_write", "f3m_cache_read", "f3m_cache_attention"):
            getattr(L, name).restype = ci
        for name in ("f3m_plan", "f3m_plan_ex", "f3m_kmvm", "direct_kmvm", "direct_kmvm_rows_f64", "f3m_plan_info",
                     "f3m_plan_get_perm", "f3m_plan_get_point_keys", "f3m_plan_get_boxes", "f3m_plan_get_list",
                     "f3m_stage_times", "f3m_level_times", "f3m_plan_xy", "direct_kmvm_xy", "direct_kmvm_xy_rows_f64",
                     "f3m_plan_source_info", "f3m_plan_get_source_perm", "f3m_plan_get_source_boxes",
                     "direct_kmvm_rows_f64_static", "f3m_plan_product_info", "f3m_plan_near_weighted"):
            getattr(L, name).restype = ci
        _lib = L
    return _lib


def _check(status):
    if status != 0:
        raise F3MError(status, lib().f3m_last_error().decode())


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _dev_f32(t, name):
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == torch.float32 and t.is_contiguous()):
        raise TypeError("%s must be a contiguous float32 device tensor" % name)
    return ctypes.c_void_p(t.data_ptr())


def _np_ptr(a):
    return a.ctypes.data_as(ctypes.c_void_p)


class Plan:
    """f3m_plan / f3m_plan_ex: the partition and interaction lists of one point set;
    with Y given, f3m_plan_xy: targets X and sources Y, for v = K(X, Y) b."""

    def __init__(self, X, lengthscale, interp_nodes, eta=2.0, leaf_max=0, max_depth=0, force_all_near=False,
                 overlap=False, stream=None, eta_smooth=0.0, adaptive_far=False, small_field=0, Y=None,
                 route_min_points=0):
        n, D = X.shape
        self.n, self.D = int(n), int(D)
        self.ns = self.n
        self._h = ctypes.c_void_p()
        opt = Options(int(leaf_max), int(max_depth), int(bool(force_all_near)), int(bool(overlap)),
                      float(eta_smooth), int(bool(adaptive_far)), int(small_field), int(route_min_points))
        xp = _dev_f32(X, "X") if n > 0 else ctypes.c_void_p()
        if Y is None:
            _check(lib().f3m_plan_ex(xp, self.n, self.D, float(lengthscale), int(interp_nodes), float(eta),
                                     ctypes.byref(opt), _stream(stream), ctypes.byref(self._h)))
        else:
            if Y.shape[1] != D:
                raise ValueError("X and Y must have the same number of columns")
            self.ns = int(Y.shape[0])
            yp = _dev_f32(Y, "Y") if self.ns > 0 else ctypes.c_void_p()
            _check(lib().f3m_plan_xy(xp, self.n, yp, self.ns, self.D, float(lengthscale), int(interp_nodes),
                                     float(eta), ctypes.byref(opt), _stream(stream), ctypes.byref(self._h)))

    def close(self):
        h, self._h = getattr(self, "_h", None), None
        if h and _lib is not None:      # _lib is already gone when the interpreter shuts down
            _lib.f3m_destroy(h)

    __del__ = close

    def kmvm(self, b, y=None, stream=None):
        """f3m_kmvm: y ~= K(X,X) b, or K(X,Y) b for a two-set plan (asynchronous on the stream)."""
        if y is None:
            y = torch.empty(self.n, dtype=torch.float32, device=b.device)
        if self.n == 0:
            return y
        if b.numel() != self.ns or y.numel() != self.n:
            raise ValueError("b must have one entry per source and y one per target")
        _check(lib().f3m_kmvm(self._h, _dev_f32(b, "b") if self.ns else None, _dev_f32(y, "y"), _stream(stream)))
        return y

    def kmvm_multi(self, B, Y=None, stream=None):
        """f3m_kmvm_multi: B is an (m, sources) tensor, one right-hand side per ROW (each row contiguous);
        returns Y of shape (m, n) with Y[j] = product of B[j]."""
        m = int(B.shape[0])
        if B.dim() != 2 or B.shape[1] != self.ns:
            raise ValueError("B must have shape (m, sources)")
        if Y is None:
            Y = torch.empty((m, self.n), dtype=torch.float32, device=B.device)
        if Y.shape != (m, self.n):
            raise ValueError("Y must have shape (m, n)")
        if m and self.n:
            _check(lib().f3m_kmvm_multi(self._h, _dev_f32(B, "B") if self.ns else None, self.ns, _dev_f32(Y, "Y"), self.n,
                                        m, _stream(stream)))
        return Y

    def cg_solve(self, b, lam, tol=1e-6, max_iter=100, x=None, stream=None):
        """f3m_cg_solve: x = (K + lam I)^{-1} b by conjugate gradients; returns (x, iterations, history)."""
        if x is None:
            x = torch.empty_like(b)
        iters = ctypes.c_int(0)
        hist = np.zeros(max_iter + 1, dtype=np.float32)
        _check(lib().f3m_cg_solve(self._h, float(lam), _dev_f32(b, "b") if self.n else None,
                                  _dev_f32(x, "x") if self.n else None, int(max_iter), float(tol), ctypes.byref(iters),
                                  _np_ptr(hist), _stream(stream)))
        return x, int(iters.value), hist[:iters.value + 1]

    def source_info(self):
        out = SourceInfo()
        _check(lib().f3m_plan_source_info(self._h, ctypes.byref(out)))
        return out

    def source_perm(self):
        out = np.empty(self.ns, dtype=np.uint32)
        _check(lib().f3m_plan_get_source_perm(self._h, _np_ptr(out)))
        return out

    def source_boxes(self, level):
        nb = int(self.source_info().nboxes[level])
        keys = np.empty(nb, dtype=np.uint32)
        starts = np.empty(nb + 1, dtype=np.uint32)
        _check(lib().f3m_plan_get_source_boxes(self._h, int(level), _np_ptr(keys), _np_ptr(starts)))
        return keys, starts

    def info(self):
        out = Info()
        _check(lib().f3m_plan_info(self._h, ctypes.byref(out)))
        return out

    def product_info(self):
        """f3m_plan_product_info: the depth at which products interpolate the near pairs (near_depth, 0: exact sums),
        and the depths whose far field goes from point to point (far_points)"""
        out = ProductInfo()
        _check(lib().f3m_plan_product_info(self._h, ctypes.byref(out)))
        return out

    def near_weighted(self):
        """f3m_plan_near_weighted: the depth whose near pairs are interpolated between weighted points, or 0"""
        return int(lib().f3m_plan_near_weighted(self._h))

    def perm(self):
        out = np.empty(self.n, dtype=np.uint32)
        _check(lib().f3m_plan_get_perm(self._h, _np_ptr(out)))
        return out

    def point_keys(self):
        out = np.empty(self.n, dtype=np.uint32)
        _check(lib().f3m_plan_get_point_keys(self._h, _np_ptr(out)))
        return out

    def boxes(self, level):
        nb = int(self.info().nboxes[level])
        keys = np.empty(nb, dtype=np.uint32)
        starts = np.empty(nb + 1, dtype=np.uint32)
        _check(lib().f3m_plan_get_boxes(self._h, int(level), _np_ptr(keys), _np_ptr(starts)))
        return keys, starts

    def interactions(self, level, kind):
        inf = self.info()
        nb = int(inf.nboxes[level])
        sz = int((inf.near_pairs, inf.far_pairs, inf.small_pairs)[kind][level])
        ptr = np.empty(nb + 1, dtype=np.uint64)
        cols = np.empty(max(sz, 1), dtype=np.uint32)
        _check(lib().f3m_plan_get_list(self._h, int(level), int(kind), _np_ptr(ptr), _np_ptr(cols)))
        return ptr, cols[:sz]

    def level_times(self, level):
        """(P2M, M2L, L2P) milliseconds of one depth in the last kmvm"""
        out = (ctypes.c_float * 3)()
        _check(lib().f3m_level_times(self._h, int(level), out))
        return tuple(float(v) for v in out)

    def stage_times(self):
        out = Times()
        _check(lib().f3m_stage_times(self._h, ctypes.byref(out)))
        return out.as_dict()


def trim_memory():
    """f3m_trim_memory: give the library's cached device blocks back to the device; returns the bytes freed."""
    return int(lib().f3m_trim_memory())


def f3m_plan(X, lengthscale, interp_nodes, eta=2.0, **kw):
    return Plan(X, lengthscale, interp_nodes, eta, **kw)


def f3m_kmvm(plan, b, y=None, stream=None):
    return plan.kmvm(b, y, stream)


def direct_kmvm(X, b, lengthscale, y=None, stream=None):
    """direct_kmvm: exact y = K(X,X) b in fp32, O(n^2)."""
    n, D = X.shape
    if y is None:
        y = torch.empty_like(b)
    _check(lib().direct_kmvm(_dev_f32(X, "X") if n else None, int(n), int(D), float(lengthscale),
                             _dev_f32(b, "b") if n else None, _dev_f32(y, "y") if n else None, _stream(stream)))
    return y


def direct_kmvm_rows_f64(X, b, lengthscale, rows, stream=None):
    """direct_kmvm_rows_f64: exact fp64 sums for the selected rows (device int64 tensor)."""
    n, D = X.shape
    rows = rows.to(device=X.device, dtype=torch.int64).contiguous()
    y64 = torch.empty(rows.numel(), dtype=torch.float64, device=X.device)
    _check(lib().direct_kmvm_rows_f64(_dev_f32(X, "X"), int(n), int(D), float(lengthscale), _dev_f32(b, "b"),
                                      ctypes.c_void_p(rows.data_ptr()), int(rows.numel()),
                                      ctypes.c_void_p(y64.data_ptr()), _stream(stream)))
    return y64


def direct_kmvm_rows_f64_static(X, b, lengthscale, rows, y64, stream=None):
    """direct_kmvm_rows_f64_static: the same sums into the caller's y64 (device float64, one entry per row);
    the library call allocates nothing (at most 16384 rows).  rows: device int64 tensor."""
    n, D = X.shape
    if not (rows.is_cuda and rows.dtype == torch.int64 and rows.is_contiguous()):
        raise TypeError("rows must be a contiguous int64 device tensor")
    if not (y64.is_cuda and y64.dtype == torch.float64 and y64.is_contiguous() and y64.numel() >= rows.numel()):
        raise TypeError("y64 must be a contiguous float64 device tensor with one entry per row")
    _check(lib().direct_kmvm_rows_f64_static(_dev_f32(X, "X"), int(n), int(D), float(lengthscale), _dev_f32(b, "b"),
                                             ctypes.c_void_p(rows.data_ptr()), int(rows.numel()),
                                             ctypes.c_void_p(y64.data_ptr()), _stream(stream)))
    return y64


def direct_kmvm_xy(X, Y, b, lengthscale, y=None, stream=None):
    """direct_kmvm_xy: exact y = K(X,Y) b in fp32."""
    nx, D = X.shape
    ny = Y.shape[0]
    if y is None:
        y = torch.empty(nx, dtype=torch.float32, device=X.device)
    _check(lib().direct_kmvm_xy(_dev_f32(X, "X") if nx else None, int(nx), _dev_f32(Y, "Y") if ny else None, int(ny),
                                int(D), float(lengthscale), _dev_f32(b, "b") if ny else None,
                                _dev_f32(y, "y") if nx else None, _stream(stream)))
    return y


def direct_kmvm_xy_rows_f64(X, Y, b, lengthscale, rows, stream=None):
    """direct_kmvm_xy_rows_f64: exact fp64 sums of K(X,Y) b for the selected rows of X."""
    nx, D = X.shape
    ny = Y.shape[0]
    rows = rows.to(device=X.device, dtype=torch.int64).contiguous()
    y64 = torch.empty(rows.numel(), dtype=torch.float64, device=X.device)
    _check(lib().direct_kmvm_xy_rows_f64(_dev_f32(X, "X"), int(nx), _dev_f32(Y, "Y") if ny else None, int(ny), int(D),
                                         float(lengthscale), _dev_f32(b, "b") if ny else None,
                                         ctypes.c_void_p(rows.data_ptr()), int(rows.numel()),
                                         ctypes.c_void_p(y64.data_ptr()), _stream(stream)))
    return y64


# ---- row-normalised products (attention) ----
# A call on a few rows takes a GPU some microseconds: the checks below ask each tensor for its shape and strides once.

_SIXTEEN = (torch.bfloat16, torch.float16)


def _on_stream(device, stream, body, *tensors):
    """body(stream handle) with the tensors' device current and the call's stream the current one, so that what the binding allocates
    belongs to it.  A stream of the caller's holds the tensors that the call uses: their memory is not given to others before it is done."""
    given = stream is not None
    if not given:
        if device.index == torch.cuda.current_device():
            return body(torch._C._cuda_getCurrentRawStream(device.index))
        stream = torch.cuda.current_stream(device)
    elif stream.device != device:
        raise ValueError("the stream is of %s, the tensors are on %s" % (stream.device, device))
    with torch.cuda.stream(stream):
        got = body(stream.cuda_stream)
    if given:
        for t in tensors:
            if t is not None:
                t.record_stream(stream)
    return got


def _rows(t, name, dtype=None, device=None, shape=None):
    """a (rows, heads, head_dim) device tensor, head_dim contiguous, as the library takes it; shape: what it has to be"""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dim() == 3 and t.dtype in _SIXTEEN):
        raise TypeError("%s must be a device tensor (rows, heads, head_dim) of bfloat16 or float16" % name)
    if dtype is not None and (t.dtype != dtype or t.device != device):
        raise ValueError("%s must have the type and the device of the other tensors" % name)
    have = t.shape
    if shape is not None and have != shape:
        raise ValueError("%s must have shape %s" % (name, tuple(shape)))
    rows, heads, dim = have
    row, head, one = t.stride()
    if one != 1 and dim > 1:
        raise ValueError("%s must be contiguous along head_dim" % name)
    if rows == 1:
        row = dim
    if heads == 1:
        head = dim
    at = t.data_ptr()
    if (at | row << 1 | head << 1) & 15 and rows * heads * dim:
        raise ValueError("%s must be 16-byte aligned, with strides that are multiples of 8" % name)
    return Rows(at or None, row, head)


def _device_array(t, name, dtype, device, shape):
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dtype and t.device == device):
        raise TypeError("%s must be a %s tensor on %s" % (name, str(dtype).replace("torch.", ""), device))
    if t.shape != shape or not t.is_contiguous():
        raise ValueError("%s must be contiguous and have shape %s" % (name, tuple(shape)))
    return t.data_ptr() or None


def _no_graph(name, *tensors):
    """results of this library carry no graph of torch's: who would expect one is told"""
    if torch.is_grad_enabled():
        for t in tensors:
            if t.requires_grad:
                warnings.warn("%s: the results carry no graph, although an argument requires gradients: those come from attention_grad(); "
                              "torch.no_grad() around the call says that this is meant" % name, stacklevel=3)
                return


def _int32(x):
    """x as the library's 32-bit integer: beyond it the largest, which is more than any length, or -1, which is refused as x would be"""
    return max(-1, min(int(x), 2 ** 31 - 1))


def _attention_args(q, shape, rq, rk, rv, kv_heads, total_k, room, q_offsets, k_offsets, max_q, max_k, scale, causal, window, sinks):
    rows, heads, dim = shape
    batch, qo = 1, None
    if q_offsets is not None:
        batch = max(0, q_offsets.shape[0] - 1) if q_offsets.dim() == 1 else 0
        qo = _device_array(q_offsets, "q_offsets", torch.int32, q.device, (batch + 1,))
    ko = None if k_offsets is None else _device_array(k_offsets, "k_offsets", torch.int32, q.device, (batch + 1,))
    if scale is None:
        scale = 1.0 / dim ** 0.5 if dim else 1.0
    return AttentionArgs(DTYPES[q.dtype], batch, heads, kv_heads, dim, 1 if causal else 0, _int32(window), _int32(sinks), scale,
                         rows if max_q is None else min(_int32(max_q), rows), room if max_k is None else min(_int32(max_k), room), rows, total_k, qo, ko, rq, rk, rv)


def _packed_args(q, k, v, q_offsets, k_offsets, max_q, max_k, scale, causal, window, sinks):
    rq = _rows(q, "q")
    shape, dtype, device = q.shape, q.dtype, q.device
    rk = _rows(k, "k", dtype, device)
    rows, heads, dim = k.shape
    if dim != shape[2]:
        raise ValueError("k must have the head_dim of q")
    rv = _rows(v, "v", dtype, device, k.shape)
    if (q_offsets is None) != (k_offsets is None):
        raise ValueError("q_offsets and k_offsets are given both or neither")
    return _attention_args(q, shape, rq, rk, rv, heads, rows, rows, q_offsets, k_offsets, max_q, max_k, scale, causal, window, sinks)


def _lse(lse, shape, device, q=None):
    if lse is None:
        return q.new_empty(shape, dtype=torch.float32)
    _device_array(lse, "lse", torch.float32, device, shape)
    return lse


def _workspace(call, a, device):
    need = call(ctypes.byref(a))
    if need <= 0:
        if need < 0:
            _check(-need)
        return None, None, 0
    w = torch.empty(need, dtype=torch.uint8, device=device)
    return w, w.data_ptr(), need


def attention(q, k, v, q_offsets=None, k_offsets=None, max_q=None, max_k=None, scale=None, causal=True, window=0, sinks=0, out=None,
              lse=None, stream=None):
    """f3m_attention: o_i = sum_j w_ij v_j, w_ij = exp(scale q_i.k_j) over its sum; returns (out, lse).

    q (rows, heads, head_dim), k and v (rows, kv_heads, head_dim) hold the sequences behind one another, rows q_offsets[b] ..
    q_offsets[b + 1] - 1 and the same of k_offsets (int32, on the device; without: one sequence).  max_q and max_k are the longest
    sequence's (default: all rows; smaller ones make for fewer work items).  causal: token i of nq sees the keys up to
    nk - nq + i; window > 0: the last `window` of those and the first `sinks`.  scale: 1/sqrt(head_dim) by default.
    lse (rows, heads) float32: logarithms of the sums, -inf where nothing is visible (and out is 0).  Rows of no sequence, and tokens from
    max_q on, keep what out and lse held; without out and lse that is whatever their memory held.
    The results carry no graph of torch's (a warning says so where q, k or v require gradients): attention_grad() gives the gradients."""
    a = _packed_args(q, k, v, q_offsets, k_offsets, max_q, max_k, scale, causal, window, sinks)
    _no_graph("attention", q, k, v)
    device, shape = q.device, q.shape

    def call(handle):
        o = torch.empty_like(q) if out is None else out
        to = _rows(o, "out", q.dtype, device, shape)
        ls = _lse(lse, shape[:2], device, q)
        L = lib()
        w, at, need = _workspace(L.f3m_attention_workspace, a, device)
        _check(L.f3m_attention(ctypes.byref(a), ctypes.byref(to), ls.data_ptr() or None, at, need, handle))
        return o, ls

    return _on_stream(device, stream, call, q, k, v, q_offsets, k_offsets, out, lse)


def attention_grad(dout, q, k, v, out, lse, q_offsets=None, k_offsets=None, max_q=None, max_k=None, scale=None, causal=True, window=0,
                   sinks=0, dq=None, dk=None, dv=None, stream=None):
    """f3m_attention_grad: (dq, dk, dv) from the gradient dout of out, with the out and lse of attention() and its arguments.  Gradients of rows
    of no sequence, of tokens from max_q and of keys from max_k on keep what dq, dk and dv held (without those, whatever their memory held)."""
    a = _packed_args(q, k, v, q_offsets, k_offsets, max_q, max_k, scale, causal, window, sinks)
    device, dtype, shape = q.device, q.dtype, q.shape
    g, o = _rows(dout, "dout", dtype, device, shape), _rows(out, "out", dtype, device, shape)
    if lse is None:
        raise TypeError("lse must be that of attention()")
    _lse(lse, shape[:2], device)

    def call(handle):
        got = [torch.empty_like(x) if y is None else y for x, y in ((q, dq), (k, dk), (v, dv))]
        to = [_rows(y, name, dtype, device, x.shape) for y, name, x in zip(got, ("dq", "dk", "dv"), (q, k, v))]
        L = lib()
        w, at, need = _workspace(L.f3m_attention_grad_workspace, a, device)
        _check(L.f3m_attention_grad(ctypes.byref(a), ctypes.byref(g), ctypes.byref(o), lse.data_ptr() or None, ctypes.byref(to[0]),
                                    ctypes.byref(to[1]), ctypes.byref(to[2]), at, need, handle))
        return tuple(got)

    return _on_stream(device, stream, call, dout, q, k, v, out, lse, q_offsets, k_offsets, dq, dk, dv)


class KVCache:
    """f3m_cache: keys and values in pages, for sequences that grow.  The tensors are the caller's:

    k, v (pages, kv_heads, page_size, head_dim), contiguous, of bfloat16, float16 or float8_e4m3fn; for the last k_exp and v_exp
    (pages, kv_heads, page_size) uint8, the rows' exponents: a value is code * 2^(byte - 127).  Slot s is row s % page_size of
    page s // page_size.  KVCache.empty makes the tensors.  A cache keeps to its tensors and to where they lie: a larger one is a new
    KVCache of new tensors."""

    def __init__(self, k, v, k_exp=None, v_exp=None):
        if not (isinstance(k, torch.Tensor) and k.is_cuda and k.dim() == 4 and k.dtype in DTYPES):
            raise TypeError("k must be a device tensor (pages, kv_heads, page_size, head_dim) of bfloat16, float16 or float8_e4m3fn")
        dtype, device, shape = k.dtype, k.device, k.shape
        at_k, at_v = _device_array(k, "k", dtype, device, shape), _device_array(v, "v", dtype, device, shape)
        at_k_exp = at_v_exp = None
        if dtype == torch.float8_e4m3fn:
            rows = shape[:3]
            at_k_exp, at_v_exp = _device_array(k_exp, "k_exp", torch.uint8, device, rows), _device_array(v_exp, "v_exp", torch.uint8, device, rows)
        elif k_exp is not None or v_exp is not None:
            raise ValueError("k_exp and v_exp belong to 8-bit caches")
        self._tensors = k, v, k_exp, v_exp
        pages, heads, page_size, dim = shape
        self._at = at_k, at_v, at_k_exp, at_v_exp
        self._c = CacheInfo(DTYPES[dtype], heads, dim, page_size, pages, *self._at)

    # without setters: calls go by the addresses of these tensors
    k, v, k_exp, v_exp = (property(lambda self, i=i: self._tensors[i]) for i in range(4))

    def _info(self):
        """what the library gets; tensors that were resized or given other memory are refused, as their old one may be gone"""
        for t, at in zip(self._tensors, self._at):
            if t is not None and t.data_ptr() != (at or 0):
                raise ValueError("the cache's tensors no longer lie where they did: make a new KVCache of them")
        return self._c

    @classmethod
    def empty(cls, pages, page_size, kv_heads, head_dim, dtype=torch.float8_e4m3fn, device="cuda"):
        """a cache of zeros"""
        def zeros(shape, dtype):
            return torch.zeros(shape, dtype=torch.uint8, device=device).view(dtype) if dtype == torch.float8_e4m3fn else torch.zeros(shape, dtype=dtype, device=device)
        shape = (pages, kv_heads, page_size, head_dim)
        exp = [torch.full(shape[:3], 127, dtype=torch.uint8, device=device) if dtype == torch.float8_e4m3fn else None for _ in range(2)]
        return cls(zeros(shape, dtype), zeros(shape, dtype), *exp)

    def _move(self, call, k, v, slots, handle):
        device, c = self.k.device, self._info()
        rk = _rows(k, "k")
        shape = k.shape
        if shape[1:] != (c.kv_heads, c.head_dim) or k.device != device:
            raise ValueError("k and v must have shape (tokens, kv_heads, head_dim) as the cache, and be on its device")
        rv = _rows(v, "v", k.dtype, device, shape)
        at = _device_array(slots, "slots", torch.int64, device, shape[:1])
        _check(call(ctypes.byref(c), DTYPES[k.dtype], ctypes.byref(rk), ctypes.byref(rv), at, shape[0], handle))

    def write(self, k, v, slots, stream=None):
        """f3m_cache_write: k, v (tokens, kv_heads, head_dim) to slots (tokens) int64, on the device; slots outside the cache are skipped.
        No slot may come twice in a call."""
        _on_stream(self.k.device, stream, lambda handle: self._move(lib().f3m_cache_write, k, v, slots, handle), k, v, slots, *self._tensors)

    def read(self, slots, dtype=None, k=None, v=None, stream=None):
        """f3m_cache_read: (k, v) of the slots, of `dtype` (default: bfloat16 from an 8-bit cache, else the cache's); zeros for slots outside"""
        dtype = (torch.bfloat16 if self._c.held == 2 else self.k.dtype) if dtype is None else dtype
        shape = (slots.numel(), self._c.kv_heads, self._c.head_dim)

        def call(handle):
            kk = slots.new_empty(shape, dtype=dtype) if k is None else k
            vv = slots.new_empty(shape, dtype=dtype) if v is None else v
            self._move(lib().f3m_cache_read, kk, vv, slots, handle)
            return kk, vv

        return _on_stream(self.k.device, stream, call, k, v, slots, *self._tensors)

    def attention(self, q, table, lengths, q_offsets=None, max_q=None, max_k=None, scale=None, causal=True, window=0, sinks=0, out=None,
                  lse=None, stream=None):
        """f3m_cache_attention: attention() of new tokens q over the sequences of the cache, their own keys included; returns (out, lse).

        Key j of sequence b lies in page table[b, j // page_size] (int32, on the device), j < lengths[b] (int32, on the device).
        q_offsets as for attention(); without, every sequence has the same number of new tokens (rows of q / sequences).
        max_k: the longest length (default: what the table has room for).  There are no gradients over a cache."""
        device, c = self.k.device, self._info()
        if not (isinstance(table, torch.Tensor) and table.is_cuda and table.dtype == torch.int32 and table.dim() == 2 and table.device == device):
            raise TypeError("table must be an int32 tensor (sequences, pages) on the cache's device")
        batch, cols = table.shape
        step, one = table.stride()
        if batch * cols and (one != 1 and cols > 1 or step < cols and batch > 1):
            raise ValueError("table must be contiguous along the pages")
        rq = _rows(q, "q")
        shape = q.shape
        if q.device != device:
            raise ValueError("q must be on the cache's device")
        _no_graph("KVCache.attention", q)
        ln = _device_array(lengths, "lengths", torch.int32, device, (batch,))

        def call(handle):
            offsets, most = q_offsets, max_q
            if offsets is None:
                if shape[0] % max(1, batch):
                    raise ValueError("without q_offsets all sequences have the same number of new tokens")
                each = shape[0] // max(1, batch)
                offsets = torch.arange(0, each * batch + 1, max(1, each), dtype=torch.int32, device=device) if each else \
                    torch.zeros(batch + 1, dtype=torch.int32, device=device)
                most = each if most is None else most
            a = _attention_args(q, shape, rq, Rows(), Rows(), c.kv_heads, 0, min(cols * c.page_size, 2 ** 31 - 65537), offsets, None, most, max_k,
                                scale, causal, window, sinks)
            if a.batch != batch:
                raise ValueError("q_offsets must have one entry more than the table has rows")
            o = torch.empty_like(q) if out is None else out
            to = _rows(o, "out", q.dtype, device, shape)
            ls = _lse(lse, shape[:2], device, q)
            L = lib()
            w, at, need = _workspace(L.f3m_attention_workspace, a, device)
            _check(L.f3m_cache_attention(ctypes.byref(c), ctypes.byref(a), table.data_ptr() or None, max(step, cols), cols, ln, ctypes.byref(to),
                                         ls.data_ptr() or None, at, need, handle))
            return o, ls

        return _on_stream(device, stream, call, q, table, lengths, q_offsets, out, lse, *self._tensors)
