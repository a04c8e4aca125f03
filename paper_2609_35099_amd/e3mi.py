"""Python binding of libe3mi (ctypes): argument marshalling only.

Every computation runs in the HIP library; this module checks tensor shapes,
dtypes and devices, passes raw device pointers and the current torch stream,
and raises E3Error on a non-OK status.  If the library has not been built the
first call raises (there is no fallback path).
"""
from __future__ import annotations

import ctypes as ct
import functools
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
# E3MI_LIB may point at another build of the same library (side-by-side builds)
LIB_PATH = os.environ.get("E3MI_LIB") or os.path.join(_HERE, "libe3mi.so")

_STATUS = {0: "E3_OK", 1: "E3_ERR_INVALID_ARG", 2: "E3_ERR_UNSUPPORTED",
           3: "E3_ERR_INDEX_OUT_OF_RANGE", 4: "E3_ERR_WORKSPACE_TOO_SMALL",
           5: "E3_ERR_HIP", 6: "E3_ERR_ALLOC"}

E3_PARITY_ALL = 0
E3_PARITY_NATURAL = 1
E3_PLAN_RECORDS = 2
E3_PLAN_COMPOSED = 4


class E3Error(RuntimeError):
    def __init__(self, status: int, where: str, detail: str = ""):
        self.status = status
        name = _STATUS.get(status, str(status))
        super().__init__(f"{where}: {name}" + (f" ({detail})" if detail else ""))


class PlanInfo(ct.Structure):
    _fields_ = [("C", ct.c_int), ("P", ct.c_int), ("D_in", ct.c_int), ("D_sh", ct.c_int),
                ("D_out", ct.c_int), ("nnz", ct.c_int), ("lmax_sh", ct.c_int),
                ("lmax_out", ct.c_int), ("supported", ct.c_int)]


_lib = None

# name -> (restype, argtypes); mirrors include/e3mi.h
_P, _I, _I64, _U, _D = ct.c_void_p, ct.c_int, ct.c_int64, ct.c_uint, ct.c_double
_U64 = ct.c_uint64
SIGNATURES = {
    "e3_plan_create": (_I, [ct.c_char_p, _I, _I, _U, ct.POINTER(_P)]),
    "e3_plan_query": (_I, [_P, ct.POINTER(PlanInfo)]),
    "e3_plan_destroy": (_I, [_P]),
    "e3_plan_paths": (_I, [_P, _P]),
    "e3_plan_records": (_I, [_P, _I64, _P, _P, _P, _P, ct.POINTER(_I64)]),
    "e3_sh_host": (_I, [_I, _P, _P, _I64]),
    "e3_graph_create": (_I, [_P, _P, _I64, _I64, ct.c_int32, _P, ct.POINTER(_P)]),
    "e3_graph_live_edges": (_I, [_P, ct.POINTER(_I64)]),
    "e3_graph_export": (_I, [_P, _P, _P, _P, _P]),
    "e3_graph_destroy": (_I, [_P]),
    "e3_sh": (_I, [_I, _P, _P, _I64, _P]),
    "e3_sh_bwd": (_I, [_I, _P, _P, _P, _I64, _P]),
    "e3_tp_fwd": (_I, [_P, _P, _P, _P, _P, _I64, _P]),
    "e3_tp_workspace_size": (_I, [_P, _I64, ct.POINTER(ct.c_size_t)]),
    "e3_tp_bwd": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _P, ct.c_size_t, _I64, _P]),
    "e3_conv_workspace_size": (_I, [_P, _P, ct.POINTER(ct.c_size_t), ct.POINTER(ct.c_size_t)]),
    "e3_linear_create": (_I, [ct.c_char_p, ct.c_char_p, ct.POINTER(ct.c_void_p)]),
    "e3_linear_query": (_I, [_P, ct.POINTER(ct.c_int64), ct.POINTER(ct.c_int), ct.POINTER(ct.c_int),
                             ct.POINTER(ct.c_int), ct.POINTER(ct.c_int)]),
    "e3_linear_destroy": (_I, [_P]),
    "e3_linear_fwd": (_I, [_P, _P, _P, _P, _I64, _P]),
    "e3_linear_workspace_size": (_I, [_P, ct.POINTER(ct.c_size_t)]),
    "e3_linear_bwd": (_I, [_P, _P, _P, _P, _P, _P, _P, ct.c_size_t, _I64, _P]),
    "e3_tpg_create": (_I, [ct.c_int, ct.c_int, ct.c_int, _I64, _P, _P, _P, _P, ct.c_int, ct.POINTER(ct.c_void_p)]),
    "e3_tpg_destroy": (_I, [_P]),
    "e3_tpg_fwd": (_I, [_P, _P, _P, _P, _I64, ct.c_int, _P]),
    "e3_tpg_workspace_size": (_I, [_P, _I64, ct.c_int, ct.POINTER(ct.c_size_t)]),
    "e3_tpg_bwd": (_I, [_P, _P, _P, _P, _P, _P, _P, ct.c_size_t, _I64, ct.c_int, _P]),
    "e3_tpg_fwd_f64": (_I, [_P, _P, _P, _P, _I64, ct.c_int, _P]),
    "e3_tpg_bwd_f64": (_I, [_P, _P, _P, _P, _P, _P, _P, ct.c_size_t, _I64, ct.c_int, _P]),
    "e3_conv_fwd_y": (_I, [_P, _P, _P, _P, _P, _P, ct.c_int, _P]),
    "e3_conv_bwd_y": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _P, ct.c_int, _P, ct.c_size_t, _P]),
    "e3_conv_bwd2": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, ct.c_size_t, _P]),
    "e3_conv_radial_workspace_size": (_I, [_P, _P, ct.c_int, ct.POINTER(ct.c_size_t)]),
    "e3_conv_fwd_radial": (_I, [_P, _P, _P, _P, _P, _P, ct.c_int, _P, _P]),
    "e3_conv_bwd_radial": (_I, [_P, _P, _P, _P, _P, _P, ct.c_int, _P, _P, _P, _P, _P, _P, ct.c_size_t, _P]),
    "e3_conv_fwd": (_I, [_P, _P, _P, _P, _P, _P, _P, ct.c_size_t, _P]),
    "e3_conv_bwd": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, ct.c_size_t, _P]),
    "e3_conv_bwd_noalloc": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _P, _P]),
    "e3_tp_fwd_f64": (_I, [_P, _P, _P, _P, _P, _I64, _P]),
    "e3_tp_workspace_size_f64": (_I, [_P, _I64, ct.POINTER(ct.c_size_t)]),
    "e3_tp_bwd_f64": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _P, ct.c_size_t, _I64, _P]),
    "e3_conv_workspace_size_f64": (_I, [_P, _P, ct.POINTER(ct.c_size_t)]),
    "e3_conv_fwd_f64": (_I, [_P, _P, _P, _P, _P, _P, _P]),
    "e3_conv_bwd_f64": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, ct.c_size_t, _P]),
    "e3_pack8": (_I, [_I, _P, _I64, _P, _P, _I64, _I64, _P]),
    "e3_unpack8": (_I, [_I, _P, _P, _P, _I64, _I64, _I64, _P]),
    "e3_layer_norm_fwd": (_I, [_I, _P, _I64, _P, _P, ct.c_float, _P, _I64, _P, _P, _P, _P, _P, _P, _I64, _I64, _P]),
    "e3_layer_norm_workspace_size": (_I, [_I, _I64, _I64, ct.POINTER(ct.c_size_t)]),
    "e3_layer_norm_bwd": (_I, [_I, _P, _I64, _P, _P, _P, _P, _I64, _P, _P, _P, _I64, _P, _P, _P, ct.c_size_t, _I64,
                               _I64, _P]),
    "e3_dense_workspace_size": (_I, [_I, _I64, _I64, _I64, ct.POINTER(ct.c_size_t), ct.POINTER(ct.c_size_t)]),
    "e3_dense_fwd": (_I, [_I, _P, _I64, _P, _P, _P, _I64, _I, _P, _I64, _P, _I64, _P, _P, _P, _P, _P, ct.c_size_t,
                          _I64, _I64, _I64, _P]),
    "e3_dense_bwd": (_I, [_I, _P, _I64, _P, _P, _P, _P, _I64, _P, _P, _I, _P, _I64, _P, _I64, _P, _P, _P, ct.c_size_t,
                          _I64, _I64, _I64, _P]),
    "e3_gated_workspace_size": (_I, [_I, _I64, _I64, _I64, ct.POINTER(ct.c_size_t), ct.POINTER(ct.c_size_t)]),
    "e3_gated_fwd": (_I, [_I, _P, _I64, _P, _P, _I, _P, _I64, _P, _I64, _P, _P, _P, _P, _P, _P, _P, ct.c_size_t, _I64,
                          _I64, _I64, _P]),
    "e3_gated_bwd": (_I, [_I, _P, _I64, _P, _P, _P, _P, _I64, _P, _P, _P, _P, _I, _P, _I64, _P, _I64, _P, _P, _P,
                          ct.c_size_t, _I64, _I64, _I64, _P]),
    "e3_dropout_fwd": (_I, [_I, _P, _I64, _P, _I64, _D, _U64, _U64, _P, _P, _I64, _I64, _I64, _P]),
    "e3_dropout_bwd": (_I, [_I, _P, _I64, _D, _U64, _U64, _P, _P, _I64, _I64, _I64, _P]),
    "e3_residual_norm_fwd": (_I, [_I, _I, _U, _P, _I64, _P, _I64, _P, _I64, ct.c_float, _D, _U64, _U64, _P, _P, _P, _P, _P,
                                  ct.c_float, _P, _I64, _P, _I64, _P, _P, _P, _P, _I64, _I64, _P]),
    "e3_residual_norm_workspace_size": (_I, [_I, _I64, _I64, ct.POINTER(ct.c_size_t)]),
    "e3_residual_norm_bwd": (_I, [_I, _I, _U, _P, _I64, _P, _I64, _P, _I64, ct.c_float, _D, _U64, _U64, _P, _P, _P, _P, _P,
                                  _P, _P, _P, _P, _I64, _P, _I64, _P, _I64, _P, _I64, _P, _I64, _P, _P, _P, _P, _P,
                                  ct.c_size_t, _I64, _I64, _P]),
    "e3_probe_stream": (_I, [_P, ct.c_size_t, _P, ct.c_size_t, _I, _I, _I, _U, ct.POINTER(ct.c_size_t),
                             ct.POINTER(ct.c_size_t), _P]),
    "e3_timing_enable": (_I, [_I]),
    "e3_timing_reset": (_I, []),
    "e3_timing_read": (_I, [_I, _P, _P, _P, ct.POINTER(_I)]),
    "e3_status_str": (ct.c_char_p, [_I]),
    "e3_last_error": (ct.c_char_p, []),
}


def lib():
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build()")
        L = ct.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def _check(status: int, where: str):
    if status != 0:
        detail = lib().e3_last_error().decode(errors="replace")
        raise E3Error(status, where, detail)


# ---------------------------------------------------------------- tensors
_modules = None   # torch and the dtypes by name, looked up once


def _torch():
    global _modules
    if _modules is None:
        import torch
        _modules = torch, {"float32": torch.float32, "float64": torch.float64, "int32": torch.int32,
                           "bfloat16": torch.bfloat16, "int8": torch.int8, "uint8": torch.uint8,
                           "int64": torch.int64}
    return _modules[0]


def _ptr(t, name, shape=None, dtype="float32"):
    torch = _torch()
    want = _modules[1][dtype]
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.dtype is not want:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on the GPU")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if shape is not None and t.shape != shape and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    return t.data_ptr() if t.numel() else None


_current = None   # torch's raw-stream and device queries


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    global _current
    if _current is None:   # torch.cuda.current_stream().cuda_stream, without the stream object (2.8 us a call)
        c = _torch()._C
        _current = c._cuda_getCurrentRawStream, c._cuda_getDevice
    return _current[0](_current[1]())


def _on_stream(fn):
    """Run a compute call with the caller's stream made current, so that the
    outputs and the workspace it allocates belong to that stream in torch's
    caching allocator (their memory is not handed out again while the kernels
    launched on that stream may still use it)."""
    @functools.wraps(fn)
    def wrapped(*args, stream=None, **kw):
        if stream is None:
            return fn(*args, **kw)
        with _torch().cuda.stream(stream):
            return fn(*args, stream=stream, **kw)
    return wrapped


# ---------------------------------------------------------------- plan
class Plan:
    """Paths, coupling tables and kernels for an irreps layout.

    `kernels` is "compiled" when a kernel variant was generated for the layout,
    "composed" when it runs block by block on generated single-block kernels,
    "records" when it runs on the record path (its coupling records uploaded
    to the current device at creation), else None (no compute).
    """

    def __init__(self, irreps: str, lmax_sh: int, lmax_out: int, natural: bool = False,
                 records: bool = False, composed: bool = False):
        h = ct.c_void_p()
        flags = ((E3_PARITY_NATURAL if natural else E3_PARITY_ALL) | (E3_PLAN_RECORDS if records else 0)
                 | (E3_PLAN_COMPOSED if composed else 0))
        _check(lib().e3_plan_create(irreps.encode(), lmax_sh, lmax_out, flags, ct.byref(h)),
               "e3_plan_create")
        self._h = h
        info = PlanInfo()
        _check(lib().e3_plan_query(h, ct.byref(info)), "e3_plan_query")
        self.info = info
        self.irreps = irreps
        self.C, self.P = info.C, info.P
        self.D_in, self.D_sh, self.D_out = info.D_in, info.D_sh, info.D_out
        self.supported = bool(info.supported)
        self.kernels = {1: "compiled", 2: "records", 3: "composed"}.get(info.supported)

    @property
    def handle(self):
        return self._h

    def paths(self) -> np.ndarray:
        out = np.zeros((self.P, 7), dtype=np.int32)
        _check(lib().e3_plan_paths(self._h, out.ctypes.data_as(ct.c_void_p)), "e3_plan_paths")
        return out

    def records(self):
        n = ct.c_int64()
        _check(lib().e3_plan_records(self._h, 0, None, None, None, None, ct.byref(n)), "e3_plan_records")
        m = n.value
        i0, i1, i2 = (np.zeros(m, np.int32) for _ in range(3))
        v = np.zeros(m, np.float64)
        _check(lib().e3_plan_records(self._h, m, i0.ctypes.data_as(ct.c_void_p), i1.ctypes.data_as(ct.c_void_p),
                                     i2.ctypes.data_as(ct.c_void_p), v.ctypes.data_as(ct.c_void_p),
                                     ct.byref(n)), "e3_plan_records")
        return i0, i1, i2, v

    def close(self):
        if getattr(self, "_h", None) and self._h.value:
            lib().e3_plan_destroy(self._h)
            self._h = ct.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def sh_host(lmax: int, u: np.ndarray) -> np.ndarray:
    """The builder's harmonic polynomials evaluated on the host (float64)."""
    u = np.ascontiguousarray(u, dtype=np.float64)
    y = np.zeros((u.shape[0], (lmax + 1) ** 2))
    _check(lib().e3_sh_host(lmax, u.ctypes.data_as(ct.c_void_p), y.ctypes.data_as(ct.c_void_p), u.shape[0]),
           "e3_sh_host")
    return y


# ---------------------------------------------------------------- graph
class Graph:
    """Receiver- and sender-sorted CSR of an edge list, built on the device."""

    def __init__(self, sender, receiver, n_nodes: int, pad_node: int = -1, stream=None):
        E = sender.shape[0]
        ps = _ptr(sender, "sender", (E,), "int32")
        pr = _ptr(receiver, "receiver", (E,), "int32")
        h = ct.c_void_p()
        _check(lib().e3_graph_create(ps, pr, n_nodes, E, pad_node, _stream(stream), ct.byref(h)),
               "e3_graph_create")
        self._h = h
        self.n_nodes, self.n_edges, self.pad_node = n_nodes, E, pad_node
        n = ct.c_int64()
        _check(lib().e3_graph_live_edges(h, ct.byref(n)), "e3_graph_live_edges")
        self.n_live = n.value

    @property
    def handle(self):
        return self._h

    def export(self):
        torch = _torch()
        dev = torch.device("cuda")
        pr = torch.empty(self.n_live, dtype=torch.int32, device=dev)
        rr = torch.empty(self.n_nodes + 1, dtype=torch.int32, device=dev)
        ps = torch.empty(self.n_live, dtype=torch.int32, device=dev)
        rs = torch.empty(self.n_nodes + 1, dtype=torch.int32, device=dev)
        torch.cuda.synchronize()
        _check(lib().e3_graph_export(self._h, _ptr(pr, "perm_r", dtype="int32"), _ptr(rr, "rowptr_r", dtype="int32"),
                                     _ptr(ps, "perm_s", dtype="int32"), _ptr(rs, "rowptr_s", dtype="int32")),
               "e3_graph_export")
        return pr, rr, ps, rs

    def close(self):
        if getattr(self, "_h", None) and self._h.value:
            lib().e3_graph_destroy(self._h)
            self._h = ct.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---------------------------------------------------------------- compute
def _empty(shape, like=None):
    torch = _torch()
    return torch.empty(shape, dtype=torch.float32, device="cuda")


@_on_stream
def sh(lmax: int, vec, out=None, stream=None):
    n = vec.shape[0]
    out = _empty((n, (lmax + 1) ** 2)) if out is None else out
    _check(lib().e3_sh(lmax, _ptr(vec, "vec", (n, 3)), _ptr(out, "y", (n, (lmax + 1) ** 2)), n, _stream(stream)),
           "e3_sh")
    return out


@_on_stream
def sh_bwd(lmax: int, vec, dy, out=None, stream=None):
    n = vec.shape[0]
    out = _empty((n, 3)) if out is None else out
    _check(lib().e3_sh_bwd(lmax, _ptr(vec, "vec", (n, 3)), _ptr(dy, "dy", (n, (lmax + 1) ** 2)),
                           _ptr(out, "dvec", (n, 3)), n, _stream(stream)), "e3_sh_bwd")
    return out


@_on_stream
def tp_fwd(plan: Plan, x, y, w, out=None, stream=None):
    R = x.shape[0]
    out = _empty((R, plan.D_out, plan.C)) if out is None else out
    _check(lib().e3_tp_fwd(plan.handle, _ptr(x, "x", (R, plan.D_in, plan.C)), _ptr(y, "y", (R, plan.D_sh)),
                           _ptr(w, "w", (R, plan.P, plan.C)), _ptr(out, "z", (R, plan.D_out, plan.C)), R,
                           _stream(stream)), "e3_tp_fwd")
    return out


def tp_workspace_size(plan: Plan, rows: int) -> int:
    b = ct.c_size_t()
    _check(lib().e3_tp_workspace_size(plan.handle, rows, ct.byref(b)), "e3_tp_workspace_size")
    return b.value


@_on_stream
def tp_bwd(plan: Plan, x, y, w, dz, dx=None, dy=None, dw=None, ws=None, stream=None):
    """(dx, dy, dw) of the weighted tensor product."""
    R = x.shape[0]
    dx = _empty((R, plan.D_in, plan.C)) if dx is None else dx
    dy = _empty((R, plan.D_sh)) if dy is None else dy
    dw = _empty((R, plan.P, plan.C)) if dw is None else dw
    if ws is None:
        ws = workspace(tp_workspace_size(plan, R))
    _check(lib().e3_tp_bwd(plan.handle, _ptr(x, "x", (R, plan.D_in, plan.C)), _ptr(y, "y", (R, plan.D_sh)),
                           _ptr(w, "w", (R, plan.P, plan.C)), _ptr(dz, "dz", (R, plan.D_out, plan.C)),
                           _ptr(dx, "dx", (R, plan.D_in, plan.C)), _ptr(dy, "dy", (R, plan.D_sh)),
                           _ptr(dw, "dw", (R, plan.P, plan.C)), ws.data_ptr(), ws.numel(), R,
                           _stream(stream)), "e3_tp_bwd")
    return dx, dy, dw


def conv_workspace_size(plan: Plan, graph: Graph):
    f, b = ct.c_size_t(), ct.c_size_t()
    _check(lib().e3_conv_workspace_size(plan.handle, graph.handle, ct.byref(f), ct.byref(b)),
           "e3_conv_workspace_size")
    return f.value, b.value


def workspace(nbytes: int):
    torch = _torch()
    return torch.empty(max(nbytes, 1), dtype=torch.uint8, device="cuda")


@_on_stream
def conv_fwd(plan: Plan, graph: Graph, x, vec, s, out=None, stream=None):
    N, E = graph.n_nodes, graph.n_edges
    out = _empty((N, plan.D_out, plan.C)) if out is None else out
    _check(lib().e3_conv_fwd(plan.handle, graph.handle, _ptr(x, "x", (N, plan.D_in, plan.C)),
                             _ptr(vec, "vec", (E, 3)), _ptr(s, "s", (E, plan.P, plan.C)),
                             _ptr(out, "m", (N, plan.D_out, plan.C)), None, 0, _stream(stream)), "e3_conv_fwd")
    return out


@_on_stream
def conv_bwd(plan: Plan, graph: Graph, x, vec, s, dm, dx=None, dvec=None, ds=None, ws=None, stream=None):
    N, E = graph.n_nodes, graph.n_edges
    dx = _empty((N, plan.D_in, plan.C)) if dx is None else dx
    dvec = _empty((E, 3)) if dvec is None else dvec
    ds = _empty((E, plan.P, plan.C)) if ds is None else ds
    if ws is None:
        ws = workspace(conv_workspace_size(plan, graph)[1])
    _check(lib().e3_conv_bwd(plan.handle, graph.handle, _ptr(x, "x", (N, plan.D_in, plan.C)),
                             _ptr(vec, "vec", (E, 3)), _ptr(s, "s", (E, plan.P, plan.C)),
                             _ptr(dm, "dm", (N, plan.D_out, plan.C)), _ptr(dx, "dx", (N, plan.D_in, plan.C)),
                             _ptr(dvec, "dvec", (E, 3)), _ptr(ds, "ds", (E, plan.P, plan.C)),
                             ws.data_ptr(), ws.numel(), _stream(stream)), "e3_conv_bwd")
    return dx, dvec, ds


# ---------------------------------------------------------------- float64 builds
def _empty64(shape):
    torch = _torch()
    return torch.empty(shape, dtype=torch.float64, device="cuda")


@_on_stream
def tp_fwd_f64(plan: Plan, x, y, w, out=None, stream=None):
    R = x.shape[0]
    out = _empty64((R, plan.D_out, plan.C)) if out is None else out
    f = "float64"
    _check(lib().e3_tp_fwd_f64(plan.handle, _ptr(x, "x", (R, plan.D_in, plan.C), f), _ptr(y, "y", (R, plan.D_sh), f),
                               _ptr(w, "w", (R, plan.P, plan.C), f), _ptr(out, "z", (R, plan.D_out, plan.C), f), R,
                               _stream(stream)), "e3_tp_fwd_f64")
    return out


@_on_stream
def tp_bwd_f64(plan: Plan, x, y, w, dz, stream=None):
    R = x.shape[0]
    f = "float64"
    dx, dy, dw = _empty64((R, plan.D_in, plan.C)), _empty64((R, plan.D_sh)), _empty64((R, plan.P, plan.C))
    b = ct.c_size_t()
    _check(lib().e3_tp_workspace_size_f64(plan.handle, R, ct.byref(b)), "e3_tp_workspace_size_f64")
    ws = workspace(b.value)
    _check(lib().e3_tp_bwd_f64(plan.handle, _ptr(x, "x", (R, plan.D_in, plan.C), f), _ptr(y, "y", (R, plan.D_sh), f),
                               _ptr(w, "w", (R, plan.P, plan.C), f), _ptr(dz, "dz", (R, plan.D_out, plan.C), f),
                               _ptr(dx, "dx", (R, plan.D_in, plan.C), f), _ptr(dy, "dy", (R, plan.D_sh), f),
                               _ptr(dw, "dw", (R, plan.P, plan.C), f), ws.data_ptr(), ws.numel(), R,
                               _stream(stream)), "e3_tp_bwd_f64")
    return dx, dy, dw


@_on_stream
def conv_fwd_f64(plan: Plan, graph: Graph, x, vec, s, out=None, stream=None):
    N, E = graph.n_nodes, graph.n_edges
    f = "float64"
    out = _empty64((N, plan.D_out, plan.C)) if out is None else out
    _check(lib().e3_conv_fwd_f64(plan.handle, graph.handle, _ptr(x, "x", (N, plan.D_in, plan.C), f),
                                 _ptr(vec, "vec", (E, 3), f), _ptr(s, "s", (E, plan.P, plan.C), f),
                                 _ptr(out, "m", (N, plan.D_out, plan.C), f), _stream(stream)), "e3_conv_fwd_f64")
    return out


@_on_stream
def conv_bwd_f64(plan: Plan, graph: Graph, x, vec, s, dm, stream=None):
    N, E = graph.n_nodes, graph.n_edges
    f = "float64"
    dx, dvec, ds = _empty64((N, plan.D_in, plan.C)), _empty64((E, 3)), _empty64((E, plan.P, plan.C))
    b = ct.c_size_t()
    _check(lib().e3_conv_workspace_size_f64(plan.handle, graph.handle, ct.byref(b)), "e3_conv_workspace_size_f64")
    ws = workspace(b.value)
    _check(lib().e3_conv_bwd_f64(plan.handle, graph.handle, _ptr(x, "x", (N, plan.D_in, plan.C), f),
                                 _ptr(vec, "vec", (E, 3), f), _ptr(s, "s", (E, plan.P, plan.C), f),
                                 _ptr(dm, "dm", (N, plan.D_out, plan.C), f), _ptr(dx, "dx", (N, plan.D_in, plan.C), f),
                                 _ptr(dvec, "dvec", (E, 3), f), _ptr(ds, "ds", (E, plan.P, plan.C), f),
                                 ws.data_ptr(), ws.numel(), _stream(stream)), "e3_conv_bwd_f64")
    return dx, dvec, ds


NOALLOC_SCRATCH_BYTES = 64 << 20


def conv_bwd_noalloc(plan: Plan, graph: Graph, x, vec, s, dm, dx, dvec, ds, stream=None):
    """conv_bwd into the caller's outputs with the library's fixed scratch
    (no allocation by the library or here; outputs must be given)."""
    N, E = graph.n_nodes, graph.n_edges
    _check(lib().e3_conv_bwd_noalloc(plan.handle, graph.handle, _ptr(x, "x", (N, plan.D_in, plan.C)),
                                     _ptr(vec, "vec", (E, 3)), _ptr(s, "s", (E, plan.P, plan.C)),
                                     _ptr(dm, "dm", (N, plan.D_out, plan.C)), _ptr(dx, "dx", (N, plan.D_in, plan.C)),
                                     _ptr(dvec, "dvec", (E, 3)), _ptr(ds, "ds", (E, plan.P, plan.C)),
                                     _stream(stream)), "e3_conv_bwd_noalloc")
    return dx, dvec, ds


def _optr(t, name, shape):
    return None if t is None else _ptr(t, name, shape)


@_on_stream
def conv_fwd_y(plan: Plan, graph: Graph, x, y, s, out=None, accumulate=False, stream=None):
    """m = conv(x, y, s) with the harmonics y [E, D_sh] given (m += ... when accumulate)."""
    N, E = graph.n_nodes, graph.n_edges
    out = _empty((N, plan.D_out, plan.C)) if out is None else out
    _check(lib().e3_conv_fwd_y(plan.handle, graph.handle, _ptr(x, "x", (N, plan.D_in, plan.C)),
                               _ptr(y, "y", (E, plan.D_sh)), _ptr(s, "s", (E, plan.P, plan.C)),
                               _ptr(out, "m", (N, plan.D_out, plan.C)), 1 if accumulate else 0, _stream(stream)),
           "e3_conv_fwd_y")
    return out


@_on_stream
def conv_bwd_y(plan: Plan, graph: Graph, x, y, s, dm, dx=None, dy=None, ds=None, want=("dx", "dy", "ds"),
               accumulate=False, ws=None, stream=None):
    """(dx, dy, ds) of eq. (conv-bwd) with y given; cotangents not in `want` are neither
    computed into memory nor returned (None)."""
    N, E = graph.n_nodes, graph.n_edges
    if "dx" in want and dx is None:
        dx = _empty((N, plan.D_in, plan.C))
    if "dy" in want and dy is None:
        dy = _empty((E, plan.D_sh))
    if "ds" in want and ds is None:
        ds = _empty((E, plan.P, plan.C))
    if ws is None:
        ws = workspace(conv_workspace_size(plan, graph)[1])
    _check(lib().e3_conv_bwd_y(plan.handle, graph.handle, _ptr(x, "x", (N, plan.D_in, plan.C)),
                               _ptr(y, "y", (E, plan.D_sh)), _ptr(s, "s", (E, plan.P, plan.C)),
                               _ptr(dm, "dm", (N, plan.D_out, plan.C)), _optr(dx, "dx", (N, plan.D_in, plan.C)),
                               _optr(dy, "dy", (E, plan.D_sh)), _optr(ds, "ds", (E, plan.P, plan.C)),
                               1 if accumulate else 0, ws.data_ptr(), ws.numel(), _stream(stream)),
           "e3_conv_bwd_y")
    return dx, dy, ds


@_on_stream
def conv_bwd2(plan: Plan, graph: Graph, x, y, s, dm, ddx, ddy, dds, ws=None, stream=None):
    """Double backward: (gx, gy, gs, gdm), the variations of (x, y, s, dm) for
    variations (ddx, ddy, dds) of the backward's outputs."""
    N, E = graph.n_nodes, graph.n_edges
    gx, gdm = _empty((N, plan.D_in, plan.C)), _empty((N, plan.D_out, plan.C))
    gy, gs = _empty((E, plan.D_sh)), _empty((E, plan.P, plan.C))
    if ws is None:
        ws = workspace(conv_workspace_size(plan, graph)[1])
    _check(lib().e3_conv_bwd2(plan.handle, graph.handle, _ptr(x, "x", (N, plan.D_in, plan.C)),
                              _ptr(y, "y", (E, plan.D_sh)), _ptr(s, "s", (E, plan.P, plan.C)),
                              _ptr(dm, "dm", (N, plan.D_out, plan.C)), _ptr(ddx, "ddx", (N, plan.D_in, plan.C)),
                              _ptr(ddy, "ddy", (E, plan.D_sh)), _ptr(dds, "dds", (E, plan.P, plan.C)),
                              _ptr(gx, "gx", (N, plan.D_in, plan.C)), _ptr(gy, "gy", (E, plan.D_sh)),
                              _ptr(gs, "gs", (E, plan.P, plan.C)), _ptr(gdm, "gdm", (N, plan.D_out, plan.C)),
                              ws.data_ptr(), ws.numel(), _stream(stream)), "e3_conv_bwd2")
    return gx, gy, gs, gdm


class RecordTP:
    """Tensor product with caller-supplied records (i0, i1, i2, value)."""

    def __init__(self, d_x: int, d_y: int, d_z: int, i0, i1, i2, val, y_per_channel: bool):
        i0, i1, i2 = (np.ascontiguousarray(a, dtype=np.int32) for a in (i0, i1, i2))
        val = np.ascontiguousarray(val, dtype=np.float64)
        h = ct.c_void_p()
        _check(lib().e3_tpg_create(d_x, d_y, d_z, val.shape[0], i0.ctypes.data_as(ct.c_void_p),
                                   i1.ctypes.data_as(ct.c_void_p), i2.ctypes.data_as(ct.c_void_p),
                                   val.ctypes.data_as(ct.c_void_p), 1 if y_per_channel else 0, ct.byref(h)),
               "e3_tpg_create")
        self.handle = h
        self.d_x, self.d_y, self.d_z, self.ypc = d_x, d_y, d_z, bool(y_per_channel)

    def close(self):
        if getattr(self, "handle", None) and self.handle.value:
            lib().e3_tpg_destroy(self.handle)
            self.handle = ct.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _yshape(self, R, C):
        return (R, self.d_y, C) if self.ypc else (R, self.d_y)

    @staticmethod
    def _kind(x):
        torch = _torch()
        return ("float64", "_f64") if x.dtype == torch.float64 else ("float32", "")

    @_on_stream
    def forward(self, x, y, out=None, stream=None):
        """z in the precision of x (float32 or float64)."""
        R, _, C = x.shape
        dt, sfx = self._kind(x)
        out = _torch().empty((R, self.d_z, C), dtype=x.dtype, device="cuda") if out is None else out
        _check(getattr(lib(), "e3_tpg_fwd" + sfx)(
            self.handle, _ptr(x, "x", (R, self.d_x, C), dt), _ptr(y, "y", self._yshape(R, C), dt),
            _ptr(out, "z", (R, self.d_z, C), dt), R, C, _stream(stream)), "e3_tpg_fwd" + sfx)
        return out

    @_on_stream
    def backward(self, x, y, dz, stream=None):
        R, _, C = x.shape
        dt, sfx = self._kind(x)
        torch = _torch()
        dx = torch.empty((R, self.d_x, C), dtype=x.dtype, device="cuda")
        dy = torch.empty(self._yshape(R, C), dtype=x.dtype, device="cuda")
        b = ct.c_size_t()
        _check(lib().e3_tpg_workspace_size(self.handle, R, C, ct.byref(b)), "e3_tpg_workspace_size")
        ws = workspace(b.value)
        _check(getattr(lib(), "e3_tpg_bwd" + sfx)(
            self.handle, _ptr(x, "x", (R, self.d_x, C), dt), _ptr(y, "y", self._yshape(R, C), dt),
            _ptr(dz, "dz", (R, self.d_z, C), dt), _ptr(dx, "dx", (R, self.d_x, C), dt),
            _ptr(dy, "dy", self._yshape(R, C), dt), ws.data_ptr(), ws.numel(), R, C,
            _stream(stream)), "e3_tpg_bwd" + sfx)
        return dx, dy


class Linear:
    """Equivariant linear mixing between two irreps layouts (weights shared over m)."""

    def __init__(self, irreps_in: str, irreps_out: str):
        h = ct.c_void_p()
        _check(lib().e3_linear_create(irreps_in.encode(), irreps_out.encode(), ct.byref(h)), "e3_linear_create")
        self.handle = h
        nw, di, do, ci, co = ct.c_int64(), ct.c_int(), ct.c_int(), ct.c_int(), ct.c_int()
        _check(lib().e3_linear_query(h, ct.byref(nw), ct.byref(di), ct.byref(do), ct.byref(ci), ct.byref(co)),
               "e3_linear_query")
        self.n_weights, self.D_in, self.D_out, self.C_in, self.C_out = nw.value, di.value, do.value, ci.value, co.value

    def close(self):
        if getattr(self, "handle", None) and self.handle.value:
            lib().e3_linear_destroy(self.handle)
            self.handle = ct.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @_on_stream
    def forward(self, x, W, out=None, stream=None):
        n = x.shape[0]
        out = _empty((n, self.D_out, self.C_out)) if out is None else out
        _check(lib().e3_linear_fwd(self.handle, _ptr(x, "x", (n, self.D_in, self.C_in)),
                                   _ptr(W, "W", (self.n_weights,)), _ptr(out, "out", (n, self.D_out, self.C_out)),
                                   n, _stream(stream)), "e3_linear_fwd")
        return out

    def workspace_size(self) -> int:
        b = ct.c_size_t()
        _check(lib().e3_linear_workspace_size(self.handle, ct.byref(b)), "e3_linear_workspace_size")
        return b.value

    @_on_stream
    def backward(self, x, W, dout, dx=None, dW=None, ws=None, stream=None):
        n = x.shape[0]
        dx = _empty((n, self.D_in, self.C_in)) if dx is None else dx
        dW = _empty((self.n_weights,)) if dW is None else dW
        if ws is None:
            ws = workspace(self.workspace_size())
        _check(lib().e3_linear_bwd(self.handle, _ptr(x, "x", (n, self.D_in, self.C_in)),
                                   _ptr(W, "W", (self.n_weights,)), _ptr(dout, "dout", (n, self.D_out, self.C_out)),
                                   _ptr(dx, "dx", (n, self.D_in, self.C_in)), _ptr(dW, "dW", (self.n_weights,)),
                                   ws.data_ptr(), ws.numel(), n, _stream(stream)), "e3_linear_bwd")
        return dx, dW


def conv_radial_workspace_size(plan: Plan, graph: Graph, K: int) -> int:
    b = ct.c_size_t()
    _check(lib().e3_conv_radial_workspace_size(plan.handle, graph.handle, K, ct.byref(b)),
           "e3_conv_radial_workspace_size")
    return b.value


@_on_stream
def conv_fwd_radial(plan: Plan, graph: Graph, x, vec, h, W, out=None, stream=None):
    """m with per-edge weights s_e = h_e W formed inside the kernel (h [E, K], W [K, P, C])."""
    N, E = graph.n_nodes, graph.n_edges
    K = W.shape[0]
    out = _empty((N, plan.D_out, plan.C)) if out is None else out
    _check(lib().e3_conv_fwd_radial(plan.handle, graph.handle, _ptr(x, "x", (N, plan.D_in, plan.C)),
                                    _ptr(vec, "vec", (E, 3)), _ptr(h, "h", (E, K)),
                                    _ptr(W, "W", (K, plan.P, plan.C)), K,
                                    _ptr(out, "m", (N, plan.D_out, plan.C)), _stream(stream)),
           "e3_conv_fwd_radial")
    return out


@_on_stream
def conv_bwd_radial(plan: Plan, graph: Graph, x, vec, h, W, dm, dx=None, dvec=None, dh=None, dW=None, ws=None,
                    stream=None):
    """(dx, dvec, dh, dW) of the convolution with fused radial weights."""
    N, E = graph.n_nodes, graph.n_edges
    K = W.shape[0]
    dx = _empty((N, plan.D_in, plan.C)) if dx is None else dx
    dvec = _empty((E, 3)) if dvec is None else dvec
    dh = _empty((E, K)) if dh is None else dh
    dW = _empty((K, plan.P, plan.C)) if dW is None else dW
    if ws is None:
        ws = workspace(conv_radial_workspace_size(plan, graph, K))
    _check(lib().e3_conv_bwd_radial(plan.handle, graph.handle, _ptr(x, "x", (N, plan.D_in, plan.C)),
                                    _ptr(vec, "vec", (E, 3)), _ptr(h, "h", (E, K)),
                                    _ptr(W, "W", (K, plan.P, plan.C)), K,
                                    _ptr(dm, "dm", (N, plan.D_out, plan.C)), _ptr(dx, "dx", (N, plan.D_in, plan.C)),
                                    _ptr(dvec, "dvec", (E, 3)), _ptr(dh, "dh", (E, K)),
                                    _ptr(dW, "dW", (K, plan.P, plan.C)), ws.data_ptr(), ws.numel(),
                                    _stream(stream)), "e3_conv_bwd_radial")
    return dx, dvec, dh, dW


# ---------------------------------------------------------------- invariant layers
ACTIVATIONS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}
_LAYER_DTYPES = {}   # torch dtype -> (e3_dtype, its name)


def _layer_dtype(t, name):
    """(e3_dtype, type's name) of a tensor the layers take."""
    try:
        return _LAYER_DTYPES[t.dtype]
    except (KeyError, AttributeError):
        torch = _torch()
        if not isinstance(t, torch.Tensor):
            raise TypeError(f"{name} must be a torch tensor") from None
        _LAYER_DTYPES.update({torch.float32: (0, "float32"), torch.bfloat16: (1, "bfloat16")})
        if t.dtype not in _LAYER_DTYPES:
            raise TypeError(f"{name} must be float32 or bfloat16, got {t.dtype}") from None
        return _LAYER_DTYPES[t.dtype]


def _rows(t, name, shape, dtype):
    """(pointer, row stride) of a matrix whose rows are contiguous; rows may be strided."""
    torch = _modules[0] if _modules else _torch()
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.dtype is not _modules[1][dtype]:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on the GPU")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    m, n = shape
    if m > 1:
        ld, one = t.stride()
        if one == 1 and ld >= n:
            return t.data_ptr(), ld
        if n > 1 and one != 1:
            raise ValueError(f"{name} must have contiguous rows")
        if ld < n:
            raise ValueError(f"{name} has overlapping rows")
        return t.data_ptr(), ld
    if m == 0:
        return None, n
    if n > 1 and t.stride(1) != 1:
        raise ValueError(f"{name} must have contiguous rows")
    return t.data_ptr(), n


class Packed8:
    """A matrix kept in 8 bits: q [rows, cols] int8 times the step 2^(c - 127) of each group of
    32 columns, c [rows, ceil(cols / 32)] uint8 (255: the group is NaN)."""

    __slots__ = ("q", "c")

    def __init__(self, q, c):
        torch = _torch()
        for t, name, dt in ((q, "q", torch.int8), (c, "c", torch.uint8)):
            if not isinstance(t, torch.Tensor) or t.dtype is not dt or t.dim() != 2:
                raise TypeError(f"{name} must be a {dt} matrix")
        if c.shape[0] != q.shape[0] or c.shape[1] != (q.shape[1] + 31) // 32:
            raise ValueError(f"c has shape {tuple(c.shape)}, expected {(q.shape[0], (q.shape[1] + 31) // 32)}")
        self.q, self.c = q, c

    @property
    def shape(self):
        return self.q.shape

    @classmethod
    def empty(cls, rows: int, cols: int) -> "Packed8":
        torch = _torch()
        p = cls.__new__(cls)
        p.q = torch.empty((rows, cols), dtype=torch.int8, device="cuda")
        p.c = torch.empty((rows, (cols + 31) // 32), dtype=torch.uint8, device="cuda")
        return p


def _packed(p, name, shape):
    """Pointers of a Packed8 of the given shape."""
    if not isinstance(p, Packed8):
        raise TypeError(f"{name} must be a Packed8")
    m, n = shape
    return _ptr(p.q, name + ".q", (m, n), "int8"), _ptr(p.c, name + ".c", (m, (n + 31) // 32), "uint8")


def _kept(t, name, shape, dtype):
    """(pointer, row stride, q, c) of an activation in full or packed."""
    if isinstance(t, Packed8):
        return (None, 0, *_packed(t, name, shape))
    return (*_rows(t, name, shape, dtype), None, None)


def _matrix(t, name):
    shape = t.shape
    if len(shape) != 2:
        raise ValueError(f"{name} must be a matrix, got shape {tuple(shape)}")
    return shape


def _scratch(ws):
    """(pointer, bytes) of a workspace, the caller's or a call's own; None: none."""
    if ws is None:
        return None, 0
    if not isinstance(ws, _torch().Tensor):
        raise TypeError("ws must be a torch tensor")
    if not ws.is_cuda:
        raise ValueError("ws must be on the GPU")
    if not ws.is_contiguous():
        raise ValueError("ws must be contiguous")
    return ws.data_ptr(), ws.numel() * ws.element_size()


@_on_stream
def pack8(x, out=None, stream=None) -> Packed8:
    """x [rows, cols] (float32 or bfloat16) in 8 bits."""
    code, dt = _layer_dtype(x, "x")
    m, n = _matrix(x, "x")
    out = Packed8.empty(m, n) if out is None else out
    _check(lib().e3_pack8(code, *_rows(x, "x", (m, n), dt), *_packed(out, "out", (m, n)), m, n, _stream(stream)),
           "e3_pack8")
    return out


@_on_stream
def unpack8(p: Packed8, dtype=None, out=None, stream=None):
    """The values of p, in float32 (or dtype; or in the type of out)."""
    torch = _torch()
    if not isinstance(p, Packed8):
        raise TypeError("p must be a Packed8")
    m, n = p.shape
    if out is None:
        out = torch.empty((m, n), dtype=dtype or torch.float32, device="cuda")
    code, dt = _layer_dtype(out, "out")
    _check(lib().e3_unpack8(code, *_packed(p, "p", (m, n)), *_rows(out, "out", (m, n), dt), m, n, _stream(stream)),
           "e3_unpack8")
    return out


def _keep_of(keep, allowed):
    keep = tuple(keep)
    for k in keep:
        if k not in allowed:
            raise ValueError(f"keep: {k!r} is none of {', '.join(allowed)}")
    return keep


@_on_stream
def layer_norm_fwd(x, gamma=None, beta=None, eps: float = 1e-5, keep=(), out=None, stream=None):
    """y = (x - mean) / sqrt(var + eps) gamma + beta over the columns of each row of x [rows, cols].

    keep adds to the result, in this order: "stats" (mean, rstd [rows], float32), "x8" (x as a
    Packed8), "y8" (y as a Packed8).
    """
    code, dt = _layer_dtype(x, "x")
    m, n = shape = _matrix(x, "x")
    keep = _keep_of(keep, ("stats", "x8", "y8"))
    y = x.new_empty(shape) if out is None else out
    got, mean, rstd, xp, yp = [y], None, None, (None, None), (None, None)
    if "stats" in keep:
        stats = _empty((2, m)).unbind(0)
        got += stats
        mean, rstd = (t.data_ptr() for t in stats)
    if "x8" in keep:
        got.append(Packed8.empty(m, n))
        xp = _packed(got[-1], "x8", shape)
    if "y8" in keep:
        got.append(Packed8.empty(m, n))
        yp = _packed(got[-1], "y8", shape)
    _check(lib().e3_layer_norm_fwd(code, *_rows(x, "x", shape, dt),
                                   None if gamma is None else _ptr(gamma, "gamma", (n,), dt),
                                   None if beta is None else _ptr(beta, "beta", (n,), dt), eps,
                                   *_rows(y, "out", shape, dt), mean, rstd, *xp, *yp, m, n, _stream(stream)),
           "e3_layer_norm_fwd")
    return tuple(got) if keep else y


@functools.lru_cache(maxsize=1024)   # a function of the sizes alone
def layer_norm_workspace_size(rows: int, cols: int, dtype="float32") -> int:
    b = ct.c_size_t()
    _check(lib().e3_layer_norm_workspace_size({"float32": 0, "bfloat16": 1}[dtype], rows, cols, ct.byref(b)),
           "e3_layer_norm_workspace_size")
    return b.value


@_on_stream
def layer_norm_bwd(x, gamma, dy, mean, rstd, want=("dx", "dgamma", "dbeta"), dx=None, ws=None, stream=None):
    """(dx, dgamma, dbeta) from dy, the forward's x (a tensor or a Packed8) and its statistics;
    cotangents not in `want` are not computed (None).  gamma may be None (ones)."""
    code, dt = _layer_dtype(dy, "dy")
    m, n = shape = _matrix(dy, "dy")
    want = _keep_of(want, ("dx", "dgamma", "dbeta"))
    if "dx" in want and dx is None:
        dx = dy.new_empty(shape)
    dg = dy.new_empty((n,)) if "dgamma" in want else None
    db = dy.new_empty((n,)) if "dbeta" in want else None
    if ws is None and (dg is not None or db is not None):
        ws = workspace(layer_norm_workspace_size(m, n, dt))
    xp, ldx, xq, xc = _kept(x, "x", shape, dt)
    _check(lib().e3_layer_norm_bwd(code, xp, ldx, xq, xc, None if gamma is None else _ptr(gamma, "gamma", (n,), dt),
                                   *_rows(dy, "dy", shape, dt), _ptr(mean, "mean", (m,)), _ptr(rstd, "rstd", (m,)),
                                   *((None, n) if dx is None else _rows(dx, "dx", shape, dt)),
                                   None if dg is None else dg.data_ptr(), None if db is None else db.data_ptr(),
                                   *_scratch(ws), m, n, _stream(stream)), "e3_layer_norm_bwd")
    return dx, dg, db


@functools.lru_cache(maxsize=1024)
def dense_workspace_size(M: int, K: int, N: int, dtype="float32"):
    """Bytes of (forward, backward)."""
    f, b = ct.c_size_t(), ct.c_size_t()
    _check(lib().e3_dense_workspace_size({"float32": 0, "bfloat16": 1}[dtype], M, K, N, ct.byref(f), ct.byref(b)),
           "e3_dense_workspace_size")
    return f.value, b.value


def _act_code(act):
    code = ACTIVATIONS.get(act)
    if code is None:
        raise ValueError(f"act: {act!r} is none of {', '.join(ACTIVATIONS)}")
    return code


@_on_stream
def dense_fwd(x, W, bias=None, res=None, act: str = "none", keep=(), out=None, ws=None, stream=None):
    """y = act(x W + bias) + res, with x [M, K], W [K, N], bias [N], res [M, N].

    keep adds to the result, in this order: "z" (z = x W + bias [M, N]), "z8" (z as a Packed8),
    "y8" (y as a Packed8).
    """
    code, dt = _layer_dtype(x, "x")
    M, K = _matrix(x, "x")
    if _matrix(W, "W")[0] != K:
        raise ValueError(f"W has shape {tuple(W.shape)}, expected {K} rows")
    N = W.shape[1]
    keep = _keep_of(keep, ("z", "z8", "y8"))
    shape = (M, N)
    y = x.new_empty(shape) if out is None else out
    got, z, zp, yp = [y], None, (None, None), (None, None)
    if "z" in keep:
        got.append(x.new_empty(shape))
        z = got[-1].data_ptr()
    if "z8" in keep:
        got.append(Packed8.empty(M, N))
        zp = _packed(got[-1], "z8", shape)
    if "y8" in keep:
        got.append(Packed8.empty(M, N))
        yp = _packed(got[-1], "y8", shape)
    if ws is None:
        nb = dense_workspace_size(M, K, N, dt)[0]
        ws = workspace(nb) if nb else None
    _check(lib().e3_dense_fwd(code, *_rows(x, "x", (M, K), dt), _ptr(W, "W", (K, N), dt),
                              None if bias is None else _ptr(bias, "bias", (N,), dt),
                              *((None, N) if res is None else _rows(res, "res", shape, dt)), _act_code(act),
                              *_rows(y, "out", shape, dt), z, N, *zp, *yp, *_scratch(ws), M, K, N, _stream(stream)),
           "e3_dense_fwd")
    return tuple(got) if keep else y


@_on_stream
def dense_bwd(x, W, dy, z=None, act: str = "none", want=("dx", "dW", "db"), dx=None, ws=None, stream=None):
    """(dx, dW, db) of a dense layer from dy and the forward's x and z, each a tensor or a Packed8 (z may be
    None for act "none"); cotangents not in `want` are not computed (None).  The residual's cotangent is dy."""
    code, dt = _layer_dtype(dy, "dy")
    M, N = shape = _matrix(dy, "dy")
    if _matrix(W, "W")[1] != N:
        raise ValueError(f"W has shape {tuple(W.shape)}, expected {N} columns")
    K = W.shape[0]
    want = _keep_of(want, ("dx", "dW", "db"))
    if "dx" in want and dx is None:
        dx = dy.new_empty((M, K))
    dW = dy.new_empty((K, N)) if "dW" in want else None
    db = dy.new_empty((N,)) if "db" in want else None
    if ws is None:
        ws = workspace(dense_workspace_size(M, K, N, dt)[1])
    xp, ldx, xq, xc = (None, K, None, None) if x is None else _kept(x, "x", (M, K), dt)
    zp, ldz, zq, zc = (None, N, None, None) if z is None else _kept(z, "z", shape, dt)
    _check(lib().e3_dense_bwd(code, xp, ldx, xq, xc, _ptr(W, "W", (K, N), dt), zp, ldz, zq, zc, _act_code(act),
                              *_rows(dy, "dy", shape, dt), *((None, K) if dx is None else _rows(dx, "dx", (M, K), dt)),
                              None if dW is None else dW.data_ptr(), None if db is None else db.data_ptr(),
                              *_scratch(ws), M, K, N, _stream(stream)), "e3_dense_bwd")
    return dx, dW, db


def _here(*tensors):
    """Launches go to the current device: every tensor has to be there."""
    device = None
    for t in tensors:
        if t is None:
            continue
        try:
            at = t.get_device()
        except AttributeError:
            raise TypeError(f"expected a torch tensor, got {type(t).__name__}") from None
        if at < 0:
            raise ValueError("tensors must be on the GPU")
        if device is None:
            if _current is None:
                _stream(None)
            device = _current[1]()
        if at != device:
            raise ValueError(f"a tensor is on GPU {at}, the current device is {device}")


# ---------------------------------------------------------------- gated dense layers
@functools.lru_cache(maxsize=1024)
def gated_workspace_size(M: int, K: int, N: int, dtype="float32"):
    """Bytes of (forward, backward) of a gated dense layer with x [M, K] and W [K, 2 N]."""
    f, b = ct.c_size_t(), ct.c_size_t()
    _check(lib().e3_gated_workspace_size({"float32": 0, "bfloat16": 1}[dtype], M, K, N, ct.byref(f), ct.byref(b)),
           "e3_gated_workspace_size")
    return f.value, b.value


def _gated_width(W, K):
    """N of W [K, 2 N]."""
    k, n2 = _matrix(W, "W")
    if k != K or n2 % 2:
        raise ValueError(f"W has shape {(k, n2)}, expected {K} rows and an even number of columns")
    return n2 // 2


@_on_stream
def gated_fwd(x, W, bias=None, act: str = "silu", keep=(), out=None, ws=None, stream=None):
    """y = act(g) u with [g | u] = x W + bias, x [M, K], W [K, 2 N], bias [2 N], y [M, N].

    keep adds to the result, in this order: "z" (z [M, 2 N], its rows g and u side by side), "z8" (a
    pair: g and u as a Packed8 each), "y8" (y as a Packed8).  z and the pair are what gated_bwd takes.
    """
    code, dt = _layer_dtype(x, "x")
    M, K = _matrix(x, "x")
    N = _gated_width(W, K)
    keep = _keep_of(keep, ("z", "z8", "y8"))
    shape = (M, N)
    y = x.new_empty(shape) if out is None else out
    _here(x, W, bias, y, ws)
    got, z, zp, yp = [y], None, (None,) * 4, (None, None)
    if "z" in keep:
        got.append(x.new_empty((M, 2 * N)))
        z = got[-1].data_ptr()
    if "z8" in keep:
        got.append((Packed8.empty(M, N), Packed8.empty(M, N)))
        zp = (*_packed(got[-1][0], "z8", shape), *_packed(got[-1][1], "z8", shape))
    if "y8" in keep:
        got.append(Packed8.empty(M, N))
        yp = _packed(got[-1], "y8", shape)
    if ws is None:
        nb = gated_workspace_size(M, K, N, dt)[0]
        ws = workspace(nb) if nb else None
    _check(lib().e3_gated_fwd(code, *_rows(x, "x", (M, K), dt), _ptr(W, "W", (K, 2 * N), dt),
                              None if bias is None else _ptr(bias, "bias", (2 * N,), dt), _act_code(act),
                              *_rows(y, "out", shape, dt), z, 2 * N, *zp, *yp, *_scratch(ws), M, K, N, _stream(stream)),
           "e3_gated_fwd")
    return tuple(got) if keep else y


@_on_stream
def gated_bwd(x, W, dy, z, act: str = "silu", want=("dx", "dW", "db"), dx=None, ws=None, stream=None):
    """(dx, dW, db) of a gated dense layer from dy and the forward's x (a tensor or a Packed8) and z (a tensor
    [M, 2 N], or the pair of "z8"); cotangents not in `want` are not computed (None).  x is needed for dW only.
    In bfloat16 dz is rounded for the products of dx and dW, but for K <= 64 and N <= 128 from a tensor z."""
    code, dt = _layer_dtype(dy, "dy")
    M, N = shape = _matrix(dy, "dy")
    K = _matrix(W, "W")[0]
    if _gated_width(W, K) != N:
        raise ValueError(f"W has shape {tuple(W.shape)}, expected {2 * N} columns")
    want = _keep_of(want, ("dx", "dW", "db"))
    if "dx" in want and dx is None:
        dx = dy.new_empty((M, K))
    dW = dy.new_empty((K, 2 * N)) if "dW" in want else None
    db = dy.new_empty((2 * N,)) if "db" in want else None
    if ws is None:
        ws = workspace(gated_workspace_size(M, K, N, dt)[1])
    xp = (None, K, None, None) if x is None else _kept(x, "x", (M, K), dt)
    if isinstance(z, (tuple, list)):
        if len(z) != 2:
            raise ValueError("z must be a tensor or a pair of Packed8")
        zp = (None, 2 * N, *_packed(z[0], "z[0]", shape), *_packed(z[1], "z[1]", shape))
        _here(W, dy, dx, ws, x.q if isinstance(x, Packed8) else x, z[0].q, z[0].c, z[1].q, z[1].c)
    else:
        zp = (*_rows(z, "z", (M, 2 * N), dt), None, None, None, None)
        _here(W, dy, dx, ws, x.q if isinstance(x, Packed8) else x, z)
    _check(lib().e3_gated_bwd(code, *xp, _ptr(W, "W", (K, 2 * N), dt), *zp, _act_code(act), *_rows(dy, "dy", shape, dt),
                              *((None, K) if dx is None else _rows(dx, "dx", (M, K), dt)),
                              None if dW is None else dW.data_ptr(), None if db is None else db.data_ptr(),
                              *_scratch(ws), M, K, N, _stream(stream)), "e3_gated_bwd")
    return dx, dW, db


# ---------------------------------------------------------------- dropout and residual norms
class Dropout:
    """What a dropout mask is made of: the probability p, a seed, an offset (both 0 to 2^64 - 1), and a counter,
    an int64 tensor of one element on the GPU whose value is added to the offset when a kernel runs (None: 0).

    The mask of a call is a function of these and of each value's row and column alone (the formula: e3_dropout_fwd
    in e3mi.h), so that a backward with an equal Dropout has its forward's mask.  Calls that shall have masks of their
    own take another seed or offset.  A captured graph draws another mask in each replay if the program counts the
    counter up in between.
    """

    __slots__ = ("p", "seed", "offset", "counter")

    def __init__(self, p: float, seed: int, offset: int = 0, counter=None):
        if not 0.0 <= p <= 1.0:
            raise ValueError(f"p must lie in [0, 1], got {p}")
        for v, name in ((seed, "seed"), (offset, "offset")):
            if not 0 <= v < 1 << 64:
                raise ValueError(f"{name} must lie in [0, 2^64), got {v}")
        self.p, self.seed, self.offset, self.counter = p, seed, offset, counter

    def _args(self):
        c = self.counter
        if c is not None:
            _here(c)
            c = _ptr(c, "counter", (1,) if c.dim() else (), "int64")
        return self.p, self.seed, self.offset, c


_NO_DROP = (0.0, 0, 0, None)


def _drop_args(drop):
    if drop is None:
        return _NO_DROP
    if not isinstance(drop, Dropout):
        raise TypeError("drop must be a Dropout")
    return drop._args()


@_on_stream
def dropout_fwd(x, drop, res=None, out=None, stream=None):
    """y = res + keep x / (1 - p) with the mask of drop (a Dropout), x and res [rows, cols]; out may be x or res."""
    code, dt = _layer_dtype(x, "x")
    m, n = shape = _matrix(x, "x")
    if not isinstance(drop, Dropout):
        raise TypeError("drop must be a Dropout")
    y = x.new_empty(shape) if out is None else out
    _here(x, res, y)
    _check(lib().e3_dropout_fwd(code, *_rows(x, "x", shape, dt),
                                *((None, n) if res is None else _rows(res, "res", shape, dt)), *drop._args(),
                                *_rows(y, "out", shape, dt), m, n, _stream(stream)), "e3_dropout_fwd")
    return y


@_on_stream
def dropout_bwd(dy, drop, dx=None, stream=None):
    """dx = keep dy / (1 - p), from the Dropout of the forward; dx may be dy.  The residual's cotangent is dy."""
    code, dt = _layer_dtype(dy, "dy")
    m, n = shape = _matrix(dy, "dy")
    if not isinstance(drop, Dropout):
        raise TypeError("drop must be a Dropout")
    dx = dy.new_empty(shape) if dx is None else dx
    _here(dy, dx)
    _check(lib().e3_dropout_bwd(code, *_rows(dy, "dy", shape, dt), *drop._args(), *_rows(dx, "dx", shape, dt), m, n,
                                _stream(stream)), "e3_dropout_bwd")
    return dx


NORMS = {"rms": 0, "layer": 1}


def _norm_code(norm):
    code = NORMS.get(norm)
    if code is None:
        raise ValueError(f"norm: {norm!r} is none of {', '.join(NORMS)}")
    return code


def _norm_weights(w, name, norm, n, dt):
    """(gamma, beta) pointers of a norm's weights: None (no norm) or a pair whose entries may be None."""
    if w is None:
        return None, None
    if not isinstance(w, (tuple, list)) or len(w) != 2:
        raise TypeError(f"{name} must be None or a pair (gamma, beta)")
    g, b = w
    if norm == "rms" and b is not None:
        raise ValueError(f"{name}: an rms norm has no beta")
    _here(g, b)
    return (None if g is None else _ptr(g, name + " gamma", (n,), dt),
            None if b is None else _ptr(b, name + " beta", (n,), dt))


def _gate(gate, shape, dt):
    """(pointer, row stride) of a gate: none, a vector (stride 0) or a matrix."""
    if gate is None:
        return None, 0
    if isinstance(gate, _torch().Tensor) and gate.dim() == 1:
        return _ptr(gate, "gate", (shape[1],), dt), 0
    return _rows(gate, "gate", shape, dt)


@_on_stream
def residual_norm_fwd(h, res=None, gate=None, scale: float = 1.0, norm: str = "rms", post=None, pre=None,
                      eps: float = 1e-5, drop=None, keep=(), out=None, y=None, stream=None):
    """s = res + scale gate drop(N1(h)) and y = N2(s), in one pass over the rows of h [rows, cols].

    post, pre: the weights (gamma, beta) of N1 (the norm after a block) and N2 (the one before the next); an
    entry may be None (1, 0), and instead of a pair None leaves the norm out.  norm: "rms" (x / sqrt(mean x^2 +
    eps) gamma, no beta) or "layer", for both.  gate: None, [cols] or [rows, cols].  drop: a Dropout.  out (s; may
    be res) and y are written where they are given.

    Returns s, with pre (s, y); keep=("stats",) adds the statistics that the backward takes, float32 rows of
    [n, rows]: for each norm that is there its rstd, before it (layer) its mean.
    """
    code, dt = _layer_dtype(h, "h")
    m, n = shape = _matrix(h, "h")
    keep = _keep_of(keep, ("stats",))
    kind = _norm_code(norm)
    s = h.new_empty(shape) if out is None else out
    if pre is None and y is not None:
        raise ValueError("y is the output of the norm that pre names")
    if pre is not None and y is None:
        y = h.new_empty(shape)
    _here(h, res, gate, s, y)
    p = [None] * 4
    stats = None
    if keep:
        stats = _empty(((1 + kind) * ((post is not None) + (pre is not None)), m))
        at, step = stats.data_ptr(), 4 * m
        for k, w in ((0, post), (2, pre)):
            if w is not None and m:
                if kind:
                    p[k], at = at, at + step
                p[k + 1], at = at, at + step
    _check(lib().e3_residual_norm_fwd(
        code, kind, (post is not None) + 2 * (pre is not None), *_rows(h, "h", shape, dt),
        *((None, n) if res is None else _rows(res, "res", shape, dt)), *_gate(gate, shape, dt), scale, *_drop_args(drop),
        *_norm_weights(post, "post", norm, n, dt), *_norm_weights(pre, "pre", norm, n, dt), eps,
        *_rows(s, "out", shape, dt), *((None, n) if y is None else _rows(y, "y", shape, dt)), *p, m, n,
        _stream(stream)), "e3_residual_norm_fwd")
    got = (s,) if y is None else (s, y)
    return (*got, stats) if keep else got if y is not None else s


@functools.lru_cache(maxsize=1024)
def residual_norm_workspace_size(rows: int, cols: int, dtype="float32") -> int:
    b = ct.c_size_t()
    _check(lib().e3_residual_norm_workspace_size({"float32": 0, "bfloat16": 1}[dtype], rows, cols, ct.byref(b)),
           "e3_residual_norm_workspace_size")
    return b.value


@_on_stream
def residual_norm_bwd(h, s, stats, dy=None, ds=None, gate=None, scale: float = 1.0, norm: str = "rms", post=None,
                      pre=None, drop=None, want=("dres", "dh", "dgate", "dpost", "dpre"), dres=None, dh=None, ws=None,
                      stream=None):
    """(dres, dh, dgate, dpost, dpre) from the cotangents dy of y and ds of s (None: 0; with pre, dy is needed)
    and the forward's h, s (needed with pre), statistics and arguments.  dpost and dpre are pairs (dgamma, dbeta);
    what was not there (a gate, a norm, a weight that was None) or is not in `want` is None.  h is needed for
    the norm after the block and for dgate.  dres and dh are written where they are given; each may be ds, dy, s
    or h itself (the same rows), but not the other."""
    ref = dy if dy is not None else ds
    if ref is None:
        raise ValueError("dy or ds must be given")
    if (dy is None) != (pre is None):
        raise ValueError("dy is the cotangent of the norm that pre names")
    code, dt = _layer_dtype(ref, "dy" if dy is not None else "ds")
    m, n = shape = _matrix(ref, "dy" if dy is not None else "ds")
    want = _keep_of(want, ("dres", "dh", "dgate", "dpost", "dpre"))
    kind = _norm_code(norm)
    if "dres" in want and dres is None:
        dres = ref.new_empty(shape)
    if "dh" in want and dh is None:
        dh = ref.new_empty(shape)
    dgate = ref.new_empty(gate.shape) if gate is not None and "dgate" in want else None
    grads = []
    for w, name in ((post, "dpost"), (pre, "dpre")):
        wanted = w is not None and name in want
        grads.append(tuple(ref.new_empty((n,)) if wanted and v is not None else None for v in (w or (None, None))))
    vectors = [v for g in grads for v in g]
    weights = (*_norm_weights(post, "post", norm, n, dt), *_norm_weights(pre, "pre", norm, n, dt))
    if ws is None and (any(v is not None for v in vectors) or (dgate is not None and dgate.dim() == 1)):
        ws = workspace(residual_norm_workspace_size(m, n, dt))
    _here(h, s, stats, dy, ds, gate, dres, dh, ws)
    count = (1 + kind) * ((post is not None) + (pre is not None))
    p = [None] * 4
    if count:
        at, step = _ptr(stats, "stats", (count, m)), 4 * m
        for k, w in ((0, post), (2, pre)):
            if w is not None and m:
                if kind:
                    p[k], at = at, at + step
                p[k + 1], at = at, at + step
    none = (None, n)
    _check(lib().e3_residual_norm_bwd(
        code, kind, (post is not None) + 2 * (pre is not None), *(none if h is None else _rows(h, "h", shape, dt)),
        *(none if s is None or pre is None else _rows(s, "s", shape, dt)), *_gate(gate, shape, dt), scale,
        *_drop_args(drop), *weights[:3], *p, *(none if dy is None else _rows(dy, "dy", shape, dt)),
        *(none if ds is None else _rows(ds, "ds", shape, dt)), *(none if dres is None else _rows(dres, "dres", shape, dt)),
        *(none if dh is None else _rows(dh, "dh", shape, dt)), None if dgate is None else dgate.data_ptr(), n,
        *(None if v is None else v.data_ptr() for v in vectors), *_scratch(ws), m, n, _stream(stream)),
        "e3_residual_norm_bwd")
    post_grads, pre_grads = (g if w is not None and name in want else None
                             for g, w, name in ((grads[0], post, "dpost"), (grads[1], pre, "dpre")))
    return dres, dh, dgate, post_grads, pre_grads


# ---------------------------------------------------------------- instrumentation
PROBE_NT_LOAD, PROBE_NT_STORE = 1, 2


@_on_stream
def probe_stream(src, dst, read_units: int, write_units: int, width: int, flags: int, stream=None):
    """One streaming probe launch; returns (bytes read, bytes written)."""
    br, bw = ct.c_size_t(), ct.c_size_t()
    sp = ct.c_void_p(src.data_ptr()) if src is not None else None
    dp = ct.c_void_p(dst.data_ptr()) if dst is not None else None
    sb = src.numel() * src.element_size() if src is not None else 0
    db = dst.numel() * dst.element_size() if dst is not None else 0
    _check(lib().e3_probe_stream(sp, sb, dp, db, read_units, write_units, width, flags, ct.byref(br),
                                 ct.byref(bw), _stream(stream)), "e3_probe_stream")
    return br.value, bw.value


# ---------------------------------------------------------------- timing
def timing_enable(on: bool = True):
    _check(lib().e3_timing_enable(1 if on else 0), "e3_timing_enable")


def timing_reset():
    _check(lib().e3_timing_reset(), "e3_timing_reset")


def timing_read() -> dict:
    """{kernel name: (summed ms, launches)} since the last reset."""
    n = ct.c_int()
    _check(lib().e3_timing_read(0, None, None, None, ct.byref(n)), "e3_timing_read")
    cap = n.value
    names = ct.create_string_buffer(32 * max(cap, 1))
    ms = np.zeros(max(cap, 1), np.float64)
    cnt = np.zeros(max(cap, 1), np.int64)
    _check(lib().e3_timing_read(cap, ct.cast(names, ct.c_void_p), ms.ctypes.data_as(ct.c_void_p),
                                cnt.ctypes.data_as(ct.c_void_p), ct.byref(n)), "e3_timing_read")
    out = {}
    for i in range(min(cap, n.value)):
        nm = names.raw[32 * i:32 * (i + 1)].split(b"\0", 1)[0].decode()
        out[nm] = (float(ms[i]), int(cnt[i]))
    return out
