"""ctypes binding of libgcn.so (include/gcn.h).

Argument marshalling only: every computation runs in the HIP library.  torch
supplies device memory (tensor.data_ptr()) and the HIP stream
(torch.cuda.current_stream().cuda_stream); nothing here computes on tensors (a
statistic whose rows or columns lie apart is copied).
If libgcn.so is missing, importing this module raises: there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgcn.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is not built; run __graft_entry__.build() (hipcc, gfx950)")

_lib = C.CDLL(LIB_PATH)

P = C.c_void_p
i32, i64, f32, f64, sz = C.c_int32, C.c_int64, C.c_float, C.c_double, C.c_size_t

OK, E_INVALID, E_RANGE, E_OVERFLOW, E_CAPACITY, E_HIP, E_UNSUPPORTED = 0, -1, -2, -3, -4, -5, -6
DENSE, SPARSE = 0, 1
ACT_NONE, ACT_RELU, ACT_SOFTMAX_CE, ACT_SILU = 0, 1, 2, 3
ORDER_AUTO, TRANSFORM_FIRST, AGGREGATE_FIRST = 0, 1, 2
AGG_NORM, AGG_SUM, AGG_MEAN, AGG_MEAN_T, AGG_MAX = 0, 1, 2, 3, 4
EPI_NONE, EPI_RELU, EPI_MASK = 0, 1, 2
OP_NN, OP_NT, OP_TN = 0, 1, 2


class GcnError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        name = _lib.gcn_status_string(status).decode()
        msg = _lib.gcn_last_error().decode()
        super().__init__(f"{where}: {name}: {msg}")


SPLIT_MIN, SPLIT_CHUNK = 4096, 2048
MUON_MAX = 16  # matrices of a gcn_muon call


class gcn_split(C.Structure):
    _fields_ = [("n_long", i32), ("n_chunk", i64), ("cap", i64), ("rows", P), ("first", P), ("owner", P),
                ("order", P)]


class gcn_graph(C.Structure):
    _fields_ = [("n", i32), ("nnz", i64), ("nnz_cap", i64), ("row_ptr", P), ("col_idx", P),
                ("deg", P), ("dinv", P), ("val", P), ("split", gcn_split), ("order", P)]


class gcn_sparse_x(C.Structure):
    _fields_ = [("n", i32), ("f", i32), ("nnz", i64), ("row_ptr", P), ("col", P), ("val", P),
                ("col_ptr", P), ("row", P), ("cval", P), ("csc_split", gcn_split)]


class gcn_feature_info(C.Structure):
    _fields_ = [("nnz", i64), ("sparsity", f64), ("mode", i32)]


class gcn_layer(C.Structure):
    _fields_ = [("f_in", i32), ("f_out", i32), ("ld_in", i64), ("ld_out", i64), ("act", i32),
                ("order", i32), ("index", i32), ("agg", i32)]


class gcn_model(C.Structure):
    _fields_ = [("n_layers", i32), ("layers", C.POINTER(gcn_layer))] + \
               [(nm, C.POINTER(P)) for nm in ("W", "b", "dW", "db", "mW", "vW", "mb", "vb", "act",
                                               "saved", "grad")] + \
               [("lr", f64), ("beta1", f64), ("beta2", f64), ("eps", f64), ("step", i32), ("d_step", P)]


class gcn_adam_tensor(C.Structure):
    _fields_ = [("param", P), ("grad", P), ("m", P), ("v", P), ("count", i64)]


class gcn_muon_tensor(C.Structure):
    _fields_ = [("param", P), ("grad", P), ("m", P), ("rows", i64), ("cols", i64), ("scale", f64)]


class gcn_profile_record(C.Structure):
    _fields_ = [("name", C.c_char * 64), ("width", i32), ("rows", i64), ("nnz", i64), ("ms", f32)]


_SIG = {
    "gcn_status_string": (C.c_char_p, [i32]),
    "gcn_last_error": (C.c_char_p, []),
    "gcn_version": (i32, []),
    "gcn_build_csr": (i32, [i32, i64, P, P, C.POINTER(gcn_graph), P, C.POINTER(sz), P]),
    "gcn_feature_stats": (i32, [P, i32, i32, i64, i32, i32, i32, P, C.POINTER(gcn_feature_info),
                                C.POINTER(gcn_sparse_x), P, C.POINTER(sz), P]),
    "gcn_layer_order": (i32, [C.POINTER(gcn_layer), i32]),
    "gcn_layer_fwd": (i32, [C.POINTER(gcn_graph), C.POINTER(gcn_layer), P, C.POINTER(gcn_sparse_x),
                            P, P, P, P, P, P, P, P, C.POINTER(sz), P]),
    "gcn_layer_bwd": (i32, [C.POINTER(gcn_graph), C.POINTER(gcn_layer), P, P, C.POINTER(gcn_sparse_x),
                            P, P, P, P, P, P, C.POINTER(sz), P]),
    "gcn_epoch": (i32, [C.POINTER(gcn_model), C.POINTER(gcn_graph), P, C.POINTER(gcn_sparse_x), P, P,
                        P, C.POINTER(sz), P]),
    "gcn_aggregate": (i32, [C.POINTER(gcn_graph), i32, i32, P, i64, P, i32, P, i64, P, i64, P, C.POINTER(sz),
                            P]),
    "gcn_row_order_used": (i32, [C.POINTER(gcn_graph), i32, i64]),
    "gcn_aggregate_max": (i32, [C.POINTER(gcn_graph), i32, P, i64, P, i64, P, i64, P, C.POINTER(sz), P]),
    "gcn_aggregate_max_bwd": (i32, [C.POINTER(gcn_graph), i32, P, i64, P, i64, P, i64, P, i64, P, C.POINTER(sz),
                                    P]),
    "gcn_gemm": (i32, [i32, i64, i64, i64, P, i64, P, i64, P, i64, P, i32, P, i64, P, C.POINTER(sz), P]),
    "gcn_gemm_static": (i32, [i32, i64, i64, i64, P, i64, P, i64, P, i64, P, i32, P, i64, P]),
    "gcn_spmm": (i32, [i64, i64, P, P, P, i64, i32, P, i64, P, i64, C.POINTER(gcn_split), P, C.POINTER(sz), P]),
    "gcn_spmm_xt": (i32, [i32, i32, i64, P, P, P, C.POINTER(gcn_split), P, i64, i32, P, i64, P, C.POINTER(sz), P]),
    "gcn_spmm_xw": (i32, [i32, i32, i64, P, P, P, P, i64, i32, P, i64, P, C.POINTER(sz), P]),
    "gcn_column_sums": (i32, [i64, i32, P, i64, P, P, P, P, C.POINTER(sz), P]),
    "gcn_group_norm_fwd": (i32, [i64, i32, i32, i32, P, i64, P, i64, P, P, f64, i32, P, i64, P, P, P, C.POINTER(sz),
                                 P]),
    "gcn_group_norm_bwd": (i32, [i64, i32, i32, i32, P, i64, P, i64, P, P, i32, P, P, P, i64, P, i64, P, P, P,
                                 C.POINTER(sz), P]),
    "gcn_adam": (i32, [C.POINTER(gcn_adam_tensor), i32, i32, f64, f64, f64, f64, P]),
    "gcn_adam_device_step": (i32, [C.POINTER(gcn_adam_tensor), i32, P, f64, f64, f64, f64, P]),
    "gcn_orthogonalize": (i32, [i64, i64, P, i64, i32, P, i64, P, C.POINTER(sz), P]),
    "gcn_muon": (i32, [C.POINTER(gcn_muon_tensor), i32, i32, f64, f64, i32, f64, P, C.POINTER(sz), P]),
    "gcn_profile_enable": (i32, [i32]),
    "gcn_profile_count": (i32, []),
    "gcn_profile_read": (i32, [i32, C.POINTER(gcn_profile_record)]),
    "gcn_profile_reset": (i32, []),
    "gcn_profile_only": (i32, [C.c_char_p]),
}
for _name, (_res, _args) in _SIG.items():
    _f = getattr(_lib, _name)
    _f.restype = _res
    _f.argtypes = _args


def _check(status, where):
    if status != OK:
        raise GcnError(status, where)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream=None):
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream


def _sectors(w: int, p: int) -> float:
    return sum((((4 * p * r) % 64) + 4 * w + 63) // 64 for r in range(16)) / 16.0


def pitch(w: int) -> int:
    """Row pitch for activations and gradients (rows the aggregation gathers): w rounded up
    to 4 floats, or to 16 where that makes a row touch fewer 64-byte sectors on average."""
    a, b = (w + 3) // 4 * 4, (w + 15) // 16 * 16
    return b if _sectors(w, b) < _sectors(w, a) else a


def padded(rows: int, w: int, device="cuda", fill=None):
    """A rows x w fp32 view with pitch(w) columns of storage (extra columns zero)."""
    buf = torch.zeros((rows, pitch(w)), dtype=torch.float32, device=device)
    return buf[:, :w]


def _ld(t):
    return t.stride(0) if t.dim() == 2 else t.shape[-1]


class _Workspace:
    """Device scratch that is kept from call to call and grows to the largest size asked for.

    A buffer serves the stream that it was allocated on.  A call on another stream gets one of its own in its
    place: calls on two streams share no scratch, and what is freed goes back to the only stream that used it.
    A call that is captured into a graph takes what is there, and a buffer that a graph uses is kept as long as
    the workspace: keep that as long as the graph, and run what shares it (replays of its graphs, calls) one
    after the other."""

    def __init__(self):
        self.buf = None
        self.stream = None  # handle of the stream that buf belongs to
        self.held = []      # buffers that a graph uses

    def hold(self):
        if not any(b is self.buf for b in self.held):
            self.held.append(self.buf)

    def kept(self, nbytes, dev, stream, capturing):
        """The buffer, if it is large enough and a call on this stream of device `dev` may use it."""
        buf = self.buf
        if buf is None or buf.get_device() != dev or buf.numel() < nbytes:
            return None
        if capturing:
            self.hold()
        elif stream != self.stream:
            return None
        return buf

    def take(self, nbytes, dev, stream, capturing):
        """The buffer for a call on `stream`, the current one (dev -1: in host memory)."""
        if self.kept(nbytes, dev, stream, capturing) is None:
            self.buf = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=dev if dev >= 0 else "cpu")
            self.stream = stream
            if capturing:
                self.hold()
        return self.buf

    def get(self, nbytes, device, stream=None):
        """The same for a call on the stream of this handle (None: the current one)."""
        if nbytes == 0:
            return None
        device = torch.device(device)
        dev = device.index if device.index is not None else torch.cuda.current_device()
        current = torch.cuda.current_stream(dev).cuda_stream
        if stream is None or stream == current:
            return self.take(nbytes, dev, current, torch.cuda.is_current_stream_capturing())
        with torch.cuda.stream(torch.cuda.ExternalStream(stream, dev) if stream else torch.cuda.default_stream(dev)):
            return self.take(nbytes, dev, stream, torch.cuda.is_current_stream_capturing())


def _run_ws(fn, args_before, args_after, where, ws: _Workspace | None, device):
    """Two-phase workspace protocol: size query, then the call with a buffer that large.  args_after begins with the
    handle of the call's stream."""
    nbytes = sz(0)
    _check(fn(*args_before, None, C.byref(nbytes), *args_after), where + " (size query)")
    ws = ws or _Workspace()
    stream = args_after[0]
    buf = ws.get(max(nbytes.value, 256), device, (stream.value or 0) if isinstance(stream, P) else stream)
    nbytes = sz(buf.numel())
    _check(fn(*args_before, buf.data_ptr(), C.byref(nbytes), *args_after), where)
    return ws


# ---------------------------------------------------------------------------
# graph and features
# ---------------------------------------------------------------------------


class SplitPlan:
    """Device buffers of a row-split plan (see gcn_split in gcn.h)."""

    def __init__(self, entries: int, dev, order: bool):
        cap = (3 * entries) // (2 * SPLIT_CHUNK) + 1  # bound on chunks (see gcn_split)
        self.rows = torch.empty(cap, dtype=torch.int32, device=dev)
        self.first = torch.empty(cap + 1, dtype=torch.int64, device=dev)
        self.owner = torch.empty(cap, dtype=torch.int32, device=dev)
        self.order = torch.empty(cap, dtype=torch.int64, device=dev) if order else None
        self.c = gcn_split(0, 0, cap, _ptr(self.rows), _ptr(self.first), _ptr(self.owner), _ptr(self.order))


class DeviceGraph:
    """A + I in CSR on the device (owning torch tensors), with its hub split plan."""

    def __init__(self, n, row_ptr, col_idx, deg, dinv, val, nnz, plan: SplitPlan | None, split_c, order=None):
        self.n = n
        self.row_ptr, self.col_idx, self.deg, self.dinv, self.val = row_ptr, col_idx, deg, dinv, val
        self.nnz = nnz
        self.plan = plan
        self.order = order  # rows in processing order (longest first), or None
        self.c = gcn_graph(n, nnz, col_idx.numel(), _ptr(row_ptr), _ptr(col_idx), _ptr(deg), _ptr(dinv),
                           _ptr(val), split_c, _ptr(order))

    @property
    def n_long(self):
        return self.c.split.n_long


def build_csr(n: int, src: torch.Tensor, dst: torch.Tensor, stream=None, split: bool = True,
              order: bool = True) -> DeviceGraph:
    """gcn_build_csr on device int32 edge arrays; returns the graph (blocking).  order: also
    build the row order of the aggregations (long rows first; results are the same)."""
    dev = src.device
    ne = src.numel()
    row_ptr = torch.empty(n + 1, dtype=torch.int64, device=dev)
    col = torch.empty(max(2 * ne + n, 1), dtype=torch.int32, device=dev)
    deg = torch.empty(max(n, 1), dtype=torch.int32, device=dev)
    dinv = torch.empty(max(n, 1), dtype=torch.float32, device=dev)
    val = torch.empty(col.numel(), dtype=torch.float32, device=dev)
    plan = SplitPlan(2 * ne + n, dev, order=False) if split else None
    ordv = torch.empty(max(n, 1), dtype=torch.int32, device=dev) if order else None
    g = gcn_graph(n, 0, col.numel(), _ptr(row_ptr), _ptr(col), _ptr(deg), _ptr(dinv), _ptr(val),
                  plan.c if plan else gcn_split(), _ptr(ordv))
    _run_ws(_lib.gcn_build_csr, (n, ne, _ptr(src), _ptr(dst), C.byref(g)), (P(_stream(stream)),),
            "gcn_build_csr", None, dev)
    return DeviceGraph(n, row_ptr, col, deg, dinv, val, g.nnz, plan, g.split, ordv)


def tune_row_order(g: DeviceGraph, width: int, reps: int = 3) -> bool:
    """Keep the graph's row order (long rows first) only where it makes the aggregation of
    this width faster on this device: times gcn_aggregate both ways, twice each, and drops
    the order when it does not win.  An aggregation that takes rows as they come says
    nothing about the order: it is then kept, untimed.  Every result is the same either way.
    Returns whether the order is kept."""
    if g.order is None or g.n == 0:
        return False
    if not _lib.gcn_row_order_used(C.byref(g.c), width, pitch(width)):
        return True
    dev = g.row_ptr.device
    M = torch.zeros((g.n, pitch(width)), dtype=torch.float32, device=dev)[:, :width]
    Z = torch.empty_like(M)
    ws = _Workspace()
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)

    def timed(order_ptr):
        g.c.order = order_ptr
        aggregate(g, M, Z, ws=ws)
        e0.record()
        for _ in range(reps):
            aggregate(g, M, Z, ws=ws)
        e1.record()
        torch.cuda.synchronize()
        return e0.elapsed_time(e1)

    on = min(timed(_ptr(g.order)), timed(_ptr(g.order)))
    off = min(timed(None), timed(None))
    keep = on < off
    g.c.order = _ptr(g.order) if keep else None
    if not keep:
        g.order = None
    return keep


class SparseFeatures:
    """X_csr (+ X_csc with its long-column split plan) on the device (owning torch tensors)."""

    def __init__(self, n, f, nnz, dev, csc=True, split=True):
        cap = max(nnz, 1)
        self.row_ptr = torch.empty(n + 1, dtype=torch.int64, device=dev)
        self.col = torch.empty(cap, dtype=torch.int32, device=dev)
        self.val = torch.empty(cap, dtype=torch.float32, device=dev)
        self.col_ptr = torch.empty(f + 1, dtype=torch.int64, device=dev) if csc else None
        self.row = torch.empty(cap, dtype=torch.int32, device=dev) if csc else None
        self.cval = torch.empty(cap, dtype=torch.float32, device=dev) if csc else None
        self.plan = SplitPlan(cap, dev, order=True) if (csc and split) else None
        self.c = gcn_sparse_x(n, f, nnz, _ptr(self.row_ptr), _ptr(self.col), _ptr(self.val),
                              _ptr(self.col_ptr), _ptr(self.row), _ptr(self.cval),
                              self.plan.c if self.plan else gcn_split())

    @property
    def nnz(self):
        return self.c.nnz


# The sparse-path threshold tau measured on MI355X (Section IV-B: tau = 1 - gamma, gamma the
# sparse product's useful-work efficiency relative to the dense one): the training step's
# dense and sparse forms of the input-feature products cross at about 6.25 % density on
# this GPU (2^21 rows, 1024 and 4096 features, width 128), so tau = 15/16.  The paper's
# testbed gave about 0.8 (pass tau=(4, 5) for that).
TAU_MI355X = (15, 16)


def feature_stats(X: torch.Tensor, tau=TAU_MI355X, force_mode=-1, materialize=None, csc=True,
                  row_nnz: torch.Tensor | None = None, stream=None):
    """Density probe (+ X_csr / X_csc when materialize is True, or None -> by mode).

    Returns (info dict, SparseFeatures or None).  Blocking.
    """
    n, f = X.shape
    ld = _ld(X)
    info = gcn_feature_info()
    st = P(_stream(stream))
    _run_ws(_lib.gcn_feature_stats, (_ptr(X), n, f, ld, tau[0], tau[1], force_mode, _ptr(row_nnz),
                                     C.byref(info), None), (st,), "gcn_feature_stats", None, X.device)
    out = dict(nnz=info.nnz, sparsity=info.sparsity, mode=info.mode)
    want = (info.mode == SPARSE) if materialize is None else materialize
    if not want:
        return out, None
    sx = SparseFeatures(n, f, info.nnz, X.device, csc=csc)
    _run_ws(_lib.gcn_feature_stats, (_ptr(X), n, f, ld, tau[0], tau[1], force_mode, None,
                                     C.byref(info), C.byref(sx.c)), (st,), "gcn_feature_stats",
            None, X.device)
    return out, sx


# ---------------------------------------------------------------------------
# lower-level steps
# ---------------------------------------------------------------------------


def aggregate(g: DeviceGraph, M: torch.Tensor, out: torch.Tensor, bias=None, epi=EPI_NONE, mask=None,
              ws: _Workspace | None = None, stream=None, agg=AGG_NORM):
    w = M.shape[1]
    _run_ws(_lib.gcn_aggregate, (C.byref(g.c), agg, w, _ptr(M), _ld(M), _ptr(bias), epi, _ptr(mask),
                                 _ld(mask) if mask is not None else 0, _ptr(out), _ld(out)),
            (P(_stream(stream)),), "gcn_aggregate", ws, out.device)
    return out


def aggregate_max(g: DeviceGraph, M: torch.Tensor, out: torch.Tensor, arg: torch.Tensor, stream=None):
    """out = max over each row of A + I of M's rows, arg = the first maximiser (int32)."""
    w = M.shape[1]
    _run_ws(_lib.gcn_aggregate_max,
            (C.byref(g.c), w, _ptr(M), _ld(M), _ptr(out), _ld(out), _ptr(arg), _ld(arg)),
            (P(_stream(stream)),), "gcn_aggregate_max", None, M.device)
    return out


def aggregate_max_bwd(g: DeviceGraph, dP: torch.Tensor, arg: torch.Tensor, dM: torch.Tensor, mask=None,
                      stream=None):
    """dM[u] = sum over u's row of dP[v] where arg[v] == u (times 1[mask > 0])."""
    w = dP.shape[1]
    _run_ws(_lib.gcn_aggregate_max_bwd, (C.byref(g.c), w, _ptr(dP), _ld(dP), _ptr(arg), _ld(arg), _ptr(mask),
                                         _ld(mask) if mask is not None else 0, _ptr(dM), _ld(dM)),
            (P(_stream(stream)),), "gcn_aggregate_max_bwd", None, dP.device)
    return dM


def gemm(op, A, B, out, bias=None, epi=EPI_NONE, mask=None, ws: _Workspace | None = None, stream=None):
    if op == OP_NN:
        m, k = A.shape
        n = B.shape[1]
    elif op == OP_NT:
        m, k = A.shape
        n = B.shape[0]
    else:
        k, m = A.shape
        n = B.shape[1]
    _run_ws(_lib.gcn_gemm, (op, m, n, k, _ptr(A), _ld(A), _ptr(B), _ld(B), _ptr(out), _ld(out),
                            _ptr(bias), epi, _ptr(mask), _ld(mask) if mask is not None else 0),
            (P(_stream(stream)),), "gcn_gemm", ws, out.device)
    return out


def gemm_static(op, A, B, out, bias=None, epi=EPI_NONE, mask=None, stream=None):
    """gcn_gemm_static: gemm with the library's static device scratch (no workspace)."""
    if op == OP_NN:
        m, k = A.shape
        n = B.shape[1]
    elif op == OP_NT:
        m, k = A.shape
        n = B.shape[0]
    else:
        k, m = A.shape
        n = B.shape[1]
    _check(_lib.gcn_gemm_static(op, m, n, k, _ptr(A), _ld(A), _ptr(B), _ld(B), _ptr(out), _ld(out), _ptr(bias),
                                epi, _ptr(mask), _ld(mask) if mask is not None else 0, P(_stream(stream))),
           "gcn_gemm_static")
    return out


def spmm(ptr, idx, val, B, out, split: gcn_split | None = None, stream=None):
    nrows = ptr.numel() - 1
    _run_ws(_lib.gcn_spmm, (nrows, idx.numel(), _ptr(ptr), _ptr(idx), _ptr(val), B.shape[0], B.shape[1], _ptr(B),
                            _ld(B), _ptr(out), _ld(out), C.byref(split) if split is not None else None),
            (P(_stream(stream)),), "gcn_spmm", None, out.device)
    return out


def spmm_xt(sx: "SparseFeatures", B: torch.Tensor, out: torch.Tensor, stream=None):
    """out (f x w) = X^T B from the CSC view of sparse features sx (Algorithm 1, Backward)."""
    n, w = B.shape
    c = sx.c
    _run_ws(_lib.gcn_spmm_xt, (c.n, c.f, c.nnz, c.col_ptr, c.row, c.cval, C.byref(c.csc_split), _ptr(B), _ld(B), w,
                               _ptr(out), _ld(out)), (P(_stream(stream)),), "gcn_spmm_xt", None, out.device)
    return out


def spmm_xw(sx: "SparseFeatures", W: torch.Tensor, out: torch.Tensor, stream=None):
    """out (n x w) = X W from the CSR view of sparse features sx (Algorithm 1, Forward)."""
    f, w = W.shape
    c = sx.c
    _run_ws(_lib.gcn_spmm_xw, (c.n, c.f, c.nnz, c.row_ptr, c.col, c.val, _ptr(W), _ld(W), w, _ptr(out), _ld(out)),
            (P(_stream(stream)),), "gcn_spmm_xw", None, out.device)
    return out


def column_sums(G, out, row_vals=None, mean=None, stream=None):
    rows, w = G.shape
    _run_ws(_lib.gcn_column_sums, (rows, w, _ptr(G), _ld(G), _ptr(out), _ptr(row_vals), _ptr(mean)),
            (P(_stream(stream)),), "gcn_column_sums", None, G.device)
    return out


def _refuse(t, shape, what):
    raise ValueError(f"{what}: fp32 {shape} with contiguous columns on the device of the call needed, got {t.dtype} "
                     f"{tuple(t.shape)}, strides {t.stride()}, on {t.device}")


def _mat(t, rows, cols, dev, what):
    """Row pitch of an fp32 matrix of this shape on device `dev`; anything else is refused: the library
    sees an address only.  (A single row's stride says nothing: its pitch is at least its width.)"""
    if t.dtype is not torch.float32 or t.get_device() != dev or t.shape != (rows, cols):
        _refuse(t, (rows, cols), what)
    ld, unit = t.stride()
    if (cols > 1 and unit != 1) or (rows > 1 and ld < cols):
        if t.numel() == 0:  # strides of nothing
            return cols
        _refuse(t, (rows, cols), what)
    return ld if rows > 1 else max(ld, cols)


def _vec(t, n, dev, what):
    """Address of an fp32 vector of n contiguous elements on device `dev` (None stays None)."""
    if t is None:
        return None
    if t.dtype is not torch.float32 or t.get_device() != dev or t.shape != (n,) or (n > 1 and t.stride(0) != 1):
        _refuse(t, (n,), what)
    return t.data_ptr()


def _stat(t, rows, cols, dev, what):
    """Address of a contiguous fp32 matrix (a single row is, whatever it is a slice of)."""
    if _mat(t, rows, cols, dev, what) != cols and rows > 1 and t.numel():
        _refuse(t, (rows, cols), what)
    return t.data_ptr()


def _stat_in(t, rows, cols, dev, what, stream):
    """A statistic that is only read, as the library takes it: one whose rows or columns have gaps between
    them (a slice, a transposed result) is copied first, on the call's stream."""
    if t.dtype is torch.float32 and t.get_device() == dev and t.shape == (rows, cols) and not t.is_contiguous():
        down, across = t.stride()
        if (cols == 1 or across == 1) and (rows == 1 or down >= cols) or down == 1 and across >= rows:
            with torch.cuda.device(dev), torch.cuda.stream(stream):
                return t.contiguous()
    _stat(t, rows, cols, dev, what)
    return t


def _device_of(t):
    if t.dim() != 2 or not t.is_cuda:
        raise ValueError("a device matrix needed")
    return t.get_device()


def _call(fn, args, where, ws, dev, stream):
    """fn(*args, workspace, its size, stream) with device `dev` current, on `stream` or that device's
    current one.  A workspace kept in ws is tried first; its size is asked for only if it is too small."""
    if stream is not None and stream.device.index != dev:
        raise ValueError(f"{where}: a stream of the tensors' device needed")
    if dev != torch.cuda.current_device():
        with torch.cuda.device(dev):
            return _call(fn, args, where, ws, dev, stream)
    st = torch.cuda.current_stream().cuda_stream
    if stream is not None and stream.cuda_stream != st:
        with torch.cuda.stream(stream):
            return _call(fn, args, where, ws, dev, None)
    buf = ws.kept(0, dev, st, torch.cuda.is_current_stream_capturing()) if ws is not None else None
    if buf is not None:
        nbytes = sz(buf.numel())
        status = fn(*args, buf.data_ptr(), C.byref(nbytes), st)
        if status == OK:
            return
        if status != E_CAPACITY:
            _check(status, where)
    _run_ws(fn, args, (st,), where, ws, torch.device("cuda", dev))


def _segments(seg_ptr, dev):
    if seg_ptr is None:
        return 1, None
    if seg_ptr.dtype is not torch.int64 or seg_ptr.get_device() != dev or seg_ptr.dim() != 1 \
            or seg_ptr.shape[0] < 1 or (seg_ptr.shape[0] > 1 and seg_ptr.stride(0) != 1):
        raise ValueError("seg_ptr: contiguous int64 offsets on the device of the call needed")
    return seg_ptr.shape[0] - 1, seg_ptr.data_ptr()


def group_norm(X, groups, gamma, beta, out, mean, rstd, seg_ptr=None, max_seg=-1, eps=1e-5, act=ACT_NONE,
               ws: _Workspace | None = None, stream=None):
    """out = act(gamma (X - mean) rstd + beta) per graph and channel group (gcn_group_norm_fwd).

    X, out: n x c (out may be X).  seg_ptr: int64 device offsets of the batch's graphs (None: one
    graph); mean, rstd: (graphs, groups), written for group_norm_bwd.  gamma, beta may be None.
    max_seg: rows of the longest graph, where the program knows it: without it (-1) a batch of small
    graphs takes up to twice as long, here and in group_norm_bwd."""
    dev = _device_of(X)
    n, c = X.shape
    k, seg = _segments(seg_ptr, dev)
    _call(_lib.gcn_group_norm_fwd,
          (n, c, groups, k, seg, max_seg, X.data_ptr(), _mat(X, n, c, dev, "X"), _vec(gamma, c, dev, "gamma"),
           _vec(beta, c, dev, "beta"), eps, act, out.data_ptr(), _mat(out, n, c, dev, "out"),
           _stat(mean, k, groups, dev, "mean"), _stat(rstd, k, groups, dev, "rstd")),
          "gcn_group_norm_fwd", ws, dev, stream)
    return out


def group_norm_bwd(X, dY, mean, rstd, groups, gamma, beta, dX=None, dgamma=None, dbeta=None, seg_ptr=None,
                   max_seg=-1, act=ACT_NONE, ws: _Workspace | None = None, stream=None):
    """Gradients of group_norm from dY = dLoss/dout, with the mean and rstd it wrote
    (gcn_group_norm_bwd): dX (may be dY), dgamma, dbeta; each may be None.  mean and rstd may have
    rows or columns apart (slices, transposed results): such a one is copied first.  max_seg as there."""
    dev = _device_of(X)
    n, c = X.shape
    k, seg = _segments(seg_ptr, dev)
    mean = _stat_in(mean, k, groups, dev, "mean", stream)
    rstd = _stat_in(rstd, k, groups, dev, "rstd", stream)
    _call(_lib.gcn_group_norm_bwd,
          (n, c, groups, k, seg, max_seg, X.data_ptr(), _mat(X, n, c, dev, "X"), _vec(gamma, c, dev, "gamma"),
           _vec(beta, c, dev, "beta"), act, mean.data_ptr(), rstd.data_ptr(),
           dY.data_ptr(), _mat(dY, n, c, dev, "dY"), _ptr(dX), _mat(dX, n, c, dev, "dX") if dX is not None else 0,
           _vec(dgamma, c, dev, "dgamma"), _vec(dbeta, c, dev, "dbeta")),
          "gcn_group_norm_bwd", ws, dev, stream)
    return dX


def adam(params, grads, ms, vs, step, lr=0.01, b1=0.9, b2=0.999, eps=1e-8, stream=None):
    arr = (gcn_adam_tensor * len(params))()
    for i, (p, g, m, v) in enumerate(zip(params, grads, ms, vs)):
        arr[i] = gcn_adam_tensor(_ptr(p), _ptr(g), _ptr(m), _ptr(v), p.numel())
    _check(_lib.gcn_adam(arr, len(params), step, lr, b1, b2, eps, P(_stream(stream))), "gcn_adam")


def orthogonalize(A, out, steps=5, ws: _Workspace | None = None, stream=None):
    """out = A with its singular values drawn towards 1 by `steps` Newton-Schulz products
    (gcn_orthogonalize); out may be A."""
    dev = _device_of(A)
    rows, cols = A.shape
    _call(_lib.gcn_orthogonalize, (rows, cols, A.data_ptr(), _mat(A, rows, cols, dev, "A"), steps, out.data_ptr(),
                                   _mat(out, rows, cols, dev, "out")), "gcn_orthogonalize", ws, dev, stream)
    return out


def muon(params, grads, ms, lr=0.02, momentum=0.95, nesterov=True, weight_decay=0.0, steps=5, scales=None,
         ws: _Workspace | None = None, stream=None):
    """One optimiser step with orthogonalised updates over weight matrices, in place (gcn_muon);
    ms: momentum buffers (zero at first).  scales: what multiplies lr for each matrix, by default
    sqrt(max(1, cols / rows)), the root of a layer's fan-out over its fan-in.  Any number of matrices: 16 share
    the launches of a call, and all are checked before the first."""
    if not params:
        return
    if not len(params) == len(grads) == len(ms) or (scales is not None and len(scales) != len(params)):
        raise ValueError("params, grads, ms and scales: one of each per matrix")
    dev = _device_of(params[0])
    arr = (gcn_muon_tensor * len(params))()
    for i, (p, g, m) in enumerate(zip(params, grads, ms)):
        if p.dim() != 2:
            raise ValueError("muon takes matrices; vectors go through adam")
        rows, cols = p.shape
        t = arr[i]
        t.param = _stat(p, rows, cols, dev, "param")
        t.grad = _stat(g, rows, cols, dev, "grad")
        t.m = _stat(m, rows, cols, dev, "m")
        t.rows, t.cols = rows, cols
        t.scale = scales[i] if scales is not None else max(1.0, cols / max(rows, 1)) ** 0.5
    how = (steps, lr, momentum, int(nesterov), weight_decay)
    size = C.sizeof(gcn_muon_tensor)
    calls = [((gcn_muon_tensor * min(MUON_MAX, len(arr) - i)).from_buffer(arr, i * size), min(MUON_MAX, len(arr) - i))
             for i in range(0, len(arr), MUON_MAX)]
    if len(calls) > 1:
        used = [t for t in arr if t.rows * t.cols]
        written = [a for t in used for a in (t.param, t.m)]
        if len(set(written)) < len(written) or not set(written).isdisjoint(t.grad for t in used):
            raise ValueError("muon: a buffer that is written is given twice")
        for some in calls:
            _check(_lib.gcn_muon(*some, *how, None, C.byref(sz(0)), None), "gcn_muon (size query)")
    for some in calls:
        _call(_lib.gcn_muon, (*some, *how), "gcn_muon", ws, dev, stream)


def layer_order(f_in, f_out, index, act, x_sparse=False, order=ORDER_AUTO, agg=AGG_NORM):
    L = gcn_layer(f_in, f_out, pitch(f_in), pitch(f_out), act, order, index, agg)
    return _lib.gcn_layer_order(C.byref(L), int(x_sparse))


def make_layer(f_in, f_out, ld_in, ld_out, act, index, order=ORDER_AUTO, agg=AGG_NORM):
    return gcn_layer(f_in, f_out, ld_in, ld_out, act, order, index, agg)


def saved_buffer(n, f_in, ld_in, agg, device="cuda"):
    """The d_saved buffer of an aggregate-first layer: n x f_in (pitch ld_in) fp32, and for a
    max layer the n x ld_in int32 maximisers after it.  Returns (buffer view, argmax view)."""
    rows = 2 * n if agg == AGG_MAX else n
    buf = torch.zeros((rows, ld_in), dtype=torch.float32, device=device)
    arg = buf[n:].view(torch.int32)[:, :f_in] if agg == AGG_MAX else None
    return buf[:n, :f_in], arg


def layer_fwd(g: DeviceGraph, L: gcn_layer, Hin, x: SparseFeatures | None, W, b, Hout, saved=None,
              labels=None, loss=None, logits=None, ws: _Workspace | None = None, stream=None):
    dev = W.device
    return _run_ws(_lib.gcn_layer_fwd,
                   (C.byref(g.c), C.byref(L), _ptr(Hin), C.byref(x.c) if x is not None else None,
                    _ptr(W), _ptr(b), _ptr(Hout), _ptr(saved), _ptr(labels), _ptr(loss), _ptr(logits)),
                   (P(_stream(stream)),), "gcn_layer_fwd", ws, dev)


def layer_bwd(g: DeviceGraph, L: gcn_layer, G, Hin, x: SparseFeatures | None, saved, W, dW, db,
              Gprev=None, ws: _Workspace | None = None, stream=None):
    dev = W.device
    return _run_ws(_lib.gcn_layer_bwd,
                   (C.byref(g.c), C.byref(L), _ptr(G), _ptr(Hin), C.byref(x.c) if x is not None else None,
                    _ptr(saved), _ptr(W), _ptr(dW), _ptr(db), _ptr(Gprev)),
                   (P(_stream(stream)),), "gcn_layer_bwd", ws, dev)


# ---------------------------------------------------------------------------
# whole model
# ---------------------------------------------------------------------------


class Model:
    """Parameters, Adam state and activation buffers of an L-layer GCN on the device.

    widths = (F, hidden..., classes).  Ws / bs: host arrays (fp32) of the initial
    parameters.  x_sparse: layer 0 reads sparse X (its order is then transform-first).
    """

    def __init__(self, n, widths, Ws, bs, device="cuda", x_sparse=False, ld_x=None, lr=0.01,
                 beta1=0.9, beta2=0.999, eps=1e-8, orders=None, device_step=False, aggs=None):
        self.n = n
        self.widths = tuple(widths)
        L = len(widths) - 1
        self.L = L
        self.x_sparse = bool(x_sparse)
        dev = torch.device(device)
        self.layers = (gcn_layer * L)()
        self.W, self.b, self.dW, self.db, self.mW, self.vW, self.mb, self.vb = ([] for _ in range(8))
        self.act, self.saved, self.grad = [], [], []
        for l in range(L):
            fi, fo = widths[l], widths[l + 1]
            ld_in = (ld_x if ld_x is not None else fi) if l == 0 else pitch(fi)
            ld_out = pitch(fo)
            act = ACT_SOFTMAX_CE if l == L - 1 else ACT_RELU
            order = orders[l] if orders is not None else ORDER_AUTO
            agg = aggs[l] if aggs is not None else AGG_NORM
            self.layers[l] = gcn_layer(fi, fo, ld_in, ld_out, act, order, l, agg)
            self.W.append(torch.as_tensor(Ws[l], dtype=torch.float32).to(dev).contiguous())
            self.b.append(torch.as_tensor(bs[l], dtype=torch.float32).to(dev).contiguous())
            self.dW.append(torch.zeros_like(self.W[-1]))
            self.db.append(torch.zeros_like(self.b[-1]))
            self.mW.append(torch.zeros_like(self.W[-1]))
            self.vW.append(torch.zeros_like(self.W[-1]))
            self.mb.append(torch.zeros_like(self.b[-1]))
            self.vb.append(torch.zeros_like(self.b[-1]))
            self.grad.append(padded(n, fo, dev))
            if l < L - 1:
                self.act.append(padded(n, fo, dev))
            resolved = _lib.gcn_layer_order(C.byref(self.layers[l]), int(x_sparse and l == 0))
            if resolved == AGGREGATE_FIRST:
                self.saved.append(saved_buffer(n, fi, ld_in, agg, dev)[0])
            else:
                self.saved.append(None)
        self.loss = torch.zeros(1, dtype=torch.float32, device=dev)
        self._ws = _Workspace()

        def arr(ts):
            a = (P * L)()
            for i, t in enumerate(ts):
                a[i] = _ptr(t) if t is not None else None
            return a

        acts = self.act + [None]
        self._arrays = dict(W=arr(self.W), b=arr(self.b), dW=arr(self.dW), db=arr(self.db),
                            mW=arr(self.mW), vW=arr(self.vW), mb=arr(self.mb), vb=arr(self.vb),
                            act=arr(acts), saved=arr(self.saved), grad=arr(self.grad))
        self.c = gcn_model()
        self.c.n_layers = L
        self.c.layers = self.layers
        for k, v in self._arrays.items():
            setattr(self.c, k, C.cast(v, C.POINTER(P)))
        self.c.lr, self.c.beta1, self.c.beta2, self.c.eps, self.c.step = lr, beta1, beta2, eps, 0
        self.d_step = torch.zeros(1, dtype=torch.int32, device=dev) if device_step else None
        self.c.d_step = _ptr(self.d_step)

    @property
    def step(self):
        return int(self.d_step.item()) if self.d_step is not None else self.c.step

    def prepare(self, g: DeviceGraph, X=None, x: SparseFeatures | None = None, labels=None):
        """Allocate the epoch workspace ahead of time (nothing may allocate during graph capture)."""
        nbytes = sz(0)
        _check(_lib.gcn_epoch(C.byref(self.c), C.byref(g.c), _ptr(X), C.byref(x.c) if x is not None else None,
                              _ptr(labels), _ptr(self.loss), None, C.byref(nbytes), None), "gcn_epoch (size query)")
        self._ws.get(max(nbytes.value, 256), self.loss.device)

    def epoch_captured(self, g: DeviceGraph, X=None, x: SparseFeatures | None = None, labels=None):
        """Enqueue one epoch with the prepared workspace and no allocation (for HIP graph capture)."""
        buf = self._ws.buf
        self._ws.hold()
        nbytes = sz(buf.numel())
        _check(_lib.gcn_epoch(C.byref(self.c), C.byref(g.c), _ptr(X), C.byref(x.c) if x is not None else None,
                              _ptr(labels), _ptr(self.loss), buf.data_ptr(), C.byref(nbytes),
                              P(_stream(None))), "gcn_epoch")
        return self.loss

    def orders(self):
        return [_lib.gcn_layer_order(C.byref(self.layers[l]), int(self.x_sparse and l == 0))
                for l in range(self.L)]

    def epoch(self, g: DeviceGraph, X=None, x: SparseFeatures | None = None, labels=None, stream=None):
        """One training epoch (asynchronous); returns the device loss tensor."""
        _run_ws(_lib.gcn_epoch, (C.byref(self.c), C.byref(g.c), _ptr(X),
                                 C.byref(x.c) if x is not None else None, _ptr(labels), _ptr(self.loss)),
                (P(_stream(stream)),), "gcn_epoch", self._ws, self.loss.device)
        return self.loss


# ---------------------------------------------------------------------------
# kernel timing
# ---------------------------------------------------------------------------


def profile_enable(capacity: int):
    _check(_lib.gcn_profile_enable(capacity), "gcn_profile_enable")


def profile_records():
    out = []
    for i in range(_lib.gcn_profile_count()):
        r = gcn_profile_record()
        _check(_lib.gcn_profile_read(i, C.byref(r)), "gcn_profile_read")
        out.append(dict(name=r.name.decode(), width=r.width, rows=r.rows, nnz=r.nnz, ms=r.ms))
    return out


def profile_reset():
    _check(_lib.gcn_profile_reset(), "gcn_profile_reset")


def profile_only(name=None):
    """Record only launches of the kernel family `name` (None: every launch)."""
    _check(_lib.gcn_profile_only(None if name is None else name.encode()), "gcn_profile_only")


def raw_lib():
    """The loaded ctypes library (for ABI tests)."""
    return _lib
