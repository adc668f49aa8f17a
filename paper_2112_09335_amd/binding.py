"""ctypes binding over the C ABI in include/cadmm.h: argument marshalling only.

Every step of the ADMM sweep runs inside libcadmm.so (HIP, gfx950).  PyTorch is used
for one thing: it allocates the device workspace and owns the stream the library
enqueues on.  If the library has not been built this module raises; there is no
CPU fallback.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import List, Optional

import numpy as np

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libcadmm.so")
_lib = None

EXPORTS = [
    "cadmm_create", "cadmm_destroy", "cadmm_last_error", "cadmm_build_graph", "cadmm_graph_sizes",
    "cadmm_get_graph", "cadmm_get_segment_order", "cadmm_set_model", "cadmm_workspace_bytes",
    "cadmm_set_workspace", "cadmm_set_data", "cadmm_init", "cadmm_run", "cadmm_eval", "cadmm_get_W",
    "cadmm_get_Z", "cadmm_get_U", "cadmm_get_steps", "cadmm_set_state", "cadmm_op_aggregate",
    "cadmm_op_aggregate_segments", "cadmm_op_transform", "cadmm_op_wgrad",
    "cadmm_profile", "cadmm_get_profile", "cadmm_profile_class_name", "cadmm_tune", "cadmm_predict",
    "cadmm_partition", "cadmm_op_calibrate", "cadmm_op_wgrad_noalloc", "cadmm_get_fista", "cadmm_op_stream",
    "cadmm_op_transform_grouped", "cadmm_op_wgrad_grouped_scratch", "cadmm_op_wgrad_grouped",
    "cadmm_op_orthogonalise_scratch", "cadmm_op_orthogonalise", "cadmm_op_muon_step",
]
PROFILE_CLASSES = 19


class CadmmError(RuntimeError):
    pass


class _Model(C.Structure):
    _fields_ = [("L", C.c_int32), ("C", C.POINTER(C.c_int32)), ("risk", C.c_int32),
                ("nu", C.c_float), ("rho", C.c_float), ("tau0", C.c_float), ("theta0", C.c_float),
                ("eta", C.c_float), ("max_backtrack", C.c_int32), ("fista_iters", C.c_int32),
                ("dual_form", C.c_int32), ("schedule", C.c_int32), ("step_policy", C.c_int32),
                ("fista_mode", C.c_int32)]


class _Stats(C.Structure):
    _fields_ = [("objective", C.c_double), ("lagrangian", C.c_double), ("risk", C.c_double),
                ("primal_res", C.c_double), ("dual_res", C.c_double), ("iter", C.c_int32),
                ("status", C.c_int32)]


def load_library():
    """dlopen libcadmm.so and check that every declared entry point is exported."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise CadmmError(f"{_LIB_PATH} is missing: run `python __graft_entry__.py` (build) first; "
                         "there is no fallback path")
    # PyTorch ships its own copy of the HIP runtime.  Load it first so that this library binds to the
    # same runtime instance: two HIP runtimes in one process do not both see the GPU.
    import torch  # noqa: F401
    lib = C.CDLL(_LIB_PATH)
    for name in EXPORTS:
        if not hasattr(lib, name):
            raise CadmmError(f"libcadmm.so does not export {name}")
    lib.cadmm_last_error.restype = C.c_char_p
    lib.cadmm_last_error.argtypes = [C.c_void_p]
    lib.cadmm_destroy.restype = None
    lib.cadmm_destroy.argtypes = [C.c_void_p]
    vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
    lib.cadmm_create.argtypes = [C.POINTER(vp), C.c_int, vp]
    lib.cadmm_build_graph.argtypes = [vp, i64, i64, vp, vp, i32, vp]
    lib.cadmm_partition.argtypes = [vp, i64, i64, vp, vp, i32, vp]
    lib.cadmm_graph_sizes.argtypes = [vp, C.POINTER(i64), C.POINTER(i64), C.POINTER(i64)]
    lib.cadmm_get_graph.argtypes = [vp] * 10
    lib.cadmm_get_segment_order.argtypes = [vp, vp]
    lib.cadmm_set_model.argtypes = [vp, C.POINTER(_Model)]
    lib.cadmm_workspace_bytes.argtypes = [vp, C.POINTER(C.c_size_t)]
    lib.cadmm_set_workspace.argtypes = [vp, vp, C.c_size_t]
    lib.cadmm_set_data.argtypes = [vp, vp, vp, C.c_int]
    lib.cadmm_init.argtypes = [vp, vp]
    lib.cadmm_run.argtypes = [vp, i32]
    lib.cadmm_eval.argtypes = [vp, C.POINTER(_Stats), vp]
    lib.cadmm_get_W.argtypes = [vp, i32, vp]
    lib.cadmm_get_Z.argtypes = [vp, i32, vp]
    lib.cadmm_get_U.argtypes = [vp, vp]
    lib.cadmm_get_steps.argtypes = [vp, vp, vp, vp, vp]
    lib.cadmm_set_state.argtypes = [vp, vp, vp, vp, vp, vp]
    lib.cadmm_get_fista.argtypes = [vp, vp, vp]
    lib.cadmm_op_aggregate.argtypes = [vp, vp, i32, vp]
    lib.cadmm_op_aggregate_segments.argtypes = [vp, vp, i32, vp]
    lib.cadmm_op_transform.argtypes = [vp, vp, i64, i32, vp, i32, vp]
    lib.cadmm_op_wgrad.argtypes = [vp, vp, vp, i64, i32, i32, vp]
    lib.cadmm_op_wgrad_noalloc.argtypes = [vp, vp, vp, i64, i32, i32, vp]
    lib.cadmm_op_stream.argtypes = [vp, vp]
    f32, sizep = C.c_float, C.POINTER(C.c_size_t)
    lib.cadmm_op_transform_grouped.argtypes = [vp, i32, vp, i64, i64, i32, vp, i32, i32, i32, vp, vp, i64]
    lib.cadmm_op_wgrad_grouped_scratch.argtypes = [vp, i64, i32, i32, i32, sizep]
    lib.cadmm_op_wgrad_grouped.argtypes = [vp, i32, vp, i64, i64, i32, vp, i64, i32, i32, vp, i32, vp, vp, C.c_size_t]
    lib.cadmm_op_orthogonalise_scratch.argtypes = [vp, i32, i32, i32, sizep]
    lib.cadmm_op_orthogonalise.argtypes = [vp, i32, vp, i32, i32, i32, i32, vp, f32, vp, vp, C.c_size_t]
    lib.cadmm_op_muon_step.argtypes = [vp, i32, vp, vp, vp, i32, i32, i32, f32, f32, i32, f32, f32, i32, vp, f32, vp, C.c_size_t]
    lib.cadmm_op_calibrate.argtypes = [vp, i32, vp, vp, i64, i32, C.POINTER(C.c_double)]
    lib.cadmm_tune.argtypes = [vp, C.c_char_p, i32]
    lib.cadmm_predict.argtypes = [vp, vp, vp, C.POINTER(C.c_double)]
    lib.cadmm_profile.argtypes = [vp, C.c_int]
    lib.cadmm_get_profile.argtypes = [vp, vp, vp, vp, vp]
    lib.cadmm_profile_class_name.argtypes = [i32]
    lib.cadmm_profile_class_name.restype = C.c_char_p
    _lib = lib
    return lib


def _ptr(a: Optional[np.ndarray]):
    return None if a is None else a.ctypes.data_as(C.c_void_p)


def _ptr_array(arrs):
    """Array of L host pointers (None entries stay null)."""
    out = (C.c_void_p * len(arrs))()
    for i, a in enumerate(arrs):
        out[i] = None if a is None else a.ctypes.data
    return out


def _rows_meet(p, q):
    """Whether two sets of rows share a byte.  A set: (address, rows, bytes from one row to the next, bytes of a row); its own rows
    are apart."""
    (a, n, step, width), (b, m, other, wide) = p, q
    if n == 0 or m == 0 or a + (n - 1) * step + width <= b or b + (m - 1) * other + wide <= a:
        return False
    if n == 1 or step == width:                               # one stretch: the other's first row that ends behind its beginning
        end, j = a + (n - 1) * step + width, max(0, (a - wide - b) // max(other, 1) + 1) if m > 1 else 0
        return j < m and b + j * other < end
    if m == 1 or other == wide:
        return _rows_meet(q, p)
    if step == other:                                         # row j of q lies at b - a + (j - i) step from row i of p
        k = max((a - b - wide) // step + 1, 1 - n)
        return k < m and b - a + k * step < width
    if n > m:
        return _rows_meet(q, p)
    for i in range(0, n, 1 << 20):                            # every row of p against q's first row that ends behind its beginning
        at = a + step * np.arange(i, min(i + (1 << 20), n), dtype=np.int64)
        j = np.maximum((at - wide - b) // other + 1, 0)
        if ((j < m) & (b + j * other < at + width)).any():
            return True
    return False


class Solver:
    """One problem instance on one GPU.  Method names mirror the C entry points."""

    def __init__(self, device: int = 0):
        self.lib = load_library()
        self.device = device
        self._types, self._gpu = None, f"cuda:{device}"
        stream_handle = None
        if device >= 0:
            import torch
            if not torch.cuda.is_available():
                raise CadmmError("no GPU visible: the HIP path cannot run (there is no CPU fallback)")
            self._torch = torch
            torch.cuda.set_device(device)
            # a stream of its own (default priority): the library can then replay an iteration as a HIP graph
            self.stream = torch.cuda.Stream(device=device)
            stream_handle = self.stream.cuda_stream
        h = C.c_void_p()
        rc = self.lib.cadmm_create(C.byref(h), device, C.c_void_p(stream_handle))
        if rc != 0:
            raise CadmmError(f"cadmm_create failed ({rc})")
        self.h = h
        self.workspace = None
        self.N = self.M = self.L = 0
        self.dims: List[int] = []

    def close(self):
        if getattr(self, "h", None):
            self.lib.cadmm_destroy(self.h)
            self.h = None
            self.workspace = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc, what):
        if rc != 0:
            msg = self.lib.cadmm_last_error(self.h)
            raise CadmmError(f"{what} failed ({rc}): {msg.decode() if msg else ''}")

    # ---- graph
    def partition(self, N, src, dst, M):
        """Communities for a graph without them: int32 [N] in [0, M) (host work, any context)."""
        src = np.ascontiguousarray(src, dtype=np.int32)
        dst = np.ascontiguousarray(dst, dtype=np.int32)
        if src.shape != dst.shape:
            raise CadmmError("edge array size mismatch")
        comm = np.empty(int(N), np.int32)
        self._check(self.lib.cadmm_partition(self.h, N, src.shape[0], _ptr(src), _ptr(dst), M, _ptr(comm)),
                    "cadmm_partition")
        return comm

    def build_graph(self, N, src, dst, M, comm=None):
        src = np.ascontiguousarray(src, dtype=np.int32)
        dst = np.ascontiguousarray(dst, dtype=np.int32)
        comm = None if comm is None else np.ascontiguousarray(comm, dtype=np.int32)
        if src.shape != dst.shape or (comm is not None and comm.shape[0] != N):
            raise CadmmError("edge / community array size mismatch")
        self._check(self.lib.cadmm_build_graph(self.h, N, src.shape[0], _ptr(src), _ptr(dst), M, _ptr(comm)),
                    "cadmm_build_graph")
        self.N, self.M = int(N), int(M)

    def graph_sizes(self):
        a, b, c = C.c_int64(), C.c_int64(), C.c_int64()
        self._check(self.lib.cadmm_graph_sizes(self.h, C.byref(a), C.byref(b), C.byref(c)), "cadmm_graph_sizes")
        return int(a.value), int(b.value), int(c.value)

    def get_graph(self):
        nnz, nseg, _ = self.graph_sizes()
        N, M = self.N, self.M
        out = dict(perm=np.empty(N, np.int32), row_ptr=np.empty(N + 1, np.int64), col=np.empty(nnz, np.int32),
                   val=np.empty(nnz, np.float32), seg_ptr=np.empty(nseg + 1, np.int64),
                   seg_row=np.empty(nseg, np.int32), seg_comm=np.empty(nseg, np.int32),
                   comm_row_ptr=np.empty(M + 1, np.int64), neighbour=np.empty(M * M, np.uint8))
        self._check(self.lib.cadmm_get_graph(self.h, *[_ptr(out[k]) for k in
                                                       ("perm", "row_ptr", "col", "val", "seg_ptr", "seg_row",
                                                        "seg_comm", "comm_row_ptr", "neighbour")]), "cadmm_get_graph")
        out["neighbour"] = out["neighbour"].reshape(M, M).astype(bool)
        return out

    def get_segment_order(self):
        _, nseg, _ = self.graph_sizes()
        order = np.empty(nseg, np.int64)
        self._check(self.lib.cadmm_get_segment_order(self.h, _ptr(order)), "cadmm_get_segment_order")
        return order

    # ---- model / workspace / data
    def set_model(self, dims, *, nu, rho, tau0, theta0, eta, max_backtrack, fista_iters, risk=0, dual_form=0,
                  schedule=0, step_policy=0, fista_mode=0):
        self.dims = [int(d) for d in dims]
        self.L = len(self.dims) - 1
        arr = (C.c_int32 * len(self.dims))(*self.dims)
        m = _Model(self.L, arr, risk, nu, rho, tau0, theta0, eta, max_backtrack, fista_iters, dual_form, schedule,
                   step_policy, fista_mode)
        self._check(self.lib.cadmm_set_model(self.h, C.byref(m)), "cadmm_set_model")

    def workspace_bytes(self):
        b = C.c_size_t()
        self._check(self.lib.cadmm_workspace_bytes(self.h, C.byref(b)), "cadmm_workspace_bytes")
        return int(b.value)

    def set_workspace(self):
        torch = self._torch
        nbytes = self.workspace_bytes()
        self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=f"cuda:{self.device}")
        base = self.workspace.data_ptr()
        aligned = (base + 255) & ~255
        self._check(self.lib.cadmm_set_workspace(self.h, C.c_void_p(aligned), nbytes), "cadmm_set_workspace")
        return nbytes

    def set_data(self, X, labels):
        X = np.ascontiguousarray(X, dtype=np.float32)
        labels = np.ascontiguousarray(labels, dtype=np.int32)
        if X.shape != (self.N, self.dims[0]) or labels.shape != (self.N,):
            raise CadmmError("X / labels shape mismatch")
        self._check(self.lib.cadmm_set_data(self.h, _ptr(X), _ptr(labels), 0), "cadmm_set_data")

    def init(self, W0):
        W0 = [np.ascontiguousarray(w, dtype=np.float32) for w in W0]
        for l, w in enumerate(W0, 1):
            if w.shape != (self.dims[l - 1], self.dims[l]):
                raise CadmmError("W0 shape mismatch")
        self._check(self.lib.cadmm_init(self.h, _ptr_array(W0)), "cadmm_init")

    # ---- iterate / read
    def run(self, k=1):
        self._check(self.lib.cadmm_run(self.h, k), "cadmm_run")

    def eval(self):
        st = _Stats()
        pen = np.zeros(max(self.L - 1, 1), np.float64)
        self._check(self.lib.cadmm_eval(self.h, C.byref(st), _ptr(pen)), "cadmm_eval")
        return dict(objective=st.objective, lagrangian=st.lagrangian, risk=st.risk, primal_res=st.primal_res,
                    dual_res=st.dual_res, iter=st.iter, status=st.status, layer_penalty=list(pen[:self.L - 1]))

    def predict(self):
        """(classes [N], logits [N, C_L], accuracy over labelled nodes) with the current weights."""
        pred = np.empty(self.N, np.int32)
        logits = np.empty((self.N, self.dims[-1]), np.float32)
        acc = C.c_double()
        self._check(self.lib.cadmm_predict(self.h, _ptr(pred), _ptr(logits), C.byref(acc)), "cadmm_predict")
        return pred, logits, float(acc.value)

    def get_W(self, l):
        out = np.empty((self.dims[l - 1], self.dims[l]), np.float32)
        self._check(self.lib.cadmm_get_W(self.h, l, _ptr(out)), "cadmm_get_W")
        return out

    def get_Z(self, l):
        out = np.empty((self.N, self.dims[l]), np.float32)
        self._check(self.lib.cadmm_get_Z(self.h, l, _ptr(out)), "cadmm_get_Z")
        return out

    def get_U(self):
        out = np.empty((self.N, self.dims[-1]), np.float32)
        self._check(self.lib.cadmm_get_U(self.h, _ptr(out)), "cadmm_get_U")
        return out

    def get_steps(self):
        nz = (self.L - 1) * self.M
        tau = np.empty(self.L, np.float64)
        theta = np.empty(nz, np.float64)
        trials = np.empty(self.L + nz, np.int32)
        sq = np.empty(self.L + nz, np.float64)
        self._check(self.lib.cadmm_get_steps(self.h, _ptr(tau), _ptr(theta), _ptr(trials), _ptr(sq)),
                    "cadmm_get_steps")
        return tau, theta, trials, sq

    def get_fista(self):
        """(L [M], candidates tested [M]) of the last solve of Z_L with backtracking (fista_mode 1)."""
        L = np.empty(self.M, np.float64)
        trials = np.empty(self.M, np.int32)
        self._check(self.lib.cadmm_get_fista(self.h, _ptr(L), _ptr(trials)), "cadmm_get_fista")
        return L, trials

    def set_state(self, W=None, Z=None, U=None, tau=None, theta=None):
        keep = []

        def prep(lst):
            if lst is None:
                return None
            arrs = [None if a is None else np.ascontiguousarray(a, dtype=np.float32) for a in lst]
            keep.append(arrs)
            return _ptr_array(arrs)
        Wp, Zp = prep(W), prep(Z)
        U = None if U is None else np.ascontiguousarray(U, dtype=np.float32)
        tau = None if tau is None else np.ascontiguousarray(tau, dtype=np.float64)
        theta = None if theta is None else np.ascontiguousarray(theta, dtype=np.float64)
        self._check(self.lib.cadmm_set_state(self.h, Wp, Zp, _ptr(U), _ptr(tau), _ptr(theta)), "cadmm_set_state")

    # ---- kernel-level calls on torch device tensors (internal row order)
    def _enter(self):
        """Tensors come from torch's current stream; the library runs on its own."""
        self.stream.wait_stream(self._torch.cuda.current_stream(self.device))

    def _leave(self):
        self._torch.cuda.current_stream(self.device).wait_stream(self.stream)

    def _on_current_stream(self):
        """Kernel-level calls are launched on torch's current stream, in order with the library's own."""
        self.lib.cadmm_op_stream(self.h, self._torch.cuda.current_stream(self.device).cuda_stream)

    def op_aggregate(self, X):
        torch = self._torch
        assert X.is_cuda and X.dtype == torch.float32 and X.is_contiguous() and X.shape[0] == self.N
        Y = torch.empty_like(X)
        self._on_current_stream()
        self._check(self.lib.cadmm_op_aggregate(self.h, X.data_ptr(), X.shape[1], Y.data_ptr()), "cadmm_op_aggregate")
        return Y

    def op_aggregate_segments(self, V):
        torch = self._torch
        assert V.is_cuda and V.dtype == torch.float32 and V.is_contiguous() and V.shape[0] == self.N
        nseg = self.graph_sizes()[1]
        P = torch.empty((nseg, V.shape[1]), dtype=torch.float32, device=V.device)
        self._on_current_stream()
        self._check(self.lib.cadmm_op_aggregate_segments(self.h, V.data_ptr(), V.shape[1], P.data_ptr()),
                    "cadmm_op_aggregate_segments")
        return P

    def op_transform(self, A, B):
        torch = self._torch
        assert A.is_cuda and B.is_cuda and A.is_contiguous() and B.is_contiguous() and A.shape[1] == B.shape[0]
        out = torch.empty((A.shape[0], B.shape[1]), dtype=torch.float32, device=A.device)
        self._on_current_stream()
        self._check(self.lib.cadmm_op_transform(self.h, A.data_ptr(), A.shape[0], A.shape[1], B.data_ptr(), B.shape[1],
                                                out.data_ptr()), "cadmm_op_transform")
        return out

    def op_calibrate(self, kind, count, reps=5):
        """'copy': GB/s of a plain device copy of `count` floats; 'update': GB/s of dst = 0.999 dst + src in place; 'mfma': TFLOP/s of register-only fp32 MFMA chains;
        'mfma_bf16': the same with bf16 MFMAs, 'mfma_bf16_valu4/6/8': with that many vector instructions after each;
        'gather' / 'gather_segments': GB/s of the aggregation's gathers alone at a row width of `count` floats."""
        torch = self._torch
        rate = C.c_double()
        self._enter()
        if kind in ("copy", "update"):
            src = torch.ones(count, dtype=torch.float32, device=f"cuda:{self.device}")
            dst = torch.zeros_like(src)
            torch.cuda.current_stream().synchronize()
            rc = self.lib.cadmm_op_calibrate(self.h, 0 if kind == "copy" else 8, C.c_void_p(src.data_ptr()),
                                             C.c_void_p(dst.data_ptr()), count, reps, C.byref(rate))
        elif kind == "mfma":
            dst = torch.empty(2048 * 256, dtype=torch.float32, device=f"cuda:{self.device}")
            rc = self.lib.cadmm_op_calibrate(self.h, 1, None, C.c_void_p(dst.data_ptr()), count, reps, C.byref(rate))
        elif kind in ("mfma_bf16", "mfma_bf16_valu4", "mfma_bf16_valu6", "mfma_bf16_valu8"):
            dst = torch.empty(2048 * 256, dtype=torch.float32, device=f"cuda:{self.device}")
            code = {"mfma_bf16": 4, "mfma_bf16_valu4": 5, "mfma_bf16_valu6": 6, "mfma_bf16_valu8": 7}[kind]
            rc = self.lib.cadmm_op_calibrate(self.h, code, None, C.c_void_p(dst.data_ptr()), count, reps, C.byref(rate))
        elif kind in ("gather", "gather_segments"):
            src = torch.randn(self.N, count, dtype=torch.float32, device=f"cuda:{self.device}")
            dst = torch.empty(2048 * 256, dtype=torch.float32, device=f"cuda:{self.device}")
            torch.cuda.current_stream().synchronize()
            rc = self.lib.cadmm_op_calibrate(self.h, 2 if kind == "gather" else 3, C.c_void_p(src.data_ptr()),
                                             C.c_void_p(dst.data_ptr()), count, reps, C.byref(rate))
        else:
            raise CadmmError(f"unknown calibration {kind}")
        self._check(rc, "cadmm_op_calibrate")
        self._leave()
        return float(rate.value)

    def op_wgrad(self, A, G):
        torch = self._torch
        assert A.is_cuda and G.is_cuda and A.is_contiguous() and G.is_contiguous() and A.shape[0] == G.shape[0]
        out = torch.empty((A.shape[1], G.shape[1]), dtype=torch.float32, device=A.device)
        self._on_current_stream()
        self._check(self.lib.cadmm_op_wgrad(self.h, A.data_ptr(), G.data_ptr(), A.shape[0], A.shape[1], G.shape[1],
                                            out.data_ptr()), "cadmm_op_wgrad")
        return out

    def op_wgrad_noalloc(self, A, G, out=None):
        """out = A^T G through the entry point that allocates nothing; `out` may be a preallocated tensor."""
        torch = self._torch
        assert A.is_cuda and G.is_cuda and A.is_contiguous() and G.is_contiguous() and A.shape[0] == G.shape[0]
        if out is None:
            out = torch.empty((A.shape[1], G.shape[1]), dtype=torch.float32, device=A.device)
        self._on_current_stream()
        self._check(self.lib.cadmm_op_wgrad_noalloc(self.h, A.data_ptr(), G.data_ptr(), A.shape[0], A.shape[1],
                                                    G.shape[1], out.data_ptr()), "cadmm_op_wgrad_noalloc")
        return out

    # Products over groups of rows and orthogonalised updates: fp32, bf16 and fp16 device tensors of this solver's GPU.  What a call
    # asks of its tensors is one expression (a call of a small product is half host time); what is wrong is looked for afterwards.
    def _value_types(self):
        if self._types is None:
            torch = self._torch
            self._types = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
        return self._types

    def _on_raw_stream(self):
        """_on_current_stream without a stream object."""
        self.lib.cadmm_op_stream(self.h, self._torch._C._cuda_getCurrentRawStream(self.device))

    def _refuse(self, what, types, rows, stacks):
        """The reason why a call's tensors do not fit.  rows: (name, matrix with dense rows, shape or None, dtype or None); stacks:
        (name, dense tensor, shape, dtypes)."""
        for name, t, *_ in rows + stacks:
            if not t.is_cuda or t.device.index != self.device:
                raise CadmmError(f"{what}: {name} is not on GPU {self.device}")
        for name, t, shape, dtype in rows:
            if t.dtype not in types or (dtype is not None and t.dtype != dtype):
                raise CadmmError(f"{what}: {name} has type {t.dtype}")
            if t.dim() != 2 or t.shape[1] < 1 or self._row_stride(t) is None:
                raise CadmmError(f"{what}: {name} must be a matrix with dense rows")
            if shape is not None and tuple(t.shape) != tuple(shape):
                raise CadmmError(f"{what}: {name} must be {tuple(shape)}, not {tuple(t.shape)}")
        for name, t, shape, dtypes in stacks:
            if t.dtype not in dtypes:
                raise CadmmError(f"{what}: {name} has type {t.dtype}")
            if tuple(t.shape) != tuple(shape) or not t.is_contiguous():
                raise CadmmError(f"{what}: {name} must be dense of shape {tuple(shape)}, not {tuple(t.shape)}")
        raise CadmmError(f"{what}: the tensors do not fit together")

    @staticmethod
    def _row_stride(t):
        """Elements from one row of a matrix to the next; None if its rows are not dense."""
        n, width = t.shape
        if n > 1:
            step, inner = t.stride()
            return step if inner == 1 or width == 1 else None
        return width if n == 0 or width == 1 or t.stride(1) == 1 else None

    def _apart(self, what, out, step, *operands):
        """A given output shares no element with what the call reads (rows that interleave do not).  operands: (name, tensor, elements from
        one row to the next); of a dense tensor the step is None."""
        def rows(name, t, step):
            size = t.element_size()
            if step is None or t.numel() == 0:
                return t.data_ptr(), min(t.numel(), 1), t.numel() * size, t.numel() * size
            if step < t.shape[1]:
                raise CadmmError(f"{what}: rows of {name} overlap each other")
            return t.data_ptr(), t.shape[0], step * size, t.shape[1] * size
        own = rows("out", out, step)
        for operand in operands:
            if _rows_meet(own, rows(*operand)):
                raise CadmmError(f"{what}: out overlaps {operand[0]}")

    def _scratch(self, query, *args):
        """Scratch of one call, from torch's allocator for the current stream: (aligned pointer, bytes, what keeps it alive)."""
        nbytes = C.c_size_t()
        self._check(query(self.h, *args, C.byref(nbytes)), query.__name__)
        if nbytes.value == 0:
            return None, 0, None
        hold = self._torch.empty(nbytes.value + 255, dtype=self._torch.uint8, device=self._gpu)
        return (hold.data_ptr() + 255) & ~255, nbytes.value, hold

    def op_transform_grouped(self, A, B, group_ptr, transposed=False, out=None):
        """out[r] = A[r] B_g for the rows r in [group_ptr[g], group_ptr[g + 1]) of every group.  A: n x K, B: groups x K x C
        (transposed: groups x C x K, and B_g is its transpose), group_ptr: int64 device tensor of groups + 1 bounds that do not
        descend.  `out` may be a preallocated n x C matrix with dense rows that shares no element with A, B or group_ptr (it may be other columns of
        A's buffer): rows of no group are left as they are there, and hold anything otherwise.  With the communities' weights in
        B: group_ptr = comm_row_ptr of get_graph.  An entry that is not finite leaves NaN or infinities where it enters."""
        torch, types, gpu = self._torch, self._types or self._value_types(), self.device
        dtype = A.dtype
        if A.dim() != 2 or B.dim() != 3 or group_ptr.dim() != 1 or group_ptr.shape[0] < 2:
            raise CadmmError("op_transform_grouped: A is a matrix, B a stack of matrices, group_ptr holds groups + 1 bounds")
        (n, K), (groups, rows, cols) = A.shape, B.shape
        if transposed:
            rows, cols = cols, rows
        lda, given = self._row_stride(A), out is not None
        fits = (dtype in types and K >= 1 and lda is not None and A.get_device() == gpu and B.get_device() == gpu and B.dtype == dtype and rows == K and
                B.is_contiguous() and group_ptr.get_device() == gpu and group_ptr.dtype == torch.int64 and
                group_ptr.shape[0] == groups + 1 and group_ptr.is_contiguous())
        if fits and out is None:
            out, ldo = torch.empty((n, cols), dtype=dtype, device=self._gpu), cols
        elif fits and out.dim() == 2:
            ldo = self._row_stride(out)
            fits = out.dtype == dtype and out.get_device() == gpu and out.shape[0] == n and out.shape[1] == cols and ldo is not None
        else:
            fits = False
        if not fits:
            groups = group_ptr.shape[0] - 1
            self._refuse("op_transform_grouped", types, [("A", A, None, None)] + ([] if out is None else [("out", out, (n, cols), dtype)]),
                         [("group_ptr", group_ptr, (groups + 1,), (torch.int64,)), ("B", B, (groups, cols, K) if transposed else (groups, K, cols), (dtype,))])
        a, b, p, o = A.data_ptr(), B.data_ptr(), group_ptr.data_ptr(), out.data_ptr()
        if given:                                             # (looked at closely only if their stretches of memory meet)
            size = 4 if dtype == torch.float32 else 2
            end = o + size * ((n - 1) * ldo + cols)
            if (o < a + size * ((n - 1) * lda + K) and a < end) or (o < b + size * groups * K * cols and b < end) or (o < p + 8 * groups + 8 and p < end):
                self._apart("op_transform_grouped", out, ldo, ("A", A, lda), ("B", B, None), ("group_ptr", group_ptr, None))
        self._on_raw_stream()
        rc = self.lib.cadmm_op_transform_grouped(self.h, types[dtype], a, n, lda, K, b, cols, 1 if transposed else 0, groups, p, o, ldo)
        if rc:
            self._check(rc, "cadmm_op_transform_grouped")
        return out

    def op_wgrad_grouped(self, A, G, group_ptr, out=None, out_dtype=None):
        """out[g] = A_g^T G_g over the rows of every group (groups x K x C): the gradient of op_transform_grouped with respect to
        B.  In fp32 unless `out` (which shares no element with A, G or group_ptr) or out_dtype (fp32 or the operands' type) says
        otherwise; zeros for a group without rows.  An entry that is not finite leaves NaN or infinities where it enters."""
        torch, types, gpu = self._torch, self._types or self._value_types(), self.device
        dtype = A.dtype
        if A.dim() != 2 or G.dim() != 2 or group_ptr.dim() != 1 or group_ptr.shape[0] < 2:
            raise CadmmError("op_wgrad_grouped: A and G are matrices, group_ptr holds groups + 1 bounds")
        (n, K), (m, width), groups = A.shape, G.shape, group_ptr.shape[0] - 1
        lda, ldg, given = self._row_stride(A), self._row_stride(G), out is not None
        wanted = (torch.float32, dtype) if out_dtype is None else (out_dtype,)
        fits = (dtype in types and G.dtype == dtype and m == n and K >= 1 and width >= 1 and lda is not None and ldg is not None and
                A.get_device() == gpu and G.get_device() == gpu and group_ptr.get_device() == gpu and group_ptr.dtype == torch.int64 and
                group_ptr.is_contiguous() and (out_dtype is None or out_dtype == torch.float32 or out_dtype == dtype))
        if fits and out is None:
            out = torch.empty((groups, K, width), dtype=out_dtype or torch.float32, device=self._gpu)
        elif fits:
            fits = out.dtype in wanted and out.get_device() == gpu and tuple(out.shape) == (groups, K, width) and out.is_contiguous()
        if not fits:
            self._refuse("op_wgrad_grouped", types, [("A", A, None, None), ("G", G, (n, width), dtype)],
                         [("group_ptr", group_ptr, (groups + 1,), (torch.int64,))] + ([] if out is None else [("out", out, (groups, K, width), wanted)]))
        a, d, p, o = A.data_ptr(), G.data_ptr(), group_ptr.data_ptr(), out.data_ptr()
        if given:                                             # (looked at closely only if their stretches of memory meet)
            size, end = 4 if dtype == torch.float32 else 2, o + (4 if out.dtype == torch.float32 else 2) * groups * K * width
            if (o < a + size * ((n - 1) * lda + K) and a < end) or (o < d + size * ((n - 1) * ldg + width) and d < end) or (o < p + 8 * groups + 8 and p < end):
                self._apart("op_wgrad_grouped", out, None, ("A", A, lda), ("G", G, ldg), ("group_ptr", group_ptr, None))
        ptr, nbytes, hold = self._scratch(self.lib.cadmm_op_wgrad_grouped_scratch, n, K, width, groups)
        self._on_raw_stream()
        rc = self.lib.cadmm_op_wgrad_grouped(self.h, types[dtype], a, n, lda, K, d, ldg, width, groups, p, types[out.dtype], o, ptr, nbytes)
        if rc:
            self._check(rc, "cadmm_op_wgrad_grouped")
        return out

    def op_orthogonalise(self, G, steps=5, coefficients=(3.4445, -4.7750, 2.0315), eps=1e-7, out=None):
        """G (K x C, or a stack batch x K x C) with the singular values of every matrix brought towards one: `steps` times
        X <- a X + (b S + c S^2) X, S = X X^T, from X = G / (||G||_F + eps).  `out` may be G itself.  X is held to 22 bits and 2^-36
        of one: by the norm as exact as in fp32, but rows or columns at 1e-8 of the others come out off by some per cent of themselves."""
        types, shape = self._types or self._value_types(), G.shape
        batch, K, width = self._matrices("op_orthogonalise", G)
        fits = G.dtype in types and G.get_device() == self.device and G.is_contiguous()
        if fits and out is None:
            out = self._torch.empty(shape, dtype=G.dtype, device=self._gpu)
        elif fits:
            fits = out.dtype == G.dtype and out.get_device() == self.device and out.shape == shape and out.is_contiguous()
        if not fits:
            self._refuse("op_orthogonalise", types, [], [("G", G, shape, types)] + ([] if out is None else [("out", out, shape, (G.dtype,))]))
        ptr, nbytes, hold = self._scratch(self.lib.cadmm_op_orthogonalise_scratch, batch, K, width)
        self._on_raw_stream()
        rc = self.lib.cadmm_op_orthogonalise(self.h, types[G.dtype], G.data_ptr(), batch, K, width, steps, self._coefficients(coefficients), eps,
                                             out.data_ptr(), ptr, nbytes)
        if rc:
            self._check(rc, "cadmm_op_orthogonalise")
        return out

    def op_muon_step(self, W, M, G, *, lr, momentum=0.95, nesterov=True, weight_decay=0.0, scale=1.0, steps=5,
                     coefficients=(3.4445, -4.7750, 2.0315), eps=1e-7):
        """One optimiser step on W (K x C, or a stack), in place: M <- momentum M + G, D = G + momentum M (nesterov) or M,
        W <- (1 - lr weight_decay) W - lr scale O with O the orthogonalised D.  W and M are fp32."""
        types, shape, f32, gpu = self._types or self._value_types(), G.shape, self._torch.float32, self.device
        batch, K, width = self._matrices("op_muon_step", G)
        if not (G.dtype in types and G.get_device() == gpu and G.is_contiguous() and W.dtype == f32 and W.get_device() == gpu and W.shape == shape and
                W.is_contiguous() and M.dtype == f32 and M.get_device() == gpu and M.shape == shape and M.is_contiguous()):
            self._refuse("op_muon_step", types, [], [("G", G, shape, types), ("W", W, shape, (f32,)), ("M", M, shape, (f32,))])
        ptr, nbytes, hold = self._scratch(self.lib.cadmm_op_orthogonalise_scratch, batch, K, width)
        self._on_raw_stream()
        rc = self.lib.cadmm_op_muon_step(self.h, types[G.dtype], G.data_ptr(), W.data_ptr(), M.data_ptr(), batch, K, width, lr, momentum,
                                         1 if nesterov else 0, weight_decay, scale, steps, self._coefficients(coefficients), eps, ptr, nbytes)
        if rc:
            self._check(rc, "cadmm_op_muon_step")

    def _coefficients(self, coefficients):
        if len(coefficients) != 3:
            raise CadmmError("three coefficients are wanted")
        return (C.c_float * 3)(*coefficients)

    def _matrices(self, what, G):
        if G.dim() not in (2, 3) or G.numel() == 0:
            raise CadmmError(f"{what}: G must be a matrix or a stack of matrices")
        return (1 if G.dim() == 2 else G.shape[0]), G.shape[-2], G.shape[-1]

    def tune(self, key, value):
        self._check(self.lib.cadmm_tune(self.h, key.encode(), int(value)), "cadmm_tune")

    # ---- per-kernel-class timing
    def profile(self, enable=True):
        self._check(self.lib.cadmm_profile(self.h, 1 if enable else 0), "cadmm_profile")

    def get_profile(self):
        n = PROFILE_CLASSES
        ms, rec = np.zeros(n, np.float64), np.zeros(n, np.int64)
        by, fl = np.zeros(n, np.float64), np.zeros(n, np.float64)
        self._check(self.lib.cadmm_get_profile(self.h, _ptr(ms), _ptr(rec), _ptr(by), _ptr(fl)), "cadmm_get_profile")
        out = {}
        for i in range(n):
            name = self.lib.cadmm_profile_class_name(i).decode()
            out[name] = dict(ms=float(ms[i]), records=int(rec[i]), bytes=float(by[i]), flops=float(fl[i]))
        return out

    # ---- convenience
    @classmethod
    def from_workload(cls, w, device=0):
        s = cls(device)
        s.build_graph(w.N, w.src, w.dst, w.M, w.comm)
        h = w.hyper
        s.set_model(w.dims, nu=h["nu"], rho=h["rho"], tau0=h["tau0"], theta0=h["theta0"], eta=h["eta"],
                    max_backtrack=h["max_backtrack"], fista_iters=h["fista_iters"], risk=h["risk"],
                    dual_form=h["dual_form"], schedule=h.get("schedule", 0),
                    step_policy=h.get("step_policy", 0), fista_mode=h.get("fista_mode", 0))
        s.set_workspace()
        s.set_data(w.X, w.labels)
        s.init(w.W0)
        return s
