"""ctypes binding of the C-ABI library (include/ttc_lqr.h, include/ttc_attention.h): argument marshalling only.

PyTorch is used for device memory and streams; every step of the path runs in the HIP library.
The library must have been built (``python -c "import __graft_entry__ as g; g.build()"``); there is
no fallback: a missing library raises.
"""
from __future__ import annotations

import ctypes
import math
import os
from ctypes import c_char_p, c_int, c_int32, c_int64, c_size_t, c_void_p

import torch

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "lib", "libttc_lqr.so")

TTC_OK, TTC_ERR_INVALID_ARG, TTC_ERR_UNSUPPORTED, TTC_ERR_WORKSPACE, TTC_ERR_DEVICE = range(5)
TTC_F32, TTC_BF16 = 0, 1
TTC_FLAG_STAGE_COST_AT_X0 = 1
TTC_FLAG_PURE_SYMPLECTIC = 2
TTC_FLAG_DOUBLING = 4

EXPORTS = ("ttc_lqr_workspace_bytes", "ttc_lqr_solve", "ttc_lqr_solve_squares", "ttc_lqr_solve_noalloc", "ttc_lqr_noalloc_scratch_bytes",
           "ttc_lqr_rollout", "ttc_lqr_solve_tv", "ttc_lqr_rollout_tv",
           "ttc_lqr_tv_rollout_workspace_bytes", "ttc_lqr_solve_cxt", "ttc_lqr_rollout_cxt",
           "ttc_lqr_cxt_rollout_workspace_bytes", "ttc_lqr_solve_tv_scan",
           "ttc_lqr_tv_scan_workspace_bytes", "ttc_lqr_tv_scan_values", "ttc_lqr_tv_scan_values_workspace_bytes",
           "ttc_lqr_backward", "ttc_lqr_backward_workspace_bytes",
           "ttc_lqr_backward_tv", "ttc_lqr_backward_tv_workspace_bytes", "ttc_lqr_backward_cxt", "ttc_lqr_backward_cxt_workspace_bytes", "ttc_block_workspace_bytes", "ttc_block_forward",
           "ttc_status_string", "ttc_version")
ATTENTION_EXPORTS = ("ttc_rope", "ttc_rope_backward", "ttc_rope_table", "ttc_kv_page_bytes", "ttc_kv_append", "ttc_kv_read",
                     "ttc_attention_workspace_bytes", "ttc_attention")


class Problem(ctypes.Structure):
    _fields_ = [("n", c_int64), ("d", c_int32), ("m", c_int32), ("T", c_int32), ("in_dtype", c_int32),
                ("flags", c_int32), ("rebase_every", c_int32),
                ("A", c_void_p), ("B", c_void_p), ("Q", c_void_p), ("R", c_void_p), ("QT", c_void_p),
                ("x0", c_void_p),
                ("sA", c_int64), ("sB", c_int64), ("sQ", c_int64), ("sR", c_int64), ("sQT", c_int64),
                ("sx0", c_int64)]


class TvProblem(ctypes.Structure):
    _fields_ = [("n", c_int64), ("d", c_int32), ("m", c_int32), ("T", c_int32), ("in_dtype", c_int32),
                ("flags", c_int32),
                ("A", c_void_p), ("B", c_void_p), ("Q", c_void_p), ("R", c_void_p), ("x0", c_void_p),
                ("sA", c_int64), ("sB", c_int64), ("sQ", c_int64), ("sR", c_int64), ("sx0", c_int64),
                ("tA", c_int64), ("tB", c_int64), ("tQ", c_int64), ("tR", c_int64)]


class CxtProblem(ctypes.Structure):
    _fields_ = [("n", c_int64), ("d", c_int32), ("r", c_int32), ("T", c_int32), ("in_dtype", c_int32),
                ("flags", c_int32),
                ("sA", c_void_p), ("sB", c_void_p), ("sQ", c_void_p), ("sQf", c_void_p), ("rinv", c_void_p),
                ("lgA", c_void_p), ("lgB", c_void_p), ("lgQ", c_void_p), ("x0", c_void_p),
                ("Bbasis", c_void_p), ("Qbasis", c_void_p)]


BLOCK_WEIGHTS = ("ln_in_gain", "ln_in_offset", "W_in", "b_in", "W_head", "b_head", "W_shared", "b_shared", "Bbasis", "Qc",
                 "ln_out_gain", "ln_out_offset", "W_out", "b_out")


class Block(ctypes.Structure):
    _fields_ = [("n_tokens", c_int64), ("C", c_int32), ("H", c_int32), ("d", c_int32), ("r", c_int32), ("T", c_int32),
                ("flags", c_int32), ("eps", ctypes.c_float)] + [(k, c_void_p) for k in BLOCK_WEIGHTS]


class Solution(ctypes.Structure):
    _fields_ = [("P0", c_void_p), ("K0", c_void_p), ("u0", c_void_p), ("value", c_void_p), ("info", c_void_p)]


class Grads(ctypes.Structure):
    _fields_ = [("gA", c_void_p), ("gB", c_void_p), ("gQ", c_void_p), ("gR", c_void_p), ("gQT", c_void_p),
                ("gx0", c_void_p), ("info", c_void_p)]


CXT_GRADS = ("gsA", "gsB", "gsQ", "gsQf", "grinv", "glgA", "glgB", "glgQ", "gx0", "gBbasis", "gQbasis", "info")


class CxtGrads(ctypes.Structure):
    _fields_ = [(k, c_void_p) for k in CXT_GRADS]


class Rope(ctypes.Structure):
    _fields_ = [("tokens", c_int64), ("heads", c_int32), ("d", c_int32), ("rot", c_int32), ("dtype", c_int32),
                ("layout", c_int32), ("x", c_void_p), ("y", c_void_p), ("x_token", c_int64), ("x_head", c_int64),
                ("y_token", c_int64), ("y_head", c_int64), ("positions", c_void_p), ("table", c_void_p), ("table_rows", c_int64)]


class KvCache(ctypes.Structure):
    _fields_ = [("data", c_void_p), ("pages", c_int64), ("heads", c_int32), ("d", c_int32), ("page", c_int32)]


class KvAppend(ctypes.Structure):
    _fields_ = [("cache", KvCache), ("tokens", c_int64), ("dtype", c_int32), ("rot", c_int32), ("layout", c_int32),
                ("k", c_void_p), ("v", c_void_p), ("k_token", c_int64), ("k_head", c_int64), ("v_token", c_int64),
                ("v_head", c_int64), ("slots", c_void_p), ("positions", c_void_p), ("table", c_void_p), ("table_rows", c_int64),
                ("q", c_void_p), ("q_out", c_void_p), ("heads_q", c_int32), ("q_token", c_int64), ("q_head", c_int64),
                ("q_out_token", c_int64), ("q_out_head", c_int64)]


class Attention(ctypes.Structure):
    _fields_ = [("cache", KvCache), ("sequences", c_int64), ("tokens", c_int64), ("heads_q", c_int32), ("dtype", c_int32),
                ("causal", c_int32), ("window", c_int32), ("scale", ctypes.c_float), ("max_q", c_int32), ("max_kv", c_int32),
                ("q", c_void_p), ("out", c_void_p), ("lse", c_void_p), ("q_token", c_int64), ("q_head", c_int64),
                ("out_token", c_int64), ("out_head", c_int64), ("cu_q", c_void_p), ("kv_len", c_void_p),
                ("block_table", c_void_p), ("table_stride", c_int64)]


class TtcError(RuntimeError):
    def __init__(self, status, text):
        super().__init__(f"ttc_lqr: {text} (status {status})")
        self.status = status


_lib = None


def load():
    """Load the shared library (once) and declare the prototypes."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(f"{LIB_PATH} is missing: build it with __graft_entry__.build()")
    lib = ctypes.CDLL(LIB_PATH)
    lib.ttc_lqr_workspace_bytes.restype = c_size_t
    lib.ttc_lqr_workspace_bytes.argtypes = [ctypes.POINTER(Problem), c_int]
    lib.ttc_lqr_solve.restype = c_int
    lib.ttc_lqr_solve.argtypes = [ctypes.POINTER(Problem), ctypes.POINTER(Solution), c_void_p, c_size_t, c_void_p]
    lib.ttc_lqr_solve_squares.restype = c_int
    lib.ttc_lqr_solve_squares.argtypes = [ctypes.POINTER(Problem)]
    lib.ttc_lqr_solve_noalloc.restype = c_int
    lib.ttc_lqr_solve_noalloc.argtypes = [ctypes.POINTER(Problem), ctypes.POINTER(Solution), c_void_p]
    lib.ttc_lqr_noalloc_scratch_bytes.restype = c_size_t
    lib.ttc_lqr_noalloc_scratch_bytes.argtypes = []
    lib.ttc_lqr_rollout.restype = c_int
    lib.ttc_lqr_rollout.argtypes = [ctypes.POINTER(Problem), c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                    c_size_t, c_void_p]
    lib.ttc_lqr_solve_tv.restype = c_int
    lib.ttc_lqr_solve_tv.argtypes = [ctypes.POINTER(TvProblem), ctypes.POINTER(Solution), c_void_p, c_size_t, c_void_p]
    lib.ttc_lqr_tv_rollout_workspace_bytes.restype = c_size_t
    lib.ttc_lqr_tv_rollout_workspace_bytes.argtypes = [ctypes.POINTER(TvProblem)]
    lib.ttc_lqr_rollout_tv.restype = c_int
    lib.ttc_lqr_rollout_tv.argtypes = [ctypes.POINTER(TvProblem), c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                       c_size_t, c_void_p]
    lib.ttc_lqr_tv_scan_workspace_bytes.restype = c_size_t
    lib.ttc_lqr_tv_scan_workspace_bytes.argtypes = [ctypes.POINTER(TvProblem)]
    lib.ttc_lqr_solve_tv_scan.restype = c_int
    lib.ttc_lqr_solve_tv_scan.argtypes = [ctypes.POINTER(TvProblem), ctypes.POINTER(Solution), c_void_p, c_size_t,
                                          c_void_p]
    lib.ttc_lqr_tv_scan_values_workspace_bytes.restype = c_size_t
    lib.ttc_lqr_tv_scan_values_workspace_bytes.argtypes = [ctypes.POINTER(TvProblem)]
    lib.ttc_lqr_tv_scan_values.restype = c_int
    lib.ttc_lqr_tv_scan_values.argtypes = [ctypes.POINTER(TvProblem), c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.ttc_lqr_solve_cxt.restype = c_int
    lib.ttc_lqr_solve_cxt.argtypes = [ctypes.POINTER(CxtProblem), ctypes.POINTER(Solution), c_void_p]
    lib.ttc_lqr_cxt_rollout_workspace_bytes.restype = c_size_t
    lib.ttc_lqr_cxt_rollout_workspace_bytes.argtypes = [ctypes.POINTER(CxtProblem)]
    lib.ttc_lqr_rollout_cxt.restype = c_int
    lib.ttc_lqr_rollout_cxt.argtypes = [ctypes.POINTER(CxtProblem), c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                        c_size_t, c_void_p]
    lib.ttc_lqr_backward_workspace_bytes.restype = c_size_t
    lib.ttc_lqr_backward_workspace_bytes.argtypes = [ctypes.POINTER(Problem)]
    lib.ttc_lqr_backward.restype = c_int
    lib.ttc_lqr_backward.argtypes = [ctypes.POINTER(Problem), c_void_p, ctypes.POINTER(Grads), c_void_p, c_size_t,
                                     c_void_p]
    lib.ttc_lqr_backward_tv_workspace_bytes.restype = c_size_t
    lib.ttc_lqr_backward_tv_workspace_bytes.argtypes = [ctypes.POINTER(TvProblem)]
    lib.ttc_lqr_backward_tv.restype = c_int
    lib.ttc_lqr_backward_tv.argtypes = [ctypes.POINTER(TvProblem), c_void_p, ctypes.POINTER(Grads), c_void_p, c_size_t,
                                        c_void_p]
    lib.ttc_lqr_backward_cxt_workspace_bytes.restype = c_size_t
    lib.ttc_lqr_backward_cxt_workspace_bytes.argtypes = [ctypes.POINTER(CxtProblem)]
    lib.ttc_lqr_backward_cxt.restype = c_int
    lib.ttc_lqr_backward_cxt.argtypes = [ctypes.POINTER(CxtProblem), c_void_p, ctypes.POINTER(CxtGrads), c_void_p, c_size_t,
                                         c_void_p]
    lib.ttc_block_workspace_bytes.restype = c_size_t
    lib.ttc_block_workspace_bytes.argtypes = [ctypes.POINTER(Block)]
    lib.ttc_block_forward.restype = c_int
    lib.ttc_block_forward.argtypes = [ctypes.POINTER(Block), c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                      c_size_t, c_void_p]
    lib.ttc_rope.restype = c_int
    lib.ttc_rope.argtypes = [ctypes.POINTER(Rope), c_void_p]
    lib.ttc_rope_backward.restype = c_int
    lib.ttc_rope_backward.argtypes = [ctypes.POINTER(Rope), c_void_p]
    lib.ttc_rope_table.restype = c_int
    lib.ttc_rope_table.argtypes = [c_void_p, c_int64, c_int32, c_void_p, ctypes.c_double, c_void_p]
    lib.ttc_kv_page_bytes.restype = c_size_t
    lib.ttc_kv_page_bytes.argtypes = [c_int32, c_int32]
    lib.ttc_kv_append.restype = c_int
    lib.ttc_kv_append.argtypes = [ctypes.POINTER(KvAppend), c_void_p]
    lib.ttc_kv_read.restype = c_int
    lib.ttc_kv_read.argtypes = [ctypes.POINTER(KvCache), c_void_p, c_int64, c_int32, c_void_p, c_void_p, c_void_p]
    lib.ttc_attention_workspace_bytes.restype = c_size_t
    lib.ttc_attention_workspace_bytes.argtypes = [ctypes.POINTER(Attention)]
    lib.ttc_attention.restype = c_int
    lib.ttc_attention.argtypes = [ctypes.POINTER(Attention), c_void_p, c_size_t, c_void_p]
    lib.ttc_status_string.restype = c_char_p
    lib.ttc_status_string.argtypes = [c_int]
    lib.ttc_version.restype = c_int
    lib.ttc_version.argtypes = []
    _lib = lib
    return lib


def ttc_version() -> int:
    return load().ttc_version()


def ttc_status_string(status: int) -> str:
    return load().ttc_status_string(status).decode()


def _check(status):
    if status != TTC_OK:
        raise TtcError(status, ttc_status_string(status))


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stride(t):
    """Elements between consecutive problems of a (n, ...) tensor whose trailing dims are contiguous."""
    if t is None:
        return 0
    if not t.is_contiguous():
        inner = 1
        for k in range(t.dim() - 1, 0, -1):
            if t.shape[k] != 1 and t.stride(k) != inner:
                raise ValueError("per-problem matrices must be contiguous row-major")
            inner *= t.shape[k]
    return t.stride(0)


_IN_DTYPES = {torch.float32: TTC_F32, torch.bfloat16: TTC_BF16}


def _in_dtype(A, *others):
    dt = A.dtype
    for t in others:
        if t is not None and t.dtype != dt:
            raise ValueError("all inputs must share one dtype")
    in_dtype = _IN_DTYPES.get(dt)
    if in_dtype is None:
        raise ValueError("inputs must be float32 or bfloat16")
    return in_dtype


def make_problem(A, B, Q, R, QT, x0, T, flags=0, rebase_every=0, n=None) -> Problem:
    """Fill the problem descriptor from tensors A (n,d,d), B (n,d,m), Q (n,d,d), R (n,m,m), QT or None,
    x0 (n,d).  A leading dimension expanded with stride 0 is passed through as a shared matrix."""
    in_dtype = _in_dtype(A, B, Q, R, x0, QT)
    shape = A.shape
    return Problem(shape[0] if n is None else n, shape[1], B.shape[2], T, in_dtype, flags, rebase_every,
                   A.data_ptr(), B.data_ptr(), Q.data_ptr(), R.data_ptr(), _ptr(QT), x0.data_ptr(),
                   _stride(A), _stride(B), _stride(Q), _stride(R), _stride(QT), _stride(x0))


def ttc_lqr_workspace_bytes(problem: Problem, for_rollout: bool = False) -> int:
    return load().ttc_lqr_workspace_bytes(ctypes.byref(problem), 1 if for_rollout else 0)


def ttc_lqr_solve_squares(problem: Problem) -> bool:
    """Whether ttc_lqr_solve composes this problem's factors by squaring (d >= 32; at d = 16 the query says no, whatever runs)."""
    return bool(load().ttc_lqr_solve_squares(ctypes.byref(problem)))


_current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_ptr(stream):
    if stream is not None:
        return stream.cuda_stream
    if _current_raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _current_raw_stream(torch.cuda.current_device())  # (the handle alone; a Stream object costs a microsecond more)


def _scratch(nbytes, dev, stream):
    """A workspace the wrapper owns: allocated for, and only released to, the stream the kernels run on (the
    caching allocator would otherwise hand the block to other work on the current stream while the launch,
    on another stream, still uses it)."""
    if stream is None or stream == torch.cuda.current_stream():
        return torch.empty((max(nbytes, 16),), dtype=torch.uint8, device=dev)
    with torch.cuda.stream(stream):
        return torch.empty((max(nbytes, 16),), dtype=torch.uint8, device=dev)


def _outputs(out, dev, f32, i32):
    """`out` (a dict or None) with a new float32, or int32, tensor for every name in f32 and i32 (name: shape) that it lacks."""
    out = dict(out or {})
    for name, shape in f32.items():
        if name not in out:
            out[name] = torch.empty(shape, dtype=torch.float32, device=dev)
    for name, shape in i32.items():
        if name not in out:
            out[name] = torch.empty(shape, dtype=torch.int32, device=dev)
    return out


def _solve_outputs(out, dev, n, d, m, want_P0, want_K0):
    shapes = {"P0": (n, d, d)} if want_P0 else {}
    if want_K0:
        shapes["K0"] = (n, m, d)
    shapes["u0"] = (n, m)
    shapes["value"] = (n,)
    out = _outputs(out, dev, shapes, {"info": (n,)})
    return out, Solution(_ptr(out.get("P0")), _ptr(out.get("K0")), _ptr(out["u0"]), _ptr(out["value"]), _ptr(out["info"]))


def ttc_lqr_solve(A, B, Q, R, QT, x0, T, *, flags=0, rebase_every=0, want_P0=True, want_K0=True,
                  out=None, workspace=None, stream=None):
    """P0 (n,d,d), K0 (n,m,d), u0 (n,m), value (n), info (n) of n LQR problems; all float32 device tensors.

    `out` may carry preallocated tensors under the same names; `workspace` a uint8 device tensor."""
    lib = load()
    prob = make_problem(A, B, Q, R, QT, x0, T, flags, rebase_every)
    dev = A.device
    out, sol = _solve_outputs(out, dev, prob.n, prob.d, prob.m, want_P0, want_K0)
    if workspace is None:
        workspace = _scratch(lib.ttc_lqr_workspace_bytes(prob, 0), dev, stream)
    _check(lib.ttc_lqr_solve(prob, sol, workspace.data_ptr(), workspace.numel(), _stream_ptr(stream)))
    return out


def ttc_lqr_solve_noalloc(A, B, Q, R, QT, x0, T, out, *, flags=0, rebase_every=0, stream=None):
    """ttc_lqr_solve through the entry point that allocates nothing: `out` must carry preallocated u0 (n,m) and,
    optionally, P0, K0, value, info; the library's own fixed scratch array serves as the workspace."""
    lib = load()
    prob = make_problem(A, B, Q, R, QT, x0, T, flags, rebase_every)
    sol = Solution(_ptr(out.get("P0")), _ptr(out.get("K0")), _ptr(out["u0"]), _ptr(out.get("value")),
                   _ptr(out.get("info")))
    _check(lib.ttc_lqr_solve_noalloc(ctypes.byref(prob), ctypes.byref(sol), _stream_ptr(stream)))
    return out


def ttc_lqr_rollout(A, B, Q, R, QT, x0, T, *, flags=0, rebase_every=0, workspace=None, stream=None):
    """U (n,T,m), X (n,T+1,d), cost (n), info (n) of n LQR problems; float32 device tensors."""
    lib = load()
    prob = make_problem(A, B, Q, R, QT, x0, T, flags, rebase_every)
    n, d, m, dev = prob.n, prob.d, prob.m, A.device
    f32 = dict(dtype=torch.float32, device=dev)
    U = torch.empty((n, T, m), **f32)
    X = torch.empty((n, T + 1, d), **f32)
    cost = torch.empty((n,), **f32)
    info = torch.empty((n,), dtype=torch.int32, device=dev)
    need = lib.ttc_lqr_workspace_bytes(ctypes.byref(prob), 1)
    if workspace is None:
        workspace = _scratch(need, dev, stream)
    _check(lib.ttc_lqr_rollout(ctypes.byref(prob), c_void_p(U.data_ptr()), c_void_p(X.data_ptr()),
                               c_void_p(cost.data_ptr()), c_void_p(info.data_ptr()),
                               c_void_p(workspace.data_ptr()), workspace.numel(), _stream_ptr(stream)))
    return {"U": U, "X": X, "cost": cost, "info": info}


def _tv_strides(t):
    """(problem stride, step stride) in elements of a (n, T, r, c) tensor whose matrices are contiguous row-major."""
    if t.dim() != 4 or (not t.is_contiguous() and
                        ((t.shape[3] != 1 and t.stride(3) != 1) or (t.shape[2] != 1 and t.stride(2) != t.shape[3]))):
        raise ValueError("expected (n, T, rows, cols) with contiguous row-major matrices")
    return t.stride()[:2]


def make_tv_problem(A, B, Q, R, x0) -> TvProblem:
    """Descriptor of a time-heterogeneous problem from A (n,T,d,d), B (n,T,d,m), Q (n,T,d,d), R (n,T,m,m), x0 (n,d);
    an axis expanded with stride 0 is passed through as shared."""
    in_dtype = _in_dtype(A, B, Q, R, x0)
    (sA, tA), (sB, tB), (sQ, tQ), (sR, tR) = _tv_strides(A), _tv_strides(B), _tv_strides(Q), _tv_strides(R)
    n, T, d, _ = A.shape
    return TvProblem(n, d, B.shape[3], T, in_dtype, 0,
                     A.data_ptr(), B.data_ptr(), Q.data_ptr(), R.data_ptr(), x0.data_ptr(),
                     sA, sB, sQ, sR, _stride(x0), tA, tB, tQ, tR)


def ttc_lqr_solve_tv(A, B, Q, R, x0, *, want_P0=True, want_K0=True, out=None, stream=None):
    """P0, K0, u0, value, info of n time-heterogeneous problems: A (n,T,d,d), B (n,T,d,m), R (n,T,m,m) and
    Q (n,T,d,d) with Q[:, s] the cost on the state step s arrives at (Q[:, T-1] is the terminal cost)."""
    lib = load()
    prob = make_tv_problem(A, B, Q, R, x0)
    out, sol = _solve_outputs(out, A.device, prob.n, prob.d, prob.m, want_P0, want_K0)
    _check(lib.ttc_lqr_solve_tv(prob, sol, None, 0, _stream_ptr(stream)))
    return out


def ttc_lqr_tv_scan_values(A, B, Q, R, x0, *, want_P=True, want_K=True, workspace=None, stream=None):
    """P (n, T, d, d) with P[:, k] = P_{k+1} and K (n, T, m, d) with K[:, s] = K_s of n time-heterogeneous problems,
    by the tree over the horizon (up-sweep and down-sweep)."""
    lib = load()
    prob = make_tv_problem(A, B, Q, R, x0)
    n, d, m, T, dev = prob.n, prob.d, prob.m, prob.T, A.device
    f32 = dict(dtype=torch.float32, device=dev)
    out = {}
    if want_P:
        out["P"] = torch.empty((n, T, d, d), **f32)
    if want_K:
        out["K"] = torch.empty((n, T, m, d), **f32)
    need = lib.ttc_lqr_tv_scan_values_workspace_bytes(ctypes.byref(prob))
    if workspace is None:
        workspace = _scratch(need, dev, stream)
    _check(lib.ttc_lqr_tv_scan_values(ctypes.byref(prob), _ptr(out.get("P")), _ptr(out.get("K")),
                                      c_void_p(workspace.data_ptr()), workspace.numel(), _stream_ptr(stream)))
    return out


def ttc_lqr_solve_tv_scan(A, B, Q, R, x0, *, want_P0=True, want_K0=True, out=None, workspace=None, stream=None):
    """ttc_lqr_solve_tv with the factors composed pairwise over the horizon (small batches, long horizons)."""
    lib = load()
    prob = make_tv_problem(A, B, Q, R, x0)
    dev = A.device
    out, sol = _solve_outputs(out, dev, prob.n, prob.d, prob.m, want_P0, want_K0)
    if workspace is None:
        workspace = _scratch(lib.ttc_lqr_tv_scan_workspace_bytes(prob), dev, stream)
    _check(lib.ttc_lqr_solve_tv_scan(prob, sol, workspace.data_ptr(), workspace.numel(), _stream_ptr(stream)))
    return out


def ttc_lqr_rollout_tv(A, B, Q, R, x0, *, workspace=None, stream=None):
    """U (n,T,m), X (n,T+1,d), cost (n), info (n) of n time-heterogeneous problems; float32 device tensors."""
    lib = load()
    prob = make_tv_problem(A, B, Q, R, x0)
    n, d, m, T, dev = prob.n, prob.d, prob.m, prob.T, A.device
    f32 = dict(dtype=torch.float32, device=dev)
    out = {"U": torch.empty((n, T, m), **f32), "X": torch.empty((n, T + 1, d), **f32),
           "cost": torch.empty((n,), **f32), "info": torch.empty((n,), dtype=torch.int32, device=dev)}
    need = lib.ttc_lqr_tv_rollout_workspace_bytes(ctypes.byref(prob))
    if workspace is None:
        workspace = _scratch(need, dev, stream)
    _check(lib.ttc_lqr_rollout_tv(ctypes.byref(prob), _ptr(out["U"]), _ptr(out["X"]), _ptr(out["cost"]),
                                  _ptr(out["info"]), c_void_p(workspace.data_ptr()), workspace.numel(),
                                  _stream_ptr(stream)))
    return out


def make_cxt_problem(sA, sB, sQ, sQf, rinv, lgA, lgB, lgQ, Bbasis, Qbasis, x0, T) -> CxtProblem:
    """Descriptor of n structured problems: sA, rinv, lgA, lgB, lgQ, x0 (n,d); sB, sQ, sQf (n,r); Bbasis, Qbasis
    (r,d,d); all contiguous and of one dtype."""
    n, d = sA.shape
    r = Bbasis.shape[0]
    shapes = {"sA": (n, d), "rinv": (n, d), "lgA": (n, d), "lgB": (n, d), "lgQ": (n, d), "x0": (n, d),
              "sB": (n, r), "sQ": (n, r), "sQf": (n, r), "Bbasis": (r, d, d), "Qbasis": (r, d, d)}
    given = dict(sA=sA, sB=sB, sQ=sQ, sQf=sQf, rinv=rinv, lgA=lgA, lgB=lgB, lgQ=lgQ, Bbasis=Bbasis, Qbasis=Qbasis, x0=x0)
    for k, t in given.items():
        if tuple(t.shape) != shapes[k] or not t.is_contiguous() or t.dtype != sA.dtype:
            raise ValueError(f"{k}: expected a contiguous {shapes[k]} tensor of dtype {sA.dtype}")
    return CxtProblem(n, d, r, T, _in_dtype(sA), 0, *(given[k].data_ptr() for k, _ in CxtProblem._fields_[6:]))


def ttc_lqr_solve_cxt(sA, sB, sQ, sQf, rinv, lgA, lgB, lgQ, Bbasis, Qbasis, x0, T, *, want_P0=True, want_K0=True,
                      out=None, stream=None):
    """P0, K0, u0, value, info of n structured, contextualised problems (float32 device tensors)."""
    lib = load()
    prob = make_cxt_problem(sA, sB, sQ, sQf, rinv, lgA, lgB, lgQ, Bbasis, Qbasis, x0, T)
    out, sol = _solve_outputs(out, sA.device, prob.n, prob.d, prob.d, want_P0, want_K0)
    _check(lib.ttc_lqr_solve_cxt(prob, sol, _stream_ptr(stream)))
    return out


def ttc_lqr_rollout_cxt(sA, sB, sQ, sQf, rinv, lgA, lgB, lgQ, Bbasis, Qbasis, x0, T, *, workspace=None, stream=None):
    """U (n,T,d), X (n,T+1,d), cost (n), info (n) of n structured problems under the optimal feedback."""
    lib = load()
    prob = make_cxt_problem(sA, sB, sQ, sQf, rinv, lgA, lgB, lgQ, Bbasis, Qbasis, x0, T)
    n, d, dev = prob.n, prob.d, sA.device
    f32 = dict(dtype=torch.float32, device=dev)
    out = {"U": torch.empty((n, T, d), **f32), "X": torch.empty((n, T + 1, d), **f32),
           "cost": torch.empty((n,), **f32), "info": torch.empty((n,), dtype=torch.int32, device=dev)}
    need = lib.ttc_lqr_cxt_rollout_workspace_bytes(ctypes.byref(prob))
    if workspace is None:
        workspace = _scratch(need, dev, stream)
    _check(lib.ttc_lqr_rollout_cxt(ctypes.byref(prob), _ptr(out["U"]), _ptr(out["X"]), _ptr(out["cost"]),
                                   _ptr(out["info"]), c_void_p(workspace.data_ptr()), workspace.numel(),
                                   _stream_ptr(stream)))
    return out


def _grads_struct(out):
    return Grads(_ptr(out["gA"]), _ptr(out["gB"]), _ptr(out["gQ"]), _ptr(out["gR"]), _ptr(out.get("gQT")),
                 _ptr(out["gx0"]), _ptr(out.get("info")))


def ttc_lqr_backward(A, B, Q, R, QT, x0, T, grad_u0, *, out=None, workspace=None, stream=None):
    """Gradients of a loss of u0 for n time-invariant problems, from grad_u0 = dl/du0 (n,m) float32: gA, gB, gQ, gR
    (n,d,d), summed over the steps, gQT (n,d,d) when QT is given, gx0 (n,d), info (n)."""
    lib = load()
    prob = make_problem(A, B, Q, R, QT, x0, T)
    n, d, dev = prob.n, prob.d, A.device
    f32 = dict(dtype=torch.float32, device=dev)
    out = dict(out or {})
    for k in ("gA", "gB", "gQ", "gR") + (("gQT",) if QT is not None else ()):
        out.setdefault(k, torch.empty((n, d, d), **f32))
    out.setdefault("gx0", torch.empty((n, d), **f32))
    out.setdefault("info", torch.empty((n,), dtype=torch.int32, device=dev))
    need = lib.ttc_lqr_backward_workspace_bytes(ctypes.byref(prob))
    if workspace is None:
        workspace = _scratch(need, dev, stream)
    gr = _grads_struct(out)
    _check(lib.ttc_lqr_backward(ctypes.byref(prob), c_void_p(grad_u0.data_ptr()), ctypes.byref(gr),
                                c_void_p(workspace.data_ptr()), workspace.numel(), _stream_ptr(stream)))
    return out


def ttc_lqr_backward_tv(A, B, Q, R, x0, grad_u0, *, out=None, workspace=None, stream=None):
    """Gradients of a loss of u0 for n time-heterogeneous problems: gA, gB, gQ, gR (n,T,d,d), gx0 (n,d), info (n)."""
    lib = load()
    prob = make_tv_problem(A, B, Q, R, x0)
    n, d, T, dev = prob.n, prob.d, prob.T, A.device
    f32 = dict(dtype=torch.float32, device=dev)
    out = dict(out or {})
    for k in ("gA", "gB", "gQ", "gR"):
        out.setdefault(k, torch.empty((n, T, d, d), **f32))
    out.setdefault("gx0", torch.empty((n, d), **f32))
    out.setdefault("info", torch.empty((n,), dtype=torch.int32, device=dev))
    need = lib.ttc_lqr_backward_tv_workspace_bytes(ctypes.byref(prob))
    if workspace is None:
        workspace = _scratch(need, dev, stream)
    gr = _grads_struct(out)
    _check(lib.ttc_lqr_backward_tv(ctypes.byref(prob), c_void_p(grad_u0.data_ptr()), ctypes.byref(gr),
                                   c_void_p(workspace.data_ptr()), workspace.numel(), _stream_ptr(stream)))
    return out


def ttc_lqr_backward_cxt(sA, sB, sQ, sQf, rinv, lgA, lgB, lgQ, Bbasis, Qbasis, x0, T, grad_u0, *, out=None, workspace=None,
                         stream=None):
    """Gradients of a loss of u0 for n structured problems, from grad_u0 = dl/du0 (n, d) float32: gsA, grinv, glgA,
    glgB, glgQ, gx0 (n, d), gsB, gsQ, gsQf (n, r), gBbasis, gQbasis (r, d, d) summed over the problems, info (n)."""
    lib = load()
    prob = make_cxt_problem(sA, sB, sQ, sQf, rinv, lgA, lgB, lgQ, Bbasis, Qbasis, x0, T)
    n, d, r, dev = prob.n, prob.d, prob.r, sA.device
    if grad_u0.dtype != torch.float32 or not grad_u0.is_contiguous() or tuple(grad_u0.shape) != (n, d):
        raise ValueError("grad_u0 must be a contiguous (n, d) float32 tensor")
    f32 = dict(dtype=torch.float32, device=dev)
    out = dict(out or {})
    for k in ("gsA", "grinv", "glgA", "glgB", "glgQ", "gx0"):
        out.setdefault(k, torch.empty((n, d), **f32))
    for k in ("gsB", "gsQ", "gsQf"):
        out.setdefault(k, torch.empty((n, r), **f32))
    for k in ("gBbasis", "gQbasis"):
        out.setdefault(k, torch.empty((r, d, d), **f32))
    out.setdefault("info", torch.empty((n,), dtype=torch.int32, device=dev))
    need = lib.ttc_lqr_backward_cxt_workspace_bytes(ctypes.byref(prob))
    if workspace is None:
        workspace = _scratch(need, dev, stream)
    grads = CxtGrads(*(_ptr(out[k]) for k in CXT_GRADS))
    _check(lib.ttc_lqr_backward_cxt(ctypes.byref(prob), _ptr(grad_u0), ctypes.byref(grads), c_void_p(workspace.data_ptr()),
                                    workspace.numel(), _stream_ptr(stream)))
    return out


TTC_BLOCK_FLAG_BF16 = 1


def make_block(weights, n_tokens, T, eps=1e-5) -> Block:
    """Descriptor of a TTC block from a dict of device tensors (keys BLOCK_WEIGHTS), float32 except that W_in and W_out
    may both be bfloat16 (then the block takes bfloat16 token features: TTC_BLOCK_FLAG_BF16); shapes are checked here,
    values never touched."""
    w = weights
    bf16 = w["W_in"].dtype == torch.bfloat16
    for k in BLOCK_WEIGHTS:
        want_dtype = torch.bfloat16 if bf16 and k in ("W_in", "W_out") else torch.float32
        if w[k].dtype != want_dtype or not w[k].is_contiguous():
            raise ValueError("block weight %s must be a contiguous %s tensor" % (k, want_dtype))
    r, d = int(w["Bbasis"].shape[0]), int(w["Bbasis"].shape[-1])
    HD, C = (int(v) for v in w["W_in"].shape)
    H = HD // d
    want = {"ln_in_gain": (C,), "ln_in_offset": (C,), "W_in": (H * d, C), "b_in": (H * d,),
            "W_head": (H, 5 * d + r, d), "b_head": (H, 5 * d + r), "W_shared": (2 * r, d), "b_shared": (2 * r,),
            "Bbasis": (r, d, d), "Qc": (r, d, d), "ln_out_gain": (H * d,), "ln_out_offset": (H * d,),
            "W_out": (C, H * d), "b_out": (C,)}
    for k, shape in want.items():
        if tuple(w[k].shape) != shape:
            raise ValueError("block weight %s has shape %s, expected %s" % (k, tuple(w[k].shape), shape))
    return Block(n_tokens, C, H, d, r, T, TTC_BLOCK_FLAG_BF16 if bf16 else 0, eps, *(w[k].data_ptr() for k in BLOCK_WEIGHTS))


def ttc_block_forward(x_in, weights, T, *, eps=1e-5, want_h0=False, want_o=False, out=None, workspace=None, stream=None):
    """x_out (n_tokens, C) of the whole TTC block for token features x_in (n_tokens, C) on the device, float32 or
    (with bfloat16 W_in, W_out) bfloat16; info (n_tokens, H); optionally the intermediate h0 and o (n_tokens, H*d), float32."""
    lib = load()
    n, dev = int(x_in.shape[0]), x_in.device
    blk = make_block(weights, n, T, eps)
    xdt = torch.bfloat16 if blk.flags & TTC_BLOCK_FLAG_BF16 else torch.float32
    if x_in.dtype != xdt or not x_in.is_contiguous() or x_in.dim() != 2:
        raise ValueError("x_in must be a contiguous (n_tokens, C) %s tensor" % xdt)
    if int(x_in.shape[1]) != blk.C:
        raise ValueError("x_in has %d features, the block expects %d" % (x_in.shape[1], blk.C))
    out = dict(out or {})
    f32 = dict(dtype=torch.float32, device=dev)
    out.setdefault("x_out", torch.empty((n, blk.C), dtype=xdt, device=dev))
    if want_h0:
        out.setdefault("h0", torch.empty((n, blk.H * blk.d), **f32))
    if want_o:
        out.setdefault("o", torch.empty((n, blk.H * blk.d), **f32))
    out.setdefault("info", torch.empty((n, blk.H), dtype=torch.int32, device=dev))
    need = lib.ttc_block_workspace_bytes(ctypes.byref(blk))
    if workspace is None:
        workspace = _scratch(need, dev, stream)
    _check(lib.ttc_block_forward(ctypes.byref(blk), _ptr(x_in), _ptr(out["x_out"]), _ptr(out.get("h0")), _ptr(out.get("o")),
                                 _ptr(out["info"]), c_void_p(workspace.data_ptr()), workspace.numel(), _stream_ptr(stream)))
    return out


# ---------------------------------------------------------------------------------------------------------------
# rotary positions, the cache in 4 bits, attention over it (include/ttc_attention.h)

_ROPE_LAYOUTS = {"half": 0, "interleaved": 1}


def _rope_layout(layout):
    code = _ROPE_LAYOUTS.get(layout)
    if code is None:
        raise ValueError("layout must be 'half' or 'interleaved'")
    return code


def _heads_strides(t, name, shape=None, dtype=None):
    """(token stride, head stride) of a (tokens, heads, d) tensor whose heads are contiguous, after its shape and type were checked."""
    have = t.shape
    if len(have) != 3 or (shape is not None and have != shape) or (dtype is not None and t.dtype is not dtype):
        raise ValueError(f"{name}: expected a {tuple(shape or ('tokens', 'heads', 'd'))} tensor" + (f" of {dtype}" if dtype else ""))
    token, head, entry = t.stride()
    if entry != 1 and have[2] > 1:
        raise ValueError(f"{name}: the entries of a head must be contiguous")
    return token, head


def _vector(t, n, dtype, name):
    if t.dtype is not dtype or t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous {dtype} tensor of {n}")
    return t.data_ptr()


def _same_device(first, *tensors):
    at = first.get_device()
    for t in tensors:
        if t is not None and t.get_device() != at:
            raise ValueError("all tensors must be on one device")


def _int32(**numbers):
    """Numbers of the caller that a descriptor holds in 32 bits, where ctypes would cut them off."""
    for name, value in numbers.items():
        if not -1 << 31 <= value < 1 << 31:
            raise ValueError(f"{name}: {value} does not fit in 32 bits")


def _on_gpu(t):
    """The last check before a launch: a kernel that is handed host memory faults."""
    if not t.is_cuda:
        raise ValueError("tensors must be on a GPU")


def _rope_table(table, d):
    rows, pairs, two = table.shape if table.dim() == 3 else (0, 0, 0)
    if two != 2 or table.dtype is not torch.float32 or not table.is_contiguous():
        raise ValueError("table: expected a contiguous float32 (rows, rot / 2, 2) tensor")
    if 2 * pairs > d:
        raise ValueError("table: more entries rotated than a head has")
    return table.data_ptr(), rows, 2 * pairs


def _new(like, shape, dtype, stream):
    """A result tensor on the device of `like`, from the memory of the stream that the kernels run on."""
    if stream is None or stream == torch.cuda.current_stream():
        return like.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


def _new_like(t, stream):
    """A contiguous tensor of the shape and type of t, likewise."""
    if stream is None and t.is_contiguous():
        return torch.empty_like(t)  # (half the time of new_empty)
    return _new(t, t.shape, t.dtype, stream)


def rope_frequencies(rot, *, base=10000.0, scaling=None, factor=1.0, trained=None, fast=32.0, slow=1.0):
    """(frequencies, scale) for ttc_rope_table: rot / 2 angles per position, float64 on the host, and the factor on cos and sin.

    scaling None: base^(-2i/rot).  For contexts `factor` times as long as the `trained` one:
      "linear"  positions are compressed: every frequency divided by factor.
      "base"    the base grows to base * factor^(rot/(rot-2)): the highest frequency stays, the lowest is divided by factor (the published
                method known as NTK-aware scaling).
      "bands"   frequencies that turn more than `fast` times within `trained` positions stay, those that turn less than `slow`
                times are divided by factor, those in between are mixed linearly over their index (the range between the whole indices that
                enclose it); the scale is 0.1 ln(factor) + 1.  This is YaRN (Peng et al., arXiv 2309.00071), with its 32, 1 and 0.1."""
    if rot < 2 or rot % 2 or factor < 1.0 or not base > 1.0:
        raise ValueError("rot must be even and positive, factor >= 1, base > 1")
    i = torch.arange(rot // 2, dtype=torch.float64)
    if scaling == "base":
        if rot < 4:
            raise ValueError("scaling 'base' needs rot >= 4")
        base = base * factor ** (rot / (rot - 2))
    freqs = torch.tensor(base, dtype=torch.float64) ** (-2.0 * i / rot)
    if scaling in (None, "base"):
        return freqs, 1.0
    if scaling == "linear":
        return freqs / factor, 1.0
    if scaling != "bands":
        raise ValueError("scaling must be None, 'linear', 'base' or 'bands'")
    if not trained or not fast > slow > 0:
        raise ValueError("scaling 'bands' needs the trained length, and fast > slow > 0")

    def index(turns):  # of the frequency that turns so often within the trained length
        return rot * math.log(trained / (2.0 * math.pi * turns)) / (2.0 * math.log(base))

    lo, hi = max(0, math.floor(index(fast))), math.ceil(index(slow))  # (hi may lie behind the last pair, which then stays mixed)
    mix = ((i - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
    return freqs * (1.0 - mix) + freqs / factor * mix, 0.1 * math.log(factor) + 1.0


def ttc_rope_table(rows, freqs, *, scale=1.0, device="cuda", out=None, stream=None):
    """float32 table (rows, pairs, 2) of scale * cos and scale * sin of position * freqs (pairs, float64; see rope_frequencies)."""
    freqs = freqs.to(device=device, dtype=torch.float64).contiguous()
    pairs = freqs.shape[0]
    if out is None:
        out = _new(freqs, (rows, pairs, 2), torch.float32, stream)
    elif tuple(out.shape) != (rows, pairs, 2) or out.dtype != torch.float32 or not out.is_contiguous() or out.device != freqs.device:
        raise ValueError("out: expected a contiguous float32 (rows, pairs, 2) tensor on the frequencies' device")
    if stream is not None and stream != torch.cuda.current_stream():
        stream.wait_stream(torch.cuda.current_stream())  # the frequencies were copied there
        freqs.record_stream(stream)
    _on_gpu(freqs)
    _check(load().ttc_rope_table(out.data_ptr(), rows, pairs, freqs.data_ptr(), scale, _stream_ptr(stream)))
    return out


def _rope(call, x, positions, table, layout, out, stream):
    dtype = _in_dtype(x)
    x_token, x_head = _heads_strides(x, "x")
    tokens, heads, d = x.shape
    table_ptr, rows, rot = _rope_table(table, d)
    pos = _vector(positions, tokens, torch.int64, "positions")
    _same_device(x, positions, table, out)
    if out is None:
        out = _new_like(x, stream)
        y_token, y_head = heads * d, d
    else:
        y_token, y_head = _heads_strides(out, "out", x.shape, x.dtype)
    if tokens and heads and d:
        _on_gpu(x)
        _check(call(Rope(tokens, heads, d, rot, dtype, _rope_layout(layout), x.data_ptr(), out.data_ptr(), x_token, x_head, y_token,
                         y_head, pos, table_ptr, rows), _stream_ptr(stream)))
    return out


def ttc_rope(x, positions, table, *, layout="half", out=None, stream=None):
    """x (tokens, heads, d) with the first 2 * table.shape[1] entries of each head turned to the tokens' positions (int64); float32 or
    bfloat16, any strides with contiguous heads (so also a part of a fused projection).  out may be x."""
    return _rope(load().ttc_rope, x, positions, table, layout, out, stream)


def ttc_rope_backward(grad, positions, table, *, layout="half", out=None, stream=None):
    """The gradient of a loss with respect to ttc_rope's x, from grad, the one with respect to its result."""
    return _rope(load().ttc_rope_backward, grad, positions, table, layout, out, stream)


def ttc_kv_page_bytes(d, page):
    """Bytes of one head of one page of `page` tokens; 0 if d or page is not supported."""
    return load().ttc_kv_page_bytes(d, page)


def make_kv_cache(pages, heads, d, page, device="cuda"):
    """An empty cache: (pages, heads, ttc_kv_page_bytes(d, page)) bytes, all zero.  What describes a cache everywhere is this tensor and d."""
    nbytes = ttc_kv_page_bytes(d, page)
    if not nbytes:
        raise ValueError("d must be 64, 128 or 256, page 16, 32, 64, 128 or 256")
    return torch.zeros((pages, heads, nbytes), dtype=torch.uint8, device=device)


def _kv_cache(cache, d):
    if cache.dtype != torch.uint8 or cache.dim() != 3 or not cache.is_contiguous():
        raise ValueError("cache: expected a contiguous uint8 (pages, heads, bytes) tensor")
    pages, heads, nbytes = cache.shape
    page = nbytes // (d + d // 16)
    if page * (d + d // 16) != nbytes:
        raise ValueError("cache: its pages are not of heads of %d" % d)
    return KvCache(cache.data_ptr(), pages, heads, d, page)


def ttc_kv_append(cache, k, v, slots, positions=None, table=None, *, layout="half", q=None, q_out=None, stream=None):
    """New tokens' keys (turned to their positions, unless table is None) and values into the cache at slots (int64; page number *
    tokens a page + token of the page; -1 leaves a token out); all of k, v (tokens, heads, d) and q (tokens, heads_q, d) float32 or
    bfloat16.  Returns the turned queries (q_out, which may be q; None without q)."""
    dtype = _in_dtype(k, v, q, q_out)
    k_token, k_head = _heads_strides(k, "k")
    tokens, heads, d = k.shape
    v_token, v_head = _heads_strides(v, "v", k.shape)
    kv = _kv_cache(cache, d)
    if kv.heads != heads:
        raise ValueError("cache: %d heads, expected %d" % (kv.heads, heads))
    at = _vector(slots, tokens, torch.int64, "slots")
    pos, table_ptr, rows, rot = None, None, 0, 0
    if table is not None:
        table_ptr, rows, rot = _rope_table(table, d)
        pos = _vector(positions, tokens, torch.int64, "positions")
    _same_device(cache, k, v, slots, positions, table, q, q_out)
    heads_q = q_token = q_head = qo_token = qo_head = 0
    if q is not None:
        q_token, q_head = _heads_strides(q, "q")
        if q.shape[0] != tokens or q.shape[2] != d:
            raise ValueError("q: expected (%d, heads_q, %d)" % (tokens, d))
        heads_q = q.shape[1]
        if q_out is None:
            q_out = _new_like(q, stream)
            qo_token, qo_head = heads_q * d, d
        else:
            qo_token, qo_head = _heads_strides(q_out, "q_out", q.shape)
    elif q_out is not None:
        raise ValueError("q_out without q")
    if tokens:
        _on_gpu(cache)
        _check(load().ttc_kv_append(KvAppend(kv, tokens, dtype, rot, _rope_layout(layout), k.data_ptr(), v.data_ptr(), k_token, k_head,
                                             v_token, v_head, at, pos, table_ptr, rows, _ptr(q), _ptr(q_out), heads_q, q_token, q_head,
                                             qo_token, qo_head), _stream_ptr(stream)))
    return q_out


def ttc_kv_read(cache, slots, d, *, dtype=torch.bfloat16, out=None, stream=None):
    """(k, v), each (n, heads, d): the numbers that the cache holds at n slots (int64); zeros for a slot outside the cache."""
    kv = _kv_cache(cache, d)
    at = _vector(slots, slots.shape[0], torch.int64, "slots")
    code = _IN_DTYPES.get(dtype)
    if code is None:
        raise ValueError("dtype must be float32 or bfloat16")
    shape = (slots.shape[0], kv.heads, d)
    if out is None:
        k = _new(cache, shape, dtype, stream)
        v = _new_like(k, stream)
        _same_device(cache, slots)
    else:
        k, v = out
        for t in (k, v):
            if tuple(t.shape) != shape or t.dtype != dtype or not t.is_contiguous():
                raise ValueError("out: expected two contiguous %s tensors of %s" % (dtype, shape))
        _same_device(cache, slots, k, v)
    if shape[0]:
        _on_gpu(cache)
        _check(load().ttc_kv_read(kv, at, shape[0], code, k.data_ptr(), v.data_ptr(), _stream_ptr(stream)))
    return k, v


def ttc_attention(q, cache, block_table, kv_len, *, cu_q=None, max_q=None, max_kv=None, scale=None, causal=True, window=0,
                  want_lse=True, out=None, workspace=None, stream=None):
    """{"out": (tokens, heads_q, d) like q, "lse": (tokens, heads_q) float32} of the queries of new tokens over a cache in 4 bits.

    Sequence s has kv_len[s] tokens in the cache (int32), the new ones the last of them, on the pages block_table[s] (int32), and the
    rows cu_q[s] .. cu_q[s+1]-1 of q (int32; without cu_q one row each).  max_q and max_kv bound the sequences' numbers of new and of all
    tokens (with cu_q max_q is needed; max_kv defaults to what block_table has room for): the work is shared out by them.  scale
    defaults to d^-1/2.  `out` may carry tensors under the same names; `workspace` a uint8 tensor."""
    lib = load()
    dtype = _in_dtype(q)
    q_token, q_head = _heads_strides(q, "q")
    tokens, heads_q, d = q.shape
    kv = _kv_cache(cache, d)
    if block_table.dtype is not torch.int32 or block_table.dim() != 2:
        raise ValueError("block_table: expected an int32 (sequences, pages) tensor")
    sequences, width = block_table.shape
    table_stride, step = block_table.stride()
    if step != 1 and width > 1:
        raise ValueError("block_table: expected contiguous rows")
    lens = _vector(kv_len, sequences, torch.int32, "kv_len")
    room = width * kv.page
    if max_kv is None:
        max_kv = min(room, 1 << 30)  # (the most that a sequence may have)
    elif max_kv > room:
        raise ValueError("max_kv: block_table has room for %d tokens" % room)
    cu = None
    if cu_q is not None:
        cu = _vector(cu_q, sequences + 1, torch.int32, "cu_q")
        if max_q is None:
            raise ValueError("max_q is needed with cu_q")
    else:
        if tokens != sequences:
            raise ValueError("q: %d rows for %d sequences" % (tokens, sequences))
        max_q = 1
    _int32(max_q=max_q, max_kv=max_kv, window=window)
    _same_device(cache, q, block_table, kv_len, cu_q, workspace)
    y = lse = None
    if out:
        y, lse = out.get("out"), out.get("lse")
        if lse is not None and (lse.shape != (tokens, heads_q) or lse.dtype is not torch.float32 or not lse.is_contiguous()):
            raise ValueError("lse: expected a contiguous float32 (tokens, heads_q) tensor")
        _same_device(cache, y, lse)
    out = dict(out) if out else {}
    if y is None:
        y = out["out"] = _new_like(q, stream)
        out_token, out_head = heads_q * d, d
    else:
        out_token, out_head = _heads_strides(y, "out", q.shape, q.dtype)
    if want_lse and lse is None:
        lse = out["lse"] = _new(q, (tokens, heads_q), torch.float32, stream)
    att = Attention(kv, sequences, tokens, heads_q, dtype, 1 if causal else 0, window, d ** -0.5 if scale is None else scale, max_q, max_kv,
                    q.data_ptr(), y.data_ptr(), _ptr(lse), q_token, q_head, out_token, out_head, cu, lens, block_table.data_ptr(),
                    table_stride)
    _on_gpu(cache)
    need = lib.ttc_attention_workspace_bytes(att)
    if need and workspace is None:
        workspace = _new(q, (need,), torch.uint8, stream)
    _check(lib.ttc_attention(att, _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream_ptr(stream)))
    return out
