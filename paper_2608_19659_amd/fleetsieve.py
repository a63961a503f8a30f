"""Thin ctypes binding of libfleetsieve (C ABI in include/fleetsieve.h).

Argument marshalling only: every step runs in the HIP library.  Device
arrays are torch tensors on a ROCm device (torch supplies memory and the
current stream); the problem statement is host data.  There is no fallback:
if ``libfleetsieve.so`` is missing or the device is not gfx950 the calls
raise.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
# FLEETSIEVE_LIB selects another build of the library (for example one whose
# host code is compiled with sanitizers); the default is the in-tree build.
LIB_PATH = os.environ.get("FLEETSIEVE_LIB") or os.path.join(_HERE, "libfleetsieve.so")

FS_OK, FS_ERR_INVALID_ARGUMENT, FS_ERR_UNSUPPORTED, FS_ERR_WORKSPACE_TOO_SMALL, FS_ERR_DEVICE, \
    FS_ERR_INTERNAL = range(6)
UNDECIDED, CERTIFIED_FEASIBLE, CERTIFIED_INFEASIBLE = 0, 1, 2
TP_NONE = 0xFF
OPT_SCORE_KERNEL = 1
OPT_KERNEL_TIMING = 2
OPT_SAMPLES_PER_LANE = 3
OPT_SCORER_WAVES = 5
OPT_SETUP = 6
OPT_LOOP_OBJECTIVE = 7
OPT_LOOP_REFIT = 8
OPT_THRESHOLD_SEARCH = 9
OPT_ATTENTION_KERNEL = 10
OBJECTIVE_MAXMIN, OBJECTIVE_LEXICOGRAPHIC = 0, 1
KERNEL_AUTO, KERNEL_WAVE, KERNEL_LANE, KERNEL_EXCLUSION = 0, 1, 2, 3

EXPORTED = ("fs_context_create", "fs_context_destroy", "fs_context_set_option", "fs_context_kernel_timing",
            "fs_last_error",
            "fs_validate_problem", "fs_workspace_size", "fs_solve_batch", "fs_score_candidates",
            "fs_certify", "fs_loop_workspace_size", "fs_profile_loop", "fs_reduce_cells", "fs_reduce_samples",
            "fs_solve_batch_lex", "fs_certify_lex", "fs_refit_intervals", "fs_loop_refit_workspace_size",
            "fs_score_lex_workspace_size", "fs_score_candidates_lex", "fs_clamp_samples",
            "fs_score_candidates_noalloc", "fs_quantize_rows", "fs_scaled_matmul_workspace_size", "fs_scaled_matmul",
            "fs_linear_workspace_size", "fs_linear", "fs_project_workspace_size", "fs_project",
            "fs_gated_project_workspace_size", "fs_gated_project", "fs_cache_append", "fs_cache_read",
            "fs_cache_attention_workspace_size", "fs_cache_attention", "fs_state_attention_workspace_size",
            "fs_state_attention")
POLICY_SCORE, POLICY_ORDER = 0, 1
CELL_SECONDS = 300.0


class FleetSieveError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"libfleetsieve status {status}: {message}")
        self.status = status


class _Problem(ctypes.Structure):
    _fields_ = [("n_classes", ctypes.c_int32), ("n_tp", ctypes.c_int32),
                ("n_levels", ctypes.c_int32), ("budget", ctypes.c_int32),
                ("tp", ctypes.c_void_p), ("levels", ctypes.c_void_p),
                ("demand", ctypes.c_void_p), ("slo", ctypes.c_void_p),
                ("floor_rps", ctypes.c_void_p)]


class _Intervals(ctypes.Structure):
    _fields_ = [("cap_lo", ctypes.c_void_p), ("cap_hi", ctypes.c_void_p),
                ("tail_lo", ctypes.c_void_p), ("tail_hi", ctypes.c_void_p),
                ("measured", ctypes.c_void_p)]


class _Alloc(ctypes.Structure):
    _fields_ = [("objective", ctypes.c_void_p), ("tp_index", ctypes.c_void_p),
                ("replicas", ctypes.c_void_p), ("floors_met", ctypes.c_void_p),
                ("goodput", ctypes.c_void_p)]


class _SloPolicy(ctypes.Structure):
    _fields_ = [("n_metrics", ctypes.c_int32), ("limit", ctypes.c_void_p), ("success_min", ctypes.c_void_p)]


class _LoopOut(ctypes.Structure):
    _fields_ = [("state", ctypes.c_void_p), ("finished", ctypes.c_void_p), ("rounds", ctypes.c_void_p),
                ("gpu_seconds", ctypes.c_void_p), ("reveals", ctypes.c_void_p), ("final_alloc", _Alloc),
                ("tau_truth", ctypes.c_void_p), ("tau_oracle", ctypes.c_void_p)]


_lib = None


def load_library():
    """Load libfleetsieve.so; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FleetSieveError(FS_ERR_INTERNAL, f"{LIB_PATH} is not built (run __graft_entry__.build())")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    P = ctypes.POINTER(_Problem)
    lib.fs_context_create.argtypes = [ctypes.c_int, ctypes.POINTER(vp)]
    lib.fs_context_destroy.argtypes = [vp]
    lib.fs_context_destroy.restype = None
    lib.fs_context_set_option.argtypes = [vp, ctypes.c_int, i64]
    lib.fs_context_kernel_timing.argtypes = [vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(i64)]
    lib.fs_last_error.restype = ctypes.c_char_p
    lib.fs_validate_problem.argtypes = [P]
    lib.fs_workspace_size.argtypes = [P, i32, i32, i32, ctypes.POINTER(sz)]
    lib.fs_solve_batch.argtypes = [vp, P, vp, vp, i64, _Alloc, vp, sz, vp]
    lib.fs_score_candidates.argtypes = [vp, P, _Intervals, i32, vp, i32, vp, vp, i32, vp, vp, vp, vp,
                                        vp, sz, vp]
    lib.fs_certify.argtypes = [vp, P, _Intervals, i32, ctypes.c_float, vp, _Alloc, _Alloc, vp, vp, sz, vp]
    lib.fs_loop_workspace_size.argtypes = [P, i32, i32, i32, ctypes.POINTER(sz)]
    lib.fs_profile_loop.argtypes = [vp, P, _Intervals, i32, vp, vp, vp, i32, vp, vp, i32, ctypes.c_float,
                                    ctypes.c_int, vp, i32, i32, _LoopOut, vp, sz, vp]
    lib.fs_score_lex_workspace_size.argtypes = [P, i32, i32, i32, ctypes.POINTER(sz)]
    lib.fs_score_candidates_lex.argtypes = [vp, P, _Intervals, i32, vp, i32, vp, vp, i32, vp, vp, vp, vp, vp, vp,
                                            sz, vp]
    lib.fs_refit_intervals.argtypes = [vp, P, _Intervals, i32, vp, vp, vp, vp]
    lib.fs_loop_refit_workspace_size.argtypes = [P, i32, i32, i32, ctypes.POINTER(sz)]
    lib.fs_clamp_samples.argtypes = [vp, P, _Intervals, i32, vp, i32, vp, vp, i32, vp, vp, vp]
    lib.fs_score_candidates_noalloc.argtypes = [vp, P, _Intervals, i32, vp, i32, vp, vp, i32, vp, vp, vp, vp, vp]
    lib.fs_solve_batch_lex.argtypes = [vp, P, vp, vp, i64, _Alloc, vp, vp, sz, vp]
    lib.fs_certify_lex.argtypes = [vp, P, _Intervals, i32, ctypes.c_float, vp, _Alloc, _Alloc, vp, vp, vp, sz, vp]
    Q = ctypes.POINTER(_SloPolicy)
    lib.fs_reduce_cells.argtypes = [vp, P, Q, vp, vp, i64, vp, vp]
    lib.fs_reduce_samples.argtypes = [vp, P, Q, vp, i32, vp, vp, i32, i32, vp, vp]
    C = ctypes.POINTER(_Cache)
    psz = ctypes.POINTER(sz)
    lib.fs_quantize_rows.argtypes = [vp, vp, i32, i64, i64, i64, vp, i64, vp, vp]
    lib.fs_scaled_matmul_workspace_size.argtypes = [i64, i64, i64, psz]
    lib.fs_scaled_matmul.argtypes = [vp, vp, i64, vp, vp, i64, vp, vp, i64, i64, i64, vp, i32, i64, vp, sz, vp]
    lib.fs_linear_workspace_size.argtypes = [i64, i64, i64, psz]
    lib.fs_linear.argtypes = [vp, vp, i32, i64, vp, i64, vp, vp, i64, i64, i64, vp, i32, i64, vp, sz, vp]
    lib.fs_state_attention_workspace_size.argtypes = [vp, i32, i64, i32, psz]
    lib.fs_state_attention.argtypes = [vp, vp, vp, i64, vp, i64, vp, i64, i32, i32, i64, i32, vp, vp, vp, i32, vp,
                                       ctypes.c_float, vp, vp, sz, vp]
    lib.fs_project_workspace_size.argtypes = lib.fs_gated_project_workspace_size.argtypes = [i64, i64, i64, psz]
    lib.fs_project.argtypes = [vp, vp, i32, i64, vp, vp, i64, vp, vp, i32, vp, i64, i64, i64, i64, vp, i32, i64, vp, sz, vp]
    lib.fs_gated_project.argtypes = [vp, vp, i32, i64, vp, vp, i64, vp, vp, i32, i64, i64, i64, vp, i32, i64, vp, sz, vp]
    lib.fs_cache_append.argtypes = [vp, C, vp, i64, vp, i64, vp, i64, i32, i32, i64, vp, vp, vp, vp, i32, i32, vp, vp]
    lib.fs_cache_read.argtypes = [vp, C, i64, vp, vp, vp, i32, vp]
    lib.fs_cache_attention_workspace_size.argtypes = [C, i32, i64, i32, psz]
    lib.fs_cache_attention.argtypes = [vp, C, vp, i64, i32, i32, i64, i32, vp, vp, vp, i64, i32, ctypes.c_float, i32,
                                       vp, vp, sz, vp]
    for name in EXPORTED:
        if name != "fs_context_destroy":
            getattr(lib, name).restype = ctypes.c_int
    lib.fs_last_error.restype = ctypes.c_char_p
    _lib = lib
    return lib


def _check(status: int):
    if status != FS_OK:
        msg = load_library().fs_last_error()
        raise FleetSieveError(status, msg.decode() if msg else "")


class _ProblemRef:
    """Host copy of a problem statement kept alive for the duration of a call."""

    def __init__(self, problem):
        self.tp = np.ascontiguousarray(problem.tp, dtype=np.int32)
        self.levels = np.ascontiguousarray(problem.levels, dtype=np.float32)
        self.demand = np.ascontiguousarray(problem.demand, dtype=np.float32)
        self.slo = np.ascontiguousarray(problem.slo, dtype=np.float32)
        fl = getattr(problem, "floor_rps", None)
        self.floor = None if fl is None else np.ascontiguousarray(fl, dtype=np.float32)
        self.K, self.NT, self.B = len(self.demand), len(self.tp), len(self.levels)
        self.N = self.K * self.NT * self.B
        self.s = _Problem(self.K, self.NT, self.B, int(problem.budget),
                          self.tp.ctypes.data, self.levels.ctypes.data, self.demand.ctypes.data,
                          self.slo.ctypes.data, None if self.floor is None else self.floor.ctypes.data)

    @property
    def ptr(self):
        return ctypes.byref(self.s)


def _torch():
    import torch
    return torch


def _dev_ptr(t, dtype, shape=None, name="array"):
    torch = _torch()
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise FleetSieveError(FS_ERR_INVALID_ARGUMENT, f"{name} must be a torch tensor on a ROCm device")
    if t.dtype != dtype:
        raise FleetSieveError(FS_ERR_INVALID_ARGUMENT, f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise FleetSieveError(FS_ERR_INVALID_ARGUMENT, f"{name} must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise FleetSieveError(FS_ERR_INVALID_ARGUMENT, f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    return t.data_ptr()


def _stream(device, stream):
    torch = _torch()
    s = stream if stream is not None else torch.cuda.current_stream(device)
    return ctypes.c_void_p(s.cuda_stream)


class Context:
    """A libfleetsieve context on one HIP device."""

    def __init__(self, device: int = 0):
        lib = load_library()
        h = ctypes.c_void_p()
        _check(lib.fs_context_create(int(device), ctypes.byref(h)))
        self.handle = h
        self.device = int(device)
        self._ws = None

    def set_option(self, option: int, value: int):
        _check(load_library().fs_context_set_option(self.handle, int(option), int(value)))

    def set_score_kernel(self, kernel: int):
        self.set_option(OPT_SCORE_KERNEL, kernel)

    def kernel_timing(self):
        """(total milliseconds, launches) of the scoring kernel since the
        last query; needs set_option(OPT_KERNEL_TIMING, n), which launches
        it n times back to back between each pair of events."""
        ms, n = ctypes.c_double(), ctypes.c_int64()
        _check(load_library().fs_context_kernel_timing(self.handle, ctypes.byref(ms), ctypes.byref(n)))
        return float(ms.value), int(n.value)

    def close(self):
        if self.handle:
            load_library().fs_context_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def workspace(self, nbytes: int):
        """A device workspace of at least nbytes, reused across calls that
        run on the same stream."""
        torch = _torch()
        if self._ws is None or self._ws.numel() < nbytes:
            self._ws = torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=f"cuda:{self.device}")
        return self._ws


def validate_problem(problem):
    ref = _ProblemRef(problem)
    _check(load_library().fs_validate_problem(ref.ptr))


def workspace_size(problem, n_orders: int = 0, n_cand: int = 0, n_samples: int = 0) -> int:
    ref = _ProblemRef(problem)
    out = ctypes.c_size_t()
    _check(load_library().fs_workspace_size(ref.ptr, int(n_orders), int(n_cand), int(n_samples),
                                            ctypes.byref(out)))
    return int(out.value)


def _alloc_tensors(n, K, device):
    torch = _torch()
    return dict(objective=torch.empty(n, dtype=torch.float32, device=device),
                tp_index=torch.empty((n, K), dtype=torch.uint8, device=device),
                replicas=torch.empty((n, K), dtype=torch.int16, device=device),
                floors_met=torch.empty(n, dtype=torch.uint8, device=device),
                goodput=torch.empty(n, dtype=torch.float32, device=device))


def _alloc_struct(d):
    return _Alloc(d["objective"].data_ptr(), d["tp_index"].data_ptr(), d["replicas"].data_ptr(),
                  d["floors_met"].data_ptr(), d["goodput"].data_ptr())


def solve_batch(ctx: Context, problem, cap, tail, stream=None, workspace=None):
    """Dense batch solve; cap, tail are float32 [n, N] device tensors.
    Returns a dict of device tensors (objective, tp_index, replicas,
    floors_met, goodput); replicas are uint16 values stored as int16."""
    torch = _torch()
    ref = _ProblemRef(problem)
    n = int(cap.shape[0]) if cap.dim() == 2 else 0
    pc = _dev_ptr(cap, torch.float32, (n, ref.N), "cap")
    pt = _dev_ptr(tail, torch.float32, (n, ref.N), "tail")
    out = _alloc_tensors(n, ref.K, cap.device)
    ws_bytes = workspace_size(problem)
    ws = workspace if workspace is not None else ctx.workspace(ws_bytes)
    _check(load_library().fs_solve_batch(ctx.handle, ref.ptr, pc, pt, n, _alloc_struct(out), ws.data_ptr(),
                                         ws.numel(), _stream(cap.device, stream)))
    return out


def solve_batch_lex(ctx: Context, problem, cap, tail, stream=None, workspace=None):
    """Dense batch solve under the whole lexicographic objective (levels
    1-4, fs_solve_batch_lex).  As solve_batch, plus goodput64: level (3)'s
    binary64 total per scenario."""
    torch = _torch()
    ref = _ProblemRef(problem)
    n = int(cap.shape[0]) if cap.dim() == 2 else 0
    pc = _dev_ptr(cap, torch.float32, (n, ref.N), "cap")
    pt = _dev_ptr(tail, torch.float32, (n, ref.N), "tail")
    out = _alloc_tensors(n, ref.K, cap.device)
    out["goodput64"] = torch.empty(n, dtype=torch.float64, device=cap.device)
    ws_bytes = workspace_size(problem)
    ws = workspace if workspace is not None else ctx.workspace(ws_bytes)
    _check(load_library().fs_solve_batch_lex(ctx.handle, ref.ptr, pc, pt, n, _alloc_struct(out),
                                             out["goodput64"].data_ptr(), ws.data_ptr(), ws.numel(),
                                             _stream(cap.device, stream)))
    return out


@dataclass
class DeviceIntervals:
    cap_lo: object
    cap_hi: object
    tail_lo: object
    tail_hi: object
    measured: object

    @staticmethod
    def from_host(iv, device):
        torch = _torch()
        return DeviceIntervals(*(torch.from_numpy(np.ascontiguousarray(a)).to(device)
                                 for a in (iv.cap_lo, iv.cap_hi, iv.tail_lo, iv.tail_hi, iv.measured)))


def _intervals_struct(iv, O, N):
    torch = _torch()
    return _Intervals(_dev_ptr(iv.cap_lo, torch.float32, (O, N), "cap_lo"),
                      _dev_ptr(iv.cap_hi, torch.float32, (O, N), "cap_hi"),
                      _dev_ptr(iv.tail_lo, torch.float32, (O, N), "tail_lo"),
                      _dev_ptr(iv.tail_hi, torch.float32, (O, N), "tail_hi"),
                      _dev_ptr(iv.measured, torch.uint8, (O, N), "measured"))


@dataclass
class ScoreOutput:
    score: object     # [O, E] float64
    gap_now: object   # [O] float64
    best: object      # [O] int32
    tau_dump: object  # [O, E, S, 2] float32 or None


class ScorePlan:
    """One fs_score_candidates call with its arguments checked and
    marshalled once.  run() enqueues the call again on the same device
    buffers (whose contents may change between runs); every run executes the
    whole scoring path on the GPU.  iv holds [O, N] device tensors, cand an
    int32 [E] device tensor, cap_s / tail_s float32 [O, E, S] device tensors."""

    def __init__(self, ctx: Context, problem, iv: DeviceIntervals, cand, cap_s, tail_s, dump: bool = False,
                 stream=None, workspace=None, out: ScoreOutput | None = None):
        torch = _torch()
        self._ref = _ProblemRef(problem)
        O = int(iv.cap_lo.shape[0])
        E = int(cand.shape[0])
        S = int(cap_s.shape[2]) if E > 0 else 0
        dev = iv.cap_lo.device
        self._ivs = _intervals_struct(iv, O, self._ref.N)
        pcand = _dev_ptr(cand, torch.int32, (E,), "cand")
        pcs = _dev_ptr(cap_s, torch.float32, (O, E, S), "cap_s")
        pts = _dev_ptr(tail_s, torch.float32, (O, E, S), "tail_s")
        if out is None:
            out = ScoreOutput(torch.empty((O, E), dtype=torch.float64, device=dev),
                              torch.empty(O, dtype=torch.float64, device=dev),
                              torch.empty(O, dtype=torch.int32, device=dev),
                              torch.empty((O, E, S, 2), dtype=torch.float32, device=dev) if dump else None)
        ws_bytes = workspace_size(problem, O, E, S)
        ws = workspace if workspace is not None else ctx.workspace(ws_bytes)
        self.out, self._ws, self._keep = out, ws, (iv, cand, cap_s, tail_s)
        self._fn = load_library().fs_score_candidates
        self._args = (ctx.handle, self._ref.ptr, self._ivs, O, pcand, E, pcs, pts, S,
                      _dev_ptr(out.score, torch.float64, (O, E), "score"),
                      _dev_ptr(out.gap_now, torch.float64, (O,), "gap_now"),
                      _dev_ptr(out.best, torch.int32, (O,), "best"),
                      _dev_ptr(out.tau_dump, torch.float32, (O, E, S, 2), "tau_dump"),
                      ws.data_ptr(), ws.numel(), _stream(dev, stream))

    def run(self) -> ScoreOutput:
        _check(self._fn(*self._args))
        return self.out


NOALLOC_SCRATCH_BYTES = 32 << 20


def score_candidates_noalloc(ctx: Context, problem, iv: DeviceIntervals, cand, cap_s, tail_s,
                             out: "ScoreOutput", stream=None) -> "ScoreOutput":
    """fs_score_candidates_noalloc: the scorer without a workspace (the
    library's static device scratch); the caller passes the outputs."""
    torch = _torch()
    ref = _ProblemRef(problem)
    O = int(iv.cap_lo.shape[0])
    E = int(cand.shape[0])
    S = int(cap_s.shape[2]) if E > 0 else 0
    ivs = _intervals_struct(iv, O, ref.N)
    _check(load_library().fs_score_candidates_noalloc(
        ctx.handle, ref.ptr, ivs, O, _dev_ptr(cand, torch.int32, (E,), "cand"),
        E, _dev_ptr(cap_s, torch.float32, (O, E, S), "cap_s"), _dev_ptr(tail_s, torch.float32, (O, E, S), "tail_s"),
        S, _dev_ptr(out.score, torch.float64, (O, E), "score"), _dev_ptr(out.gap_now, torch.float64, (O,), "gap_now"),
        _dev_ptr(out.best, torch.int32, (O,), "best"), _dev_ptr(out.tau_dump, torch.float32, (O, E, S, 2), "tau_dump"),
        _stream(iv.cap_lo.device, stream)))
    return out


def score_candidates(ctx: Context, problem, iv: DeviceIntervals, cand, cap_s, tail_s, dump: bool = False,
                     stream=None, workspace=None, out: ScoreOutput | None = None) -> ScoreOutput:
    """Acquisition scores (fs_score_candidates), one call."""
    return ScorePlan(ctx, problem, iv, cand, cap_s, tail_s, dump, stream, workspace, out).run()


@dataclass
class CertifyOutput:
    state: object
    gap: object
    cons: dict
    opt: dict


def certify(ctx: Context, problem, iv: DeviceIntervals, eps: float = 0.05, stream=None,
            workspace=None) -> CertifyOutput:
    torch = _torch()
    ref = _ProblemRef(problem)
    O = int(iv.cap_lo.shape[0])
    dev = iv.cap_lo.device
    ivs = _intervals_struct(iv, O, ref.N)
    state = torch.empty(O, dtype=torch.int32, device=dev)
    gap = torch.empty(O, dtype=torch.float64, device=dev)
    cons = _alloc_tensors(O, ref.K, dev)
    opt = _alloc_tensors(O, ref.K, dev)
    ws_bytes = workspace_size(problem, O)
    ws = workspace if workspace is not None else ctx.workspace(ws_bytes)
    _check(load_library().fs_certify(ctx.handle, ref.ptr, ivs, O, float(eps), state.data_ptr(),
                                     _alloc_struct(cons), _alloc_struct(opt), gap.data_ptr(), ws.data_ptr(),
                                     ws.numel(), _stream(dev, stream)))
    return CertifyOutput(state, gap, cons, opt)


@dataclass
class CertifyLexOutput:
    state: object
    gap_maxmin: object   # [O] float64, tau+ - tau-
    gap_goodput: object  # [O] float64, |gp+ - gp-| / max(gp+, gp-)
    cons: dict
    opt: dict


def certify_lex(ctx: Context, problem, iv: DeviceIntervals, eps: float = 0.05, stream=None,
                workspace=None) -> CertifyLexOutput:
    """Certificate with the stage-wise gap under the whole objective
    (fs_certify_lex)."""
    torch = _torch()
    ref = _ProblemRef(problem)
    O = int(iv.cap_lo.shape[0])
    dev = iv.cap_lo.device
    ivs = _intervals_struct(iv, O, ref.N)
    state = torch.empty(O, dtype=torch.int32, device=dev)
    gmm = torch.empty(O, dtype=torch.float64, device=dev)
    ggp = torch.empty(O, dtype=torch.float64, device=dev)
    cons = _alloc_tensors(O, ref.K, dev)
    opt = _alloc_tensors(O, ref.K, dev)
    ws_bytes = workspace_size(problem, O)
    ws = workspace if workspace is not None else ctx.workspace(ws_bytes)
    _check(load_library().fs_certify_lex(ctx.handle, ref.ptr, ivs, O, float(eps), state.data_ptr(),
                                         _alloc_struct(cons), _alloc_struct(opt), gmm.data_ptr(), ggp.data_ptr(),
                                         ws.data_ptr(), ws.numel(), _stream(dev, stream)))
    return CertifyLexOutput(state, gmm, ggp, cons, opt)


@dataclass
class ScoreLexOutput:
    score_maxmin: object   # [O, E] float64
    score_goodput: object  # [O, E] float64
    gap_maxmin: object     # [O] float64
    gap_goodput: object    # [O] float64
    best: object           # [O] int32


def score_lex_workspace_size(problem, n_orders: int, n_cand: int, n_samples: int) -> int:
    ref = _ProblemRef(problem)
    out = ctypes.c_size_t()
    _check(load_library().fs_score_lex_workspace_size(ref.ptr, int(n_orders), int(n_cand), int(n_samples),
                                                      ctypes.byref(out)))
    return int(out.value)


class ScoreLexPlan:
    """One fs_score_candidates_lex call with its arguments checked and
    marshalled once; run() enqueues the call again on the same device
    buffers.  Shapes as in ScorePlan."""

    def __init__(self, ctx: Context, problem, iv: DeviceIntervals, cand, cap_s, tail_s, stream=None,
                 workspace=None):
        torch = _torch()
        self._ref = _ProblemRef(problem)
        O = int(iv.cap_lo.shape[0])
        E = int(cand.shape[0])
        S = int(cap_s.shape[2]) if E > 0 else 0
        dev = iv.cap_lo.device
        self._ivs = _intervals_struct(iv, O, self._ref.N)
        pcand = _dev_ptr(cand, torch.int32, (E,), "cand")
        pcs = _dev_ptr(cap_s, torch.float32, (O, E, S), "cap_s")
        pts = _dev_ptr(tail_s, torch.float32, (O, E, S), "tail_s")
        out = ScoreLexOutput(torch.empty((O, E), dtype=torch.float64, device=dev),
                             torch.empty((O, E), dtype=torch.float64, device=dev),
                             torch.empty(O, dtype=torch.float64, device=dev),
                             torch.empty(O, dtype=torch.float64, device=dev),
                             torch.empty(O, dtype=torch.int32, device=dev))
        ws_bytes = score_lex_workspace_size(problem, O, E, S)
        ws = workspace if workspace is not None else ctx.workspace(ws_bytes)
        self.out, self._ws, self._keep = out, ws, (iv, cand, cap_s, tail_s)
        self._fn = load_library().fs_score_candidates_lex
        self._args = (ctx.handle, self._ref.ptr, self._ivs, O, pcand, E, pcs, pts, S,
                      out.score_maxmin.data_ptr(), out.score_goodput.data_ptr(), out.gap_maxmin.data_ptr(),
                      out.gap_goodput.data_ptr(), out.best.data_ptr(), ws.data_ptr(), ws.numel(),
                      _stream(dev, stream))

    def run(self) -> ScoreLexOutput:
        _check(self._fn(*self._args))
        return self.out


def score_candidates_lex(ctx: Context, problem, iv: DeviceIntervals, cand, cap_s, tail_s, stream=None,
                         workspace=None) -> ScoreLexOutput:
    """The stage-wise score under the whole objective
    (fs_score_candidates_lex); shapes as in score_candidates."""
    return ScoreLexPlan(ctx, problem, iv, cand, cap_s, tail_s, stream, workspace).run()


def refit_intervals(ctx: Context, problem, iv: DeviceIntervals, stream=None) -> DeviceIntervals:
    """Algorithm 1's fit step (fs_refit_intervals) on [O, N] device
    intervals; returns new intervals (cap_hi and measured shared with iv)."""
    torch = _torch()
    ref = _ProblemRef(problem)
    O = int(iv.cap_lo.shape[0])
    ivs = _intervals_struct(iv, O, ref.N)
    out = DeviceIntervals(torch.empty_like(iv.cap_lo), iv.cap_hi, torch.empty_like(iv.tail_lo),
                          torch.empty_like(iv.tail_hi), iv.measured)
    _check(load_library().fs_refit_intervals(ctx.handle, ref.ptr, ivs, O, out.cap_lo.data_ptr(),
                                             out.tail_lo.data_ptr(), out.tail_hi.data_ptr(),
                                             _stream(iv.cap_lo.device, stream)))
    return out


def clamp_samples(ctx: Context, problem, iv: DeviceIntervals, cand, cap_s, tail_s, stream=None):
    """The candidates' samples clamped into their current intervals
    (fs_clamp_samples); returns new (cap_s, tail_s) tensors [O, E, S]."""
    torch = _torch()
    ref = _ProblemRef(problem)
    O = int(iv.cap_lo.shape[0])
    E = int(cand.shape[0])
    S = int(cap_s.shape[2]) if E > 0 else 0
    ivs = _intervals_struct(iv, O, ref.N)
    pcand = _dev_ptr(cand, torch.int32, (E,), "cand")
    pcs = _dev_ptr(cap_s, torch.float32, (O, E, S), "cap_s")
    pts = _dev_ptr(tail_s, torch.float32, (O, E, S), "tail_s")
    cs_out, ts_out = torch.empty_like(cap_s), torch.empty_like(tail_s)
    _check(load_library().fs_clamp_samples(ctx.handle, ref.ptr, ivs, O, pcand, E, pcs, pts, S, cs_out.data_ptr(),
                                           ts_out.data_ptr(), _stream(iv.cap_lo.device, stream)))
    return cs_out, ts_out


def loop_refit_workspace_size(problem, n_orders: int, n_cand: int, n_samples: int) -> int:
    ref = _ProblemRef(problem)
    out = ctypes.c_size_t()
    _check(load_library().fs_loop_refit_workspace_size(ref.ptr, int(n_orders), int(n_cand), int(n_samples),
                                                       ctypes.byref(out)))
    return int(out.value)


def loop_workspace_size(problem, n_orders: int, n_cand: int, n_samples: int) -> int:
    ref = _ProblemRef(problem)
    out = ctypes.c_size_t()
    _check(load_library().fs_loop_workspace_size(ref.ptr, int(n_orders), int(n_cand), int(n_samples),
                                                 ctypes.byref(out)))
    return int(out.value)


@dataclass
class LoopOutput:
    state: object        # [O] int32
    finished: object     # [O] uint8
    rounds: object       # [O] int32
    gpu_seconds: object  # [O] float64
    reveals: object      # [O, max_rounds] int32
    final: dict          # [O] allocation tensors (objective, tp_index, replicas, floors_met, goodput)
    tau_truth: object    # [O] float32
    tau_oracle: object   # [O] float32


def profile_loop(ctx: Context, problem, iv: DeviceIntervals, truth_cap, truth_tail, cand, cap_s, tail_s,
                 eps: float = 0.05, policy: int = POLICY_SCORE, order=None, max_rounds: int | None = None,
                 check_every: int = 4, stream=None, workspace=None, refit: bool = False) -> LoopOutput:
    """The profiling loop (fs_profile_loop) for O trajectories.  iv holds
    the initial designs [O, N]; truth_cap / truth_tail are float32 [O, N]
    device tensors; order is an int32 [O, E] device tensor (policy
    POLICY_ORDER) or None.  max_rounds defaults to E."""
    torch = _torch()
    ref = _ProblemRef(problem)
    O = int(iv.cap_lo.shape[0])
    E = int(cand.shape[0])
    S = int(cap_s.shape[2]) if (E > 0 and policy == POLICY_SCORE) else 0
    R = E if max_rounds is None else int(max_rounds)
    dev = iv.cap_lo.device
    ivs = _intervals_struct(iv, O, ref.N)
    ptc = _dev_ptr(truth_cap, torch.float32, (O, ref.N), "truth_cap")
    ptt = _dev_ptr(truth_tail, torch.float32, (O, ref.N), "truth_tail")
    pcand = _dev_ptr(cand, torch.int32, (E,), "cand")
    pcs = _dev_ptr(cap_s, torch.float32, (O, E, S), "cap_s") if S else None
    pts = _dev_ptr(tail_s, torch.float32, (O, E, S), "tail_s") if S else None
    pord = _dev_ptr(order, torch.int32, (O, E), "order") if order is not None else None
    out = LoopOutput(torch.empty(O, dtype=torch.int32, device=dev), torch.empty(O, dtype=torch.uint8, device=dev),
                     torch.empty(O, dtype=torch.int32, device=dev), torch.empty(O, dtype=torch.float64, device=dev),
                     torch.empty((O, R), dtype=torch.int32, device=dev), _alloc_tensors(O, ref.K, dev),
                     torch.empty(O, dtype=torch.float32, device=dev), torch.empty(O, dtype=torch.float32, device=dev))
    lo = _LoopOut(out.state.data_ptr(), out.finished.data_ptr(), out.rounds.data_ptr(), out.gpu_seconds.data_ptr(),
                  out.reveals.data_ptr() if R > 0 else None, _alloc_struct(out.final), out.tau_truth.data_ptr(),
                  out.tau_oracle.data_ptr())
    ws_bytes = (loop_refit_workspace_size if refit else loop_workspace_size)(problem, O, E, S)
    ws = workspace if workspace is not None else ctx.workspace(ws_bytes)
    ctx.set_option(OPT_LOOP_REFIT, 1 if refit else 0)
    _check(load_library().fs_profile_loop(ctx.handle, ref.ptr, ivs, O, ptc, ptt, pcand, E, pcs, pts, S,
                                          float(eps), int(policy), pord, R, int(check_every), lo, ws.data_ptr(),
                                          ws.numel(), _stream(dev, stream)))
    return out


class _PolicyRef:
    """Host copy of a class policy (limit [K][M], success_min [K] or None)."""

    def __init__(self, policy, K):
        self.limit = np.ascontiguousarray(np.asarray(policy.limit, dtype=np.float32).reshape(K, -1))
        sm = getattr(policy, "success_min", None)
        self.smin = None if sm is None else np.ascontiguousarray(sm, dtype=np.float32)
        self.M = int(self.limit.shape[1])
        self.s = _SloPolicy(self.M, self.limit.ctypes.data, None if self.smin is None else self.smin.ctypes.data)

    @property
    def ptr(self):
        return ctypes.byref(self.s)


class ReducePlan:
    """One fs_reduce_cells or fs_reduce_samples call with its arguments
    checked and marshalled once; run() enqueues it again on the same device
    buffers."""

    def __init__(self, fn, args, out, keep):
        self._fn, self._args, self.out, self._keep = fn, args, out, keep

    def run(self):
        _check(self._fn(*self._args))
        return self.out

    @staticmethod
    def cells(ctx: Context, problem, policy, tails, success=None, out=None, stream=None) -> "ReducePlan":
        """tails float32 [R, N, M], success float32 [R, N] or None, out [R, N]."""
        torch = _torch()
        ref = _ProblemRef(problem)
        pol = _PolicyRef(policy, ref.K)
        R = int(tails.shape[0])
        dev = tails.device
        pt = _dev_ptr(tails, torch.float32, (R, ref.N, pol.M), "tails")
        ps = _dev_ptr(success, torch.float32, (R, ref.N), "success") if success is not None else None
        if out is None:
            out = torch.empty((R, ref.N), dtype=torch.float32, device=dev)
        po = _dev_ptr(out, torch.float32, (R, ref.N), "out")
        return ReducePlan(load_library().fs_reduce_cells,
                          (ctx.handle, ref.ptr, pol.ptr, pt, ps, R, po, _stream(dev, stream)),
                          out, (ref, pol, tails, success))

    @staticmethod
    def samples(ctx: Context, problem, policy, cand, tail_s, succ_s=None, out=None, stream=None) -> "ReducePlan":
        """cand int32 [E], tail_s float32 [O, E, S, M], succ_s [O, E, S] or None, out [O, E, S]."""
        torch = _torch()
        ref = _ProblemRef(problem)
        pol = _PolicyRef(policy, ref.K)
        O, E, S = (int(x) for x in tail_s.shape[:3])
        dev = tail_s.device
        pc = _dev_ptr(cand, torch.int32, (E,), "cand")
        pt = _dev_ptr(tail_s, torch.float32, (O, E, S, pol.M), "tail_s")
        ps = _dev_ptr(succ_s, torch.float32, (O, E, S), "succ_s") if succ_s is not None else None
        if out is None:
            out = torch.empty((O, E, S), dtype=torch.float32, device=dev)
        po = _dev_ptr(out, torch.float32, (O, E, S), "out")
        return ReducePlan(load_library().fs_reduce_samples,
                          (ctx.handle, ref.ptr, pol.ptr, pc, E, pt, ps, O, S, po, _stream(dev, stream)),
                          out, (ref, pol, cand, tail_s, succ_s))


def reduce_cells(ctx: Context, problem, policy, tails, success=None, out=None, stream=None):
    """Pseudo-tails of cells under a class policy (fs_reduce_cells): tails is
    a float32 [R, N, M] device tensor, success float32 [R, N] or None;
    returns float32 [R, N] holding 0 (feasible) or +inf."""
    return ReducePlan.cells(ctx, problem, policy, tails, success, out, stream).run()


def reduce_samples(ctx: Context, problem, policy, cand, tail_s, succ_s=None, out=None, stream=None):
    """Pseudo-tails of candidate samples (fs_reduce_samples): tail_s is a
    float32 [O, E, S, M] device tensor, succ_s float32 [O, E, S] or None;
    returns float32 [O, E, S]."""
    return ReducePlan.samples(ctx, problem, policy, cand, tail_s, succ_s, out, stream).run()


# ------------------------------------------------------- serving operators --
F32, F16, BF16 = 0, 1, 2
MAX_INNER = 131071
MAX_SEQUENCES = 4096


class _Cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("n_pages", ctypes.c_int32), ("n_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("page_size", ctypes.c_int32)]


def _invalid(message):
    return FleetSieveError(FS_ERR_INVALID_ARGUMENT, message)


def _element_type(dtype):
    torch = _torch()
    types = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}
    if dtype not in types:
        raise _invalid(f"elements must be float32, float16 or bfloat16, got {dtype}")
    return types[dtype]


def _rows(t, shape, name, dtype=None):
    """(pointer, stride of the first dimension) of a device tensor of this
    shape (None: any size) whose other dimensions are adjacent in memory."""
    torch = _torch()
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise _invalid(f"{name} must be a torch tensor on a ROCm device")
    if dtype is not None and t.dtype != dtype:
        raise _invalid(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() != len(shape) or any(want is not None and want != got for want, got in zip(shape, t.shape)):
        raise _invalid(f"{name} must have shape {tuple('any' if n is None else n for n in shape)}, got {tuple(t.shape)}")
    step = 1
    for size, stride in zip(reversed(t.shape[1:]), reversed(t.stride()[1:])):
        if size > 1 and stride != step:
            raise _invalid(f"{name} must be contiguous in all but its first dimension")
        step *= size
    # a single row's stride is of no account
    return t.data_ptr(), (int(t.stride(0)) if t.shape[0] > 1 else step)


def _same_device(ctx, **tensors):
    for name, t in tensors.items():
        if getattr(t, "is_cuda", False) and t.device.index != ctx.device:  # what is no device tensor is refused by name
            raise _invalid(f"{name} is on {t.device}, the context on cuda:{ctx.device}")


def _empty(shape, dtype, device, stream):
    """A new output.  For a stream other than the current one its memory is
    that stream's own: what the current one still has to do with memory of its
    own is not waited for."""
    torch = _torch()
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    current = torch.cuda.current_stream(device)
    with torch.cuda.stream(stream):
        out = torch.empty(shape, dtype=dtype, device=device)
    out.record_stream(current)
    return out


def _workspace(ctx, workspace, need, stream):
    torch = _torch()
    if workspace is not None:
        return workspace
    ws = ctx.workspace(need)
    # a larger one may take its place while this stream works on it
    ws.record_stream(stream if stream is not None else torch.cuda.current_stream(ctx.device))
    return ws


def _keep_for(stream, *tensors):
    """Memory given back while `stream` still works on it waits for it."""
    if stream is not None:
        for t in tensors:
            if t is not None:
                t.record_stream(stream)


def quantize_rows(ctx: Context, x, stream=None):
    """(codes int8 [rows, cols], scale float32 [rows]) of a matrix with a
    scale for each row (fs_quantize_rows)."""
    torch = _torch()
    p, stride = _rows(x, (None, None), "x")
    rows, cols = (int(n) for n in x.shape)
    _same_device(ctx, x=x)
    codes = _empty((rows, cols), torch.int8, x.device, stream)
    scale = _empty(rows, torch.float32, x.device, stream)
    _check(load_library().fs_quantize_rows(ctx.handle, p, _element_type(x.dtype), rows, cols, stride, codes.data_ptr(),
                                           cols, scale.data_ptr(), _stream(x.device, stream)))
    _keep_for(stream, x)
    return codes, scale


def _size(fn, *args):
    out = ctypes.c_size_t()
    _check(fn(*args, ctypes.byref(out)))
    return int(out.value)


class _Plan:
    """A call with its arguments checked and marshalled once; run() enqueues
    it again on the same device buffers, whose contents may change between
    runs, and returns its output.  It does so on `stream`, or on the stream that
    is current when the plan is made.  Without a workspace it takes the
    context's, which all its calls share: plans whose runs may overlap need
    workspaces of their own."""

    def run(self):
        _check(self._fn(*self._args))
        return self.out


class MatmulPlan(_Plan):
    """out[m, n] = (sum_k a[m, k] w[n, k]) a_scale[m] w_scale[n] + bias[n]
    (fs_scaled_matmul): a int8 [M, K], w int8 [N, K], float32 scales and bias."""

    def __init__(self, ctx: Context, a, a_scale, w, w_scale, bias=None, out_dtype=None, out=None, stream=None,
                 workspace=None):
        torch = _torch()
        pa, sa = _rows(a, (None, None), "a", torch.int8)
        M, K = (int(n) for n in a.shape)
        pw, sw = _rows(w, (None, K), "w", torch.int8)
        N = int(w.shape[0])
        if out is None:
            out = _empty((M, N), out_dtype or torch.bfloat16, a.device, stream)
        po, so = _rows(out, (M, N), "out", out_dtype)
        lib = load_library()
        need = _size(lib.fs_scaled_matmul_workspace_size, M, N, K)
        ws = _workspace(ctx, workspace, need, stream)
        _same_device(ctx, a=a, a_scale=a_scale, w=w, w_scale=w_scale, bias=bias, out=out, workspace=ws)
        self.out, self._keep = out, (a, a_scale, w, w_scale, bias, ws)
        self._fn = lib.fs_scaled_matmul
        self._args = (ctx.handle, pa, sa, _dev_ptr(a_scale, torch.float32, (M,), "a_scale"), pw, sw,
                      _dev_ptr(w_scale, torch.float32, (N,), "w_scale"), _dev_ptr(bias, torch.float32, (N,), "bias"),
                      M, N, K, po, _element_type(out.dtype), so, _dev_ptr(ws, torch.uint8, None, "workspace"), ws.numel(),
                      _stream(a.device, stream))
        _keep_for(stream, out, *self._keep)


def scaled_matmul(ctx: Context, a, a_scale, w, w_scale, bias=None, out_dtype=None, out=None, stream=None,
                  workspace=None):
    """fs_scaled_matmul, one call (see MatmulPlan)."""
    return MatmulPlan(ctx, a, a_scale, w, w_scale, bias, out_dtype, out, stream, workspace).run()


class LinearPlan(_Plan):
    """A projection in 8-bit integers (fs_linear): x [M, K] is quantised with
    a scale for each row and multiplied by w int8 [N, K] with w_scale [N]."""

    def __init__(self, ctx: Context, x, w, w_scale, bias=None, out_dtype=None, out=None, stream=None, workspace=None):
        torch = _torch()
        px, sx = _rows(x, (None, None), "x")
        M, K = (int(n) for n in x.shape)
        pw, sw = _rows(w, (None, K), "w", torch.int8)
        N = int(w.shape[0])
        if out is None:
            out = _empty((M, N), out_dtype or x.dtype, x.device, stream)
        po, so = _rows(out, (M, N), "out", out_dtype)
        lib = load_library()
        need = _size(lib.fs_linear_workspace_size, M, N, K)
        ws = _workspace(ctx, workspace, need, stream)
        _same_device(ctx, x=x, w=w, w_scale=w_scale, bias=bias, out=out, workspace=ws)
        self.out, self._keep = out, (x, w, w_scale, bias, ws)
        self._fn = lib.fs_linear
        self._args = (ctx.handle, px, _element_type(x.dtype), sx, pw, sw,
                      _dev_ptr(w_scale, torch.float32, (N,), "w_scale"), _dev_ptr(bias, torch.float32, (N,), "bias"),
                      M, N, K, po, _element_type(out.dtype), so, _dev_ptr(ws, torch.uint8, None, "workspace"), ws.numel(),
                      _stream(x.device, stream))
        _keep_for(stream, out, *self._keep)


def linear(ctx: Context, x, w, w_scale, bias=None, out_dtype=None, out=None, stream=None, workspace=None):
    """fs_linear, one call (see LinearPlan)."""
    return LinearPlan(ctx, x, w, w_scale, bias, out_dtype, out, stream, workspace).run()


ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}


class _Norm(ctypes.Structure):
    _fields_ = [("gain", ctypes.c_void_p), ("eps", ctypes.c_float)]


@dataclass
class Norm:
    """The RMS norm of a projection's rows, x * gain / sqrt(mean x^2 + eps):
    gain float32 [K], None for ones."""
    gain: object = None
    eps: float = 1e-6

    def _struct(self, K):
        torch = _torch()
        return _Norm(_dev_ptr(self.gain, torch.float32, (K,), "gain"), float(self.eps))


def _activation(name):
    if name not in ACTIVATIONS:
        raise _invalid(f"activation must be one of {', '.join(ACTIVATIONS)}, got {name!r}")
    return ACTIVATIONS[name]


class ProjectPlan(_Plan):
    """act(y) + residual, y the projection of x [M, K] (LinearPlan) behind the
    rows' norm (fs_project).  residual [M, N] has out's type and may be out
    itself: then the call adds to it."""

    def __init__(self, ctx: Context, x, w, w_scale, norm: Norm | None = None, bias=None, activation: str = "none",
                 residual=None, out_dtype=None, out=None, stream=None, workspace=None):
        torch = _torch()
        px, sx = _rows(x, (None, None), "x")
        M, K = (int(n) for n in x.shape)
        pw, sw = _rows(w, (None, K), "w", torch.int8)
        N = int(w.shape[0])
        if out is None:
            out = _empty((M, N), out_dtype or x.dtype, x.device, stream)
        po, so = _rows(out, (M, N), "out", out_dtype)
        pr, sr = _rows(residual, (M, N), "residual", out.dtype) if residual is not None else (None, 0)
        lib = load_library()
        need = _size(lib.fs_project_workspace_size, M, N, K)
        ws = _workspace(ctx, workspace, need, stream)
        gain = norm.gain if norm is not None else None
        _same_device(ctx, x=x, gain=gain, w=w, w_scale=w_scale, bias=bias, residual=residual, out=out, workspace=ws)
        self._norm = norm._struct(K) if norm is not None else None
        self.out, self._keep = out, (x, gain, w, w_scale, bias, residual, ws)
        self._fn = lib.fs_project
        self._args = (ctx.handle, px, _element_type(x.dtype), sx, None if norm is None else ctypes.byref(self._norm), pw, sw,
                      _dev_ptr(w_scale, torch.float32, (N,), "w_scale"), _dev_ptr(bias, torch.float32, (N,), "bias"),
                      _activation(activation), pr, sr, M, N, K, po, _element_type(out.dtype), so,
                      _dev_ptr(ws, torch.uint8, None, "workspace"), ws.numel(), _stream(x.device, stream))
        _keep_for(stream, out, *self._keep)


def project(ctx: Context, x, w, w_scale, norm: Norm | None = None, bias=None, activation: str = "none", residual=None,
            out_dtype=None, out=None, stream=None, workspace=None):
    """fs_project, one call (see ProjectPlan)."""
    return ProjectPlan(ctx, x, w, w_scale, norm, bias, activation, residual, out_dtype, out, stream, workspace).run()


class GatedProjectPlan(_Plan):
    """act(g) * u, g and u the projections of x [M, K] behind the rows' norm by
    w int8 [2 N, K]: the gates' N rows, then the values' (fs_gated_project);
    w_scale and bias [2 N]."""

    def __init__(self, ctx: Context, x, w, w_scale, norm: Norm | None = None, bias=None, activation: str = "silu",
                 out_dtype=None, out=None, stream=None, workspace=None):
        torch = _torch()
        px, sx = _rows(x, (None, None), "x")
        M, K = (int(n) for n in x.shape)
        pw, sw = _rows(w, (None, K), "w", torch.int8)
        rows = int(w.shape[0])
        if rows % 2:
            raise _invalid(f"w must have a gate's and a value's row for each channel, got {rows} rows")
        N = rows // 2
        if out is None:
            out = _empty((M, N), out_dtype or x.dtype, x.device, stream)
        po, so = _rows(out, (M, N), "out", out_dtype)
        lib = load_library()
        need = _size(lib.fs_gated_project_workspace_size, M, N, K)
        ws = _workspace(ctx, workspace, need, stream)
        gain = norm.gain if norm is not None else None
        _same_device(ctx, x=x, gain=gain, w=w, w_scale=w_scale, bias=bias, out=out, workspace=ws)
        self._norm = norm._struct(K) if norm is not None else None
        self.out, self._keep = out, (x, gain, w, w_scale, bias, ws)
        self._fn = lib.fs_gated_project
        self._args = (ctx.handle, px, _element_type(x.dtype), sx, None if norm is None else ctypes.byref(self._norm), pw, sw,
                      _dev_ptr(w_scale, torch.float32, (rows,), "w_scale"),
                      _dev_ptr(bias, torch.float32, (rows,), "bias"), _activation(activation), M, N, K, po,
                      _element_type(out.dtype), so, _dev_ptr(ws, torch.uint8, None, "workspace"), ws.numel(),
                      _stream(x.device, stream))
        _keep_for(stream, out, *self._keep)


def gated_project(ctx: Context, x, w, w_scale, norm: Norm | None = None, bias=None, activation: str = "silu",
                  out_dtype=None, out=None, stream=None, workspace=None):
    """fs_gated_project, one call (see GatedProjectPlan)."""
    return GatedProjectPlan(ctx, x, w, w_scale, norm, bias, activation, out_dtype, out, stream, workspace).run()


@dataclass
class KVCache:
    """A paged cache of keys and values in 8 bits with a scale for each page
    and head: k int8 [pages, heads, page_size, head_dim], v int8 [pages, heads,
    head_dim, page_size], k_scale and v_scale float32 [pages, heads]."""
    k: object
    v: object
    k_scale: object
    v_scale: object

    @staticmethod
    def empty(n_pages: int, n_heads: int, head_dim: int, page_size: int, device) -> "KVCache":
        torch = _torch()
        z = lambda shape, dtype: torch.zeros(shape, dtype=dtype, device=device)
        return KVCache(z((n_pages, n_heads, page_size, head_dim), torch.int8),
                       z((n_pages, n_heads, head_dim, page_size), torch.int8),
                       z((n_pages, n_heads), torch.float32), z((n_pages, n_heads), torch.float32))

    @property
    def page_size(self) -> int:
        return int(self.k.shape[2])

    @property
    def n_heads(self) -> int:
        return int(self.k.shape[1])

    @property
    def head_dim(self) -> int:
        return int(self.k.shape[3])

    def _tensors(self):
        return dict(k_codes=self.k, v_codes=self.v, k_scale=self.k_scale, v_scale=self.v_scale)

    def _struct(self):
        torch = _torch()
        if self.k.dim() != 4:
            raise _invalid("k must be [pages, heads, page_size, head_dim]")
        P, H, S, D = (int(n) for n in self.k.shape)
        return _Cache(_dev_ptr(self.k, torch.int8, (P, H, S, D), "k"), _dev_ptr(self.v, torch.int8, (P, H, D, S), "v"),
                      _dev_ptr(self.k_scale, torch.float32, (P, H), "k_scale"),
                      _dev_ptr(self.v_scale, torch.float32, (P, H), "v_scale"), P, H, D, S)


class AppendPlan(_Plan):
    """Rotates a step's queries and keys to their positions and appends keys
    and values to the cache (fs_cache_append).  k, v [T, heads, head_dim] and
    q [T, query heads, head_dim] may be parts of wider rows; slots and
    positions int32 [T]; cos, sin float32 [positions, rotary_dim / 2], None for
    no rotation.  run() returns the rotated queries (None without q)."""

    def __init__(self, ctx: Context, cache: KVCache, k, v, slots, q=None, positions=None, cos=None, sin=None,
                 q_out=None, stream=None):
        torch = _torch()
        self._cache = cache._struct()
        T = int(k.shape[0])
        shape = (T, cache.n_heads, cache.head_dim)
        pk, sk = _rows(k, shape, "k")
        pv, sv = _rows(v, shape, "v", k.dtype)
        pq, sq, po, heads = None, 0, None, 0
        if q is not None:
            pq, sq = _rows(q, (T, None, cache.head_dim), "q", k.dtype)
            heads = int(q.shape[1])
            if q_out is None:
                q_out = _empty((T, heads, cache.head_dim), q.dtype, q.device, stream)
            po = _dev_ptr(q_out, q.dtype, (T, heads, cache.head_dim), "q_out")
        reach = half = 0
        if cos is not None:
            if sin is None or positions is None:
                raise _invalid("a rotation needs positions, cos and sin")
            if cos.dim() != 2:
                raise _invalid("cos must be [positions, rotary_dim / 2]")
            reach, half = (int(n) for n in cos.shape)
        _same_device(ctx, k=k, v=v, q=q, slots=slots, positions=positions, cos=cos, sin=sin, q_out=q_out, **cache._tensors())
        self.out, self._keep = (q_out if q is not None else None), (*cache._tensors().values(), k, v, q, slots, positions, cos, sin)
        self._fn = load_library().fs_cache_append
        self._args = (ctx.handle, ctypes.byref(self._cache), pk, sk, pv, sv, pq, sq, heads, _element_type(k.dtype), T,
                      _dev_ptr(slots, torch.int32, (T,), "slots"), _dev_ptr(positions, torch.int32, (T,), "positions"),
                      _dev_ptr(cos, torch.float32, (reach, half), "cos"),
                      _dev_ptr(sin, torch.float32, (reach, half), "sin") if cos is not None else None, reach, 2 * half,
                      po, _stream(k.device, stream))
        _keep_for(stream, self.out, *self._keep)


def cache_append(ctx: Context, cache: KVCache, k, v, slots, q=None, positions=None, cos=None, sin=None, q_out=None,
                 stream=None):
    """fs_cache_append, one call (see AppendPlan)."""
    return AppendPlan(ctx, cache, k, v, slots, q, positions, cos, sin, q_out, stream).run()


class ReadPlan(_Plan):
    """The values that the cache holds at slots int32 [T] (fs_cache_read):
    run() returns (k, v) [T, heads, head_dim], float32 by default."""

    def __init__(self, ctx: Context, cache: KVCache, slots, dtype=None, out=None, stream=None):
        torch = _torch()
        self._cache = cache._struct()
        T = int(slots.shape[0])
        shape = (T, cache.n_heads, cache.head_dim)
        dtype = dtype or torch.float32
        if out is None:
            out = tuple(_empty(shape, dtype, cache.k.device, stream) for _ in range(2))
        _same_device(ctx, slots=slots, k_out=out[0], v_out=out[1], **cache._tensors())
        self.out, self._keep = out, (*cache._tensors().values(), slots)
        self._fn = load_library().fs_cache_read
        self._args = (ctx.handle, ctypes.byref(self._cache), T, _dev_ptr(slots, torch.int32, (T,), "slots"),
                      _dev_ptr(out[0], dtype, shape, "k_out"), _dev_ptr(out[1], dtype, shape, "v_out"),
                      _element_type(dtype), _stream(cache.k.device, stream))
        _keep_for(stream, *out, *self._keep)


def cache_read(ctx: Context, cache: KVCache, slots, dtype=None, out=None, stream=None):
    """fs_cache_read, one call (see ReadPlan)."""
    return ReadPlan(ctx, cache, slots, dtype, out, stream).run()


class AttentionPlan(_Plan):
    """Causal attention of packed new tokens over the cache
    (fs_cache_attention): q [T, query heads, head_dim] (may be part of wider
    rows), block_table int32 [sequences, width], ctx_lens int32 [sequences]
    (tokens in the cache, the new ones among them), cu_q int32 [sequences + 1],
    max_q the largest number of new tokens of a sequence.  scale defaults to
    head_dim ** -0.5; window 0 means none."""

    def __init__(self, ctx: Context, cache: KVCache, q, block_table, ctx_lens, cu_q, max_q: int, scale=None,
                 window: int = 0, out=None, stream=None, workspace=None):
        torch = _torch()
        self._cache = cache._struct()
        pq, sq = _rows(q, (None, None, cache.head_dim), "q")
        T, heads = int(q.shape[0]), int(q.shape[1])
        S = int(ctx_lens.shape[0])
        if block_table.dim() != 2:
            raise _invalid("block_table must be [sequences, width]")
        width = int(block_table.shape[1])
        if out is None:
            out = _empty((T, heads, cache.head_dim), q.dtype, q.device, stream)
        po = _dev_ptr(out, q.dtype, (T, heads, cache.head_dim), "out")
        lib = load_library()
        need = _size(lib.fs_cache_attention_workspace_size, ctypes.byref(self._cache), heads, T, S)
        ws = _workspace(ctx, workspace, need, stream)
        _same_device(ctx, q=q, block_table=block_table, ctx_lens=ctx_lens, cu_q=cu_q, out=out, workspace=ws, **cache._tensors())
        self.out, self._keep = out, (*cache._tensors().values(), q, block_table, ctx_lens, cu_q, ws)
        self._fn = lib.fs_cache_attention
        self._args = (ctx.handle, ctypes.byref(self._cache), pq, sq, _element_type(q.dtype), heads, T, S,
                      _dev_ptr(cu_q, torch.int32, (S + 1,), "cu_q"), _dev_ptr(ctx_lens, torch.int32, (S,), "ctx_lens"),
                      _dev_ptr(block_table, torch.int32, (S, width), "block_table"), width, int(max_q),
                      float(cache.head_dim ** -0.5 if scale is None else scale), int(window), po,
                      _dev_ptr(ws, torch.uint8, None, "workspace"), ws.numel(), _stream(q.device, stream))
        _keep_for(stream, out, *self._keep)


def cache_attention(ctx: Context, cache: KVCache, q, block_table, ctx_lens, cu_q, max_q: int, scale=None,
                    window: int = 0, out=None, stream=None, workspace=None):
    """fs_cache_attention, one call (see AttentionPlan)."""
    return AttentionPlan(ctx, cache, q, block_table, ctx_lens, cu_q, max_q, scale, window, out, stream, workspace).run()


class _StatePool(ctypes.Structure):
    _fields_ = [("s", ctypes.c_void_p), ("n_states", ctypes.c_int32), ("n_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32)]


class StateAttentionPlan(_Plan):
    """Attention of packed new tokens over one decaying matrix a head
    (fs_state_attention).  states float32 [states, heads, head_dim, head_dim] is
    the pool, updated in place; q [T, query heads, head_dim], k and v [T, heads,
    head_dim] may be parts of wider rows; state_index int32 [sequences] (negative:
    starts from zeros, not kept), ctx_lens, cu_q and max_q as in AttentionPlan (a
    sequence whose ctx_lens is its number of new tokens starts from zeros);
    log_decay float32 [heads], at most 0.  scale defaults to head_dim ** -0.5."""

    def __init__(self, ctx: Context, states, q, k, v, state_index, ctx_lens, cu_q, max_q: int, log_decay, scale=None,
                 out=None, stream=None, workspace=None):
        torch = _torch()
        if states.dim() != 4:
            raise _invalid("states must be [states, heads, head_dim, head_dim]")
        P, H, D = (int(n) for n in states.shape[:3])
        self._pool = _StatePool(_dev_ptr(states, torch.float32, (P, H, D, D), "states"), P, H, D)
        pq, sq = _rows(q, (None, None, D), "q")
        T, heads = int(q.shape[0]), int(q.shape[1])
        pk, sk = _rows(k, (T, H, D), "k", q.dtype)
        pv, sv = _rows(v, (T, H, D), "v", q.dtype)
        S = int(state_index.shape[0])
        if out is None:
            out = _empty((T, heads, D), q.dtype, q.device, stream)
        po = _dev_ptr(out, q.dtype, (T, heads, D), "out")
        lib = load_library()
        need = _size(lib.fs_state_attention_workspace_size, ctypes.byref(self._pool), heads, T, S)
        ws = _workspace(ctx, workspace, need, stream)
        _same_device(ctx, states=states, q=q, k=k, v=v, state_index=state_index, ctx_lens=ctx_lens, cu_q=cu_q,
                     log_decay=log_decay, out=out, workspace=ws)
        self.out, self._keep = out, (states, q, k, v, state_index, ctx_lens, cu_q, log_decay, ws)
        self._fn = lib.fs_state_attention
        self._args = (ctx.handle, ctypes.byref(self._pool), pq, sq, pk, sk, pv, sv, _element_type(q.dtype), heads, T, S,
                      _dev_ptr(cu_q, torch.int32, (S + 1,), "cu_q"), _dev_ptr(ctx_lens, torch.int32, (S,), "ctx_lens"),
                      _dev_ptr(state_index, torch.int32, (S,), "state_index"), int(max_q),
                      _dev_ptr(log_decay, torch.float32, (H,), "log_decay"), float(D ** -0.5 if scale is None else scale),
                      po, _dev_ptr(ws, torch.uint8, None, "workspace"), ws.numel(), _stream(q.device, stream))
        _keep_for(stream, out, *self._keep)


def state_attention(ctx: Context, states, q, k, v, state_index, ctx_lens, cu_q, max_q: int, log_decay, scale=None,
                    out=None, stream=None, workspace=None):
    """fs_state_attention, one call (see StateAttentionPlan)."""
    return StateAttentionPlan(ctx, states, q, k, v, state_index, ctx_lens, cu_q, max_q, log_decay, scale, out, stream,
                              workspace).run()
