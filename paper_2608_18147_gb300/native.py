"""Thin ctypes binding of include/ecasq.h.

Every function here has the C entry point's name and only marshals
arguments: torch CUDA tensors become device pointers, the current torch
stream becomes the cudaStream_t, and host results come back as Python
values.  All arithmetic runs in libecasq.so; there is no fallback -- if the
library cannot be loaded, every call raises.
"""
from __future__ import annotations

import ctypes as C
import os
import threading

import numpy as np

from . import build as _build

OK, EINVAL, ENONFINITE, EINFEASIBLE, EWORKSPACE, ECUDA, ETIMEOUT, ERANGE = 0, -1, -2, -3, -4, -5, -6, -7
F32, F16, BF16 = 0, 1, 2  # element types of the operators on 4-bit codes
BAD_PAGE, BAD_LENGTH, BAD_COUNT, BAD_VALUE, BAD_WAIT = 1, 2, 4, 8, 16  # bits of their status word
EXACT_S, NO_REFINE_GUARD, DP_REFERENCE, TIME_KERNELS, EXACT_TABLES, RESIDENT_COSTS, STREAMED_COSTS = 1, 2, 4, 8, 16, 32, 64
ONE_PART_PUBLISH = 128  # accepted, without effect
UNSEEDED_SEARCH = 256  # fast DP search: no seeded tile skipping (same results)
TEST_STALL = 1 << 30  # test hook of the bounded waits (include/ecasq.h)
TEST_SHORT_PARTS = 1 << 28  # test hook: far segments of the fast DP in parts of three tiles (same results)
TEST_LOST_WAIT = 1 << 30  # test hook of ecasq_matvec, in its `type`: blocks go on as if a wait of their first round had run out
TEST_SELF_SEED = 1 << 29  # test hook: a fixed-multiplier pass seeded with its own fp32 minima (same results)

_lock = threading.Lock()
_lib = None
_torch_module = None


class Params(C.Structure):
    _fields_ = [("s", C.c_int32), ("flags", C.c_uint32), ("budget_bits", C.c_double), ("lambda_", C.c_double),
                ("lambda_lo", C.c_double), ("lambda_hi", C.c_double), ("search_rounds", C.c_int32),
                ("refine_max_rounds", C.c_int32), ("refine_rel_tol", C.c_double)]


class Result(C.Structure):
    _fields_ = [("status", C.c_int32), ("m", C.c_int32), ("passes", C.c_int32), ("lambdas_evaluated", C.c_int32),
                ("refine_rounds", C.c_int32), ("reserved", C.c_int32), ("d", C.c_int64), ("p", C.c_int64),
                ("lambda_", C.c_double), ("lambda_prime", C.c_double), ("norm2", C.c_double), ("mse", C.c_double),
                ("vnmse", C.c_double), ("h_surrogate", C.c_double), ("h_exact", C.c_double), ("r_tot", C.c_double),
                ("objective", C.c_double), ("candidates", C.c_int64), ("rescored", C.c_int64),
                ("dp_kernel_ms", C.c_double), ("dp_kernel_launches", C.c_int32), ("reserved2", C.c_int32),
                ("refine_last_rel", C.c_double)]

    def as_dict(self):
        out = {}
        for name, _ in self._fields_:
            key = "lambda" if name == "lambda_" else name
            out[key] = getattr(self, name)
        return out


class Timeshare(C.Structure):
    _fields_ = [("beta", C.c_double), ("lambda_plus", C.c_double), ("mse", C.c_double), ("vnmse", C.c_double),
                ("h_surrogate", C.c_double), ("h_exact", C.c_double), ("plus_mse", C.c_double),
                ("plus_h_surrogate", C.c_double), ("plus_h_exact", C.c_double), ("m_plus", C.c_int32),
                ("reserved", C.c_int32)]

    def as_dict(self):
        return {name: getattr(self, name) for name, _ in self._fields_}


class Cache(C.Structure):
    _fields_ = [("rows", C.c_void_p), ("levels", C.c_void_p), ("row_page", C.c_int64), ("row_slot", C.c_int64),
                ("row_head", C.c_int64), ("level_page", C.c_int64), ("level_slot", C.c_int64),
                ("level_head", C.c_int64), ("pages", C.c_int64), ("page_size", C.c_int32), ("heads", C.c_int32),
                ("d", C.c_int32), ("type", C.c_int32), ("levels_n", C.c_int32), ("reserved", C.c_int32)]


class EcasqError(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        msg = lib().ecasq_strerror(code).decode() if _lib is not None else str(code)
        super().__init__("%s: %s (status %d)" % (where, msg, code))


def lib_path() -> str:
    return _build.LIB


def lib():
    """Load libecasq.so (building it first if it is missing or stale)."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is not None:
            return _lib
        path = _build.build()
        L = C.CDLL(path)
        vp, i32, i64, u32, u64, dbl, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_uint32, C.c_uint64, C.c_double, C.c_size_t
        pd = C.POINTER(C.c_double)
        pi32 = C.POINTER(C.c_int32)
        pi64 = C.POINTER(C.c_int64)
        PP = C.POINTER(Params)
        PR = C.POINTER(Result)
        PC = C.POINTER(Cache)
        sig = {
            "ecasq_version": (C.c_int, []),
            "ecasq_strerror": (C.c_char_p, [C.c_int]),
            "ecasq_workspace_size": (sz, [i64, i32, i64]),
            "ecasq_workspace_size_flags": (sz, [i64, i32, i64, u32]),
            "ecasq_solve": (C.c_int, [vp, i64, PP, vp, sz, vp, PR, vp]),
            "ecasq_solve_grid": (C.c_int, [vp, i64, vp, i64, PP, vp, sz, vp, PR, vp]),
            "ecasq_workspace_size_grid": (sz, [i64, i64, i32, u32]),
            "ecasq_workspace_size_opt": (sz, [i64, i64, i32, i32]),
            "ecasq_workspace_size_prep": (sz, [i64]),
            "ecasq_opt_dp": (C.c_int, [vp, i64, vp, i64, i32, pd, i32, u32, vp, sz, vp, pi32, pd, vp]),
            "ecasq_solve_timeshare": (C.c_int, [vp, i64, vp, i64, PP, vp, sz, vp, vp, PR, C.POINTER(Timeshare), vp]),
            "ecasq_quantize_timeshare": (C.c_int, [vp, i64, vp, i32, vp, i32, dbl, u64, u64, vp, vp, vp, vp, sz, pd,
                                                   vp]),
            "ecasq_dp_pass": (C.c_int, [vp, i64, i32, pd, i32, u32, vp, sz, vp, pi32, pd, vp]),
            "ecasq_dp_tables": (C.c_int, [vp, sz, i32, vp, vp, pi64, vp]),
            "ecasq_workspace_size_linear": (sz, [i64]),
            "ecasq_dp_linear": (C.c_int, [vp, i64, i32, dbl, u32, vp, sz, vp, pi32, pd, vp]),
            "ecasq_refine": (C.c_int, [vp, i64, vp, i32, dbl, dbl, i32, dbl, u32, vp, sz, PR, vp]),
            "ecasq_evaluate": (C.c_int, [vp, i64, vp, i32, vp, sz, pd, vp]),
            "ecasq_quantize": (C.c_int, [vp, i64, vp, i32, u64, vp, vp, vp, sz, pd, vp]),
            "ecasq_quantize_noalloc": (C.c_int, [vp, i64, vp, i32, u64, vp, vp, pd, vp]),
            "ecasq_solve_batched": (C.c_int, [vp, i64, i64, PP, vp, sz, vp, vp, PR, vp]),
            "ecasq_prepare": (C.c_int, [vp, i64, vp, sz, vp, vp, vp, vp, vp, pi64, vp]),
            "ecasq_pack": (C.c_int, [vp, i64, i64, i64, vp, i64, vp]),
            "ecasq_matvec": (C.c_int, [vp, i64, i32, i64, vp, i64, vp, i32, vp, i64, i32, i64, i64, i32, vp, i64, vp,
                                       vp]),
            "ecasq_workspace_size_project": (sz, [i64, i64, i64, i32]),
            "ecasq_project_plan": (C.c_int, [i64, i64, i64, i32, i32, i32, pi64]),
            "ecasq_project_rings": (C.c_int, [i32, i32, i32, pi32]),
            "ecasq_project": (C.c_int, [vp, i64, i32, i64, vp, i64, vp, i32, vp, i64, i32, i64, i64, i32, vp, i32, vp, i64, vp, i64,
                                        vp, sz, vp, vp]),
            "ecasq_gated": (C.c_int, [vp, i64, i32, i64, vp, i64, vp, i32, vp, i64, i32, i64, i64, i32, i32, vp, i64, vp, sz, vp,
                                      vp]),
            "ecasq_norm": (C.c_int, [vp, i64, i32, i64, i64, vp, i64, vp, i32, C.c_float, i64, vp, i64, vp, i64, vp, i64, vp]),
            "ecasq_cache_write": (C.c_int, [vp, i32, i64, i64, i64, vp, i32, vp, vp, PC, u64, vp, vp]),
            "ecasq_workspace_size_attend": (sz, [i64, i32, i32, i32, i64]),
            "ecasq_attend": (C.c_int, [vp, i64, i64, i64, i32, PC, PC, vp, i64, vp, vp, i64, C.c_float, vp, i64, i64,
                                       vp, vp, sz, vp, vp]),
            "ecasq_kernel_launches": (i64, []),
        }
        for name, (res, args) in sig.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
        return L


def exported_symbols():
    """Names declared in include/ecasq.h that the loaded library exports."""
    L = lib()
    names = []
    for name in ("ecasq_version", "ecasq_strerror", "ecasq_workspace_size", "ecasq_workspace_size_flags",
                 "ecasq_solve", "ecasq_solve_grid", "ecasq_workspace_size_grid", "ecasq_solve_timeshare",
                 "ecasq_quantize_timeshare", "ecasq_workspace_size_opt", "ecasq_workspace_size_prep", "ecasq_opt_dp",
                 "ecasq_dp_pass",
                 "ecasq_dp_tables", "ecasq_workspace_size_linear", "ecasq_dp_linear", "ecasq_refine", "ecasq_evaluate", "ecasq_quantize", "ecasq_quantize_noalloc",
                 "ecasq_solve_batched",
                 "ecasq_prepare", "ecasq_pack", "ecasq_matvec", "ecasq_workspace_size_project", "ecasq_project", "ecasq_gated",
                 "ecasq_norm", "ecasq_cache_write", "ecasq_workspace_size_attend",
                 "ecasq_attend", "ecasq_kernel_launches"):
        if hasattr(L, name):
            names.append(name)
    return names


# ------------------------------------------------------------------ helpers

def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _stream():
    torch = _torch()
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _ptr(t):
    return C.c_void_p(t.data_ptr())


def _dev_f32(x):
    torch = _torch()
    if not isinstance(x, torch.Tensor):
        x = torch.as_tensor(np.ascontiguousarray(x, dtype=np.float32))
    if x.dtype != torch.float32:
        raise TypeError("x must be float32")
    if not x.is_cuda:
        x = x.cuda()
    return x.contiguous()


def _check(rc, where, ok=(OK,)):
    if rc not in ok:
        raise EcasqError(rc, where)
    return rc


def ws_status(ws):
    """Counters the library leaves at the start of a workspace after a call
    (unique values, device-side flags, fast-DP statistics)."""
    raw = ws[:120].cpu().numpy().tobytes()
    (p, nonfinite, range_err, timeout, bound_viol, norm2, rescored, overflow, last_s, last_G, last_d, members,
     big_bands, tiles_run, tiles_skipped, grid_nL, grid_nR, tiles_fetched) = __import__("struct").unpack("<qiiiidqqiiqqqqqqqq", raw)
    return dict(p=p, nonfinite=nonfinite, range_err=range_err, timeout=timeout, bound_viol=bound_viol, norm2=norm2,
                rescored=rescored, overflow=overflow, last_s=last_s, last_G=last_G, last_d=last_d, members=members,
                big_bands=big_bands, tiles_run=tiles_run, tiles_skipped=tiles_skipped, grid_nL=grid_nL,
                grid_nR=grid_nR, tiles_fetched=tiles_fetched)


def ecasq_workspace_size(d, s, rows=1) -> int:
    return int(lib().ecasq_workspace_size(int(d), int(s), int(rows)))


def ecasq_workspace_size_flags(d, s, rows=1, flags=0) -> int:
    return int(lib().ecasq_workspace_size_flags(int(d), int(s), int(rows), int(flags)))


def workspace(d, s, rows=1, flags=0):
    """A device workspace (torch uint8 tensor; CUDA allocations are 256-byte aligned)."""
    torch = _torch()
    n = ecasq_workspace_size_flags(d, s, rows, flags)
    if n == 0:
        raise EcasqError(EINVAL, "ecasq_workspace_size")
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def make_params(s, budget_bits=0.0, lambda_=-1.0, lambda_lo=0.0, lambda_hi=0.0, search_rounds=0,
                refine_max_rounds=0, refine_rel_tol=0.0, flags=0):
    return Params(int(s), int(flags), float(budget_bits), float(lambda_), float(lambda_lo), float(lambda_hi),
                  int(search_rounds), int(refine_max_rounds), float(refine_rel_tol))


# --------------------------------------------------------------- entry points

def ecasq_solve(x, s, budget_bits=0.0, lambda_=-1.0, ws=None, **kw):
    """Budgeted (or fixed-multiplier) solve; returns (Q tensor [m], result dict)."""
    torch = _torch()
    x = _dev_f32(x)
    d = x.numel()
    if ws is None:
        ws = workspace(d, s, flags=kw.get("flags", 0))
    prm = make_params(s, budget_bits, lambda_, **kw)
    Q = torch.zeros(s, dtype=torch.float32, device="cuda")
    res = Result()
    rc = lib().ecasq_solve(_ptr(x), d, C.byref(prm), _ptr(ws), ws.numel(), _ptr(Q), C.byref(res), _stream())
    _check(rc, "ecasq_solve", ok=(OK, EINFEASIBLE))
    return Q[:res.m].clone(), res.as_dict()


def ecasq_solve_grid(x, P, s, budget_bits=0.0, lambda_=-1.0, ws=None, **kw):
    """Budgeted solve with the codebook drawn from the candidate set P (strictly ascending,
    P[0] <= min x, P[-1] >= max x)."""
    torch = _torch()
    x = _dev_f32(x)
    P = _dev_f32(P)
    d, n = x.numel(), P.numel()
    if ws is None:
        nb = int(lib().ecasq_workspace_size_grid(d, n, int(s), int(kw.get("flags", 0))))
        if nb == 0:
            raise EcasqError(EINVAL, "ecasq_workspace_size_grid")
        ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    prm = make_params(s, budget_bits, lambda_, **kw)
    Q = torch.zeros(s, dtype=torch.float32, device="cuda")
    res = Result()
    rc = lib().ecasq_solve_grid(_ptr(x), d, _ptr(P), n, C.byref(prm), _ptr(ws), ws.numel(), _ptr(Q), C.byref(res),
                                _stream())
    _check(rc, "ecasq_solve_grid", ok=(OK, EINFEASIBLE))
    return Q[:res.m].clone(), res.as_dict()


def ecasq_solve_timeshare(x, s, budget_bits, P=None, ws=None, **kw):
    """Budgeted solve with two-way time-sharing (Sec. 7): (Q- tensor, Q+ tensor or empty,
    result dict of Q-, time-sharing dict).  P: optional permissible set as in ecasq_solve_grid."""
    torch = _torch()
    x = _dev_f32(x)
    d = x.numel()
    flags = int(kw.get("flags", 0))
    if P is not None:
        P = _dev_f32(P)
        n = P.numel()
        nb = int(lib().ecasq_workspace_size_grid(d, n, int(s), flags))
    else:
        n = 0
        nb = int(lib().ecasq_workspace_size_flags(d, int(s), 1, flags))
    if ws is None:
        if nb == 0:
            raise EcasqError(EINVAL, "workspace size")
        ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    prm = make_params(s, budget_bits, -1.0, **kw)
    Qm = torch.zeros(s, dtype=torch.float32, device="cuda")
    Qp = torch.zeros(s, dtype=torch.float32, device="cuda")
    res = Result()
    ts = Timeshare()
    rc = lib().ecasq_solve_timeshare(_ptr(x), d, _ptr(P) if P is not None else None, n, C.byref(prm), _ptr(ws),
                                     ws.numel(), _ptr(Qm), _ptr(Qp), C.byref(res), C.byref(ts), _stream())
    _check(rc, "ecasq_solve_timeshare", ok=(OK, EINFEASIBLE))
    return Qm[:res.m].clone(), Qp[:ts.m_plus].clone(), res.as_dict(), ts.as_dict()


def ecasq_quantize_timeshare(x, Qm, Qp, beta, seed, seed_ts, ws=None, with_sel=True):
    """Time-shared stochastic quantization (Sec. 7): (idx, sel or None, counts [mm + mp], rate)."""
    torch = _torch()
    x = _dev_f32(x)
    d = x.numel()
    Qm = _dev_f32(Qm)
    Qp = _dev_f32(Qp) if Qp is not None and len(Qp) else None
    mm, mp = Qm.numel(), (Qp.numel() if Qp is not None else 0)
    if ws is None:
        ws = torch.empty(256, dtype=torch.uint8, device="cuda")
    idx = torch.empty(d, dtype=torch.uint8, device="cuda")
    sel = torch.empty(d, dtype=torch.uint8, device="cuda") if with_sel else None
    counts = torch.empty(mm + mp, dtype=torch.int32, device="cuda")
    rate = C.c_double()
    rc = lib().ecasq_quantize_timeshare(_ptr(x), d, _ptr(Qm), mm, _ptr(Qp) if Qp is not None else None, mp,
                                        float(beta), C.c_uint64(int(seed) & 0xFFFFFFFFFFFFFFFF),
                                        C.c_uint64(int(seed_ts) & 0xFFFFFFFFFFFFFFFF), _ptr(idx),
                                        _ptr(sel) if sel is not None else None, _ptr(counts), _ptr(ws), ws.numel(),
                                        C.byref(rate), _stream())
    _check(rc, "ecasq_quantize_timeshare")
    return idx, sel, counts, rate.value


def ecasq_opt_dp(x, s, lambdas, P=None, flags=0, ws=None):
    """Optimal DP of Sec. 4 at up to 8 fixed multipliers (vNMSE scale): (Q [G, s] tensor,
    m list, metrics [G, 4] = optimum, MSE, H(I,B), H(Xhat)).  P: optional permissible set."""
    torch = _torch()
    x = _dev_f32(x)
    d = x.numel()
    lams = np.ascontiguousarray(np.atleast_1d(lambdas), dtype=np.float64)
    G = lams.size
    n = 0
    if P is not None:
        P = _dev_f32(P)
        n = P.numel()
    if ws is None:
        nb = int(lib().ecasq_workspace_size_opt(d, n if P is not None else d, int(s), G))
        if nb == 0:
            raise EcasqError(EINVAL, "ecasq_workspace_size_opt")
        ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    Q = torch.zeros((G, s), dtype=torch.float32, device="cuda")
    m = (C.c_int32 * G)()
    met = np.zeros(4 * G, np.float64)
    rc = lib().ecasq_opt_dp(_ptr(x), d, _ptr(P) if P is not None else None, n, int(s),
                            lams.ctypes.data_as(C.POINTER(C.c_double)), G, int(flags), _ptr(ws), ws.numel(), _ptr(Q),
                            m, met.ctypes.data_as(C.POINTER(C.c_double)), _stream())
    _check(rc, "ecasq_opt_dp")
    return Q, list(m), met.reshape(G, 4)


def uniform_grid(x, n):
    """n equally spaced fp32 candidates from min x to max x, both endpoints exact."""
    x = np.asarray(x, dtype=np.float32)
    lo, hi = float(x.min()), float(x.max())
    g = np.linspace(lo, hi, n).astype(np.float32)
    g[0], g[-1] = np.float32(lo), np.float32(hi)
    return np.unique(g)


def ecasq_dp_pass(x, s, lambdas, flags=0, ws=None):
    """One DP pass at up to 8 multipliers: (Q [G, s] tensor, m list, metrics [G, 4])."""
    torch = _torch()
    x = _dev_f32(x)
    d = x.numel()
    lams = np.ascontiguousarray(lambdas, dtype=np.float64)
    G = lams.size
    if ws is None:
        ws = workspace(d, s, flags=flags)
    Q = torch.zeros((G, s), dtype=torch.float32, device="cuda")
    m = (C.c_int32 * G)()
    met = np.zeros(4 * G, np.float64)
    rc = lib().ecasq_dp_pass(_ptr(x), d, int(s), lams.ctypes.data_as(C.POINTER(C.c_double)), G, int(flags),
                             _ptr(ws), ws.numel(), _ptr(Q), m, met.ctypes.data_as(C.POINTER(C.c_double)), _stream())
    _check(rc, "ecasq_dp_pass")
    return Q, list(m), met.reshape(G, 4)


def ecasq_dp_linear(x, s, lambda_, flags=0, ws=None):
    """Linear-space traceback of the approximate DP at one multiplier (vNMSE scale):
    (Q tensor [m], metrics [4] = dp(m, p-1), MSE, H(I,B), H(Xhat))."""
    torch = _torch()
    x = _dev_f32(x)
    d = x.numel()
    if ws is None:
        nb = int(lib().ecasq_workspace_size_linear(d))
        if nb == 0:
            raise EcasqError(EINVAL, "ecasq_workspace_size_linear")
        ws = torch.empty(nb, dtype=torch.uint8, device=x.device)
    Q = torch.zeros(s, dtype=torch.float32, device=x.device)
    m = C.c_int32()
    met = np.zeros(4, np.float64)
    rc = lib().ecasq_dp_linear(_ptr(x), d, int(s), float(lambda_), int(flags), _ptr(ws), ws.numel(), _ptr(Q),
                               C.byref(m), met.ctypes.data_as(C.POINTER(C.c_double)), _stream())
    _check(rc, "ecasq_dp_linear")
    return Q[:m.value].clone(), met


def ecasq_dp_tables(ws, g, s, p_max):
    """DP tables of multiplier g of the last pass: (dp [(s+1), p] f64, bp [(s+1), p] i32) tensors."""
    torch = _torch()
    dp = torch.empty((s + 1) * p_max, dtype=torch.float64, device="cuda")
    bp = torch.empty((s + 1) * p_max, dtype=torch.int32, device="cuda")
    p = C.c_int64()
    rc = lib().ecasq_dp_tables(_ptr(ws), ws.numel(), int(g), _ptr(dp), _ptr(bp), C.byref(p), _stream())
    _check(rc, "ecasq_dp_tables")
    n = (s + 1) * p.value
    return dp[:n].view(s + 1, p.value), bp[:n].view(s + 1, p.value)


def ecasq_refine(x, Q, lambda_, budget_bits=-1.0, max_rounds=5, rel_tol=0.0, flags=0, ws=None):
    """Three-colour refinement (Sec. 6) of Q at multiplier lambda_; returns (Q, result dict)."""
    torch = _torch()
    x = _dev_f32(x)
    d = x.numel()
    Q = _dev_f32(Q).clone()
    m = Q.numel()
    if ws is None:
        ws = workspace(d, 2)
    res = Result()
    rc = lib().ecasq_refine(_ptr(x), d, _ptr(Q), m, float(lambda_), float(budget_bits), int(max_rounds),
                            float(rel_tol), int(flags), _ptr(ws), ws.numel(), C.byref(res), _stream())
    _check(rc, "ecasq_refine")
    return Q, res.as_dict()


def ecasq_evaluate(x, Q, ws=None):
    """(MSE, H(I,B), H(Xhat)) of a codebook Q subset of x."""
    x = _dev_f32(x)
    d = x.numel()
    Q = _dev_f32(Q)
    if ws is None:
        ws = workspace(d, 2)
    out = np.zeros(3, np.float64)
    rc = lib().ecasq_evaluate(_ptr(x), d, _ptr(Q), Q.numel(), _ptr(ws), ws.numel(),
                              out.ctypes.data_as(C.POINTER(C.c_double)), _stream())
    _check(rc, "ecasq_evaluate")
    return float(out[0]), float(out[1]), float(out[2])


def ecasq_quantize(x, Q, seed, ws=None, idx=None, counts=None):
    """Stochastic quantization (Sec. 2): (idx uint8 tensor, counts tensor, empirical entropy)."""
    torch = _torch()
    x = _dev_f32(x)
    d = x.numel()
    Q = _dev_f32(Q)
    m = Q.numel()
    if ws is None:
        ws = torch.empty(256, dtype=torch.uint8, device="cuda")
    if idx is None:
        idx = torch.empty(d, dtype=torch.uint8, device=x.device)
    if counts is None:
        counts = torch.empty(m, dtype=torch.int32, device=x.device)
    _out_tensor(idx, d, (torch.uint8,), "ecasq_quantize", "idx")
    _out_tensor(counts, m, _count_dtypes(), "ecasq_quantize", "counts")
    if not (idx.device == x.device == counts.device == ws.device):
        raise EcasqError(EINVAL, "ecasq_quantize: x, idx, counts and ws must be on one device")
    he = C.c_double()
    rc = lib().ecasq_quantize(_ptr(x), d, _ptr(Q), m, C.c_uint64(int(seed) & 0xFFFFFFFFFFFFFFFF), _ptr(idx),
                              _ptr(counts), _ptr(ws), ws.numel(), C.byref(he), _stream())
    _check(rc, "ecasq_quantize")
    return idx, counts, he.value


def _out_tensor(t, n, dtypes, where, name):
    """An output buffer the kernel writes through a raw pointer: a contiguous CUDA tensor
    of one of `dtypes` with at least n elements (else EINVAL before any device work)."""
    torch = _torch()
    ok = (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype in dtypes and t.is_contiguous()
          and t.numel() >= n)
    if not ok:
        raise EcasqError(EINVAL, "%s: %s must be a contiguous CUDA tensor of %s with at least %d elements"
                         % (where, name, "/".join(str(d) for d in dtypes), n))
    return t


def _count_dtypes():
    torch = _torch()
    u32 = getattr(torch, "uint32", None)
    return (torch.int32,) + ((u32,) if u32 is not None else ())


def ecasq_quantize_noalloc(x, Q, seed, idx, counts):
    """ecasq_quantize without a workspace; idx (uint8 [d]) and counts (int32 [m])
    are the caller's device tensors, on the device of x.  Returns the empirical entropy."""
    torch = _torch()
    where = "ecasq_quantize_noalloc"
    _out_tensor(idx, 0, (torch.uint8,), where, "idx")
    _out_tensor(counts, 0, _count_dtypes(), where, "counts")
    x = _dev_f32(x)
    Q = _dev_f32(Q)
    _out_tensor(idx, x.numel(), (torch.uint8,), where, "idx")
    _out_tensor(counts, Q.numel(), _count_dtypes(), where, "counts")
    if not (idx.device == x.device == Q.device == counts.device):
        raise EcasqError(EINVAL, "%s: x, Q, idx and counts must be on one device" % where)
    he = C.c_double()
    rc = lib().ecasq_quantize_noalloc(_ptr(x), x.numel(), _ptr(Q), Q.numel(),
                                      C.c_uint64(int(seed) & 0xFFFFFFFFFFFFFFFF), _ptr(idx), _ptr(counts),
                                      C.byref(he), _stream())
    _check(rc, "ecasq_quantize_noalloc")
    return he.value


class BatchResults:
    """The per-row results of ecasq_solve_batched as a read-only sequence of dicts, each
    built from the C records when it is read (building 10^4 dicts up front costs more
    than the solve of short rows)."""

    def __init__(self, records):
        self._records = records

    def __len__(self):
        return len(self._records)

    def __getitem__(self, i):
        if isinstance(i, slice):
            return [self._records[t].as_dict() for t in range(*i.indices(len(self._records)))]
        return self._records[i].as_dict()

    def __iter__(self):
        for r in self._records:
            yield r.as_dict()

    def field(self, name):
        """One field of every row, as a numpy array."""
        return np.array([getattr(r, "lambda_" if name == "lambda" else name) for r in self._records])


def ecasq_solve_batched(X, s, budget_bits=0.0, lambda_=-1.0, ws=None, **kw):
    """Independent budgeted solves of the rows of X [rows, d]: (Q [rows, s], m [rows], results);
    results is a BatchResults sequence (one dict per row, built when read)."""
    torch = _torch()
    X = _dev_f32(X)
    rows, d = X.shape
    if ws is None:
        ws = workspace(d, s, rows, flags=kw.get("flags", 0))
    prm = make_params(s, budget_bits, lambda_, **kw)
    Q = torch.zeros((rows, s), dtype=torch.float32, device="cuda")
    m = torch.zeros(rows, dtype=torch.int32, device="cuda")
    res = (Result * rows)()
    rc = lib().ecasq_solve_batched(_ptr(X), rows, d, C.byref(prm), _ptr(ws), ws.numel(), _ptr(Q), _ptr(m), res,
                                   _stream())
    _check(rc, "ecasq_solve_batched", ok=(OK, EINFEASIBLE))
    return Q, m, BatchResults(res)


def ecasq_prepare(x, ws=None):
    """Weighted histogram and App. E prefix sums: dict of tensors v, w, N, S, S2 and p."""
    torch = _torch()
    x = _dev_f32(x)
    d = x.numel()
    if ws is None:
        ws = torch.empty(int(lib().ecasq_workspace_size_prep(d)), dtype=torch.uint8, device="cuda")
    v = torch.empty(d, dtype=torch.float32, device="cuda")
    w = torch.empty(d, dtype=torch.int64, device="cuda")
    N = torch.empty(d + 1, dtype=torch.int64, device="cuda")
    S = torch.empty(2 * (d + 1), dtype=torch.float64, device="cuda")
    S2 = torch.empty(2 * (d + 1), dtype=torch.float64, device="cuda")
    p = C.c_int64()
    rc = lib().ecasq_prepare(_ptr(x), d, _ptr(ws), ws.numel(), _ptr(v), _ptr(w), _ptr(N), _ptr(S), _ptr(S2),
                             C.byref(p), _stream())
    _check(rc, "ecasq_prepare")
    p = p.value
    return dict(p=p, v=v[:p], w=w[:p], N=N[:p + 1], S_hi=S[:p + 1], S_lo=S[p + 1:2 * p + 2],
                S2_hi=S2[:p + 1], S2_lo=S2[p + 1:2 * p + 2])


# ------------------------------------------------------ operators on 4-bit codes
#
# These calls are short, so what is in front of them is C too (csrc/binding.c, built beside the library): it looks at the
# tensors and calls the C entry point.  What it does not take comes back as None, and is looked at here once more to say why.
# They serve: none has a gradient, and tensors that want one are refused.

_TYPES = {}
_codes = None


def _ready():
    """The extension, set up with the library's entry points and torch."""
    global _codes
    L = lib()
    with _lock:
        if _codes is None:
            import importlib.machinery
            import importlib.util
            torch = _torch()
            _TYPES.update({torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16})
            path = _build.build_binding()
            loader = importlib.machinery.ExtensionFileLoader("_codes", path)
            module = importlib.util.module_from_spec(importlib.util.spec_from_file_location("_codes", path, loader=loader))
            loader.exec_module(module)
            address = lambda fn: C.cast(fn, C.c_void_p).value  # noqa: E731
            module.setup(address(L.ecasq_matvec), address(L.ecasq_cache_write), address(L.ecasq_attend), address(L.ecasq_project),
                         address(L.ecasq_gated), address(L.ecasq_workspace_size_project), address(L.ecasq_norm), torch.Tensor, torch.empty,
                         torch.cuda.current_device, torch._C._cuda_getCurrentRawStream, workspace_attend,
                         torch.is_grad_enabled, torch.autograd.forward_ad,
                         (torch.float32, torch.float16, torch.bfloat16, torch.uint8, torch.int32, torch.int64,
                          torch.float8_e4m3fn))
            _codes = module
    return _codes


def _refuse(where, what):
    raise EcasqError(EINVAL, "%s: %s" % (where, what))


def _need(where, *wanted):
    """Raises for the first of (condition, what it means) that does not hold; a condition is a function, as it may not
    even be computable."""
    for holds, what in wanted:
        try:
            ok = holds()
        except (AttributeError, TypeError, IndexError, RuntimeError):
            ok = False
        if not ok:
            _refuse(where, what)


def _here(where, *tensors):
    """The index of the CUDA device that all the given tensors (None allowed) are on: the current one, whose stream the call
    uses."""
    torch = _torch()
    devices = {t.get_device() if isinstance(t, torch.Tensor) else -1 for t in tensors if t is not None}
    if len(devices) != 1 or -1 in devices or torch.cuda.current_device() not in devices:
        _refuse(where, "tensors must be on the current CUDA device")


def _no_gradients(where, *tensors):
    """These operators serve: a tensor (None allowed) whose gradient or tangent is asked for is refused."""
    torch = _torch()
    for t in tensors:
        if isinstance(t, torch.Tensor) and ((torch.is_grad_enabled() and t.requires_grad)
                                            or torch.autograd.forward_ad.unpack_dual(t).tangent is not None):
            _refuse(where, "no gradients: call it under torch.no_grad() or with detached tensors")


def ecasq_pack(idx):
    """Indices [n, k] (uint8, < 16) of a weight matrix as the packed rows that ecasq_matvec reads: uint8
    [n, 64 ceil(k / 128)]."""
    torch = _torch()
    where = "ecasq_pack"
    L = lib()
    _here(where, idx)
    if idx.dtype != torch.uint8 or idx.dim() != 2 or (idx.shape[1] > 1 and idx.stride(1) != 1):
        _refuse(where, "idx must be uint8 [n, k] with contiguous rows")
    n, k = idx.shape
    codes = torch.empty((n, 64 * -(-k // 128)), dtype=torch.uint8, device=idx.device)
    rc = L.ecasq_pack(idx.data_ptr(), idx.stride(0) if n > 1 else k, n, k, codes.data_ptr(), codes.shape[1], _stream())
    _check(rc, where)
    return codes


def _product_needs(torch, x, codes, levels, scales, group):
    """What a product with a coded matrix wants of its operands, for _need()."""
    k = lambda: x.shape[-1]  # noqa: E731
    return ((lambda: x.dtype in _TYPES and x.dim() in (1, 2) and (k() < 2 or x.stride(-1) == 1),
             "x must be [b, k] or [k] of float32, float16 or bfloat16 with contiguous rows"),
            (lambda: codes.dtype == torch.uint8 and codes.dim() == 2 and codes.stride(1) == 1 and codes.shape[1] >= 64 * -(-k() // 128),
             "codes must be uint8 [n, 64 ceil(k / 128)] with contiguous rows"),
            (lambda: levels.dtype == x.dtype and levels.dim() == 1 and levels.is_contiguous() and 1 <= levels.numel() <= 16,
             "levels must be 1 to 16 values of x's type"),
            (lambda: group >= 32 and group % 32 == 0, "group must be a multiple of 32"),
            (lambda: scales.dtype in (x.dtype, torch.float32) and scales.dim() == 2 and scales.shape[0] == codes.shape[0]
             and scales.shape[1] >= -(-k() // group) and (scales.shape[1] < 2 or scales.stride(1) == 1),
             "scales must be [n, ceil(k / group)] of x's type or float32 with contiguous rows"))


def _rows_like(t, x, n, dtype):
    """Whether t is [b, n] (or [n], as x is) of dtype with contiguous rows."""
    return t.dtype == dtype and t.shape == x.shape[:-1] + (n,) and (n < 2 or t.stride(-1) == 1)


def _matvec_refused(torch, x, codes, levels, scales, group, out, status):
    where = "ecasq_matvec"
    _here(where, x, codes, levels, scales, out)
    _no_gradients(where, x, levels, scales, out)
    _need(where, *_product_needs(torch, x, codes, levels, scales, group),
          (lambda: out is None or _rows_like(out, x, codes.shape[0], x.dtype), "out must be [b, n] (or [n]) of x's type with contiguous rows"),
          (lambda: _is_status(status, x), "status must be an int32 tensor on the device of the others"))
    _refuse(where, "bad arguments")


def ecasq_matvec(x, codes, levels, scales, group, out=None, status=None):
    """y = x W^T for the 4-bit matrix W[r, c] = scales[r, c // group] * levels[code[r, c]].

    x [b, k] or [k] (float32, float16 or bfloat16), codes [n, 64 ceil(k / 128)] as ecasq_pack gives them,
    levels [m <= 16] of x's type, scales [n, ceil(k / group)] of x's type or float32, group a multiple of 32.
    status: int32 tensor that BAD_* bits are or-ed into.  Returns y [b, n] or [n] of x's type (`out` if given).
    No gradients: a tensor that requires one is refused while they are recorded."""
    y = (_codes or _ready()).matvec(x, codes, levels, scales, group, out, status)
    if y is None:
        _matvec_refused(_torch(), x, codes, levels, scales, group, out, status)
    if y.__class__ is int:
        _check(y, "ecasq_matvec")
    return y


ACTIVATIONS = {None: 0, "none": 0, "relu": 1, "silu": 2, "gelu": 3, "gelu_tanh": 4}  # ECASQ_ACT_*


def _activation(where, name):
    try:
        return ACTIVATIONS[name]
    except (KeyError, TypeError):
        _refuse(where, "activation must be one of %s" % ", ".join(str(a) for a in ACTIVATIONS))


def workspace_project(b, n, k, dtype):
    """A device workspace for ecasq_project, or ecasq_gated, with a matrix of n rows and k columns and up to b rows of x of `dtype`
    (it may be empty)."""
    torch = _torch()
    _ready()
    if dtype not in _TYPES:
        _refuse("workspace_project", "dtype must be float32, float16 or bfloat16")
    room = int(lib().ecasq_workspace_size_project(int(b), int(n), int(k), _TYPES[dtype]))
    return torch.empty(room, dtype=torch.uint8, device="cuda")


def _layer_product_refused(torch, where, x, codes, levels, scales, group, bias, residual, out, ws, status, halves):
    _here(where, x, codes, levels, scales, bias, residual, out, ws)
    _no_gradients(where, x, levels, scales, bias, residual, out)
    n = lambda: codes.shape[0] // halves  # noqa: E731
    _need(where, *_product_needs(torch, x, codes, levels, scales, group),
          (lambda: codes.shape[0] % halves == 0, "codes must have an even number of rows: the gate's, then the other half's"),
          (lambda: bias is None or (bias.dtype == x.dtype and bias.shape == (n(),) and bias.is_contiguous()),
           "bias must be contiguous [n] of x's type"),
          (lambda: residual is None or _rows_like(residual, x, n(), x.dtype),
           "residual must be [b, n] (or [n]) of x's type with contiguous rows"),
          (lambda: out is None or _rows_like(out, x, n(), x.dtype), "out must be [b, n] (or [n]) of x's type with contiguous rows"),
          (lambda: ws is None or (ws.dtype == torch.uint8 and ws.is_contiguous()), "ws must be contiguous uint8"),
          (lambda: _is_status(status, x), "status must be an int32 tensor on the device of the others"))
    _refuse(where, "bad arguments")


def ecasq_project(x, codes, levels, scales, group, bias=None, activation=None, residual=None, out=None, ws=None, status=None):
    """y = activation(x W^T + bias) + residual for the 4-bit matrix W of ecasq_matvec, in one call.

    x, codes, levels, scales, group, status as for ecasq_matvec; bias [n] and residual [b, n] (or [n]) of x's type or None;
    activation None, "relu", "silu", "gelu" or "gelu_tanh".  ws: workspace_project(b, n, k, x.dtype), or None (one is made
    where one is needed: for float32, and for rows of x off 16-byte boundaries).  Returns y [b, n] or [n] of x's type (`out` if given, which may be the
    residual itself, not x).  No gradients: a tensor that requires one is refused while they are recorded."""
    act = _activation("ecasq_project", activation)
    y = (_codes or _ready()).project(x, codes, levels, scales, group, bias, act, residual, out, ws, status)
    if y is None:
        _layer_product_refused(_torch(), "ecasq_project", x, codes, levels, scales, group, bias, residual, out, ws, status, 1)
    if y.__class__ is int:
        _check(y, "ecasq_project")
    return y


def ecasq_gated(x, codes, levels, scales, group, activation="silu", out=None, ws=None, status=None):
    """h = activation(x G^T) * (x U^T), the first half of a gated feed-forward block, in one call.

    codes, levels, scales: one coded matrix of 2n rows, those of G and then those of U; x, group and status as for
    ecasq_matvec; activation and ws (workspace_project(b, 2 * n, k, x.dtype)) as for ecasq_project.  Returns h [b, n] or
    [n] of x's type (`out` if given, not x).  No gradients: a tensor that requires one is refused while they are recorded."""
    act = _activation("ecasq_gated", activation)
    y = (_codes or _ready()).gated(x, codes, levels, scales, group, act, out, ws, status)
    if y is None:
        _layer_product_refused(_torch(), "ecasq_gated", x, codes, levels, scales, group, None, None, out, ws, status, 2)
    if y.__class__ is int:
        _check(y, "ecasq_gated")
    return y


def _norm_refused(torch, x, weight, eps, residual, group, out, out_sum, out_scales):
    where = "ecasq_norm"
    _here(where, x, weight, residual, out, out_sum, out_scales)
    _no_gradients(where, x, weight, residual, out, out_sum, out_scales)
    k = lambda: x.shape[-1]  # noqa: E731
    _need(where,
          (lambda: x.dtype in _TYPES and x.dim() in (1, 2) and k() > 0 and (k() < 2 or x.stride(-1) == 1),
           "x must be [b, k] or [k] of float32, float16 or bfloat16 with contiguous rows"),
          (lambda: weight.dtype in (x.dtype, torch.float32) and weight.shape == (k(),) and weight.is_contiguous(),
           "weight must be contiguous [k] of x's type or float32"),
          (lambda: eps >= 0, "eps must not be negative"),
          (lambda: residual is None or _rows_like(residual, x, k(), x.dtype), "residual must be like x"),
          (lambda: group is None or group >= k() or (group > 0 and group % 16 == 0), "group must be None, a multiple of 16 or at least k"),
          (lambda: out is None or _rows_like(out, x, k(), x.dtype if group is None else torch.float8_e4m3fn),
           "out must be like x, or of float8_e4m3fn with a group"),
          (lambda: out_sum is None or (residual is not None and _rows_like(out_sum, x, k(), x.dtype)),
           "out_sum must be like x, and needs a residual"),
          (lambda: out_scales is None or (group is not None and _rows_like(out_scales, x, -(-k() // group), torch.float32)),
           "out_scales must be float32 [b, ceil(k / group)] (or [ceil(k / group)]) with contiguous rows, and needs a group"))
    _refuse(where, "bad arguments")


def ecasq_norm(x, weight, eps=1e-6, residual=None, group=None, out=None, out_sum=None, out_scales=None):
    """Root-mean-square norm of the rows of x [b, k] or [k], after the residual's addition: s = x + residual rounded to x's type
    (x without one), y = s / sqrt(mean(s^2) + eps) * weight.

    weight [k] of x's type or float32.  With `group` (a multiple of 16, or at least k: one scale a row) y is coded to 8 bits:
    float8_e4m3fn values y / scale, scale = max |y| / 448 of each group of columns.  Returns y, (y, scales), (y, s) or
    (y, scales, s); out, out_scales and out_sum are taken for them where given.  out_sum, and out without a group, may be x or
    the residual itself, but not both the same.  No gradients: a tensor that requires one is refused while they are recorded."""
    y = (_codes or _ready()).norm(x, weight, eps, residual, group, out, out_sum, out_scales)
    if y is None:
        _norm_refused(_torch(), x, weight, eps, residual, group, out, out_sum, out_scales)
    if y.__class__ is int:
        _check(y, "ecasq_norm")
    return y


def _is_status(status, like):
    return status is None or (status.dtype == _torch().int32 and status.numel() > 0 and status.get_device() == like.get_device())


def _cache_type(rows, levels):
    """(type, row length) of one side of a paged cache; (None, 0) if it is not one."""
    torch = _torch()
    if rows.dim() != 4 or rows.stride(3) != 1:
        return None, 0
    if levels is None:
        return (rows.dtype, rows.shape[3]) if rows.dtype in _TYPES else (None, 0)
    ok = (rows.dtype == torch.uint8 and levels.dim() == 4 and levels.stride(3) == 1 and levels.shape[:3] == rows.shape[:3]
          and levels.shape[3] in (8, 16) and levels.dtype in (torch.float16, torch.bfloat16))
    return (levels.dtype, 2 * rows.shape[3]) if ok else (None, 0)


_CACHE_IS = ("a cache is [pages, page_size, heads, d] of float32, float16 or bfloat16, or coded uint8 [..., d / 2] with levels "
             "[pages, page_size, heads, 8 or 16] of float16 or bfloat16, with contiguous rows")


def _write_refused(torch, x, Q, m, slots, codes, levels, status):
    where = "ecasq_cache_write"
    _here(where, x, Q, m, slots, codes, levels)
    _no_gradients(where, x, Q, levels)
    rows = lambda: slots.numel() * codes.shape[2]  # noqa: E731
    _need(where,
          (lambda: levels is not None and _cache_type(codes, levels)[0] is not None, _CACHE_IS),
          (lambda: slots.dtype == torch.int64 and slots.is_contiguous(), "slots must be contiguous int64 [n]"),
          (lambda: x.dtype in (torch.float32, levels.dtype) and x.stride(2) == 1
           and x.shape == (slots.numel(), codes.shape[2], 2 * codes.shape[3]),
           "x must be [n, heads, d] of float32 or the cache's type with contiguous entries"),
          (lambda: Q.dtype == torch.float32 and Q.is_contiguous() and 1 <= Q.shape[-1] <= levels.shape[3]
           and Q.numel() == rows() * Q.shape[-1], "Q must be contiguous float32 [n * heads, s], s at most the cache's levels"),
          (lambda: m is None or (m.dtype == torch.int32 and m.is_contiguous() and m.numel() == rows()),
           "m must be contiguous int32 [n * heads]"),
          (lambda: _is_status(status, x), "status must be an int32 tensor on the device of the others"))
    _refuse(where, "bad arguments")


def ecasq_cache_write(x, Q, m, slots, codes, levels, seed, status=None):
    """Encodes new rows x [n, heads, d] into a coded cache, each with its own codebook, by the rounding of ecasq_quantize.

    Q float32 [n * heads, s] or [n, heads, s] and m int32 [n * heads] (or None) as ecasq_solve_batched gives them,
    slots int64 [n] (page * page_size + slot, negative: not written), codes uint8 [pages, page_size, heads, d / 2],
    levels [pages, page_size, heads, 8 or 16] of float16 or bfloat16; x float32 or of levels' type.  status: int32
    tensor that BAD_* bits are or-ed into.  Returns (codes, levels), written in place.
    No gradients: a tensor that requires one is refused while they are recorded."""
    rc = (_codes or _ready()).cache_write(x, Q, m, slots, codes, levels, seed, status)
    if rc is None:
        _write_refused(_torch(), x, Q, m, slots, codes, levels, status)
    if rc:
        _check(rc, "ecasq_cache_write")
    return codes, levels


def workspace_attend(b, heads, kv_heads, d, max_len):
    """A device workspace for ecasq_attend with these sizes or smaller ones, kv_heads and d the same (it may be empty)."""
    torch = _torch()
    n = int(lib().ecasq_workspace_size_attend(int(b), int(heads), int(kv_heads), int(d), int(max_len)))
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def _attend_refused(torch, q, k, v, table, lengths, starts, k_levels, v_levels, max_len, out, ws, status):
    where = "ecasq_attend"
    _here(where, q, k, v, table, lengths, starts, k_levels, v_levels, out, ws)
    _no_gradients(where, q, k, v, k_levels, v_levels, out)
    row = lambda t: t.dtype == torch.int32 and t.shape == q.shape[:1] and t.is_contiguous()  # noqa: E731
    _need(where,
          (lambda: (k_levels is None) == (v_levels is None), "k and v must both be plain or both be coded"),
          (lambda: _cache_type(k, k_levels)[0] is not None and _cache_type(k, k_levels) == _cache_type(v, v_levels)
           and (k_levels is None or k_levels.shape[3] == v_levels.shape[3]), _CACHE_IS + ", k and v alike"),
          (lambda: q.dim() == 3 and q.stride(2) == 1 and (q.dtype, q.shape[2]) == _cache_type(k, k_levels),
           "q must be [b, heads, d] of the cache's type and row length with contiguous entries"),
          (lambda: table.dtype == torch.int32 and table.dim() == 2 and table.shape[0] == q.shape[0]
           and (table.shape[1] < 2 or table.stride(1) == 1), "table must be int32 [b, pages of a sequence] with contiguous rows"),
          (lambda: row(lengths), "lengths must be contiguous int32 [b]"),
          (lambda: starts is None or row(starts), "starts must be contiguous int32 [b]"),
          (lambda: max_len is None or 0 <= max_len <= table.shape[1] * k.shape[1], "the table has too few pages for max_len"),
          (lambda: out is None or (out.dtype == q.dtype and out.shape == q.shape and out.stride(2) == 1), "out must be like q"),
          (lambda: ws is None or (ws.dtype == torch.uint8 and ws.is_contiguous()), "ws must be contiguous uint8"),
          (lambda: _is_status(status, q), "status must be an int32 tensor on the device of the others"))
    _refuse(where, "bad arguments")


def ecasq_attend(q, k, v, table, lengths, scale=None, starts=None, k_levels=None, v_levels=None, max_len=None, out=None,
                 ws=None, status=None):
    """Attention of one new token a sequence over a paged cache of plain or coded rows: (out, lse).

    q [b, heads, d]; k, v [pages, page_size, kv_heads, d] of q's type, or uint8 [..., d / 2] with k_levels, v_levels
    [..., 8 or 16] of q's type; table int32 [b, pages of a sequence]; lengths int32 [b], starts int32 [b] or None: the
    keys [starts, lengths) are seen.  scale: 1 / sqrt(d) if None.  max_len: host bound of the lengths (None: what the table
    holds).  status: int32 tensor that BAD_* bits are or-ed into.  out [b, heads, d] of q's type, lse float32 [b, heads]
    (natural logarithm; -inf where no key is seen, with out = 0).  No gradients: a tensor that requires one is refused while they are
    recorded."""
    both = (_codes or _ready()).attend(q, k, v, table, lengths, scale, starts, k_levels, v_levels, max_len, out, ws, status)
    if both is None:
        _attend_refused(_torch(), q, k, v, table, lengths, starts, k_levels, v_levels, max_len, out, ws, status)
    if both.__class__ is int:
        _check(both, "ecasq_attend")
    return both


def ecasq_kernel_launches() -> int:
    """Kernels the library has launched in this process so far."""
    return int(lib().ecasq_kernel_launches())
