"""Python binding of liberc.so (the C ABI in include/erc.h): argument marshalling only.

Every function here has the name of the C entry point it calls and does nothing but allocate
torch tensors for outputs / workspace, pass raw device pointers and the current CUDA stream, and
turn error codes into exceptions.  All arithmetic runs in the library's CUDA kernels; there is no
CPU path, and loading fails loudly when the library has not been built.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "liberc.so")

ERC_OK = 0
ERC_ERR_INVALID_ARG = 1
ERC_ERR_CUDA = 2
ERC_ERR_CAPACITY = 3
ERC_ERR_NOT_CONVERGED = 4
ERC_ERR_NUMERIC = 5
ERC_ERR_TIMEOUT = 6
ERC_DUP_SUM = 0
ERC_DUP_FIRST = 1
ERC_PRECOND_NONE = 0
ERC_PRECOND_JACOBI = 1

_c_p = ctypes.c_void_p
_i32 = ctypes.c_int32
_i64 = ctypes.c_int64
_u64 = ctypes.c_uint64
_f32 = ctypes.c_float
_sz = ctypes.c_size_t


class ErcError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"erc status {status}: {message}")
        self.status = status


class ErcGraphC(ctypes.Structure):
    _fields_ = [("n", _i32), ("m", _i64), ("row_ptr", _c_p), ("col", _c_p), ("val", _c_p),
                ("deg", _c_p), ("csr_eid", _c_p), ("eu", _c_p), ("ev", _c_p), ("ew", _c_p)]


class ErcSampleRuleC(ctypes.Structure):
    _fields_ = [("temperature", _f32), ("top_k", _i32), ("top_p", _f32), ("min_p", _f32),
                ("temperature_rows", _c_p), ("top_k_rows", _c_p), ("top_p_rows", _c_p),
                ("min_p_rows", _c_p)]


class ErcRouteRuleC(ctypes.Structure):
    _fields_ = [("experts", _i32), ("k", _i32), ("score", _i32), ("groups", _i32),
                ("top_groups", _i32), ("group_best", _i32), ("renorm", _i32), ("scale", _f32)]


class ErcFfnShapeC(ctypes.Structure):
    _fields_ = [("slots", _i64), ("experts", _i32), ("width", _i32), ("inner", _i32), ("act", _i32),
                ("type", _i32)]


class ErcParamsC(ctypes.Structure):
    _fields_ = [("seed", _u64), ("K", _i32), ("kc", _i32), ("eps", _f32), ("tol", _f32),
                ("max_iter", _i32), ("eta", _f32), ("dup_policy", _i32), ("precond", _i32)]


_SIGS = {
    "erc_version": (ctypes.c_char_p, []),
    "erc_last_error": (ctypes.c_char_p, []),
    "erc_kernel_launches": (ctypes.c_uint64, []),
    "erc_set_wait_limit": (None, [ctypes.c_uint32]),
    "erc_build_laplacian_workspace_size": (_sz, [_i32, _i64]),
    "erc_build_laplacian": (_i32, [_i32, _c_p, _c_p, _c_p, _i64, _i32, _c_p, _c_p, _c_p, _c_p,
                                   _c_p, _c_p, _c_p, _c_p, ctypes.POINTER(_i64), _c_p, _sz, _c_p]),
    "erc_build_laplacian_ex": (_i32, [_i32, _c_p, _c_p, _c_p, _i64, _i32, _c_p, _c_p, _c_p, _c_p,
                                      _c_p, _c_p, _c_p, _c_p, ctypes.POINTER(_i64),
                                      ctypes.POINTER(_i32), _c_p, _sz, _c_p]),
    "erc_jl_rhs": (_i32, [ctypes.POINTER(ErcGraphC), _u64, _i32, _i32, _i32, _c_p, _i32, _c_p]),
    "erc_batched_cg_workspace_size": (_sz, [_i32, _i32]),
    "erc_batched_cg": (_i32, [ctypes.POINTER(ErcGraphC), _f32, _c_p, _c_p, _i32, _i32, _f32,
                              _i32, _c_p, _c_p, _c_p, _sz, _c_p]),
    "erc_batched_cg_timed": (_i32, [ctypes.POINTER(ErcGraphC), _f32, _c_p, _c_p, _i32, _i32,
                                    _f32, _i32, _c_p, _c_p, _c_p, _sz, ctypes.POINTER(_f32),
                                    ctypes.POINTER(_i32), _c_p]),
    "erc_batched_pcg": (_i32, [ctypes.POINTER(ErcGraphC), _f32, _c_p, _c_p, _i32, _i32, _f32,
                               _i32, _c_p, _c_p, _c_p, _sz, _c_p]),
    "erc_batched_pcg_timed": (_i32, [ctypes.POINTER(ErcGraphC), _f32, _c_p, _c_p, _i32, _i32,
                                     _f32, _i32, _c_p, _c_p, _c_p, _sz, ctypes.POINTER(_f32),
                                     ctypes.POINTER(_i32), _c_p]),
    "erc_edge_resistance": (_i32, [ctypes.POINTER(ErcGraphC), _c_p, _i32, _i32, _c_p, _c_p]),
    "erc_curvature": (_i32, [ctypes.POINTER(ErcGraphC), _c_p, _c_p, _c_p, _c_p]),
    "erc_sampling_probs_workspace_size": (_sz, [_i32, _i64]),
    "erc_sampling_probs": (_i32, [ctypes.POINTER(ErcGraphC), _c_p, _f32, _c_p, _c_p, _c_p, _sz,
                                  _c_p]),
    "erc_sampling_probs_noalloc": (_i32, [ctypes.POINTER(ErcGraphC), _c_p, _f32, _c_p, _c_p,
                                          _c_p]),
    "erc_sample_workspace_size": (_sz, [_i32, _i64, _i64]),
    "erc_sample_subgraph": (_i32, [ctypes.POINTER(ErcGraphC), _i32, _c_p, _i64, _u64, _i64, _i32,
                                   _c_p, ctypes.POINTER(_i32), _c_p, ctypes.POINTER(_i64), _c_p,
                                   _sz, _c_p]),
    "erc_saint_counts": (_i32, [ctypes.POINTER(ErcGraphC), _c_p, _i32, _c_p, _i64, _c_p, _c_p,
                                _c_p]),
    "erc_saint_norm": (_i32, [ctypes.POINTER(ErcGraphC), _c_p, _c_p, _i32, _c_p, _c_p, _c_p]),
    "erc_laplacian_apply_workspace_size": (_sz, [_i32, _i32]),
    "erc_laplacian_apply": (_i32, [ctypes.POINTER(ErcGraphC), _f32, _c_p, _c_p, _i32, _i32, _c_p,
                                   _c_p, _sz, _c_p]),
    "erc_laplacian_apply_timed": (_i32, [ctypes.POINTER(ErcGraphC), _f32, _c_p, _c_p, _i32,
                                         _i32, _c_p, _i32, ctypes.POINTER(_f32), _c_p, _sz,
                                         _c_p]),
    "erc_philox_signs": (_i32, [_u64, _i64, _i64, _i32, _i32, _c_p, _c_p]),
    "erc_run_workspace_size": (_sz, [_i32, _i64, _i32]),
    "erc_run": (_i32, [ctypes.POINTER(ErcParamsC), _i32, _c_p, _c_p, _c_p, _i64,
                       ctypes.POINTER(_i64), _c_p, _c_p, _c_p, _c_p, _c_p, _c_p, _c_p, _c_p, _c_p,
                       _c_p, _sz, _c_p]),
    "erc_run_host_workspace_size": (_sz, [_i32, _i64, _i32, _i32]),
    "erc_run_host": (_i32, [ctypes.POINTER(ErcParamsC), _i32, _c_p, _c_p, _c_p, _i64,
                            ctypes.POINTER(_i64), _c_p, _c_p, _c_p, _c_p, _c_p, _c_p, _c_p, _c_p,
                            _c_p, _c_p, _sz, _c_p]),
    "erc_sample_rows": (_i32, [_i64, _i64, _c_p, _i32, _i64, _c_p, ctypes.POINTER(ErcSampleRuleC),
                               _c_p, _c_p, _c_p, _c_p]),
    "erc_route": (_i32, [_i64, _c_p, _i32, _i64, _c_p, ctypes.POINTER(ErcRouteRuleC), _c_p, _c_p,
                         _c_p]),
    "erc_route_backward": (_i32, [_i64, _c_p, _i32, _i64, _c_p, _c_p,
                                  ctypes.POINTER(ErcRouteRuleC), _c_p, _c_p]),
    "erc_expert_plan_workspace_size": (_sz, [_i64, _i32, _i32]),
    "erc_expert_plan": (_i32, [_i64, _i32, _i32, _c_p, _c_p, _c_p, _c_p, _c_p, _sz, _c_p]),
    "erc_expert_gather": (_i32, [_i64, _i32, _i64, _c_p, _i32, _c_p, _c_p, _c_p, _c_p]),
    "erc_expert_combine": (_i32, [_i64, _i32, _i64, _c_p, _i32, _c_p, _c_p, _c_p, _c_p]),
    "erc_expert_combine_backward": (_i32, [_i64, _i32, _i64, _c_p, _c_p, _i32, _c_p, _c_p, _c_p,
                                           _c_p, _c_p, _c_p]),
    "erc_score_rows_workspace_size": (_sz, [_i64, _i64, _i32, _i32]),
    "erc_score_rows": (_i32, [_i64, _i64, _c_p, _i32, _i64, _c_p, _f32, _i32, _c_p, _c_p, _c_p,
                              _c_p, _c_p, _c_p, _sz, _c_p]),
    "erc_score_rows_backward": (_i32, [_i64, _i64, _c_p, _i32, _i64, _c_p, _f32, _c_p, _c_p, _c_p,
                                       _c_p, _c_p, _c_p]),
    "erc_expert_ffn_workspace_size": (_sz, [ctypes.POINTER(ErcFfnShapeC)]),
    "erc_expert_ffn": (_i32, [ctypes.POINTER(ErcFfnShapeC), _c_p, _c_p, _c_p, _c_p, _c_p, _c_p,
                              _c_p, _sz, _c_p]),
    "erc_expert_ffn_backward_workspace_size": (_sz, [ctypes.POINTER(ErcFfnShapeC)]),
    "erc_expert_ffn_backward": (_i32, [ctypes.POINTER(ErcFfnShapeC), _c_p, _c_p, _c_p, _c_p, _c_p,
                                       _c_p, _c_p, _c_p, _c_p, _c_p, _sz, _c_p]),
    "erc_dropout": (_i32, [_i64, _c_p, _i32, _c_p, ctypes.c_double, _u64, _c_p, _i64, _c_p, _c_p]),
}

_lib = None


def lib():
    """The loaded liberc.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build(); "
                               "there is no CPU fallback")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGS.items():
            f = getattr(L, name)
            f.restype = res
            f.argtypes = args
        _lib = L
    return _lib


def exported_symbols():
    return list(_SIGS)


def _check(status, allow=()):
    if status != ERC_OK and status not in allow:
        raise ErcError(status, lib().erc_last_error().decode(errors="replace"))
    return status


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _workspace(nbytes, device):
    return torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device=device)


def erc_version():
    return lib().erc_version().decode()


def erc_kernel_launches():
    return int(lib().erc_kernel_launches())


def erc_set_wait_limit(polls):
    """Polls every bounded device-side wait makes before giving up (0 restores the defaults)."""
    lib().erc_set_wait_limit(int(polls))


@dataclass
class Graph:
    """Tensors of a graph built by erc_build_laplacian plus the matching C struct."""

    n: int
    m: int
    row_ptr: torch.Tensor
    col: torch.Tensor
    val: torch.Tensor
    deg: torch.Tensor
    csr_eid: torch.Tensor
    eu: torch.Tensor
    ev: torch.Tensor
    ew: torch.Tensor
    unit_weights: bool

    def c(self):
        g = ErcGraphC()
        g.n, g.m = self.n, self.m
        g.row_ptr, g.col, g.deg, g.csr_eid = (_ptr(self.row_ptr), _ptr(self.col), _ptr(self.deg),
                                              _ptr(self.csr_eid))
        g.val = None if self.unit_weights else _ptr(self.val)
        g.ew = None if self.unit_weights else _ptr(self.ew)
        g.eu, g.ev = _ptr(self.eu), _ptr(self.ev)
        return g


def erc_build_laplacian(n, src, dst, w=None, dup_policy=ERC_DUP_SUM):
    """Device int32 src/dst (and float32 w or None) -> Graph (see include/erc.h)."""
    dev = src.device
    m_in = src.numel()
    cap2, cap1 = max(2 * m_in, 1), max(m_in, 1)
    row_ptr = torch.empty(n + 1, dtype=torch.int64, device=dev)
    col = torch.empty(cap2, dtype=torch.int32, device=dev)
    val = torch.empty(cap2, dtype=torch.float32, device=dev)
    deg = torch.empty(n, dtype=torch.float32, device=dev)
    csr_eid = torch.empty(cap2, dtype=torch.int32, device=dev)
    eu = torch.empty(cap1, dtype=torch.int32, device=dev)
    ev = torch.empty(cap1, dtype=torch.int32, device=dev)
    ew = torch.empty(cap1, dtype=torch.float32, device=dev)
    ws = _workspace(lib().erc_build_laplacian_workspace_size(n, m_in), dev)
    m = _i64(0)
    unit = _i32(0)
    _check(lib().erc_build_laplacian_ex(n, _ptr(src), _ptr(dst), _ptr(w), m_in, dup_policy,
                                        _ptr(row_ptr), _ptr(col), _ptr(val), _ptr(deg),
                                        _ptr(csr_eid), _ptr(eu), _ptr(ev), _ptr(ew),
                                        ctypes.byref(m), ctypes.byref(unit), _ptr(ws), ws.numel(),
                                        _stream()))
    m = m.value
    return Graph(n, m, row_ptr, col[:2 * m], val[:2 * m], deg, csr_eid[:2 * m], eu[:m], ev[:m],
                 ew[:m], bool(unit.value))


def padded_ld(kc):
    return (kc + 3) // 4 * 4


def erc_jl_rhs(g, seed, K, c0, kc, ld=None, out=None):
    ld = padded_ld(kc) if ld is None else ld
    Y = torch.empty(g.n, ld, dtype=torch.float32, device=g.row_ptr.device) if out is None else out
    gc = g.c()
    _check(lib().erc_jl_rhs(ctypes.byref(gc), seed, K, c0, kc, _ptr(Y), ld, _stream()))
    return Y


def _solve(fn, g, eps, Y, kc, tol, max_iter, X, ws, timed):
    n, ld = Y.shape
    dev = Y.device
    X = torch.empty_like(Y) if X is None else X
    iters = torch.empty(kc, dtype=torch.int32, device=dev)
    relres = torch.empty(kc, dtype=torch.float32, device=dev)
    if ws is None:
        ws = _workspace(lib().erc_batched_cg_workspace_size(n, ld), dev)
    gc = g.c()
    args = [ctypes.byref(gc), eps, _ptr(Y), _ptr(X), ld, kc, tol, max_iter, _ptr(iters),
            _ptr(relres), _ptr(ws), ws.numel()]
    if not timed:
        st = _check(getattr(lib(), fn)(*args, _stream()), allow=(ERC_ERR_NOT_CONVERGED,))
        return X, iters, relres, st
    us = _f32(0)
    path = _i32(0)
    st = _check(getattr(lib(), fn)(*args, ctypes.byref(us), ctypes.byref(path), _stream()),
                allow=(ERC_ERR_NOT_CONVERGED,))
    return X, iters, relres, st, float(us.value), int(path.value)


def erc_batched_cg(g, eps, Y, kc, tol, max_iter=20000, X=None, ws=None):
    """Returns (X, iters, relres, status); status is ERC_OK or ERC_ERR_NOT_CONVERGED."""
    return _solve("erc_batched_cg", g, eps, Y, kc, tol, max_iter, X, ws, False)


def erc_batched_cg_timed(g, eps, Y, kc, tol, max_iter=20000, X=None, ws=None):
    """erc_batched_cg plus (solve microseconds, path): 2 = cluster column-group solver, 1 = resident
    cooperative solver, 0 = multi-kernel graph loop."""
    return _solve("erc_batched_cg_timed", g, eps, Y, kc, tol, max_iter, X, ws, True)


def erc_batched_pcg(g, eps, Y, kc, tol, max_iter=20000, X=None, ws=None):
    """Jacobi-preconditioned variant of erc_batched_cg (an option, not the paper's solver)."""
    return _solve("erc_batched_pcg", g, eps, Y, kc, tol, max_iter, X, ws, False)


def erc_batched_pcg_timed(g, eps, Y, kc, tol, max_iter=20000, X=None, ws=None):
    """erc_batched_pcg plus (solve microseconds, path: 1 resident, 0 multi-kernel)."""
    return _solve("erc_batched_pcg_timed", g, eps, Y, kc, tol, max_iter, X, ws, True)


def erc_edge_resistance(g, X, kc, R_acc):
    gc = g.c()
    _check(lib().erc_edge_resistance(ctypes.byref(gc), _ptr(X), X.shape[1], kc, _ptr(R_acc),
                                     _stream()))
    return R_acc


def erc_curvature(g, R):
    dev = R.device
    p = torch.empty(g.n, dtype=torch.float32, device=dev)
    kappa = torch.empty(max(g.m, 1), dtype=torch.float32, device=dev)[:g.m]
    gc = g.c()
    _check(lib().erc_curvature(ctypes.byref(gc), _ptr(R), _ptr(p), _ptr(kappa), _stream()))
    return p, kappa


def erc_sampling_probs(g, kappa, eta=1e-8):
    dev = kappa.device
    pn = torch.empty(g.n, dtype=torch.float32, device=dev)
    pe = torch.empty(max(g.m, 1), dtype=torch.float32, device=dev)[:g.m]
    ws = _workspace(lib().erc_sampling_probs_workspace_size(g.n, g.m), dev)
    gc = g.c()
    _check(lib().erc_sampling_probs(ctypes.byref(gc), _ptr(kappa), eta, _ptr(pn), _ptr(pe),
                                    _ptr(ws), ws.numel(), _stream()))
    return pn, pe


ERC_SAMPLE_NODES, ERC_SAMPLE_EDGES = 0, 1


def erc_sample_subgraph(g, kind, prob, budget, seed, first_draw=0, induced=True, ws=None):
    """One curvature-guided subgraph (see include/erc.h): (nodes int32, edges int32) on device."""
    dev = g.row_ptr.device
    nodes = torch.empty(max(g.n, 1), dtype=torch.int32, device=dev)
    edges = torch.empty(max(g.m, 1), dtype=torch.int32, device=dev)
    if ws is None:
        ws = _workspace(lib().erc_sample_workspace_size(g.n, g.m, budget), dev)
    n_s, m_s = _i32(0), _i64(0)
    gc = g.c()
    _check(lib().erc_sample_subgraph(ctypes.byref(gc), kind, _ptr(prob), budget, seed, first_draw,
                                     int(bool(induced)), _ptr(nodes), ctypes.byref(n_s),
                                     _ptr(edges), ctypes.byref(m_s), _ptr(ws), ws.numel(),
                                     _stream()))
    return nodes[:n_s.value], edges[:m_s.value]


def erc_saint_counts(g, nodes, edges, node_count, edge_count):
    gc = g.c()
    _check(lib().erc_saint_counts(ctypes.byref(gc), _ptr(nodes), nodes.numel(), _ptr(edges),
                                  edges.numel(), _ptr(node_count), _ptr(edge_count), _stream()))


def erc_saint_norm(g, node_count, edge_count, N):
    dev = g.row_ptr.device
    lam = torch.empty(g.n, dtype=torch.float32, device=dev)
    alpha = torch.empty(max(2 * g.m, 1), dtype=torch.float32, device=dev)[:2 * g.m]
    gc = g.c()
    _check(lib().erc_saint_norm(ctypes.byref(gc), _ptr(node_count), _ptr(edge_count), N,
                                _ptr(lam), _ptr(alpha), _stream()))
    return lam, alpha


def erc_sampling_probs_noalloc(g, kappa, eta=1e-8, out=None):
    """erc_sampling_probs without a workspace: the library's static device scratch is used.

    For callers that cannot allocate device memory; pass preallocated `out` = (prob_node,
    prob_edge) to keep the call itself free of allocations on the Python side too.
    """
    dev = kappa.device
    if out is None:
        out = (torch.empty(g.n, dtype=torch.float32, device=dev),
               torch.empty(max(g.m, 1), dtype=torch.float32, device=dev)[:g.m])
    pn, pe = out
    gc = g.c()
    _check(lib().erc_sampling_probs_noalloc(ctypes.byref(gc), _ptr(kappa), eta, _ptr(pn),
                                            _ptr(pe), _stream()))
    return pn, pe


def erc_laplacian_apply(g, eps, P, kc, want_pap=False):
    n, ld = P.shape
    AP = torch.empty_like(P)
    pap = torch.empty(kc, dtype=torch.float64, device=P.device) if want_pap else None
    ws = _workspace(lib().erc_laplacian_apply_workspace_size(n, ld), P.device)
    gc = g.c()
    _check(lib().erc_laplacian_apply(ctypes.byref(gc), eps, _ptr(P), _ptr(AP), ld, kc, _ptr(pap),
                                     _ptr(ws), ws.numel(), _stream()))
    return AP, pap


def erc_laplacian_apply_timed(g, eps, P, kc, reps=50):
    """Mean duration (microseconds) of the operator kernel over `reps` back-to-back launches."""
    n, ld = P.shape
    AP = torch.empty_like(P)
    pap = torch.empty(kc, dtype=torch.float64, device=P.device)
    ws = _workspace(lib().erc_laplacian_apply_workspace_size(n, ld), P.device)
    us = _f32(0)
    gc = g.c()
    _check(lib().erc_laplacian_apply_timed(ctypes.byref(gc), eps, _ptr(P), _ptr(AP), ld, kc,
                                           _ptr(pap), reps, ctypes.byref(us), _ptr(ws),
                                           ws.numel(), _stream()))
    return float(us.value)


def erc_philox_signs(seed, e0, e1, c0, c1, device="cuda"):
    out = torch.empty(max((e1 - e0) * (c1 - c0), 1), dtype=torch.int32, device=device)
    _check(lib().erc_philox_signs(seed, e0, e1, c0, c1, _ptr(out), _stream()))
    return out[:(e1 - e0) * (c1 - c0)].view(e1 - e0, c1 - c0)


@dataclass
class Params:
    K: int
    kc: int
    eps: float = 1e-3
    tol: float = 1e-6
    seed: int = 0xE2C1
    max_iter: int = 20000
    eta: float = 1e-8
    dup_policy: int = ERC_DUP_SUM
    precond: int = ERC_PRECOND_NONE

    def c(self):
        p = ErcParamsC()
        p.seed, p.K, p.kc, p.eps, p.tol = self.seed, self.K, self.kc, self.eps, self.tol
        p.max_iter, p.eta, p.dup_policy = self.max_iter, self.eta, self.dup_policy
        p.precond = self.precond
        return p


def _run_outputs(n, m_in, K, device, pin=False):
    kw = dict(device=device) if not pin else dict(pin_memory=True)
    c1 = max(m_in, 1)
    return dict(eu=torch.empty(c1, dtype=torch.int32, **kw),
                ev=torch.empty(c1, dtype=torch.int32, **kw),
                R=torch.empty(c1, dtype=torch.float32, **kw),
                p=torch.empty(n, dtype=torch.float32, **kw),
                kappa=torch.empty(c1, dtype=torch.float32, **kw),
                prob_node=torch.empty(n, dtype=torch.float32, **kw),
                prob_edge=torch.empty(c1, dtype=torch.float32, **kw),
                iters=torch.empty(K, dtype=torch.int32, **kw),
                relres=torch.empty(K, dtype=torch.float32, **kw))


def _trim(out, m):
    for k in ("eu", "ev", "R", "kappa", "prob_edge"):
        out[k] = out[k][:m]
    out["m"] = m
    return out


def erc_run_workspace(n, m_in, params, device="cuda"):
    return _workspace(lib().erc_run_workspace_size(n, m_in, params.kc), device)


def erc_run(n, src, dst, w, params, ws=None, out=None):
    """The whole path on device-resident inputs; returns a dict of device tensors + status."""
    dev = src.device
    m_in = src.numel()
    if ws is None:
        ws = erc_run_workspace(n, m_in, params, dev)
    o = _run_outputs(n, m_in, params.K, dev) if out is None else out
    m = _i64(0)
    pc = params.c()
    st = _check(lib().erc_run(ctypes.byref(pc), n, _ptr(src), _ptr(dst), _ptr(w), m_in,
                              ctypes.byref(m), _ptr(o["eu"]), _ptr(o["ev"]), _ptr(o["R"]),
                              _ptr(o["p"]), _ptr(o["kappa"]), _ptr(o["prob_node"]),
                              _ptr(o["prob_edge"]), _ptr(o["iters"]), _ptr(o["relres"]),
                              _ptr(ws), ws.numel(), _stream()), allow=(ERC_ERR_NOT_CONVERGED,))
    res = _trim(dict(o), m.value)
    res["status"] = st
    return res


def erc_run_host_workspace(n, m_in, params, device="cuda"):
    return _workspace(lib().erc_run_host_workspace_size(n, m_in, params.kc, params.K), device)


def erc_run_host(n, src, dst, w, params, ws=None, out=None):
    """The whole path from host (ideally pinned) inputs to host outputs, copies included."""
    m_in = src.numel()
    if ws is None:
        ws = erc_run_host_workspace(n, m_in, params)
    o = _run_outputs(n, m_in, params.K, None, pin=True) if out is None else out
    m = _i64(0)
    pc = params.c()
    st = _check(lib().erc_run_host(ctypes.byref(pc), n, _ptr(src), _ptr(dst), _ptr(w), m_in,
                                   ctypes.byref(m), _ptr(o["eu"]), _ptr(o["ev"]), _ptr(o["R"]),
                                   _ptr(o["p"]), _ptr(o["kappa"]), _ptr(o["prob_node"]),
                                   _ptr(o["prob_edge"]), _ptr(o["iters"]), _ptr(o["relres"]),
                                   _ptr(ws), ws.numel(), _stream()),
                allow=(ERC_ERR_NOT_CONVERGED,))
    res = _trim(dict(o), m.value)
    res["status"] = st
    return res


# ------------------------------------------------------------------------------------------------
# row-wise choices: the argument checks that need the tensors' types, shapes and devices are made
# here (the C entry points see raw pointers), and raise ErcError with ERC_ERR_INVALID_ARG.  All tensors
# are on the current device.  Results carry no autograd history: a caller that differentiates wraps
# a call and its gradient in a torch.autograd.Function
# ------------------------------------------------------------------------------------------------
ERC_F32, ERC_BF16, ERC_F16 = 0, 1, 2
ERC_SCORE_SOFTMAX, ERC_SCORE_SIGMOID = 0, 1
_TYPES = {torch.float32: ERC_F32, torch.bfloat16: ERC_BF16, torch.float16: ERC_F16}


def _refuse(message):
    raise ErcError(ERC_ERR_INVALID_ARG, message)


def _need(t, name, dtype, shape, device):
    """`t` is a dense tensor of this type and shape on `device`."""
    if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape
            and t.device == device and t.is_contiguous()):
        _refuse(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {device}")


def _integer(v, name):
    """`v` as an int, of any size."""
    if type(v) is int:
        return v
    try:
        n = int(v)
    except (TypeError, ValueError, OverflowError):
        n = None
    if n is None or n != v:
        _refuse(f"{name} must be a whole number")
    return n


def _whole(v, name):
    """`v` as an int32; a ctypes field would wrap a number that does not fit."""
    if type(v) is int and -2**31 <= v < 2**31:
        return v
    try:
        n = int(v)
    except (TypeError, ValueError, OverflowError):
        n = None
    if n is None or n != v or not -2**31 <= n < 2**31:
        _refuse(f"{name} must be a whole number of 32 bits")
    return n


def _on_current_device(t, name):
    """The library launches on the current device, whichever device a pointer or a stream belongs to."""
    if t.device.index != torch.cuda.current_device():
        _refuse(f"{name} is on {t.device}, which is not the current device")


def _rows_of(t, name):
    """(rows, n, type, row stride) of a matrix of scores with unit element stride."""
    kind = _TYPES.get(t.dtype) if isinstance(t, torch.Tensor) and t.is_cuda else None
    if kind is None or t.dim() != 2:
        _refuse(f"{name} must be a 2-d float32, bfloat16 or float16 CUDA tensor")
    _on_current_device(t, name)
    rows, n = t.shape
    stride, unit = t.stride()
    if n > 1 and unit != 1:
        _refuse(f"the rows of {name} must have unit element stride")
    return rows, n, kind, stride if rows > 1 else n


def _stream_of(t):
    # the raw handle: the Stream object of torch.cuda.current_stream costs 2 us a call
    return torch._C._cuda_getCurrentRawStream(t.device.index)


def erc_sample_rows(logits, words, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One draw from each row of logits [rows, n] (see include/erc.h): (ids int32, logp float32,
    kept int32), each [rows].

    words int64 [rows] holds 64 random bits a row; temperature, top_k, top_p and min_p are numbers,
    or tensors [rows] (float32, int32, float32, float32) with a value for each row.
    """
    rows, n, kind, stride = _rows_of(logits, "logits")
    dev = logits.device
    _need(words, "words", torch.int64, (rows,), dev)
    rule = ErcSampleRuleC(1.0, 0, 1.0, 0.0)
    for name, v, dtype in (("temperature", temperature, torch.float32),
                           ("top_k", top_k, torch.int32), ("top_p", top_p, torch.float32),
                           ("min_p", min_p, torch.float32)):
        if isinstance(v, torch.Tensor):
            _need(v, name, dtype, (rows,), dev)
            setattr(rule, name + "_rows", v.data_ptr())
        elif name == "top_k":
            rule.top_k = _whole(2**31 - 1 if v >= 2**31 else v, name)
        else:
            setattr(rule, name, float(v))
    ids = torch.empty(rows, dtype=torch.int32, device=dev)
    logp = torch.empty(rows, dtype=torch.float32, device=dev)
    kept = torch.empty(rows, dtype=torch.int32, device=dev)
    _check(lib().erc_sample_rows(rows, n, logits.data_ptr(), kind, stride, words.data_ptr(),
                                 ctypes.byref(rule), ids.data_ptr(), logp.data_ptr(),
                                 kept.data_ptr(), _stream_of(logits)))
    return ids, logp, kept


def erc_route(logits, k, score=ERC_SCORE_SOFTMAX, bias=None, groups=1, top_groups=1, group_best=2,
              renorm=True, scale=1.0):
    """k experts of each row of logits [rows, E] (see include/erc.h): (experts int32, weights
    float32), each [rows, k]; bias float32 [E] or None."""
    rows, E, kind, stride = _rows_of(logits, "logits")
    dev = logits.device
    if bias is not None:
        _need(bias, "bias", torch.float32, (E,), dev)
    k = _whole(k, "k")
    rule = ErcRouteRuleC(_whole(E, "E"), k, _whole(score, "score"), _whole(groups, "groups"),
                         _whole(top_groups, "top_groups"), _whole(group_best, "group_best"),
                         int(bool(renorm)), scale)
    experts = torch.empty(rows, max(k, 0), dtype=torch.int32, device=dev)
    weights = torch.empty(rows, max(k, 0), dtype=torch.float32, device=dev)
    _check(lib().erc_route(rows, logits.data_ptr(), kind, stride, _ptr(bias), ctypes.byref(rule),
                           experts.data_ptr(), _ptr(weights), _stream_of(logits)))
    return experts, weights


def erc_route_backward(logits, experts, dweights, score=ERC_SCORE_SOFTMAX, renorm=True, scale=1.0):
    """The gradient of erc_route's weights with respect to logits, for the experts it chose."""
    rows, E, kind, stride = _rows_of(logits, "logits")
    dev = logits.device
    if not (isinstance(experts, torch.Tensor) and experts.dim() == 2):
        _refuse("experts must be [rows, k]")
    k = experts.shape[1]
    _need(experts, "experts", torch.int32, (rows, k), dev)
    _need(dweights, "dweights", torch.float32, (rows, k), dev)
    rule = ErcRouteRuleC(_whole(E, "E"), _whole(k, "k"), _whole(score, "score"), 1, 1, 1, int(bool(renorm)), scale)
    dlogits = torch.empty(rows, E, dtype=logits.dtype, device=dev)
    _check(lib().erc_route_backward(rows, logits.data_ptr(), kind, stride, experts.data_ptr(),
                                    dweights.data_ptr(), ctypes.byref(rule), dlogits.data_ptr(),
                                    _stream_of(logits)))
    return dlogits


def erc_expert_plan(experts, n_experts, ws=None):
    """The pairs of experts int32 [rows, k] in expert order (see include/erc.h): (offsets int64
    [n_experts + 1], order int32 [rows * k], slot int32 [rows, k]).  ws: a uint8 workspace of
    erc_expert_plan_workspace_size bytes, or None."""
    if not (isinstance(experts, torch.Tensor) and experts.is_cuda and experts.dim() == 2):
        _refuse("experts must be a CUDA tensor [rows, k]")
    _on_current_device(experts, "experts")
    rows, k = experts.shape
    dev = experts.device
    _need(experts, "experts", torch.int32, (rows, k), dev)
    k, n_experts = _whole(k, "k"), _whole(n_experts, "n_experts")
    if n_experts < 1:
        _refuse("n_experts out of range")
    offsets = torch.empty(n_experts + 1, dtype=torch.int64, device=dev)
    order = torch.empty(rows * k, dtype=torch.int32, device=dev)
    slot = torch.empty(rows, k, dtype=torch.int32, device=dev)
    if ws is None:
        need = lib().erc_expert_plan_workspace_size(rows, k, n_experts)
        ws = _workspace(need, dev) if need else None
    elif not (isinstance(ws, torch.Tensor) and ws.dtype is torch.uint8 and ws.device == dev
              and ws.is_contiguous()):
        _refuse(f"ws must be a contiguous uint8 tensor on {dev}")
    _check(lib().erc_expert_plan(rows, k, n_experts, experts.data_ptr(), offsets.data_ptr(),
                                 order.data_ptr(), slot.data_ptr(), _ptr(ws),
                                 0 if ws is None else ws.numel(), _stream_of(experts)))
    return offsets, order, slot


def _matrix(t, name):
    kind = _TYPES.get(t.dtype) if isinstance(t, torch.Tensor) and t.is_cuda else None
    if kind is None or t.dim() != 2 or not t.is_contiguous():
        _refuse(f"{name} must be a contiguous 2-d float32, bfloat16 or float16 CUDA tensor")
    _on_current_device(t, name)
    return t.shape[0], t.shape[1], kind


def _slots(slot, rows, dev):
    if not (isinstance(slot, torch.Tensor) and slot.dim() == 2):
        _refuse("slot must be [rows, k]")
    rows = slot.shape[0] if rows is None else rows
    _need(slot, "slot", torch.int32, (rows, slot.shape[1]), dev)
    return rows, _whole(slot.shape[1], "k")


def _placed(offsets, dev):
    if not (isinstance(offsets, torch.Tensor) and offsets.dim() == 1 and offsets.numel() > 0):
        _refuse("offsets must be [n_experts + 1]")
    _need(offsets, "offsets", torch.int64, offsets.shape, dev)
    return offsets.data_ptr() + 8 * (offsets.numel() - 1)


def erc_expert_gather(x, slot, offsets):
    """Rows of x [rows, width] at the slots of their pairs: xs [rows * k, width], zeros from
    offsets[-1] on.  The gradient is erc_expert_combine(dxs, slot)."""
    rows, width, kind = _matrix(x, "x")
    _, k = _slots(slot, rows, x.device)
    xs = torch.empty(rows * k, width, dtype=x.dtype, device=x.device)
    _check(lib().erc_expert_gather(rows, k, width, x.data_ptr(), kind, slot.data_ptr(),
                                   _placed(offsets, x.device), xs.data_ptr(), _stream_of(x)))
    return xs


def erc_expert_combine(y, slot, weights=None):
    """The weighted sum over each row's pairs of y [rows * k, width]: out [rows, width].  The gradient
    is erc_expert_combine_backward, or erc_expert_gather(dout, slot, offsets) where weights is None."""
    slots, width, kind = _matrix(y, "y")
    rows, k = _slots(slot, None, y.device)
    if slots != rows * k:
        _refuse("y must have rows * k rows")
    if weights is not None:
        _need(weights, "weights", torch.float32, (rows, k), y.device)
    out = torch.empty(rows, width, dtype=y.dtype, device=y.device)
    _check(lib().erc_expert_combine(rows, k, width, y.data_ptr(), kind, slot.data_ptr(), _ptr(weights),
                                    out.data_ptr(), _stream_of(y)))
    return out


def erc_expert_combine_backward(dout, y, slot, offsets, weights):
    """The gradient of erc_expert_combine: (dy [rows * k, width], dweights float32 [rows, k])."""
    rows, width, kind = _matrix(dout, "dout")
    dev = dout.device
    _, k = _slots(slot, rows, dev)
    _need(y, "y", dout.dtype, (rows * k, width), dev)
    _need(weights, "weights", torch.float32, (rows, k), dev)
    dy = torch.empty_like(y)
    dweights = torch.empty(rows, k, dtype=torch.float32, device=dev)
    _check(lib().erc_expert_combine_backward(rows, k, width, dout.data_ptr(), y.data_ptr(), kind, slot.data_ptr(),
                                             _placed(offsets, dev), _ptr(weights), dy.data_ptr(),
                                             dweights.data_ptr(), _stream_of(dout)))
    return dy, dweights


# ------------------------------------------------------------------------------------------------
# training and answering: given entries of rows of scores, the experts' products, dropout
# ------------------------------------------------------------------------------------------------
ERC_SCORE_MAX_K = 32
ERC_ACT_SILU, ERC_ACT_GELU, ERC_ACT_RELU = 0, 1, 2


def _given_workspace(ws, need, device):
    """`ws` or a fresh workspace of `need` bytes."""
    if ws is None:
        return torch.empty(need, dtype=torch.uint8, device=device) if need else None
    if not (isinstance(ws, torch.Tensor) and ws.dtype is torch.uint8 and ws.device == device
            and ws.is_contiguous()):
        _refuse(f"ws must be a contiguous uint8 tensor on {device}")
    return ws


def _at(t):
    """The address of a tensor as a plain number, which ctypes takes faster than a c_void_p; None is NULL."""
    return None if t is None else t.data_ptr()


def erc_score_rows(logits, ids=None, temperature=1.0, k=0, ws=None):
    """What each row of logits [rows, n] says about the entry ids[row] (see include/erc.h):
    (logp float32 [rows], entropy float32 [rows], norm float32 [rows, 2], top_ids int32 [rows, k],
    top_logp float32 [rows, k]); logp is None without ids, the last two without k.

    ids int32 [rows]; an id outside [0, n) gives 0.  norm is what erc_score_rows_backward takes.  ws: a
    uint8 workspace of erc_score_rows_workspace_size bytes, or None.
    """
    rows, n, kind, stride = _rows_of(logits, "logits")
    dev = logits.device
    if ids is not None:
        _need(ids, "ids", torch.int32, (rows,), dev)
    k = _whole(k, "k")
    if not 0 <= k <= ERC_SCORE_MAX_K:
        _refuse(f"k must be in [0, {ERC_SCORE_MAX_K}]")
    logp = torch.empty(rows, dtype=torch.float32, device=dev) if ids is not None else None
    entropy = torch.empty(rows, dtype=torch.float32, device=dev)
    norm = torch.empty((rows, 2), dtype=torch.float32, device=dev)
    top_ids = torch.empty((rows, k), dtype=torch.int32, device=dev) if k else None
    top_logp = torch.empty((rows, k), dtype=torch.float32, device=dev) if k else None
    L = lib()
    need = L.erc_score_rows_workspace_size(rows, n, kind, k)
    if need or ws is not None:
        ws = _given_workspace(ws, need, dev)
    status = L.erc_score_rows(rows, n, logits.data_ptr(), kind, stride, _at(ids), temperature, k, _at(logp),
                              entropy.data_ptr(), norm.data_ptr(), _at(top_ids), _at(top_logp), _at(ws),
                              0 if ws is None else ws.numel(), _stream_of(logits))
    if status:
        _check(status)
    return logp, entropy, norm, top_ids, top_logp


def erc_score_rows_backward(logits, ids, norm, dlogp=None, entropy=None, dentropy=None, temperature=1.0):
    """The gradient of erc_score_rows' logp and entropy: dlogits [rows, n] from dlogp and dentropy
    float32 [rows] (None: 0), with the forward call's norm and entropy."""
    rows, n, kind, stride = _rows_of(logits, "logits")
    dev = logits.device
    _need(norm, "norm", torch.float32, (rows, 2), dev)
    for name, t, dtype in (("ids", ids, torch.int32), ("dlogp", dlogp, torch.float32),
                           ("entropy", entropy, torch.float32), ("dentropy", dentropy, torch.float32)):
        if t is not None:
            _need(t, name, dtype, (rows,), dev)
    dlogits = torch.empty(rows, n, dtype=logits.dtype, device=dev)
    _check(lib().erc_score_rows_backward(rows, n, logits.data_ptr(), kind, stride, _at(ids), temperature,
                                         norm.data_ptr(), _at(entropy), _at(dlogp), _at(dentropy),
                                         dlogits.data_ptr(), _stream_of(logits)))
    return dlogits


def _ffn_shape(x, name, offsets, w_in, w_out, act):
    """The shape of a block, with its weights and offsets checked against x [slots, width]."""
    slots, width, kind = _matrix(x, name)
    dev, dtype = x.device, x.dtype
    if not (isinstance(offsets, torch.Tensor) and offsets.dtype is torch.int64 and offsets.dim() == 1
            and offsets.device == dev and offsets.is_contiguous() and offsets.numel() > 0):
        _refuse(f"offsets must be a contiguous int64 tensor [n_experts + 1] on {dev}")
    experts = offsets.numel() - 1
    if not (isinstance(w_out, torch.Tensor) and w_out.dim() == 3):
        _refuse("w_out must be [experts, width, inner]")
    inner = w_out.shape[2]
    _need(w_out, "w_out", dtype, (experts, width, inner), dev)
    _need(w_in, "w_in", dtype, (experts, 2 * inner, width), dev)
    return ErcFfnShapeC(slots, experts, _whole(width, "width"), _whole(inner, "inner"), _whole(act, "act"), kind)


def erc_expert_ffn(xs, offsets, w_in, w_out, act=ERC_ACT_SILU, keep=False, ws=None):
    """The gated feed-forward block of each expert on its rows of xs [slots, width] (see include/erc.h):
    (y [slots, width], pre [slots, 2 inner] or None).

    offsets int64 [experts + 1] as from erc_expert_plan (a dense block: [0, slots]); w_in [experts,
    2 inner, width], w_out [experts, width, inner].  keep: also return pre, which the gradient takes.
    ws: a uint8 workspace of erc_expert_ffn_workspace_size bytes, or None; it holds the status of the
    device's waits.  Where one ran out, results that were not reached are NaN.
    """
    shape = _ffn_shape(xs, "xs", offsets, w_in, w_out, act)
    dev = xs.device
    y = torch.empty_like(xs)
    pre = torch.empty(shape.slots, 2 * shape.inner, dtype=xs.dtype, device=dev) if keep else None
    L, ref = lib(), ctypes.byref(shape)
    ws = _given_workspace(ws, L.erc_expert_ffn_workspace_size(ref), dev)
    status = L.erc_expert_ffn(ref, xs.data_ptr(), offsets.data_ptr(), w_in.data_ptr(), w_out.data_ptr(), y.data_ptr(),
                              _at(pre), _at(ws), 0 if ws is None else ws.numel(), _stream_of(xs))
    if status:
        _check(status)
    return y, pre


def erc_expert_ffn_backward(dy, xs, pre, offsets, w_in, w_out, act=ERC_ACT_SILU, dxs=True, dw=True, ws=None):
    """The gradient of erc_expert_ffn from dy [slots, width] and the forward call's pre: (dxs, dw_in,
    dw_out); dxs, dw: which of the rows' and the weights' to form (None for the others)."""
    shape = _ffn_shape(xs, "xs", offsets, w_in, w_out, act)
    dev = xs.device
    _need(dy, "dy", xs.dtype, xs.shape, dev)
    _need(pre, "pre", xs.dtype, (shape.slots, 2 * shape.inner), dev)
    out = (torch.empty_like(xs) if dxs else None, torch.empty_like(w_in) if dw else None,
           torch.empty_like(w_out) if dw else None)
    L, ref = lib(), ctypes.byref(shape)
    ws = _given_workspace(ws, L.erc_expert_ffn_backward_workspace_size(ref), dev)
    _check(L.erc_expert_ffn_backward(ref, dy.data_ptr(), xs.data_ptr(), pre.data_ptr(), offsets.data_ptr(),
                                     w_in.data_ptr(), w_out.data_ptr(), _at(out[0]), _at(out[1]), _at(out[2]),
                                     _at(ws), 0 if ws is None else ws.numel(), _stream_of(xs)))
    return out


def erc_dropout(x, p, key, residual=None, first=0):
    """Dropout of a contiguous tensor from the generator's stream of `key`, plus the residual (see
    include/erc.h).  The gradient of x is the same call on out's gradient, without the residual.

    key: a whole number (mod 2^64), or an int64 tensor [1], read when the kernel runs; first: the
    stream's number of x's first entry, a multiple of 4.
    """
    kind = _TYPES.get(x.dtype) if isinstance(x, torch.Tensor) and x.is_cuda else None
    if kind is None or not x.is_contiguous():
        _refuse("x must be a contiguous float32, bfloat16 or float16 CUDA tensor")
    _on_current_device(x, "x")
    if residual is not None:
        _need(residual, "residual", x.dtype, x.shape, x.device)
    if isinstance(key, torch.Tensor):
        _need(key, "key", torch.int64, (1,), x.device)
        number, at = 0, key.data_ptr()
    else:
        number, at = _integer(key, "key") % 2**64, None
    first = _integer(first, "first")
    if not 0 <= first < 2**62:
        _refuse("first must be in [0, 2^62)")
    out = torch.empty_like(x)
    status = lib().erc_dropout(x.numel(), x.data_ptr(), kind, _at(residual), p, number, at, first, out.data_ptr(),
                               _stream_of(x))
    if status:
        _check(status)
    return out
