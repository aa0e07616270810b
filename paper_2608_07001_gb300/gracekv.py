"""Python binding of the GraceKV compression library (include/gracekv.h).

Argument marshalling only: every step of the compression pass runs in the
CUDA kernels of libgracekv.so.  Tensors are torch CUDA tensors (device
memory); calls are enqueued on the current torch stream.  There is no CPU
fallback: importing this module fails if the library is missing.
"""
from __future__ import annotations

import ctypes as C
import dataclasses
import os
import struct
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIBPATH = os.path.join(_HERE, "libgracekv.so")

GKV_OK, GKV_EINVAL, GKV_EBUDGET, GKV_ENOMEM, GKV_ECUDA, GKV_ETIMEOUT = 0, 1, 2, 3, 4, 5
GKV_ENONFINITE, GKV_ESTATE, GKV_EUNSUPPORTED, GKV_ECAPACITY = 6, 7, 8, 9
GKV_F32, GKV_BF16 = 0, 1


class GkvParams(C.Structure):
    _fields_ = [
        ("L", C.c_int32), ("G", C.c_int32), ("Hq", C.c_int32), ("T", C.c_int32),
        ("d", C.c_int32), ("W", C.c_int32), ("dtype", C.c_int32),
        ("ctx_start", C.c_int32), ("ctx_end", C.c_int32), ("recent", C.c_int32),
        ("budget", C.c_int64), ("rope_base", C.c_double),
        ("n_min", C.c_int32), ("n_max", C.c_int32), ("n0", C.c_int32),
        ("lambda_stab", C.c_double), ("lambda_s", C.c_double), ("lambda_d", C.c_double),
        ("lambda_n", C.c_double), ("c_cut", C.c_double),
        ("seg_layers", C.c_int32 * 8), ("n_seg_layers", C.c_int32),
        ("windows", C.c_int32 * 4), ("n_windows", C.c_int32),
        ("k_cand", C.c_int32),
        ("lambda_kappa", C.c_double), ("lambda_Z", C.c_double), ("lambda_M", C.c_double),
        ("eps", C.c_double), ("base_frac", C.c_double),
        ("lambda_graph", C.c_double), ("alpha_floor", C.c_double),
        ("seg_mode", C.c_int32), ("quota_alloc", C.c_int32),
        ("floor_c", C.c_double), ("floor_gamma", C.c_double), ("floor_eta", C.c_double),
        ("floor_half", C.c_int32),
        ("eta_seed", C.c_double), ("rho_hop", C.c_double), ("m_seed", C.c_int32), ("r_hop", C.c_int32),
        ("dp_warmup", C.c_int32),
    ]


class GkvDecodeCache(C.Structure):
    _fields_ = [
        ("L", C.c_int32), ("G", C.c_int32), ("Hq", C.c_int32), ("d", C.c_int32),
        ("dtype", C.c_int32), ("K", C.c_void_p), ("V", C.c_void_p), ("log_m", C.c_void_p),
        ("offsets", C.c_void_p), ("n_entries", C.c_int64), ("K_app", C.c_void_p),
        ("V_app", C.c_void_p), ("app_cap", C.c_int32),
    ]


class GkvPrompt(C.Structure):
    _fields_ = [
        ("G", C.c_int32), ("Hq", C.c_int32), ("d", C.c_int32), ("dtype", C.c_int32), ("n_seqs", C.c_int32),
        ("n_q", C.c_int64), ("n_k", C.c_int64), ("cu_q", C.c_void_p), ("cu_k", C.c_void_p),
        ("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p), ("out", C.c_void_p), ("lse", C.c_void_p),
    ] + [(n, C.c_int64) for n in ("q_ts", "q_hs", "k_ts", "k_hs", "v_ts", "v_hs", "o_ts", "o_hs")]


class GkvPagedCache(C.Structure):
    _fields_ = [
        ("L", C.c_int32), ("B", C.c_int32), ("G", C.c_int32), ("Hq", C.c_int32), ("d", C.c_int32),
        ("dtype", C.c_int32), ("page_size", C.c_int32), ("max_pages", C.c_int32), ("n_pages", C.c_int64),
        ("K", C.c_void_p), ("V", C.c_void_p), ("log_m", C.c_void_p), ("table", C.c_void_p),
        ("lens", C.c_void_p), ("rope_base", C.c_double),
    ]


class GkvPagedTokens(C.Structure):
    _fields_ = [("n_tokens", C.c_int32)] + [(n, C.c_void_p) for n in ("cu_new", "pos", "k", "v", "q", "q_out")] + [
        (n, C.c_int64) for n in ("k_ts", "k_hs", "v_ts", "v_hs", "q_ts", "q_hs", "qo_ts", "qo_hs")]


class GkvPagedScales(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p)]


class GkvPagedRows(C.Structure):
    _fields_ = [("n_tokens", C.c_int32)] + [(n, C.c_void_p) for n in ("cu_new", "k", "v")] + [
        (n, C.c_int64) for n in ("k_ts", "k_hs", "v_ts", "v_hs")]


# the structures that every call fills, packed in one go
_PROMPT, _TOKENS, _ROWS = struct.Struct("@5i4x2q7P8q"), struct.Struct("@i4x6P8q"), struct.Struct("@i4x3P4q")
assert _PROMPT.size == C.sizeof(GkvPrompt) and _TOKENS.size == C.sizeof(GkvPagedTokens) and _ROWS.size == C.sizeof(GkvPagedRows)


class GraceKVError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"gracekv status {status}: {msg}")
        self.status = status


_lib = None

EXPORTED = ["gracekv_default_params", "gracekv_budget_for_ratio", "gracekv_graph_layers",
            "gracekv_create",
            "gracekv_destroy", "gracekv_last_error", "gracekv_status_string", "gracekv_query",
            "gracekv_segment", "gracekv_score", "gracekv_build_trees", "gracekv_allocate", "gracekv_gather",
            "gracekv_export", "gracekv_profile", "gracekv_stats", "gracekv_row_stats_noalloc",
            "gracekv_compress_host", "gracekv_export_floor", "gracekv_head_sensitivity",
            "gracekv_set_graph_queries", "gracekv_decode_workspace_size", "gracekv_decode_append",
            "gracekv_decode_attention", "gracekv_decode_status",
            "gracekv_prompt_workspace_size", "gracekv_prompt_attention", "gracekv_prompt_status",
            "gracekv_paged_workspace_size", "gracekv_paged_load", "gracekv_paged_advance",
            "gracekv_paged_append", "gracekv_paged_attention", "gracekv_paged_status",
            "gracekv_quant_load", "gracekv_quant_append", "gracekv_quant_attention", "gracekv_paged_read", "gracekv_paged_unload",
            "gracekv_shared_workspace_size", "gracekv_shared_attention", "gracekv_shared_status"]


def lib() -> C.CDLL:
    """Load libgracekv.so (built by __graft_entry__.build()); raises if absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIBPATH):
        raise ImportError(f"{LIBPATH} is missing: build it with __graft_entry__.build()")
    L = C.CDLL(LIBPATH)
    vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
    L.gracekv_default_params.argtypes = [C.POINTER(GkvParams)]
    L.gracekv_budget_for_ratio.argtypes = [i32, i32, i32, C.c_double]
    L.gracekv_budget_for_ratio.restype = i64
    L.gracekv_graph_layers.argtypes = [i32, C.POINTER(i32)]
    L.gracekv_graph_layers.restype = i32
    L.gracekv_create.argtypes = [C.POINTER(GkvParams), C.POINTER(vp)]
    L.gracekv_destroy.argtypes = [vp]
    L.gracekv_destroy.restype = None
    L.gracekv_last_error.argtypes = [vp]
    L.gracekv_last_error.restype = C.c_char_p
    L.gracekv_status_string.argtypes = [C.c_int]
    L.gracekv_status_string.restype = C.c_char_p
    L.gracekv_query.argtypes = [vp, C.POINTER(i32), C.POINTER(i32), C.POINTER(i64), C.POINTER(i32)]
    L.gracekv_segment.argtypes = [vp, vp, vp, i32, vp, vp, i32, C.POINTER(i32), vp, vp]
    L.gracekv_build_trees.argtypes = [vp, vp, vp, vp, vp, vp, i32, vp]
    L.gracekv_score.argtypes = [vp, vp, vp, vp]
    L.gracekv_compress_host.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i64, C.POINTER(i64), vp]
    L.gracekv_allocate.argtypes = [vp, C.POINTER(i64), vp]
    L.gracekv_gather.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i64, vp]
    L.gracekv_export.argtypes = [vp, i64, C.POINTER(i64)] + [vp] * 18 + [vp]
    L.gracekv_export_floor.argtypes = [vp, vp, vp, C.POINTER(i64), vp]
    L.gracekv_set_graph_queries.argtypes = [vp, vp, i32]
    L.gracekv_head_sensitivity.argtypes = [vp, vp] + [i32] * 7 + [vp, vp, vp]
    L.gracekv_profile.argtypes = [vp, i32]
    L.gracekv_stats.argtypes = [vp, vp, i32, C.POINTER(i64), vp, i32]
    L.gracekv_row_stats_noalloc.argtypes = [vp, vp] + [i32] * 9 + [vp, vp, vp, vp]
    dcp = C.POINTER(GkvDecodeCache)
    L.gracekv_decode_workspace_size.argtypes = [dcp, C.POINTER(C.c_size_t)]
    L.gracekv_decode_append.argtypes = [dcp, i32, i32, i32, vp, vp, vp]
    L.gracekv_decode_attention.argtypes = [dcp, i32, i32, i32, vp, vp, vp, vp]
    L.gracekv_decode_status.argtypes = [vp, vp]
    prp, pcp = C.POINTER(GkvPrompt), C.POINTER(GkvPagedCache)
    L.gracekv_prompt_workspace_size.argtypes = [prp, C.POINTER(C.c_size_t)]
    L.gracekv_prompt_attention.argtypes = [prp, vp, vp]
    L.gracekv_prompt_status.argtypes = [vp, vp]
    L.gracekv_paged_workspace_size.argtypes = [pcp, C.POINTER(C.c_size_t)]
    L.gracekv_paged_load.argtypes = [pcp, i32, vp, vp, vp, vp, i64, vp, vp]
    L.gracekv_paged_advance.argtypes = [pcp, vp, vp]
    L.gracekv_paged_append.argtypes = [pcp, i32, C.POINTER(GkvPagedTokens), vp, vp]
    L.gracekv_paged_attention.argtypes = [pcp, i32, vp, vp, vp, vp]
    L.gracekv_paged_status.argtypes = [vp, vp]
    scp = C.POINTER(GkvPagedScales)
    L.gracekv_quant_load.argtypes = [pcp, scp, i32, vp, vp, vp, vp, i64, vp, vp]
    L.gracekv_quant_append.argtypes = [pcp, scp, i32, C.POINTER(GkvPagedTokens), vp, vp]
    L.gracekv_quant_attention.argtypes = [pcp, scp, i32, vp, vp, vp, vp]
    L.gracekv_paged_read.argtypes = [pcp, scp, i32, C.POINTER(GkvPagedRows), vp, vp]
    L.gracekv_paged_unload.argtypes = [pcp, scp, i32, vp, vp, vp, vp, i64, vp, vp]
    L.gracekv_shared_workspace_size.argtypes = [pcp, pcp, C.POINTER(C.c_size_t)]
    L.gracekv_shared_attention.argtypes = [pcp, scp, pcp, scp, i32, vp, vp, vp, vp, vp]
    L.gracekv_shared_status.argtypes = [vp, vp]
    _lib = L
    return L


def gracekv_default_params() -> GkvParams:
    p = GkvParams()
    lib().gracekv_default_params(C.byref(p))
    return p


def gracekv_budget_for_ratio(L: int, G: int, n_ctx: int, x: float) -> int:
    return int(lib().gracekv_budget_for_ratio(L, G, n_ctx, float(x)))


def gracekv_graph_layers(L: int) -> list:
    """The multi-hop relevance's graph layers for an L-layer model."""
    out = (C.c_int32 * 2)()
    n = int(lib().gracekv_graph_layers(int(L), out))
    if n < 0:
        _raise(GKV_EINVAL)
    return [int(out[k]) for k in range(n)]


graph_layers = gracekv_graph_layers


def gracekv_row_stats_noalloc(K, Q, c_lo: int, c_hi: int, row_m, row_Z, row_ZC, stream=None):
    """Row statistics without a context and without any device allocation.

    For callers that cannot call cudaMalloc (an engine owning the device's
    memory pool, or a loop that cannot afford an allocation's synchronisation):
    the scratch is a fixed 4 MiB array inside the library.  Outputs are
    caller-provided [L, Hq, W] fp32 CUDA tensors.  Overlapping calls race.
    Every argument is checked here before the library is called (a wrong
    element size or a short output would otherwise become an out-of-bounds
    device access); a mismatch raises GraceKVError(GKV_EINVAL).
    """
    def bad(why):
        return GraceKVError(GKV_EINVAL, "row_stats_noalloc: " + why)

    if K.dim() != 4 or Q.dim() != 4:
        raise bad("K is [L, G, T, d] and Q is [L, Hq, W, d]")
    L, G, T, d = K.shape
    Hq, W = Q.shape[1], Q.shape[2]
    if K.dtype not in (torch.bfloat16, torch.float32):
        raise bad(f"K must be bf16 or fp32, not {K.dtype}")
    if Q.dtype != K.dtype:
        raise bad(f"Q must have K's dtype {K.dtype}, not {Q.dtype}")
    if Q.shape[0] != L or Q.shape[3] != d:
        raise bad(f"Q {tuple(Q.shape)} does not match K {tuple(K.shape)} in L or d")
    for name, o in (("row_m", row_m), ("row_Z", row_Z), ("row_ZC", row_ZC)):
        if o.dtype != torch.float32 or o.numel() < L * Hq * W:
            raise bad(f"{name} must be fp32 with at least L*Hq*W = {L * Hq * W} elements")
        if o.device != K.device:
            raise bad(f"{name} is on {o.device}, K on {K.device}")
    if Q.device != K.device:
        raise bad(f"Q is on {Q.device}, K on {K.device}")
    dt = GKV_BF16 if K.dtype == torch.bfloat16 else GKV_F32
    st = lib().gracekv_row_stats_noalloc(_ptr(K), _ptr(Q), L, G, Hq, T, d, W, dt, c_lo, c_hi,
                                         _ptr(row_m), _ptr(row_Z), _ptr(row_ZC), _stream(stream))
    if st != GKV_OK:
        raise GraceKVError(st, lib().gracekv_status_string(st).decode())


def gracekv_head_sensitivity(W_O, o, G: int, stream=None):
    """omega [L, G] (fp32, device) from W_O [L, D, Hq*d] and o [L, Hq, U, d] (bf16)."""
    L, D, _ = W_O.shape
    _, Hq, U, d = o.shape
    om = torch.empty(L, G, dtype=torch.float32, device=W_O.device)
    scratch = torch.empty(L * G * 65, dtype=torch.float32, device=W_O.device)
    st = lib().gracekv_head_sensitivity(_ptr(W_O), _ptr(o), L, G, Hq, d, D, U, GKV_BF16, _ptr(om),
                                        _ptr(scratch), _stream(stream))
    if st != GKV_OK:
        raise GraceKVError(st, lib().gracekv_status_string(st).decode())
    return om


def _host_ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if t.is_cuda or not t.is_contiguous():
        raise ValueError("tensors must be contiguous host tensors")
    return C.c_void_p(t.data_ptr())


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("tensors must be contiguous CUDA tensors")
    return C.c_void_p(t.data_ptr())


def _stream(stream=None):
    s = stream if stream is not None else torch.cuda.current_stream()
    return C.c_void_p(s.cuda_stream)


def make_params(L, G, Hq, T, d, W, *, dtype, budget, rope_base, ctx_start=0, ctx_end=None,
                **overrides) -> GkvParams:
    p = gracekv_default_params()
    p.L, p.G, p.Hq, p.T, p.d, p.W = L, G, Hq, T, d, W
    p.dtype = GKV_BF16 if dtype in (torch.bfloat16, "bf16") else GKV_F32
    p.ctx_start = ctx_start
    p.ctx_end = T if ctx_end is None else ctx_end
    p.budget = int(budget)
    p.rope_base = float(rope_base)
    for k, v in overrides.items():
        if k == "windows":
            for i, w in enumerate(v):
                p.windows[i] = w
            p.n_windows = len(v)
        elif k == "seg_layers":
            for i, w in enumerate(v):
                p.seg_layers[i] = w
            p.n_seg_layers = len(v)
        else:
            setattr(p, k, v)
    return p


class Context:
    """Owns a gracekv_ctx; the four stage calls follow the C ABI one to one."""

    def __init__(self, params: GkvParams):
        self.params = params
        h = C.c_void_p()
        st = lib().gracekv_create(C.byref(params), C.byref(h))
        if st != GKV_OK:
            raise GraceKVError(st, lib().gracekv_status_string(st).decode())
        self.h = h
        r, nc, bf, js = C.c_int32(), C.c_int32(), C.c_int64(), C.c_int32()
        lib().gracekv_query(self.h, C.byref(r), C.byref(nc), C.byref(bf), C.byref(js))
        self.recent, self.n_c, self.b_free = r.value, nc.value, bf.value

    def close(self):
        if getattr(self, "h", None):
            lib().gracekv_destroy(self.h)
            self.h = None

    __del__ = close

    def _check(self, st: int):
        if st != GKV_OK:
            msg = lib().gracekv_last_error(self.h).decode()
            raise GraceKVError(st, msg or lib().gracekv_status_string(st).decode())

    def gracekv_segment(self, V, slot_starts, hidden=None, surprisal=None, kappa=None, stream=None) -> int:
        n = C.c_int32()
        Dh = 0 if hidden is None else hidden.shape[-1]
        self._check(lib().gracekv_segment(self.h, _ptr(V), _ptr(hidden), Dh, _ptr(surprisal),
                                          _ptr(slot_starts), slot_starts.numel() - 1, C.byref(n),
                                          _ptr(kappa), _stream(stream)))
        return n.value

    def gracekv_compress_host(self, K, V, Q, out: "Cache", omega=None, stream=None) -> int:
        """The whole pass from host tensors (pinned for the full copy rate)
        into the host cache `out`; returns the number of entries."""
        n = C.c_int64()
        hp = [_host_ptr(t) for t in (K, V, Q, omega, out.K, out.V, out.pos, out.log_m, out.src_lo,
                                     out.src_hi, out.offsets)]
        self._check(lib().gracekv_compress_host(self.h, *hp, out.K.shape[0], C.byref(n), _stream(stream)))
        return n.value

    def gracekv_score(self, K, Q, stream=None):
        self._check(lib().gracekv_score(self.h, _ptr(K), _ptr(Q), _stream(stream)))

    def gracekv_build_trees(self, K, V, Q, omega=None, slot_starts=None, n_slots=0, stream=None):
        self._check(lib().gracekv_build_trees(self.h, _ptr(K), _ptr(V), _ptr(Q), _ptr(omega),
                                              _ptr(slot_starts), n_slots, _stream(stream)))

    def gracekv_allocate(self, stream=None) -> int:
        n = C.c_int64()
        self._check(lib().gracekv_allocate(self.h, C.byref(n), _stream(stream)))
        return n.value

    def gracekv_gather(self, K, V, out: "Cache", stream=None):
        self._check(lib().gracekv_gather(self.h, _ptr(K), _ptr(V), _ptr(out.K), _ptr(out.V),
                                         _ptr(out.pos), _ptr(out.log_m), _ptr(out.src_lo),
                                         _ptr(out.src_hi), _ptr(out.offsets), out.K.shape[0],
                                         _stream(stream)))

    STAGES = ("segment", "row_stats", "token_values", "unit_trees", "allocate", "gather", "floor",
              "multihop")

    def gracekv_set_graph_queries(self, Qg):
        """Qg [n_graph, Hq, T, d] bf16: queries of every position at the graph layers."""
        self._check(lib().gracekv_set_graph_queries(self.h, _ptr(Qg), Qg.shape[0]))
        self._Qg = Qg

    def gracekv_export_floor(self, stream=None) -> dict:
        """The singleton floor of the last tree build (host arrays)."""
        import numpy as np
        p = self.params
        LG = p.L * p.G
        acc = np.zeros((LG, self.n_c), np.uint8)
        f = np.zeros((LG, self.n_c), np.float32)
        bf = C.c_int64()
        self._check(lib().gracekv_export_floor(self.h, C.c_void_p(acc.ctypes.data), C.c_void_p(f.ctypes.data),
                                               C.byref(bf), _stream(stream)))
        return dict(accepted=acc, f=f, B_floor=bf.value)

    def gracekv_profile(self, enable: bool = True):
        self._check(lib().gracekv_profile(self.h, int(enable)))

    def gracekv_stats(self):
        """(per-stage ms since the last call, kernels launched so far, tree work counters)."""
        import numpy as np
        ms = np.zeros(len(self.STAGES), np.float32)
        work = np.zeros(6, np.uint64)
        n = C.c_int64()
        self._check(lib().gracekv_stats(self.h, C.c_void_p(ms.ctypes.data), len(ms), C.byref(n),
                                        C.c_void_p(work.ctypes.data), len(work)))
        names = ("scan_steps", "cand_evals", "cand_len_sum", "units", "dp_chunks", "dp_rerun")
        return dict(zip(self.STAGES, ms.tolist())), n.value, dict(zip(names, map(int, work)))

    def gracekv_export(self, node_cap: Optional[int] = None, stream=None) -> dict:
        """Host copy of the trees and selection (introspection for tests)."""
        import numpy as np
        p = self.params
        js = C.c_int32()
        lib().gracekv_query(self.h, None, None, None, C.byref(js))
        J = js.value
        nu = p.L * p.G * J
        cap = node_cap or p.L * p.G * 2 * self.n_c
        nrow = p.L * p.Hq * p.W
        arr = dict(unit_first=np.zeros(nu + 1, np.int64), unit_Uadd=np.zeros(nu, np.float32),
                   unit_Ddrop=np.zeros(nu, np.float32), add_sel=np.zeros(nu, np.uint8),
                   a=np.zeros(cap, np.int32), b=np.zeros(cap, np.int32),
                   child0=np.zeros(cap, np.int32), nchild=np.zeros(cap, np.int32),
                   cost=np.zeros(cap, np.int32), D=np.zeros(cap, np.float32),
                   R=np.zeros(cap, np.float32), U=np.zeros(cap, np.float32),
                   kappa=np.zeros(cap, np.float32), split_sel=np.zeros(cap, np.uint8),
                   row_m=np.zeros(nrow, np.float32), row_Z=np.zeros(nrow, np.float32),
                   row_ZC=np.zeros(nrow, np.float32), rtok=np.zeros(p.L * p.G * self.n_c, np.float32))
        order = ["unit_first", "unit_Uadd", "unit_Ddrop", "add_sel", "a", "b", "child0", "nchild",
                 "cost", "D", "R", "U", "kappa", "split_sel", "row_m", "row_Z", "row_ZC", "rtok"]
        nn = C.c_int64()
        self._check(lib().gracekv_export(self.h, cap, C.byref(nn),
                                         *[C.c_void_p(arr[k].ctypes.data) for k in order],
                                         _stream(stream)))
        n = nn.value
        for k in ["a", "b", "child0", "nchild", "cost", "D", "R", "U", "kappa", "split_sel"]:
            arr[k] = arr[k][:n]
        arr["J"] = J
        return arr


@dataclasses.dataclass
class Cache:
    """Ragged compressed cache (device tensors, capacity rows)."""
    K: torch.Tensor
    V: torch.Tensor
    pos: torch.Tensor
    log_m: torch.Tensor
    src_lo: torch.Tensor
    src_hi: torch.Tensor
    offsets: torch.Tensor

    @staticmethod
    def empty_host(cap: int, d: int, LG: int, dtype) -> "Cache":
        """Page-locked host arrays (the output of gracekv_compress_host)."""
        c = Cache.empty(cap, d, LG, dtype, device="cpu")
        return Cache(*(t.pin_memory() for t in (c.K, c.V, c.pos, c.log_m, c.src_lo, c.src_hi, c.offsets)))

    @staticmethod
    def empty(cap: int, d: int, LG: int, dtype, device="cuda") -> "Cache":
        i32 = dict(dtype=torch.int32, device=device)
        return Cache(torch.empty(cap, d, dtype=dtype, device=device),
                     torch.empty(cap, d, dtype=dtype, device=device),
                     torch.empty(cap, **i32), torch.empty(cap, dtype=torch.float32, device=device),
                     torch.empty(cap, **i32), torch.empty(cap, **i32),
                     torch.empty(LG + 1, dtype=torch.int64, device=device))


class Compressor:
    """Runs the four stages on one context with preallocated outputs."""

    def __init__(self, params: GkvParams, device="cuda"):
        self.ctx = Context(params)
        p = params
        self.params = p
        dt = torch.bfloat16 if p.dtype == GKV_BF16 else torch.float32
        self.slots = torch.empty(self.ctx.n_c + 2, dtype=torch.int32, device=device)
        self.kappa = torch.empty(p.T, dtype=torch.float32, device=device)
        cap = p.budget + p.L * p.G * (p.T - (p.ctx_end - p.ctx_start)) + 8
        self.cache = Cache.empty(cap, p.d, p.L * p.G, dt, device)
        self.n_slots = 0
        self.n_entries = 0
        self._side = None

    def __call__(self, K, V, Q, omega=None, hidden=None, surprisal=None, slot_starts=None,
                 stream=None, Qg=None) -> "Cache":
        c = self.ctx
        if Qg is not None:          # multi-hop relevance: the graph layers' queries
            c.gracekv_set_graph_queries(Qg)
        # the score passes (K, Q only) run on a second stream while the
        # segmentation runs; the tree build waits for them
        main = stream if stream is not None else torch.cuda.current_stream()
        if self._side is None:
            self._side = torch.cuda.Stream(device=K.device)
        self._side.wait_stream(main)
        c.gracekv_score(K, Q, self._side)
        K.record_stream(self._side)
        Q.record_stream(self._side)
        self.n_slots = c.gracekv_segment(V, self.slots, hidden, surprisal, self.kappa, main)
        if slot_starts is not None:
            c.gracekv_build_trees(K, V, Q, omega, slot_starts, slot_starts.numel() - 1, stream)
        else:
            c.gracekv_build_trees(K, V, Q, omega, None, 0, stream)
        self.n_entries = c.gracekv_allocate(stream)
        c.gracekv_gather(K, V, self.cache, stream)
        return self.cache


def _raise(st: int):
    if st != GKV_OK:
        raise GraceKVError(st, lib().gracekv_status_string(st).decode())


class Decoder:
    """Decoding attention on a packed cache (gracekv_decode_* of the C ABI).

    K, V [E, d], log_m [E] fp32 and offsets [L*G + 1] int64 are the device
    outputs of gracekv_gather (or any cache in that layout); the append area
    [L, G, app_cap, d] and the workspace are allocated here.  ``n_app`` counts
    the appended rows; ``append`` adds one row to every (l, g) of the layers
    it is given and ``attention`` reads the packed entries plus the first
    ``n_app`` appended rows.
    """

    def __init__(self, K, V, log_m, offsets, *, L: int, G: int, Hq: int, app_cap: int = 0):
        d = K.shape[1]
        if K.numel() == 0:              # no packed entry at all: pass a valid address
            K = V = torch.zeros(1, d, dtype=K.dtype, device=K.device)
            log_m = torch.zeros(1, dtype=torch.float32, device=K.device)
        self.dtype = K.dtype
        dt = GKV_BF16 if K.dtype == torch.bfloat16 else GKV_F32
        self.K_app = torch.empty(L, G, max(app_cap, 1), d, dtype=K.dtype, device=K.device)
        self.V_app = torch.empty_like(self.K_app)
        self._keep = (K, V, log_m, offsets)
        ptr = lambda t: _ptr(t).value
        self.desc = GkvDecodeCache(L, G, Hq, d, dt, ptr(K), ptr(V), ptr(log_m), ptr(offsets),
                                   K.shape[0], ptr(self.K_app), ptr(self.V_app), app_cap)
        n = C.c_size_t()
        _raise(lib().gracekv_decode_workspace_size(C.byref(self.desc), C.byref(n)))
        self.workspace = torch.zeros(n.value, dtype=torch.uint8, device=K.device)
        self.L, self.G, self.Hq, self.d = L, G, Hq, d
        self.n_app = 0

    def append(self, k_new, v_new, l0: int = 0, stream=None):
        """k_new, v_new [n_layers, G, d]: row n_app of layers l0.. (n_app is
        advanced when the call covers the last layer)."""
        nl = k_new.shape[0]
        _raise(lib().gracekv_decode_append(C.byref(self.desc), l0, nl, self.n_app, _ptr(k_new),
                                           _ptr(v_new), _stream(stream)))
        if l0 + nl == self.L:
            self.n_app += 1

    def attention(self, q, l0: int = 0, out=None, stream=None):
        """q [n_layers, Hq, d] -> out [n_layers, Hq, d] fp32."""
        nl = q.shape[0]
        if out is None:
            out = torch.empty(nl, self.Hq, self.d, dtype=torch.float32, device=q.device)
        _raise(lib().gracekv_decode_attention(C.byref(self.desc), l0, nl, self.n_app, _ptr(q),
                                              _ptr(out), _ptr(self.workspace), _stream(stream)))
        return out

    def status(self, stream=None):
        _raise(lib().gracekv_decode_status(_ptr(self.workspace), _stream(stream)))


# ---- serving: the prompt's attention and the paged cache --------------------
_DTYPES = {torch.float32: GKV_F32, torch.bfloat16: GKV_BF16}


def _bad(why: str):
    return GraceKVError(GKV_EINVAL, why)


def _refuse(name: str, t: torch.Tensor, shape, dtype, device):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    raise _bad(f"{name} is {t.dtype} {tuple(t.shape)} on {t.device}, not {dtype} {tuple(shape)} on {device}")


def _rows(name: str, t: torch.Tensor, n: int, heads: int, d: int, dtype, device):
    """(pointer, token stride, head stride) of [n, heads, d] rows with contiguous channels."""
    if t.dtype is not dtype or t.shape != (n, heads, d) or t.device != device:
        _refuse(name, t, (n, heads, d), dtype, device)
    ts, hs, cs = t.stride()
    if cs != 1:
        raise _bad(f"the channels of {name} must be contiguous")
    # the stride of an axis of one element is arbitrary and never used
    return t.data_ptr(), ts if n > 1 else 0, hs if heads > 1 else 0


def _words(name: str, t: torch.Tensor, shape, dtype, device):
    """Pointer of a contiguous index or statistics array."""
    if t.dtype is not dtype or t.shape != shape or t.device != device:
        _refuse(name, t, shape, dtype, device)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous CUDA tensor")
    return t.data_ptr()


class _Workspace:
    """A zeroed workspace, usable on any one stream at a time: its zeros are there
    before the constructor returns, and it and what else the object made stay alive
    for the streams that they are used on."""

    def _make_workspace(self, n: int, device):
        self.workspace = torch.zeros(n, dtype=torch.uint8, device=device)
        self._device, self._ws = self.workspace.device, self.workspace.data_ptr()
        own = torch.cuda.current_stream(self._device)
        own.synchronize()
        self._own_stream = own.cuda_stream
        self._made, self._used_on = [self.workspace], set()

    def _run(self, call, *args):
        """A call of the library with the tensors' device current: it launches on the current one."""
        if torch._C._cuda_getDevice() == self._device.index:
            _raise(call(*args))
        else:
            with torch.cuda.device(self._device):
                _raise(call(*args))

    def _on(self, stream, *tensors):
        """The raw stream of a call; tensors used on an explicit stream stay alive for it."""
        if stream is None:
            raw = torch._C._cuda_getCurrentRawStream(self._device.index)
            if raw != self._own_stream and raw not in self._used_on:
                for t in self._made:
                    t.record_stream(torch.cuda.current_stream(self._device))
                self._used_on.add(raw)
            return raw
        if stream.device != self._device:
            raise _bad(f"the stream is on {stream.device}, the tensors are on {self._device}")
        self.workspace.record_stream(stream)
        for t in tensors:
            if t is not None:
                t.record_stream(stream)
        return stream.cuda_stream


def _empty_like_on(stream, shape, dtype, device):
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


class PromptAttention(_Workspace):
    """Causal attention of packed prompts (gracekv_prompt_* of the C ABI).

    One object holds the workspace of one stream.  q [N, Hq, d], k and v
    [Nk, G, d] with any token and head strides of whole 16 bytes (a slice of a
    fused projection, or K[l].transpose(0, 1) of a [L, G, T, d] cache);
    cu_q, cu_k int32 device row bounds of the sequences (cu_k = cu_q when not
    given).  A sequence with more keys than queries continues a prompt: its
    queries are the last ones.
    """

    def __init__(self, *, G: int, Hq: int, d: int, dtype, device="cuda"):
        if dtype not in _DTYPES:
            raise _bad(f"dtype must be bf16 or fp32, not {dtype}")
        self.G, self.Hq, self.d, self.dtype, self._code = G, Hq, d, dtype, _DTYPES[dtype]
        self._buf = bytearray(C.sizeof(GkvPrompt))
        self.desc = GkvPrompt.from_buffer(self._buf)
        _PROMPT.pack_into(self._buf, 0, G, Hq, d, self._code, *[0] * 18)
        n = C.c_size_t()
        _raise(lib().gracekv_prompt_workspace_size(C.byref(self.desc), C.byref(n)))
        self._make_workspace(n.value, device)
        self._ref = C.byref(self.desc)
        self._call = lib().gracekv_prompt_attention

    def __call__(self, q, k, v, cu_q, cu_k=None, *, out=None, lse=None, return_lse=False, stream=None):
        """out [N, Hq, d] of q's dtype (or (out, lse [N, Hq] fp32) with return_lse)."""
        dev, G, Hq, d, dt = self._device, self.G, self.Hq, self.d, self.dtype
        n_q, n_k, n1 = q.shape[0], k.shape[0], cu_q.shape[0]
        qp, q_ts, q_hs = _rows("q", q, n_q, Hq, d, dt, dev)
        kp, k_ts, k_hs = _rows("k", k, n_k, G, d, dt, dev)
        vp, v_ts, v_hs = _rows("v", v, n_k, G, d, dt, dev)
        cq = _words("cu_q", cu_q, (n1,), torch.int32, dev)
        ck = cq if cu_k is None else _words("cu_k", cu_k, (n1,), torch.int32, dev)
        if out is None:
            out = _empty_like_on(stream, (n_q, Hq, d), dt, dev)
            op, o_ts, o_hs = out.data_ptr(), Hq * d, d
        else:
            op, o_ts, o_hs = _rows("out", out, n_q, Hq, d, dt, dev)
        lp = 0
        if lse is not None:
            lp = _words("lse", lse, (n_q, Hq), torch.float32, dev)
        elif return_lse:
            lse = _empty_like_on(stream, (n_q, Hq), torch.float32, dev)
            lp = lse.data_ptr()
        _PROMPT.pack_into(self._buf, 0, G, Hq, d, self._code, n1 - 1, n_q, n_k, cq, ck, qp, kp, vp, op, lp,
                          q_ts, q_hs, k_ts, k_hs, v_ts, v_hs, o_ts, o_hs)
        self._run(self._call, self._ref, self._ws, self._on(stream, q, k, v, cu_q, cu_k, out, lse))
        return (out, lse) if return_lse else out

    def status(self, stream=None):
        self._run(lib().gracekv_prompt_status, self._ws, self._on(stream))


class PagedCache(_Workspace):
    """A paged cache of many requests (gracekv_paged_* of the C ABI).

    K, V [n_pages, page_size, d], log_m [n_pages, page_size] fp32 (or None),
    table [L, B, G, max_pages] int32 and lens [L, B, G] int32 are the caller's
    device tensors; `PagedCache.allocate` makes them and then also hands out
    the pages (`load`, `advance`, `release`).  A dense [L, G, T, d] cache is one
    too: L G pages of T entries.  One object holds the workspace of one stream.

    Pages of torch.float8_e4m3fn with k_scale, v_scale [n_pages, page_size] uint8
    are quantised (gracekv_quant_* of the C ABI): a row stands for its codes times
    2^(byte - 127).  Every call takes and gives rows of `dtype` (bf16 or fp32)
    then too, and the writing ones quantise.
    """

    def __init__(self, K, V, table, lens, *, Hq: int, log_m=None, rope_base: float = 0.0, k_scale=None, v_scale=None, dtype=None):
        quant = K.dtype is torch.float8_e4m3fn
        if dtype is None:
            dtype = torch.bfloat16 if quant else K.dtype
        if dtype not in _DTYPES or not (quant or dtype is K.dtype):
            raise _bad(f"K must be bf16, fp32 or e4m3 with rows of either, not {K.dtype} with rows of {dtype}")
        if (k_scale is not None) != quant or (v_scale is not None) != quant:
            raise _bad("quantised pages, and no others, have scales of their keys and of their values")
        if K.dim() != 3 or table.dim() != 4:
            raise _bad("K is [n_pages, page_size, d] and table [L, B, G, max_pages]")
        dev = K.device
        n_pages, ps, d = K.shape
        L, B, G, mp = table.shape
        self.K, self.V, self.log_m, self.table, self.lens = K, V, log_m, table, lens
        self.L, self.B, self.G, self.Hq, self.d, self.dtype = L, B, G, Hq, d, dtype
        self.page_size, self.max_pages, self.n_pages = ps, mp, n_pages
        self.k_scale, self.v_scale, self.quantised = k_scale, v_scale, quant
        self._pool = (K, V, log_m, table, lens, k_scale, v_scale)
        self.desc = GkvPagedCache(
            L, B, G, Hq, d, _DTYPES[dtype], ps, mp, n_pages, _words("K", K, K.shape, K.dtype, dev),
            _words("V", V, K.shape, K.dtype, dev),
            None if log_m is None else _words("log_m", log_m, (n_pages, ps), torch.float32, dev),
            _words("table", table, table.shape, torch.int32, dev), _words("lens", lens, (L, B, G), torch.int32, dev),
            float(rope_base))
        self._scales = None
        if quant:
            self._scales = GkvPagedScales(*(_words(x, t, (n_pages, ps), torch.uint8, dev)
                                            for x, t in (("k_scale", k_scale), ("v_scale", v_scale))))
        n = C.c_size_t()
        _raise(lib().gracekv_paged_workspace_size(C.byref(self.desc), C.byref(n)))
        self._make_workspace(n.value, dev)
        self._buf, self._row_buf = bytearray(C.sizeof(GkvPagedTokens)), bytearray(C.sizeof(GkvPagedRows))
        self._tokens = C.byref(GkvPagedTokens.from_buffer(self._buf))
        self._rows = C.byref(GkvPagedRows.from_buffer(self._row_buf))
        # the cache's own arguments of a call that takes both kinds, and of one of its kind
        self._both = (C.byref(self.desc), None if self._scales is None else C.byref(self._scales))
        self._ref = self._both if quant else self._both[:1]
        L_, kind = lib(), "gracekv_quant_" if quant else "gracekv_paged_"
        self._load, self._append, self._attention = (getattr(L_, kind + x) for x in ("load", "append", "attention"))
        self._read, self._unload = L_.gracekv_paged_read, L_.gracekv_paged_unload
        self._free = None

    @staticmethod
    def allocate(*, L: int, B: int, G: int, Hq: int, d: int, dtype, n_pages: int, max_pages: int,
                 page_size: int = 64, log_m: bool = True, rope_base: float = 0.0, device="cuda",
                 quantised: bool = False) -> "PagedCache":
        """An empty cache that hands out its own pages."""
        import numpy as np
        kind = torch.float8_e4m3fn if quantised else dtype
        scale = dict(dtype=torch.uint8, device=device)
        c = PagedCache(torch.empty(n_pages, page_size, d, dtype=kind, device=device),
                       torch.empty(n_pages, page_size, d, dtype=kind, device=device),
                       torch.full((L, B, G, max_pages), -1, dtype=torch.int32, device=device),
                       torch.zeros(L, B, G, dtype=torch.int32, device=device), Hq=Hq, rope_base=rope_base, dtype=dtype,
                       k_scale=torch.empty(n_pages, page_size, **scale) if quantised else None,
                       v_scale=torch.empty(n_pages, page_size, **scale) if quantised else None,
                       log_m=torch.empty(n_pages, page_size, device=device) if log_m else None)
        c._made += [t for t in c._pool if t is not None]
        c._free = np.arange(n_pages - 1, -1, -1, dtype=np.int32)     # a stack: the last one goes next
        c._n_free = n_pages
        c._host_lens = np.zeros((L, B, G), np.int64)
        c._host_table = np.full((L, B, G, max_pages), -1, np.int32)
        return c

    def _own_pages(self):
        if self._free is None:
            raise GraceKVError(GKV_ESTATE, "this cache's pages are the caller's (PagedCache.allocate hands them out)")

    def _grow(self, new_lens, stream):
        """Pages for the host lengths to become new_lens."""
        import numpy as np
        ps = self.page_size
        have, need = -(-self._host_lens // ps), -(-new_lens // ps)
        if need.max(initial=0) > self.max_pages:
            raise GraceKVError(GKV_ECAPACITY, "a sequence needs more than max_pages pages")
        n = int((need - have).sum())
        if n > self._n_free:
            raise GraceKVError(GKV_ECAPACITY, f"{n} pages needed, {self._n_free} free")
        if n:
            more = (need - have).reshape(-1)
            seq = np.repeat(np.arange(more.size), more)
            step = np.arange(n) - np.repeat(np.cumsum(more) - more, more)
            at = seq * self.max_pages + have.reshape(-1)[seq] + step
            pages = self._free[self._n_free - n:self._n_free][::-1].copy()
            self._n_free -= n
            self._host_table.reshape(-1)[at] = pages
            with torch.cuda.stream(stream):
                self.table.view(-1).index_copy_(0, torch.from_numpy(at).to(self.table.device),
                                                torch.from_numpy(pages).to(self.table.device))
        self._host_lens = new_lens

    def _packed(self, b: int, K, V, log_m, offsets):
        """The checked arguments of gracekv_paged_load from b to n_entries."""
        dev, E = self._device, K.shape[0]
        if not 0 <= b < self.B:
            raise _bad(f"request {b} of {self.B}")
        if log_m is not None and self.log_m is None:
            raise _bad("log m, and this cache keeps none")
        ptrs = (_words("K", K, (E, self.d), self.dtype, dev), _words("V", V, (E, self.d), self.dtype, dev),
                None if log_m is None else _words("log_m", log_m, (E,), torch.float32, dev),
                _words("offsets", offsets, (self.L * self.G + 1,), torch.int64, dev))
        if E >= 1 << 31 or (E and (ptrs[0] % 16 or ptrs[1] % 16)):
            raise _bad("K and V are at most 2^31 - 1 entries, on 16 bytes")
        return b, *ptrs, E

    def load_packed(self, b: int, K, V, log_m, offsets, stream=None):
        """The packed cache K, V [E, d], log_m [E] or None, offsets [L G + 1] int64
        becomes request b's entries (the table already holds their pages)."""
        self._run(self._load, *self._ref, *self._packed(b, K, V, log_m, offsets), self._ws,
                  self._on(stream, K, V, log_m, offsets, *self._pool))

    def unload_packed(self, b: int, n_entries: int, out=None, stream=None):
        """Request b's entries, at most n_entries, as a packed cache: (K, V [n_entries, d]
        of `dtype`, log_m [n_entries], offsets [L G + 1] int64), new or the four tensors
        `out`.  What load_packed takes, but that a cache without log m gives zeros for it
        and loads with None.  The pages stay as they are."""
        dev, E, n1 = self._device, n_entries, self.L * self.G + 1
        if not 0 <= b < self.B or not 0 <= E < 1 << 31:
            raise _bad(f"request {b} of {self.B}, {E} entries")
        if out is None:
            out = K, V, log_m, offsets = (
                _empty_like_on(stream, (E, self.d), self.dtype, dev), _empty_like_on(stream, (E, self.d), self.dtype, dev),
                _empty_like_on(stream, (E,), torch.float32, dev), _empty_like_on(stream, (n1,), torch.int64, dev))
            kp, vp, mp, op = K.data_ptr(), V.data_ptr(), log_m.data_ptr(), offsets.data_ptr()
        else:
            K, V, log_m, offsets = out
            kp, vp = _words("K", K, (E, self.d), self.dtype, dev), _words("V", V, (E, self.d), self.dtype, dev)
            mp, op = _words("log_m", log_m, (E,), torch.float32, dev), _words("offsets", offsets, (n1,), torch.int64, dev)
            if E and (kp % 16 or vp % 16):
                raise _bad("K and V are on 16 bytes")
        self._run(self._unload, *self._both, b, kp, vp, mp, op, E, self._ws,
                  self._on(stream, K, V, log_m, offsets, *self._pool))
        return out

    def unload(self, b: int, stream=None) -> Cache:
        """Request b's entries as a packed cache, to be loaded again (here, into another
        cache, of another kind of pages) after its pages went back (`release`).  Its
        positions and source intervals are not kept in pages: None."""
        self._own_pages()
        if not 0 <= b < self.B:
            raise _bad(f"request {b} of {self.B}")
        K, V, log_m, offsets = self.unload_packed(b, int(self._host_lens[:, b].sum()), None, stream)
        return Cache(K, V, None, log_m, None, None, offsets)

    def load(self, b: int, cache: Cache, n_entries: int, stream=None):
        """A compressed cache (Compressor's output) as request b, replacing what the
        slot held; refused, the slot keeps it.  Reads the offsets back to the host once."""
        import numpy as np
        self._own_pages()
        if not 0 <= n_entries <= cache.K.shape[0]:
            raise _bad(f"{n_entries} entries of {cache.K.shape[0]}")
        args = (cache.K[:n_entries], cache.V[:n_entries], None if self.log_m is None else cache.log_m[:n_entries], cache.offsets)
        self._packed(b, *args)
        self._on(stream)
        s = stream if stream is not None else torch.cuda.current_stream(self.K.device)
        with torch.cuda.stream(s):
            off = cache.offsets.cpu().numpy()
            if self.log_m is None and bool((cache.log_m[:n_entries] != 0).any()):
                raise _bad("entries of several tokens (log m above 0), and this cache keeps no log m")
        counts = np.diff(off)
        if off[0] < 0 or counts.min() < 0 or off[-1] > n_entries:
            raise _bad("the cache's offsets do not fit its entries")
        need = -(-counts // self.page_size)
        held = int((self._host_table[:, b] >= 0).sum())
        if need.max() > self.max_pages or need.sum() > self._n_free + held:
            raise GraceKVError(GKV_ECAPACITY, f"{int(need.sum())} pages needed, {self._n_free + held} free")
        self.release(b, stream)
        new = self._host_lens.copy()
        new[:, b] = counts.reshape(self.L, self.G)
        self._grow(new, s)
        self.load_packed(b, *args, stream)

    def advance(self, counts=None, stream=None):
        """The next step's tokens: counts[b] of each request.  Lengths grow, pages are
        assigned; returns the device cu_new of the appends.  Default: one token for
        every request with entries, in all its heads, and None.  (Where the pages are
        the caller's, for every head with entries: gracekv_paged_advance without cu_new.)"""
        import numpy as np
        self._on(stream)
        s = stream if stream is not None else torch.cuda.current_stream(self.K.device)
        n = counts
        if counts is not None:
            n = counts = np.asarray(counts, dtype=np.int64)
            if counts.shape != (self.B,) or counts.min() < 0:
                raise _bad("counts is one token count per request")
        if self._free is not None:
            if counts is None:
                held = self._host_lens > 0
                active = held.any(axis=(0, 2))
                if not held[:, active].all():         # a head without entries: the library would leave it idle
                    n = active
                self._grow(self._host_lens + active[None, :, None], s)
            else:
                self._grow(self._host_lens + counts[None, :, None], s)
        cu = None
        if n is not None:
            with torch.cuda.stream(s):
                cu = torch.from_numpy(np.concatenate([[0], np.cumsum(n)]).astype(np.int32)).to(self.K.device)
        self.advance_by(cu, stream)
        return None if counts is None else cu

    def advance_by(self, cu_new=None, stream=None):
        """Lengths alone, from a device cu_new [B + 1] (gracekv_paged_advance)."""
        p = None if cu_new is None else _words("cu_new", cu_new, (self.B + 1,), torch.int32, self.K.device)
        self._run(lib().gracekv_paged_advance, self._both[0], p, self._on(stream, self.table, self.lens, cu_new))

    def release(self, b: int, stream=None):
        """Request b's pages return to the pool; the slot is idle."""
        import numpy as np
        self._own_pages()
        if not 0 <= b < self.B:
            raise _bad(f"request {b} of {self.B}")
        self._on(stream, self.table, self.lens)
        s = stream if stream is not None else torch.cuda.current_stream(self.K.device)
        held = self._host_table[:, b]
        pages = held[held >= 0]
        self._free[self._n_free:self._n_free + pages.size] = pages
        self._n_free += pages.size
        held[...] = -1
        self._host_lens = np.array(self._host_lens)
        self._host_lens[:, b] = 0
        with torch.cuda.stream(s):
            self.lens[:, b] = 0
            self.table[:, b] = -1           # the pages are another request's next: no word leads to them

    def append(self, l: int, k, v, pos, q=None, cu_new=None, out=None, stream=None):
        """Layer l's new tokens: k, v [N, G, d] into the pages (k rotated to pos [N]
        int32); returns q [N, Hq, d] rotated (into `out`, which may be q), or None."""
        dev, N, dt, d = self._device, k.shape[0], self.dtype, self.d
        kp, k_ts, k_hs = _rows("k", k, N, self.G, d, dt, dev)
        vp, v_ts, v_hs = _rows("v", v, N, self.G, d, dt, dev)
        qp = op = q_ts = q_hs = o_ts = o_hs = 0
        if q is not None:
            qp, q_ts, q_hs = _rows("q", q, N, self.Hq, d, dt, dev)
            if out is None:
                out = _empty_like_on(stream, (N, self.Hq, d), dt, dev)
                op, o_ts, o_hs = out.data_ptr(), self.Hq * d, d
            else:
                op, o_ts, o_hs = _rows("out", out, N, self.Hq, d, dt, dev)
        _TOKENS.pack_into(self._buf, 0, N,
                          0 if cu_new is None else _words("cu_new", cu_new, (self.B + 1,), torch.int32, dev),
                          _words("pos", pos, (N,), torch.int32, dev), kp, vp, qp, op,
                          k_ts, k_hs, v_ts, v_hs, q_ts, q_hs, o_ts, o_hs)
        self._run(self._append, *self._ref, l, self._tokens, self._ws,
                  self._on(stream, k, v, pos, q, cu_new, out, *self._pool))
        return out

    def read(self, l: int, n: int, cu=None, k=None, v=None, stream=None):
        """Layer l's last entries as n rows of tokens (k, v [n, G, d] of `dtype`, new or
        the tensors given, with strides as append's): the last cu[b + 1] - cu[b] of
        every head of request b, as rows cu[b]...; without cu one of each request.
        Zeros where a head has fewer; rows of no request are not written."""
        dev, dt, shape = self._device, self.dtype, (n, self.G, self.d)
        if n < 0:
            raise _bad(f"{n} rows")
        whole = self.G * self.d
        if k is None:
            k = _empty_like_on(stream, shape, dt, dev)
            kp, k_ts, k_hs = k.data_ptr(), whole, self.d
        else:
            kp, k_ts, k_hs = _rows("k", k, *shape, dt, dev)
        if v is None:
            v = _empty_like_on(stream, shape, dt, dev)
            vp, v_ts, v_hs = v.data_ptr(), whole, self.d
        else:
            vp, v_ts, v_hs = _rows("v", v, *shape, dt, dev)
        _ROWS.pack_into(self._row_buf, 0, n, 0 if cu is None else _words("cu", cu, (self.B + 1,), torch.int32, dev), kp, vp,
                        k_ts, k_hs, v_ts, v_hs)
        self._run(self._read, *self._both, l, self._rows, self._ws, self._on(stream, k, v, cu, *self._pool))
        return k, v

    def attention(self, l: int, q, out=None, stream=None):
        """q [B, Hq, d], one rotated query per request slot -> out [B, Hq, d] of the
        cache's dtype over layer l (zeros for an idle slot)."""
        dev, shape = self._device, (self.B, self.Hq, self.d)
        qp = _words("q", q, shape, self.dtype, dev)
        if out is None:
            out = _empty_like_on(stream, shape, self.dtype, dev)
            op = out.data_ptr()
        else:
            op = _words("out", out, shape, self.dtype, dev)
        self._run(self._attention, *self._ref, l, qp, op, self._ws, self._on(stream, q, out, *self._pool))
        return out

    def status(self, stream=None):
        self._run(lib().gracekv_paged_status, self._ws, self._on(stream))


class SharedAttention(_Workspace):
    """Decoding attention of requests that share prefixes (gracekv_shared_* of the C ABI).

    cache holds the requests' own entries, prefix (a PagedCache of the same L, G, Hq,
    d and dtype; either may be quantised) one prefix a slot, read once for all the
    requests that share it.  One object holds the workspace of one stream.

    Three launches: for bf16 rows worth it from about 50000 requests x prefix entries
    of a KV head on (32 heads, 8 of KV), for fp32 from 32 requests on 1024 entries, 16
    on 4096, 8 on longer ones.  Below, PagedCache.attention over tables that begin with
    the prefix's pages is faster.
    """

    def __init__(self, cache: PagedCache, prefix: PagedCache):
        if prefix._device != cache._device:
            raise _bad(f"the prefix is on {prefix._device}, the cache on {cache._device}")
        self.cache, self.prefix = cache, prefix
        n = C.c_size_t()
        _raise(lib().gracekv_shared_workspace_size(cache._both[0], prefix._both[0], C.byref(n)))
        self._make_workspace(n.value, cache._device)
        self._call = lib().gracekv_shared_attention

    def __call__(self, l: int, q, cu_prefix=None, out=None, stream=None):
        """q [B, Hq, d], one rotated query per request slot -> out [B, Hq, d] over layer l:
        requests cu_prefix[p]... cu_prefix[p + 1] (int32 [prefix.B + 1]; None with one
        prefix slot: all) attend prefix slot p's entries and then their own."""
        c, x, dev = self.cache, self.prefix, self._device
        shape = (c.B, c.Hq, c.d)
        qp = _words("q", q, shape, c.dtype, dev)
        cp = None
        if cu_prefix is not None:
            cp = _words("cu_prefix", cu_prefix, (x.B + 1,), torch.int32, dev)
        elif x.B != 1:
            raise _bad(f"{x.B} prefix slots and no cu_prefix")
        if out is None:
            out = _empty_like_on(stream, shape, c.dtype, dev)
            op = out.data_ptr()
        else:
            op = _words("out", out, shape, c.dtype, dev)
        c._on(stream, *c._pool)
        x._on(stream, *x._pool)
        self._run(self._call, *c._both, *x._both, l, cp, qp, op, self._ws, self._on(stream, q, cu_prefix, out))
        return out

    def status(self, stream=None):
        self._run(lib().gracekv_shared_status, self._ws, self._on(stream))
