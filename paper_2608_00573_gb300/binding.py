"""ctypes binding of include/trimmoe.h (argument marshalling only).

Every step of the layer runs in the CUDA library; this module only converts
torch tensors / numpy arrays into the C structs and calls the entry points.
It raises if the compiled library is missing: there is no fallback path.
"""
from __future__ import annotations

import array
import ctypes as C
import os
import threading
from typing import Optional

import numpy as np

from . import workload as W

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "_build", "libtrimmoe.so")

TRIMMOE_OK = 0
STATUS_NAMES = {0: "OK", -1: "ERR_ARG", -2: "ERR_UNSUPPORTED", -3: "ERR_OOM", -4: "ERR_CUDA",
                -5: "ERR_COVERAGE", -6: "ERR_DEVICE_TIMEOUT", -7: "ERR_CACHE"}
EXEC, SKIP, EXIT, DEAD = 0, 1, 2, 3


class TrimmoeError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


class trimmoe_config(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("N", "d", "E", "k", "F", "F_sh", "C", "M", "H", "act",
                                       "renorm_topk", "n_sub", "T_max")] + \
               [(n, C.c_float) for n in ("omega_T", "omega_D", "d_ref_ms", "phi_beta")] + \
               [("profile", C.c_int), ("norm_eps", C.c_float), ("n_centroids", C.c_int)] + \
               [(n, C.c_int) for n in ("attn_heads", "attn_kv_heads", "head_dim", "attn_seq")] + \
               [("rope_theta", C.c_float), ("graphs", C.c_int)]


class trimmoe_weights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("W_r", "b_r", "W_x", "b_x", "W13", "W2", "W13_sh", "W2_sh",
                                          "W_norm", "centroids", "W_attn_norm", "W_qkv", "W_o")]


class trimmoe_tables(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("place", "sim", "sub_thresh", "trans_ms", "comp_ms", "P",
                                          "theta", "lambda_", "eps", "centroid_exit")]


class trimmoe_tokens(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("hidden", "s", "Dhat", "Dbar", "pJ", "alive", "last_exec",
                                          "xi_last", "exit_layer")]


class trimmoe_layer_out(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("topk_idx", "topk_g", "I", "xi", "action", "exp_sel",
                                          "srv_sel", "perm", "group_off", "lhat", "h_attn")]


class trimmoe_stats_t(C.Structure):
    _fields_ = [(n, C.c_uint64) for n in ("layer_tokens", "exec_tokens", "skipped", "exited",
                                          "pairs_local_exact", "pairs_local_sub", "pairs_remote_exact",
                                          "pairs_remote_sub", "shared_rows")] + \
               [("delay_ms", C.c_double), ("remote_hops", C.c_double), ("max_budget_ratio", C.c_float),
                ("device_error", C.c_int), ("launches", C.c_uint64), ("layer_calls", C.c_uint64),
                ("gemm_flops", C.c_double)] + \
               [(n, C.c_double) for n in ("ms_decide", "ms_compact", "ms_gather", "ms_gemm_up",
                                          "ms_gemm_down", "ms_combine")] + \
               [("n_gemm_up", C.c_uint64), ("n_gemm_down", C.c_uint64),
                ("flops_gemm_up", C.c_double), ("flops_gemm_down", C.c_double), ("ms_router", C.c_double),
                ("bytes_gemm_up", C.c_double), ("bytes_gemm_down", C.c_double),
                ("lookahead_shared", C.c_uint64),
                ("ms_attn", C.c_double), ("ms_attn_gemm", C.c_double), ("flops_attn", C.c_double),
                ("flops_attn_gemm", C.c_double), ("pairs_executed", C.c_uint64),
                ("bytes_expert_weights", C.c_double)]

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_}


class trimmoe_feedback_cfg(C.Structure):
    _fields_ = [("user_size", C.c_int), ("eta", C.c_float), ("p_min", C.c_float), ("kappa", C.c_float)]


class trimmoe_feedback_out(C.Structure):
    _fields_ = [("omega_T", C.c_float), ("omega_D", C.c_float), ("T_norm", C.c_double), ("D_util", C.c_double),
                ("users_updated", C.c_int), ("window_delay_ms", C.c_double), ("window_ref_slots", C.c_double)]

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_}


class trimmoe_calibration_t(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("trans", "alive", "resid", "act", "above", "P", "pi", "sigma",
                                          "act_freq", "lambda_", "rho")]


class trimmoe_cache_config(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("layers", "q_heads", "kv_heads", "head_dim", "page_size", "n_pages",
                                       "max_seqs", "max_pages", "T_max")]


class trimmoe_cache_state(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("k", "v", "table", "length", "ref")]


class trimmoe_append_args(C.Structure):
    _fields_ = [("qkv", C.c_void_p), ("ld_qkv", C.c_int), ("q_out", C.c_void_p), ("ld_q", C.c_int),
                ("gamma_q", C.c_void_p), ("gamma_k", C.c_void_p), ("norm_eps", C.c_float),
                ("rope_theta", C.c_float), ("pos", C.c_void_p)]


class trimmoe_attend_args(C.Structure):
    _fields_ = [("q", C.c_void_p), ("ld_q", C.c_int), ("out", C.c_void_p), ("ld_out", C.c_int),
                ("tree", C.c_void_p), ("scale", C.c_float)]


class trimmoe_cache_stats_t(C.Structure):
    _fields_ = [("device_error", C.c_int), ("free_pages", C.c_int), ("launches", C.c_uint64)]


EXPORTS = ("trimmoe_create", "trimmoe_layer_step", "trimmoe_forward", "trimmoe_forward_host",
           "trimmoe_stats", "trimmoe_reset_stats", "trimmoe_last_error", "trimmoe_destroy",
           "trimmoe_compact_noalloc", "trimmoe_feedback", "trimmoe_calibration_begin",
           "trimmoe_calibration_end", "trimmoe_replicate", "trimmoe_watchdog_selftest",
           "trimmoe_cache_create", "trimmoe_cache_step", "trimmoe_cache_append", "trimmoe_cache_attend",
           "trimmoe_cache_fork", "trimmoe_cache_truncate", "trimmoe_cache_accept", "trimmoe_cache_compact",
           "trimmoe_cache_stats", "trimmoe_cache_last_error", "trimmoe_cache_destroy")

_lib = None
_lock = threading.Lock()


def lib():
    """Load the CUDA library (raises if it has not been built)."""
    global _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(LIB_PATH):
                raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                                   "`python -m paper_2608_00573_gb300.build`")
            L = C.CDLL(LIB_PATH)
            vp, i = C.c_void_p, C.c_int
            L.trimmoe_create.argtypes = [vp, vp, vp, C.POINTER(vp)]
            L.trimmoe_create.restype = i
            L.trimmoe_layer_step.argtypes = [vp, i, i, vp, vp, vp]
            L.trimmoe_layer_step.restype = i
            L.trimmoe_forward.argtypes = [vp, i, vp, vp]
            L.trimmoe_forward.restype = i
            L.trimmoe_forward_host.argtypes = [vp, i, vp, vp]
            L.trimmoe_forward_host.restype = i
            L.trimmoe_stats.argtypes = [vp, vp]
            L.trimmoe_stats.restype = i
            L.trimmoe_reset_stats.argtypes = [vp]
            L.trimmoe_reset_stats.restype = i
            L.trimmoe_watchdog_selftest.argtypes = [vp, i, vp]
            L.trimmoe_watchdog_selftest.restype = i
            L.trimmoe_last_error.argtypes = [vp]
            L.trimmoe_last_error.restype = C.c_char_p
            L.trimmoe_destroy.argtypes = [vp]
            L.trimmoe_destroy.restype = None
            L.trimmoe_compact_noalloc.argtypes = [vp, vp, i, i, i, i, vp, vp, vp, vp, vp]
            L.trimmoe_feedback.argtypes = [vp, vp, i, vp, vp, vp]
            L.trimmoe_feedback.restype = i
            L.trimmoe_calibration_begin.argtypes = [vp]
            L.trimmoe_calibration_begin.restype = i
            L.trimmoe_calibration_end.argtypes = [vp, C.c_longlong, vp]
            L.trimmoe_calibration_end.restype = i
            L.trimmoe_replicate.argtypes = [i, i, i, vp, vp, vp, vp, vp, vp, vp]
            L.trimmoe_replicate.restype = i
            L.trimmoe_compact_noalloc.restype = i
            _lib = L
    return _lib


def _check(rc, handle=None):
    if rc != TRIMMOE_OK:
        msg = lib().trimmoe_last_error(handle)
        raise TrimmoeError(rc, msg.decode() if msg else "")


# ----------------------------------------------------------- thin wrappers

def trimmoe_create(cfg: trimmoe_config, w: trimmoe_weights, tab: trimmoe_tables) -> C.c_void_p:
    h = C.c_void_p()
    _check(lib().trimmoe_create(C.byref(cfg), C.byref(w), C.byref(tab), C.byref(h)))
    return h


def trimmoe_layer_step(h, layer: int, T: int, tok: trimmoe_tokens, out: Optional[trimmoe_layer_out],
                       stream: int = 0):
    _check(lib().trimmoe_layer_step(h, layer, T, C.byref(tok), C.byref(out) if out is not None else None,
                                    C.c_void_p(stream)), h)


def trimmoe_forward(h, T: int, tok: trimmoe_tokens, stream: int = 0):
    _check(lib().trimmoe_forward(h, T, C.byref(tok), C.c_void_p(stream)), h)


def trimmoe_forward_host(h, T: int, tok: trimmoe_tokens, stream: int = 0):
    _check(lib().trimmoe_forward_host(h, T, C.byref(tok), C.c_void_p(stream)), h)


def trimmoe_stats(h) -> dict:
    s = trimmoe_stats_t()
    rc = lib().trimmoe_stats(h, C.byref(s))
    d = s.as_dict()
    d["status"] = rc
    return d


def trimmoe_reset_stats(h):
    _check(lib().trimmoe_reset_stats(h), h)


def trimmoe_watchdog_selftest(h, timeout_us: int, stream: int = 0) -> int:
    """Run the bounded-wait self-check; returns the status code (DEVICE_TIMEOUT when the
    wait ran out as designed) instead of raising."""
    return lib().trimmoe_watchdog_selftest(h, timeout_us, C.c_void_p(stream))


def trimmoe_last_error(h=None) -> str:
    m = lib().trimmoe_last_error(h)
    return m.decode() if m else ""


def trimmoe_destroy(h):
    lib().trimmoe_destroy(h)


def trimmoe_feedback(h, fb: trimmoe_feedback_cfg, T: int, tok: trimmoe_tokens, stream: int = 0) -> dict:
    out = trimmoe_feedback_out()
    _check(lib().trimmoe_feedback(h, C.byref(fb), T, C.byref(tok), C.byref(out), C.c_void_p(stream)), h)
    return out.as_dict()


def trimmoe_calibration_begin(h):
    _check(lib().trimmoe_calibration_begin(h), h)


def trimmoe_calibration_end(h, T_cal: int, N: int, E: int, M: int) -> dict:
    """Counts and statistics of the offline stage as numpy arrays."""
    o = dict(trans=np.zeros((max(N - 1, 1), E, E), np.uint64), alive=np.zeros(N, np.uint64),
             resid=np.zeros((N, M), np.uint64), act=np.zeros((N, E), np.uint64), above=np.zeros((N, E), np.uint64),
             P=np.zeros((max(N - 1, 1), E, E), np.float32), pi=np.zeros(N, np.float32),
             sigma=np.zeros((N, E), np.float32), act_freq=np.zeros((N, E), np.float32),
             lam=np.zeros((N, E), np.float32), rho=np.zeros((N, M), np.float32))
    st = trimmoe_calibration_t(trans=_ptr(o["trans"]), alive=_ptr(o["alive"]), resid=_ptr(o["resid"]),
                               act=_ptr(o["act"]), above=_ptr(o["above"]), P=_ptr(o["P"]), pi=_ptr(o["pi"]),
                               sigma=_ptr(o["sigma"]), act_freq=_ptr(o["act_freq"]), lambda_=_ptr(o["lam"]),
                               rho=_ptr(o["rho"]))
    _check(lib().trimmoe_calibration_end(h, int(T_cal), C.byref(st)), h)
    return o


def trimmoe_replicate(lam, rho, trans, expert_bytes, capacity, place):
    """Greedy replication (Eq. 28) on a copy of place (host arrays); returns (place, added)."""
    N, E = place.shape
    M = trans.shape[0]
    pl = np.array(place, dtype=np.uint16, copy=True)
    arrs = [np.ascontiguousarray(a, dt) for a, dt in ((lam, np.float32), (rho, np.float32), (trans, np.float32),
                                                        (expert_bytes, np.float64), (capacity, np.float64))]
    added = C.c_int(0)
    _check(lib().trimmoe_replicate(N, E, M, *[_ptr(a) for a in arrs], _ptr(pl), C.byref(added)))
    return pl, added.value


def trimmoe_compact_noalloc(action, exp_sel, T: int, k: int, E: int, has_shared: int, perm, group_off,
                            pos_pair, pos_sh, stream: int = 0):
    """Compaction into caller-owned outputs with no device allocation (device tensors)."""
    _check(lib().trimmoe_compact_noalloc(_ptr(action), _ptr(exp_sel), T, k, E, has_shared, _ptr(perm),
                                         _ptr(group_off), _ptr(pos_pair), _ptr(pos_sh), C.c_void_p(stream)))


# ----------------------------------------------------------- engine

TOKEN_FIELDS = ("hidden", "s", "Dhat", "Dbar", "pJ", "alive", "last_exec", "xi_last", "exit_layer")


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, np.ndarray):
        return t.ctypes.data
    return t.data_ptr()


class Engine:
    """Owns a trimmoe handle plus the torch tensors it borrows."""

    def __init__(self, cfg: W.WorkloadConfig, tables: dict, small: dict, experts: dict, T_max: int,
                 device="cuda", profile=False, graphs: bool = False):
        import torch
        self.torch = torch
        self.cfg = cfg
        self.device = torch.device(device)
        dev = self.device

        def dt(a, dtype):
            if isinstance(a, torch.Tensor):
                return a.to(dev).contiguous()
            a = np.ascontiguousarray(a)
            if a.dtype == np.uint16:
                return torch.from_numpy(a.view(np.int16)).to(dev).view(torch.bfloat16).contiguous()
            return torch.from_numpy(a).to(dev, dtype=dtype).contiguous()

        self.w = {
            "W_r": dt(small["W_r"], torch.bfloat16), "b_r": dt(small["b_r"], torch.float32),
            "W_x": dt(small["W_x"], torch.bfloat16), "b_x": dt(small["b_x"], torch.float32),
            "W13": dt(experts["W13"], torch.bfloat16), "W2": dt(experts["W2"], torch.bfloat16),
            "W13_sh": dt(experts["W13_sh"], torch.bfloat16) if cfg.F_sh else None,
            "W2_sh": dt(experts["W2_sh"], torch.bfloat16) if cfg.F_sh else None,
            "W_norm": dt(small["W_norm"], torch.bfloat16) if small.get("W_norm") is not None else None,
            "centroids": dt(small["centroids"], torch.bfloat16) if cfg.n_centroids else None,
            "W_attn_norm": dt(small["W_attn_norm"], torch.bfloat16) if cfg.attn_heads else None,
            "W_qkv": dt(experts["W_qkv"], torch.bfloat16) if cfg.attn_heads else None,
            "W_o": dt(experts["W_o"], torch.bfloat16) if cfg.attn_heads else None,
        }
        self.tables = {k: np.ascontiguousarray(v) for k, v in tables.items() if k != "d_ref"}
        self.c_cfg = trimmoe_config(
            N=cfg.N, d=cfg.d, E=cfg.E, k=cfg.k, F=cfg.F, F_sh=cfg.F_sh, C=cfg.C, M=cfg.M, H=cfg.H,
            act=cfg.act, renorm_topk=cfg.renorm_topk, n_sub=cfg.n_sub, T_max=T_max,
            omega_T=cfg.omega_T, omega_D=cfg.omega_D, d_ref_ms=float(tables["d_ref"]),
            phi_beta=cfg.phi_beta, profile=int(profile), norm_eps=cfg.norm_eps,
            n_centroids=cfg.n_centroids, attn_heads=cfg.attn_heads, attn_kv_heads=cfg.attn_kv_heads,
            head_dim=cfg.head_dim, attn_seq=cfg.attn_seq, rope_theta=cfg.rope_theta, graphs=1 if graphs else 0)
        self.c_w = trimmoe_weights(**{k: _ptr(v) for k, v in self.w.items()})
        t = self.tables
        P = t["P"].astype(np.float32) if t["P"].size else None
        self._P = P
        self.c_tab = trimmoe_tables(
            place=_ptr(t["place"].astype(np.uint16)), sim=_ptr(t["sim"]), sub_thresh=_ptr(t["sub_thresh"]),
            trans_ms=_ptr(t["trans"]), comp_ms=_ptr(t["comp"]), P=_ptr(P), theta=_ptr(t["theta"]),
            lambda_=_ptr(t["lam"]), eps=_ptr(t["eps"]))
        self._keep_place = t["place"].astype(np.uint16)
        self.c_tab.place = _ptr(self._keep_place)
        if cfg.n_centroids:
            self._cexit = np.ascontiguousarray(small["centroid_exit"], dtype=np.float32)
            self.c_tab.centroid_exit = _ptr(self._cexit)
        self.T_max = T_max
        self.handle = trimmoe_create(self.c_cfg, self.c_w, self.c_tab)

    # token state ----------------------------------------------------------
    def tokens_to_device(self, tok: dict):
        torch = self.torch
        out = {}
        for k in TOKEN_FIELDS:
            a = tok["h" if k == "hidden" else k]
            if isinstance(a, torch.Tensor):
                out[k] = a.to(self.device).contiguous()
            else:
                a = np.ascontiguousarray(a)
                if k == "hidden":
                    out[k] = torch.from_numpy(a.view(np.int16)).to(self.device).view(torch.bfloat16)
                else:
                    out[k] = torch.from_numpy(a).to(self.device)
        return out

    @staticmethod
    def tokens_to_host(tok: dict) -> dict:
        import torch
        out = {}
        for k, v in tok.items():
            v = v.detach().cpu()
            if k == "hidden":
                out["h"] = v.view(torch.int16).numpy().view(np.uint16).copy()
            else:
                out[k] = v.numpy().copy()
        return out

    def c_tokens(self, tok: dict) -> trimmoe_tokens:
        return trimmoe_tokens(**{k: _ptr(tok[k]) for k in TOKEN_FIELDS})

    def alloc_layer_out(self, T: int) -> dict:
        torch = self.torch
        K, E, dev = self.cfg.k, self.cfg.E, self.device
        return dict(
            topk_idx=torch.empty(T * K, dtype=torch.int32, device=dev),
            topk_g=torch.empty(T * K, dtype=torch.float32, device=dev),
            I=torch.empty(T, dtype=torch.float32, device=dev),
            xi=torch.empty(T, dtype=torch.float32, device=dev),
            action=torch.empty(T, dtype=torch.uint8, device=dev),
            exp_sel=torch.empty(T * K, dtype=torch.uint8, device=dev),
            srv_sel=torch.empty(T * K, dtype=torch.uint8, device=dev),
            perm=torch.full((T * K + T,), -1, dtype=torch.int32, device=dev),
            group_off=torch.empty(E + 2, dtype=torch.int32, device=dev),
            lhat=torch.empty(T, dtype=torch.int16, device=dev),
            h_attn=(torch.empty((T, self.cfg.d), dtype=torch.bfloat16, device=dev) if self.cfg.attn_heads
                    else None))

    def stream_ptr(self, stream=None) -> int:
        torch = self.torch
        s = stream if stream is not None else torch.cuda.current_stream(self.device)
        return int(s.cuda_stream)

    def layer_step(self, layer: int, tok: dict, T: Optional[int] = None, out: Optional[dict] = None,
                   stream=None):
        T = tok["s"].shape[0] if T is None else T
        c_out = trimmoe_layer_out(**{k: _ptr(v) for k, v in out.items()}) if out is not None else None
        trimmoe_layer_step(self.handle, layer, T, self.c_tokens(tok), c_out, self.stream_ptr(stream))
        return out

    def forward(self, tok: dict, T: Optional[int] = None, stream=None):
        T = tok["s"].shape[0] if T is None else T
        trimmoe_forward(self.handle, T, self.c_tokens(tok), self.stream_ptr(stream))

    def forward_host(self, host_tok: dict, T: Optional[int] = None, stream=None):
        """host_tok: dict of pinned CPU torch tensors keyed by TOKEN_FIELDS."""
        T = host_tok["s"].shape[0] if T is None else T
        trimmoe_forward_host(self.handle, T, self.c_tokens(host_tok), self.stream_ptr(stream))

    def stats(self) -> dict:
        return trimmoe_stats(self.handle)

    def calibration_begin(self):
        trimmoe_calibration_begin(self.handle)

    def calibration_end(self, T_cal: int) -> dict:
        return trimmoe_calibration_end(self.handle, T_cal, self.cfg.N, self.cfg.E, self.cfg.M)

    def feedback(self, tok: dict, user_size: int, eta: float, p_min: float, kappa: float,
                 T: Optional[int] = None, stream=None) -> dict:
        """Eq. (37) / (43) at the end of an observation window (updates tok['pJ'] in place)."""
        T = tok["s"].shape[0] if T is None else T
        fb = trimmoe_feedback_cfg(user_size=user_size, eta=eta, p_min=p_min, kappa=kappa)
        return trimmoe_feedback(self.handle, fb, T, self.c_tokens(tok), self.stream_ptr(stream))

    def reset_stats(self):
        trimmoe_reset_stats(self.handle)

    def close(self):
        if getattr(self, "handle", None):
            trimmoe_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ----------------------------------------------------------- paged cache

def _cache_lib():
    """The library with the prototypes of the cache's entry points."""
    L = lib()
    if not getattr(L, "_cache_prototypes", False):
        vp, i = C.c_void_p, C.c_int
        for name, args in (("create", [vp, vp, C.POINTER(vp)]), ("step", [vp, i, vp, vp, vp]),
                           ("append", [vp, i, vp, vp]), ("attend", [vp, i, vp, vp]), ("fork", [vp, i, vp, vp, vp]),
                           ("truncate", [vp, i, vp, vp, vp]), ("accept", [vp, i, vp, vp, vp, i, vp]),
                           ("compact", [vp, vp]), ("stats", [vp, vp, i])):
            f = getattr(L, "trimmoe_cache_" + name)
            f.argtypes, f.restype = args, i
        L.trimmoe_cache_last_error.argtypes = [vp]
        L.trimmoe_cache_last_error.restype = C.c_char_p
        L.trimmoe_cache_destroy.argtypes = [vp]
        L.trimmoe_cache_destroy.restype = None
        L._cache_prototypes = True
    return L


def trimmoe_cache_create(cfg: trimmoe_cache_config, st: trimmoe_cache_state) -> C.c_void_p:
    h = C.c_void_p()
    _check(_cache_lib().trimmoe_cache_create(C.byref(cfg), C.byref(st), C.byref(h)))
    return h


class PagedCache:
    """Keys and values of sequences kept between steps, and the attention over them.

    Owns a trimmoe_cache handle and borrows the caller's tensors (all on one
    GPU, contiguous): k, v bfloat16 [layers][n_pages][kv_heads][page][head_dim],
    table int32 [max_seqs][max_pages] (-1: none), length int32 [max_seqs], ref
    int32 [n_pages].  ``PagedCache.empty`` makes them for a new cache.  Calls are
    queued on the current stream (or ``stream``); see include/trimmoe.h for
    their rules.  Sequence lists are host sequences of ints.  With ``stream``, what
    wrote the inputs has to be ordered before the call and what reads the result
    behind it, as for any work on two streams; the inputs' memory is kept from
    other uses until that stream has read them, and a result is of that stream.
    """

    def __init__(self, k, v, table, length, ref, q_heads: int, T_max: int):
        import torch
        self.torch = torch
        self.handle = None
        self._lib = _cache_lib()
        self._bf16 = torch.bfloat16
        self._raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        self._Tensor, self._empty, self._int32, self._int64 = torch.Tensor, torch.empty, torch.int32, torch.int64
        self._append_args, self._attend_args = trimmoe_append_args(), trimmoe_attend_args()
        self._append_at, self._attend_at = C.addressof(self._append_args), C.addressof(self._attend_args)
        self._c_append, self._c_attend = self._lib.trimmoe_cache_append, self._lib.trimmoe_cache_attend
        if k.dim() != 5 or k.shape != v.shape or table.dim() != 2 or length.dim() != 1 or ref.dim() != 1:
            raise TrimmoeError(-1, "cache: k and v are [layers][n_pages][kv_heads][page][head_dim], table is "
                                   "[max_seqs][max_pages], length and ref are vectors")
        self.layers, self.n_pages, self.kv_heads, self.page, self.head_dim = k.shape
        self.max_seqs, self.max_pages = table.shape
        self.q_heads, self.T_max, self.device = int(q_heads), int(T_max), k.device
        if length.shape[0] != self.max_seqs or ref.shape[0] != self.n_pages:
            raise TrimmoeError(-1, "cache: length has one entry per table row, ref one per page")
        for t, dt in ((k, torch.bfloat16), (v, torch.bfloat16), (table, torch.int32), (length, torch.int32),
                      (ref, torch.int32)):
            self._tensor(t, dt, None, "cache")
            if not t.is_contiguous():
                raise TrimmoeError(-1, "cache: tensors must be contiguous")
        self.k, self.v, self.table, self.length, self.ref = k, v, table, length, ref
        self.T = 0
        self._index = self.device.index
        self._q_cols, self._qkv_cols = self.q_heads * self.head_dim, (self.q_heads + 2 * self.kv_heads) * self.head_dim
        cfg = trimmoe_cache_config(layers=self.layers, q_heads=self.q_heads, kv_heads=self.kv_heads,
                                   head_dim=self.head_dim, page_size=self.page, n_pages=self.n_pages,
                                   max_seqs=self.max_seqs, max_pages=self.max_pages, T_max=self.T_max)
        st = trimmoe_cache_state(k=_ptr(k), v=_ptr(v), table=_ptr(table), length=_ptr(length), ref=_ptr(ref))
        with torch.cuda.device(self.device):
            self.handle = trimmoe_cache_create(cfg, st)

    @classmethod
    def empty(cls, layers: int, n_pages: int, q_heads: int, kv_heads: int, head_dim: int, page: int, max_seqs: int,
              max_pages: int, T_max: int, device="cuda"):
        """A cache of n_pages free pages (page contents are left unset)."""
        import torch
        shape = (layers, n_pages, kv_heads, page, head_dim)
        return cls(torch.empty(shape, dtype=torch.bfloat16, device=device),
                   torch.empty(shape, dtype=torch.bfloat16, device=device),
                   torch.full((max_seqs, max_pages), -1, dtype=torch.int32, device=device),
                   torch.zeros(max_seqs, dtype=torch.int32, device=device),
                   torch.zeros(n_pages, dtype=torch.int32, device=device), q_heads, T_max)

    # checks and calls ------------------------------------------------------
    # A decode step calls append and attend once per layer, and on the GPU they take a
    # few microseconds: the checks below are ordered and kept so that a call costs about
    # as much on the host.
    def _tensor(self, t, dtype, shape, what):
        if t is None:
            return
        if not isinstance(t, self.torch.Tensor) or t.device != self.device or t.device.type != "cuda":
            raise TrimmoeError(-1, f"{what}: tensors must be on the cache's GPU")
        if t.dtype != dtype:
            raise TrimmoeError(-1, f"{what}: expected {dtype}, got {t.dtype}")
        if shape is not None and (tuple(t.shape) != tuple(shape) or (t.numel() and not t.is_contiguous())):
            raise TrimmoeError(-1, f"{what}: expected a contiguous tensor of shape {tuple(shape)}, got {tuple(t.shape)}")

    def _rows(self, t, cols, what):
        """Row stride of a [T][cols] tensor (of a single row: its length, whatever a view of it says)."""
        if isinstance(t, self._Tensor) and t.dtype is self._bf16 and t.get_device() == self._index and \
                t.shape == (self.T, cols):
            ld, one = t.stride()
            if one == 1 or not self.T:
                return ld if self.T > 1 else cols
        self._tensor(t, self._bf16, None, what)
        raise TrimmoeError(-1, f"{what}: expected shape {(self.T, cols)} with contiguous rows, got {tuple(t.shape)}")

    def _vector(self, t, dtype, n, what):
        """Address of a vector of n values, None without one."""
        if t is None:
            return None
        if not (isinstance(t, self._Tensor) and t.dtype is dtype and t.get_device() == self._index and t.shape == (n,) and
                (n < 2 or t.stride(0) == 1)):
            self._tensor(t, dtype, (n,), what)
        return t.data_ptr()

    def _new(self, cols, stream):
        """A [T][cols] result, allocated on the stream that writes it."""
        if stream is None:
            return self._empty((self.T, cols), dtype=self._bf16, device=self.device)
        with self.torch.cuda.stream(stream):
            return self._empty((self.T, cols), dtype=self._bf16, device=self.device)

    @staticmethod
    def _list(v):
        """Host int32 list: (object that owns it, address, length, values)."""
        if isinstance(v, np.ndarray):
            if v.ndim != 1 or v.dtype.kind not in "iu":
                raise TrimmoeError(-1, "cache: sequence lists are one-dimensional, of integers")
            v = v.tolist()
        try:
            a = array.array("i", v)
        except (TypeError, OverflowError) as e:
            raise TrimmoeError(-1, f"cache: sequence lists hold 32-bit integers ({e})") from None
        return a, a.buffer_info()[0], len(a)

    def _pair(self, a, b, what):
        a, b = self._list(a), self._list(b)
        if a[2] != b[2]:
            raise TrimmoeError(-1, f"{what}: lists of different lengths")
        return a, b

    def _stream(self, stream):
        if stream is not None:
            return int(stream.cuda_stream)
        if self._raw_stream is not None:
            return self._raw_stream(self._index)
        return int(self.torch.cuda.current_stream(self.device).cuda_stream)

    @staticmethod
    def _keep(stream, *tensors):
        """The caller may drop these at once: their memory is used again only behind `stream`."""
        for t in tensors:
            if t is not None:
                t.record_stream(stream)

    def _done(self, rc):
        if rc != TRIMMOE_OK:
            raise TrimmoeError(rc, self._lib.trimmoe_cache_last_error(self.handle).decode())

    def step(self, seq, q_len, stream=None):
        """Room for q_len[i] new tokens of sequence seq[i]; the work list of append and attend."""
        seq, q_len = self._pair(seq, q_len, "step")
        self._done(self._lib.trimmoe_cache_step(self.handle, seq[2], seq[1], q_len[1], self._stream(stream)))
        self.T = sum(q_len[0])

    def append(self, layer: int, qkv, q_out=None, gamma_q=None, gamma_k=None, eps: float = 1e-6, theta: float = 1e6,
               pos=None, stream=None):
        """Norm (with gammas) and rotate the step's queries and keys of qkv [T][(q + 2 kv heads) * head_dim], write
        its keys and values into the cache; returns the queries [T][q_heads * head_dim] (q_out, which may be a
        view of qkv's query columns)."""
        a, cols = self._append_args, self._q_cols
        a.ld_qkv = self._rows(qkv, self._qkv_cols, "append")
        if q_out is None:
            q_out = self._new(cols, stream)
            a.ld_q = cols
        else:
            a.ld_q = self._rows(q_out, cols, "append")
        a.gamma_q = self._vector(gamma_q, self._bf16, self.head_dim, "append")
        a.gamma_k = self._vector(gamma_k, self._bf16, self.head_dim, "append")
        a.pos = self._vector(pos, self._int32, self.T, "append")
        a.qkv = qkv.data_ptr()
        a.q_out = q_out.data_ptr()
        a.norm_eps = eps
        a.rope_theta = theta
        rc = self._c_append(self.handle, layer, self._append_at, self._stream(stream))
        if rc:
            self._done(rc)
        if stream is not None:
            self._keep(stream, qkv, q_out, gamma_q, gamma_k, pos)
        return q_out

    def attend(self, layer: int, q, out=None, tree=None, scale: float = 0.0, stream=None):
        """Attention of the step's queries [T][q_heads * head_dim] over their sequences; tree: int64 [T] words, bit j
        = sees new token j of its sequence (default: causal)."""
        a, cols = self._attend_args, self._q_cols
        a.ld_q = self._rows(q, cols, "attend")
        if out is None:
            out = self._new(cols, stream)
            a.ld_out = cols
        else:
            a.ld_out = self._rows(out, cols, "attend")
        a.tree = self._vector(tree, self._int64, self.T, "attend")
        a.q = q.data_ptr()
        a.out = out.data_ptr()
        a.scale = scale
        rc = self._c_attend(self.handle, layer, self._attend_at, self._stream(stream))
        if rc:
            self._done(rc)
        if stream is not None:
            self._keep(stream, q, out, tree)
        return out

    def fork(self, src, dst, stream=None):
        """Sequences dst[i] become continuations of src[i] and share its pages."""
        src, dst = self._pair(src, dst, "fork")
        self._done(self._lib.trimmoe_cache_fork(self.handle, dst[2], src[1], dst[1], self._stream(stream)))

    def truncate(self, seq, length, stream=None):
        """Cut sequences to at most length[i] positions (0 frees them)."""
        seq, length = self._pair(seq, length, "truncate")
        self._done(self._lib.trimmoe_cache_truncate(self.handle, seq[2], seq[1], length[1], self._stream(stream)))

    def accept(self, seq, n_acc, path, stream=None):
        """Keep the drafts path[i][:n_acc[i]] of the last step (int32 tensors [n] and [n][depth]), moved to the front."""
        seq = self._list(seq)
        self._tensor(n_acc, self.torch.int32, (seq[2],), "accept")
        if path.dim() != 2:
            raise TrimmoeError(-1, "accept: path is [n][depth]")
        self._tensor(path, self.torch.int32, (seq[2], path.shape[1]), "accept")
        self._done(self._lib.trimmoe_cache_accept(self.handle, seq[2], seq[1], n_acc.data_ptr(), path.data_ptr(),
                                                  path.shape[1], self._stream(stream)))
        if stream is not None:
            self._keep(stream, n_acc, path)

    def compact(self, stream=None):
        """Move the pages in use to the lowest indices, except those that the program holds itself (ref above the
        page's holders in table): these stay where they are."""
        self._done(self._lib.trimmoe_cache_compact(self.handle, self._stream(stream)))

    def stats(self, reset: bool = False) -> dict:
        """Synchronises; {status, device_error, free_pages, launches}."""
        s = trimmoe_cache_stats_t()
        rc = self._lib.trimmoe_cache_stats(self.handle, C.byref(s), int(reset))
        return dict(status=rc, device_error=s.device_error, free_pages=s.free_pages, launches=s.launches)

    def close(self):
        if getattr(self, "handle", None):
            _cache_lib().trimmoe_cache_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
