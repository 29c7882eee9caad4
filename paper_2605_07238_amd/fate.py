"""Thin ctypes binding of libfate (include/fate.h).

Argument marshalling only: numpy host arrays are passed by pointer, device
buffers are torch tensors (torch is used for device memory and streams), and
every step of the scoring path runs in libfate's HIP kernels.  There is no
fallback: if the library is missing or a call fails, an exception is raised.

Entry points mirror the C names: :func:`fate_pack_dags`,
:func:`fate_pack_state`, :func:`fate_score_frontier`, :func:`fate_topk`, plus
the host-only :func:`fate_layout_dags` / :func:`fate_layout_state`.  The calls
that a device makes for a plan's stages are :func:`fate_kv_reserve`,
:func:`fate_kv_append` (:func:`fate_kv_append_axes`), :func:`fate_attn_paged` and
:func:`fate_attn_prompt` (their scores shaped: :func:`fate_attn_paged_shaped`,
:func:`fate_attn_prompt_shaped`), :func:`fate_sample` and :func:`fate_kv_trim`;
a whole step of them can be captured in a graph.
"""

from __future__ import annotations

import ctypes as C
import functools
import math
import os
from typing import NamedTuple, Optional

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
# FATE_LIBRARY names another build of the same sources (the sanitizer build).
LIB_PATH = os.environ.get("FATE_LIBRARY") or os.path.join(HERE, "libfate.so")

FATE_OK = 0
FATE_EINVAL, FATE_ERANGE, FATE_ECYCLE, FATE_ENOFEAS, FATE_ESIZE, FATE_ESTATE, FATE_EHIP = -1, -2, -3, -4, -5, -6, -7
STATUS_NAMES = {0: "FATE_OK", -1: "FATE_EINVAL", -2: "FATE_ERANGE", -3: "FATE_ECYCLE", -4: "FATE_ENOFEAS",
                -5: "FATE_ESIZE", -6: "FATE_ESTATE", -7: "FATE_EHIP"}

# Every symbol declared in include/fate.h.
EXPORTS = ["fate_version", "fate_strerror", "fate_pack_dags_size", "fate_pack_dags", "fate_layout_dags",
           "fate_pack_state_size", "fate_pack_state", "fate_layout_state", "fate_score_ws_size",
           "fate_score_frontier", "fate_score_topk", "fate_topk", "fate_pack_state_advance_size",
           "fate_pack_state_advance", "fate_commit_ws_size", "fate_commit_advance", "fate_commit_advance_noalloc",
           "fate_pack_dags_opt_size",
           "fate_pack_dags_opt", "fate_layout_dags_opt", "fate_score_sweep", "fate_topk_sweep", "fate_plan_wave",
           "fate_simulate", "fate_place_baseline", "fate_sim_ws_size", "fate_simulate_device",
           "fate_place_baseline_device", "fate_kv_append", "fate_attn_paged_ws_size", "fate_attn_paged",
           "fate_attn_prompt", "fate_kv_reserve", "fate_kv_trim", "fate_kv_append_axes",
           "fate_attn_paged_shaped", "fate_attn_prompt_shaped", "fate_sample_ws_size", "fate_sample"]

# Scoring variants and packing options (fate_params_t.flags, fate_pack_opts_t.levels).
FATE_MEAN_PER_LEVEL, FATE_NO_WINDOWS = 1, 2
FATE_LEVELS_HOP, FATE_LEVELS_TOPO = 0, 1
FATE_MAX_SWEEP = 16
FATE_PLACE_ROUND_ROBIN, FATE_PLACE_HEFT = 0, 1
FATE_BF16, FATE_F16, FATE_F32 = 0, 1, 2
FATE_NOALLOC_WS_BYTES = 32 << 20  # workspace the library holds per GPU for fate_commit_advance_noalloc


class FateError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__("%s failed: %s (%s)" % (what, STATUS_NAMES.get(status, status), _strerror(status)))


class Cluster(C.Structure):
    _fields_ = [("D", C.c_int32), ("M", C.c_int32), ("exec", C.c_void_p), ("switch_s", C.c_void_p),
                ("weight_bytes", C.c_void_p), ("cap_bytes", C.c_void_p), ("beta", C.c_void_p)]


class DagBatch(C.Structure):
    _fields_ = [("B", C.c_int32), ("stage_off", C.c_void_p), ("par_off", C.c_void_p), ("par_idx", C.c_void_p),
                ("model", C.c_void_p), ("elig", C.c_void_p), ("shard_max", C.c_void_p),
                ("prefix_hash", C.c_void_p), ("prefix_tokens", C.c_void_p), ("out_bytes", C.c_void_p)]


class State(C.Structure):
    _fields_ = [("K", C.c_int32), ("resident", C.c_void_p), ("prefix_cache", C.c_void_p),
                ("holders", C.c_void_p), ("status", C.c_void_p), ("tau_free", C.c_void_p),
                ("t_now", C.c_void_p)]


class Params(C.Structure):
    _fields_ = [("lam_q", C.c_float), ("lam_s", C.c_float), ("lam_tr", C.c_float), ("lam_c", C.c_float),
                ("lam_p", C.c_float), ("kappa_prefix", C.c_float), ("gamma", C.c_float), ("H", C.c_int32),
                ("lam_m", C.c_float), ("flags", C.c_int32)]


class SimMetrics(C.Structure):
    _fields_ = [("tasks", C.c_int64), ("makespan", C.c_double), ("p95", C.c_double), ("xdev_edges", C.c_int64),
                ("cache_hits", C.c_int64), ("model_cont", C.c_int64)]


class PackOpts(C.Structure):
    _fields_ = [("H", C.c_int32), ("levels", C.c_int32), ("level_weights", C.c_int32)]


class Dags(C.Structure):
    _fields_ = [("B", C.c_int32), ("D", C.c_int32), ("M", C.c_int32), ("H", C.c_int32),
                ("N", C.c_int64), ("E", C.c_int64), ("n_desc", C.c_int64),
                ("beta_uniform", C.c_int32), ("beta0", C.c_float),
                ("base", C.c_void_p), ("bytes", C.c_size_t),
                ("exec", C.c_void_p), ("switch_s", C.c_void_p), ("beta", C.c_void_p),
                ("weight", C.c_void_p), ("cap", C.c_void_p), ("fits", C.c_void_p),
                ("records", C.c_void_p), ("par_idx", C.c_void_p), ("desc_off", C.c_void_p),
                ("desc", C.c_void_p), ("stage_off", C.c_void_p), ("levels", C.c_int32), ("desc_w", C.c_void_p),
                ("max_r", C.c_int32), ("ch_off", C.c_void_p), ("ch_idx", C.c_void_p),
                ("max_stages", C.c_int64), ("row_records", C.c_void_p)]


class StateH(C.Structure):
    _fields_ = [("B", C.c_int32), ("D", C.c_int32), ("K", C.c_int32), ("max_shard", C.c_int32),
                ("N", C.c_int64), ("n_frontier", C.c_int64), ("n_cand", C.c_int64),
                ("base", C.c_void_p), ("bytes", C.c_size_t),
                ("resident", C.c_void_p), ("prefix_cache", C.c_void_p), ("holders", C.c_void_p),
                ("tau_free", C.c_void_p), ("t_now", C.c_void_p),
                ("frontier", C.c_void_p), ("cand_off", C.c_void_p),
                ("n_slices", C.c_int64), ("slices", C.c_void_p),
                ("n_done_edges", C.c_int64), ("done_n", C.c_void_p), ("done", C.c_void_p),
                ("advance", C.c_int32), ("status", C.c_void_p), ("counts", C.c_void_p), ("finish", C.c_void_p),
                ("slice", C.c_int32), ("fr_off", C.c_void_p), ("order", C.c_void_p)]


class Heads(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("heads_q", C.c_int32), ("heads_kv", C.c_int32), ("head_dim", C.c_int32)]


class Rows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("token", C.c_int64), ("head", C.c_int64)]


class KvCache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("page", C.c_int64), ("head", C.c_int64),
                ("token", C.c_int64), ("n_pages", C.c_int32), ("page_size", C.c_int32)]


class Seqs(C.Structure):
    _fields_ = [("B", C.c_int32), ("max_pages", C.c_int32), ("T", C.c_int64), ("pages_stride", C.c_int64),
                ("off", C.c_void_p), ("kv_len", C.c_void_p), ("pages", C.c_void_p)]


class Axes(C.Structure):
    _fields_ = [("n_axes", C.c_int32), ("pair_axis", C.c_void_p), ("positions", C.c_void_p), ("stride", C.c_int64)]


class Scores(C.Structure):
    _fields_ = [("cap", C.c_float), ("slopes", C.c_void_p), ("prefix", C.c_void_p), ("start", C.c_void_p)]


class KvTables(C.Structure):
    _fields_ = [("B", C.c_int32), ("max_pages", C.c_int32), ("page_size", C.c_int32), ("n_pages", C.c_int32),
                ("pages_stride", C.c_int64), ("pages", C.c_void_p), ("free", C.c_void_p), ("n_free", C.c_void_p),
                ("kv_len", C.c_void_p)]


class Sampling(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("rows", C.c_int32), ("vocab", C.c_int32), ("stride", C.c_int64),
                ("logits", C.c_void_p), ("u", C.c_void_p), ("temperature", C.c_void_p), ("top_k", C.c_void_p),
                ("top_p", C.c_void_p), ("min_p", C.c_void_p), ("temperature_all", C.c_float), ("top_k_all", C.c_int32),
                ("top_p_all", C.c_float), ("min_p_all", C.c_float)]


_lib = None


def load(path: Optional[str] = None):
    """Load libfate.so; raises if it has not been built."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise RuntimeError("libfate.so not found at %s; build it with `python -m paper_2605_07238_amd.build`" % p)
    lib = C.CDLL(p)
    P = C.POINTER
    st = C.c_int
    lib.fate_version.restype = C.c_char_p
    lib.fate_strerror.restype = C.c_char_p
    lib.fate_strerror.argtypes = [st]
    lib.fate_pack_dags_size.argtypes = [P(Cluster), P(DagBatch), C.c_int32, P(C.c_size_t)]
    lib.fate_pack_dags.argtypes = [P(Cluster), P(DagBatch), C.c_int32, C.c_void_p, C.c_size_t, C.c_void_p, P(Dags)]
    lib.fate_layout_dags.argtypes = [P(Cluster), P(DagBatch), C.c_int32, C.c_void_p, C.c_size_t, P(Dags)]
    lib.fate_pack_state_size.argtypes = [P(Dags), P(DagBatch), P(State), C.c_int32, P(C.c_size_t),
                                         P(C.c_int64), P(C.c_int64)]
    lib.fate_pack_state.argtypes = [P(Dags), P(DagBatch), P(State), C.c_int32, C.c_void_p, C.c_size_t,
                                    C.c_void_p, P(StateH)]
    lib.fate_layout_state.argtypes = [P(Dags), P(DagBatch), P(State), C.c_int32, C.c_void_p, C.c_size_t, P(StateH)]
    lib.fate_score_ws_size.argtypes = [P(Dags), P(StateH), P(C.c_size_t)]
    lib.fate_score_frontier.argtypes = [P(Dags), P(StateH), P(Params), C.c_void_p, C.c_int64, C.c_void_p,
                                        C.c_size_t, C.c_void_p]
    lib.fate_score_topk.argtypes = [P(Dags), P(StateH), P(Params), C.c_void_p, C.c_int64, C.c_int32, C.c_void_p,
                                    C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    lib.fate_topk.argtypes = [P(StateH), C.c_void_p, C.c_int64, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]
    lib.fate_pack_state_advance_size.argtypes = [P(Dags), P(DagBatch), P(State), C.c_int32, P(C.c_size_t)]
    lib.fate_pack_state_advance.argtypes = [P(Dags), P(DagBatch), P(State), C.c_int32, C.c_void_p, C.c_size_t,
                                            C.c_void_p, P(StateH)]
    lib.fate_commit_ws_size.argtypes = [P(Dags), P(StateH), P(C.c_size_t)]
    lib.fate_commit_advance.argtypes = [P(Dags), P(StateH), C.c_void_p, C.c_int32, C.c_void_p, C.c_size_t,
                                        C.c_void_p]
    lib.fate_commit_advance_noalloc.argtypes = [P(Dags), P(StateH), C.c_void_p, C.c_int32, C.c_void_p]
    lib.fate_pack_dags_opt_size.argtypes = [P(Cluster), P(DagBatch), P(PackOpts), P(C.c_size_t)]
    lib.fate_pack_dags_opt.argtypes = [P(Cluster), P(DagBatch), P(PackOpts), C.c_void_p, C.c_size_t, C.c_void_p,
                                       P(Dags)]
    lib.fate_layout_dags_opt.argtypes = [P(Cluster), P(DagBatch), P(PackOpts), C.c_void_p, C.c_size_t, P(Dags)]
    lib.fate_score_sweep.argtypes = [P(Dags), P(StateH), P(Params), C.c_int32, C.c_void_p, C.c_int64, C.c_int64,
                                     C.c_void_p, C.c_size_t, C.c_void_p]
    lib.fate_topk_sweep.argtypes = [P(StateH), C.c_void_p, C.c_int64, C.c_int64, C.c_int32, C.c_int32, C.c_void_p,
                                    C.c_void_p, C.c_void_p]
    lib.fate_plan_wave.argtypes = [P(StateH), C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p]
    lib.fate_simulate.argtypes = [P(Cluster), P(DagBatch), P(State), C.c_void_p, C.c_void_p, C.c_float,
                                  P(SimMetrics)]
    lib.fate_place_baseline.argtypes = [P(Cluster), P(DagBatch), P(State), C.c_int32, C.c_float, C.c_void_p,
                                        C.c_void_p]
    lib.fate_sim_ws_size.argtypes = [P(Dags), P(C.c_size_t)]
    lib.fate_simulate_device.argtypes = [P(Dags), P(StateH), C.c_void_p, C.c_void_p, C.c_float, C.c_void_p,
                                         C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    lib.fate_place_baseline_device.argtypes = [P(Dags), P(StateH), C.c_int32, C.c_float, C.c_void_p, C.c_void_p,
                                               C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    lib.fate_kv_append.argtypes = [P(Heads), P(Seqs), P(Rows), P(Rows), P(Rows), C.c_void_p, C.c_int64, C.c_int32,
                                   C.c_int32, P(KvCache), P(Rows), C.c_void_p, C.c_void_p]
    lib.fate_attn_paged_ws_size.argtypes = [P(Heads), P(Seqs), P(KvCache), C.c_int64, P(C.c_size_t)]
    lib.fate_attn_paged.argtypes = [P(Heads), P(Seqs), P(Rows), P(KvCache), C.c_int64, C.c_float, P(Rows),
                                    C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    lib.fate_attn_prompt.argtypes = [P(Heads), P(Seqs), P(Rows), P(Rows), P(Rows), C.c_float, P(Rows), C.c_void_p,
                                     C.c_void_p, C.c_void_p]
    lib.fate_kv_append_axes.argtypes = [P(Heads), P(Seqs), P(Rows), P(Rows), P(Rows), C.c_void_p, C.c_int64, C.c_int32,
                                        C.c_int32, P(Axes), P(KvCache), P(Rows), C.c_void_p, C.c_void_p]
    lib.fate_attn_paged_shaped.argtypes = [P(Heads), P(Seqs), P(Rows), P(KvCache), C.c_int64, C.c_float, P(Scores), P(Rows),
                                           C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    lib.fate_attn_prompt_shaped.argtypes = [P(Heads), P(Seqs), P(Rows), P(Rows), P(Rows), C.c_float, P(Scores), P(Rows),
                                            C.c_void_p, C.c_void_p, C.c_void_p]
    lib.fate_kv_reserve.argtypes = [P(KvTables), C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                    C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
    lib.fate_kv_trim.argtypes = [P(KvTables), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
    lib.fate_sample_ws_size.argtypes = [P(Sampling), P(C.c_size_t)]
    lib.fate_sample.argtypes = [P(Sampling), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    for name in EXPORTS[2:]:
        getattr(lib, name).restype = st
    if path is None:
        _lib = lib
    return lib


def _strerror(status: int) -> str:
    try:
        return load().fate_strerror(status).decode()
    except Exception:  # noqa: BLE001 - best effort in an error path
        return "?"


def _check(status: int, what: str):
    if status != FATE_OK:
        raise FateError(status, what)


def version() -> str:
    return load().fate_version().decode()


def _c(a, dt):
    return np.ascontiguousarray(a, dtype=dt)


class HostInputs:
    """C views of a workload's host arrays (kept alive by this object)."""

    def __init__(self, w):
        self.keep = dict(
            exec=_c(w.exec, np.float32), switch_s=_c(w.switch_s, np.float32),
            weight=_c(w.weight_bytes, np.int64), cap=_c(w.cap_bytes, np.int64), beta=_c(w.beta, np.float32),
            stage_off=_c(w.stage_off, np.int64), par_off=_c(w.par_off, np.int64), par_idx=_c(w.par_idx, np.int32),
            model=_c(w.model, np.int32), elig=_c(w.elig, np.uint64), shard=_c(w.shard_max, np.int32),
            hash=_c(w.prefix_hash, np.uint64), tokens=_c(w.prefix_tokens, np.float32),
            sigma=_c(w.out_bytes, np.float32),
            resident=_c(w.resident, np.uint64), cache=_c(w.prefix_cache, np.uint64),
            holders=_c(w.holders, np.uint64), status=_c(w.status, np.uint8),
            tau=_c(w.tau_free, np.float32), t_now=_c(w.t_now, np.float32),
        )
        k = self.keep
        ptr = lambda a: a.ctypes.data if a.size else None
        self.cluster = Cluster(int(w.D), int(w.M), ptr(k["exec"]), ptr(k["switch_s"]), ptr(k["weight"]),
                               ptr(k["cap"]), ptr(k["beta"]))
        self.batch = DagBatch(int(w.B), k["stage_off"].ctypes.data, ptr(k["par_off"]), ptr(k["par_idx"]),
                              ptr(k["model"]), ptr(k["elig"]), ptr(k["shard"]), ptr(k["hash"]), ptr(k["tokens"]),
                              ptr(k["sigma"]))
        self.state = State(int(w.K), ptr(k["resident"]), ptr(k["cache"]), ptr(k["holders"]), ptr(k["status"]),
                           ptr(k["tau"]), ptr(k["t_now"]))


def _stream_ptr(stream):
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream


class PackedDags:
    def __init__(self, buf, handle: Dags, host: HostInputs):
        self.buf = buf          # torch uint8 device tensor owning the memory
        self.handle = handle
        self.host = host


class PackedState:
    def __init__(self, buf, handle: StateH, host: HostInputs):
        self.buf = buf
        self.handle = handle
        self.host = host

    @property
    def n_frontier(self) -> int:
        return int(self.handle.n_frontier)

    @property
    def n_cand(self) -> int:
        return int(self.handle.n_cand)

    @property
    def advance(self) -> bool:
        return bool(self.handle.advance)

    def counts(self):
        """Current (frontier stages, candidates, slices, rejected selections):
        read from the device for a planning state (synchronises)."""
        import torch
        h = self.handle
        if not h.advance:
            return int(h.n_frontier), int(h.n_cand), int(h.n_slices), 0
        off = h.counts - self.buf.data_ptr()
        c = self.buf[off:off + 16].view(torch.int32).cpu().numpy().astype(np.int64)
        return int(c[0]), int(c[1]), int(c[2]), int(c[3])


def fate_pack_dags_size(w, H: int) -> int:
    hi = HostInputs(w)
    nbytes = C.c_size_t(0)
    _check(load().fate_pack_dags_size(C.byref(hi.cluster), C.byref(hi.batch), int(H), C.byref(nbytes)),
           "fate_pack_dags_size")
    return int(nbytes.value)


def _pack_opts(w, H, levels, level_weights) -> PackOpts:
    p = dict(w.params) if w is not None else {}
    lv = int(levels if levels is not None else (FATE_LEVELS_TOPO if p.get("topo_levels") else FATE_LEVELS_HOP))
    lw = int(bool(level_weights if level_weights is not None else p.get("mean_levels", 0)))
    return PackOpts(int(w.H if H is None else H), lv, lw)


def fate_pack_dags(w, H: Optional[int] = None, device="cuda", stream=None, levels: Optional[int] = None,
                   level_weights: Optional[bool] = None) -> PackedDags:
    """Validate and pack workload ``w``'s DAG batch into a device buffer.
    ``levels`` (FATE_LEVELS_HOP / _TOPO) and ``level_weights`` default to the
    workload's ``topo_levels`` / ``mean_levels`` parameters."""
    import torch
    o = _pack_opts(w, H, levels, level_weights)
    lib = load()
    hi = HostInputs(w)
    nbytes = C.c_size_t(0)
    _check(lib.fate_pack_dags_opt_size(C.byref(hi.cluster), C.byref(hi.batch), C.byref(o), C.byref(nbytes)),
           "fate_pack_dags_opt_size")
    buf = torch.empty(max(1, nbytes.value), dtype=torch.uint8, device=device)
    h = Dags()
    _check(lib.fate_pack_dags_opt(C.byref(hi.cluster), C.byref(hi.batch), C.byref(o), C.c_void_p(buf.data_ptr()),
                                  nbytes.value, C.c_void_p(_stream_ptr(stream)), C.byref(h)), "fate_pack_dags_opt")
    return PackedDags(buf, h, hi)


def fate_layout_dags(w, H: Optional[int] = None, levels: Optional[int] = None,
                     level_weights: Optional[bool] = None):
    """Host-only packed image of the DAG batch: (numpy uint8 buffer, Dags handle)."""
    o = _pack_opts(w, H, levels, level_weights)
    lib = load()
    hi = HostInputs(w)
    nbytes = C.c_size_t(0)
    _check(lib.fate_pack_dags_opt_size(C.byref(hi.cluster), C.byref(hi.batch), C.byref(o), C.byref(nbytes)),
           "fate_pack_dags_opt_size")
    buf = np.zeros(max(1, nbytes.value), np.uint8)
    h = Dags()
    _check(lib.fate_layout_dags_opt(C.byref(hi.cluster), C.byref(hi.batch), C.byref(o), buf.ctypes.data,
                                    nbytes.value, C.byref(h)), "fate_layout_dags_opt")
    return buf, h, hi


def fate_pack_state(packed: PackedDags, w, max_shard: Optional[int] = None, device="cuda",
                    stream=None, advance: bool = False) -> PackedState:
    """Validate the state of ``w`` against ``packed`` and pack state + frontier.
    ``advance`` packs a planning state for fate_commit_advance."""
    import torch
    ms = int(w.max_shard if max_shard is None else max_shard)
    lib = load()
    hi = HostInputs(w)
    nbytes = C.c_size_t(0)
    if advance:
        _check(lib.fate_pack_state_advance_size(C.byref(packed.handle), C.byref(hi.batch), C.byref(hi.state), ms,
                                                C.byref(nbytes)), "fate_pack_state_advance_size")
        buf = torch.empty(max(1, nbytes.value), dtype=torch.uint8, device=device)
        h = StateH()
        _check(lib.fate_pack_state_advance(C.byref(packed.handle), C.byref(hi.batch), C.byref(hi.state), ms,
                                           C.c_void_p(buf.data_ptr()), nbytes.value,
                                           C.c_void_p(_stream_ptr(stream)), C.byref(h)), "fate_pack_state_advance")
        return PackedState(buf, h, hi)
    nf, nc = C.c_int64(0), C.c_int64(0)
    _check(lib.fate_pack_state_size(C.byref(packed.handle), C.byref(hi.batch), C.byref(hi.state), ms,
                                    C.byref(nbytes), C.byref(nf), C.byref(nc)), "fate_pack_state_size")
    buf = torch.empty(max(1, nbytes.value), dtype=torch.uint8, device=device)
    h = StateH()
    _check(lib.fate_pack_state(C.byref(packed.handle), C.byref(hi.batch), C.byref(hi.state), ms,
                               C.c_void_p(buf.data_ptr()), nbytes.value, C.c_void_p(_stream_ptr(stream)),
                               C.byref(h)), "fate_pack_state")
    return PackedState(buf, h, hi)


def fate_layout_state(dags_handle: Dags, w, max_shard: Optional[int] = None):
    """Host-only packed state image: (numpy uint8 buffer, StateH handle)."""
    ms = int(w.max_shard if max_shard is None else max_shard)
    lib = load()
    hi = HostInputs(w)
    nbytes = C.c_size_t(0)
    nf, nc = C.c_int64(0), C.c_int64(0)
    _check(lib.fate_pack_state_size(C.byref(dags_handle), C.byref(hi.batch), C.byref(hi.state), ms,
                                    C.byref(nbytes), C.byref(nf), C.byref(nc)), "fate_pack_state_size")
    buf = np.zeros(max(1, nbytes.value), np.uint8)
    h = StateH()
    _check(lib.fate_layout_state(C.byref(dags_handle), C.byref(hi.batch), C.byref(hi.state), ms, buf.ctypes.data,
                                 nbytes.value, C.byref(h)), "fate_layout_state")
    return buf, h, hi


def make_params(w=None, H: Optional[int] = None, **over) -> Params:
    from . import synth
    p = dict(synth.DEFAULT_PARAMS)
    if w is not None:
        p.update(w.params)
    p.update({k: v for k, v in over.items() if k != "H"})
    Hv = int(H if H is not None else (w.H if w is not None else 0))
    flags = (FATE_MEAN_PER_LEVEL if p.get("mean_levels") else 0) | (FATE_NO_WINDOWS if p.get("no_windows") else 0)
    return Params(p["lam_q"], p["lam_s"], p["lam_tr"], p["lam_c"], p["lam_p"], p["kappa_prefix"], p["gamma"], Hv,
                  float(p.get("lam_m", 0.0)), flags)


def fate_score_frontier(packed: PackedDags, state: PackedState, params: Params, out=None, stream=None):
    """Score every candidate; returns a float32 device tensor [n_cand]."""
    import torch
    lib = load()
    nc = state.n_cand
    if out is None:
        out = torch.empty(max(1, nc), dtype=torch.float32, device=packed.buf.device)
    ws = C.c_size_t(0)
    _check(lib.fate_score_ws_size(C.byref(packed.handle), C.byref(state.handle), C.byref(ws)), "fate_score_ws_size")
    wsbuf = torch.empty(max(1, ws.value), dtype=torch.uint8, device=packed.buf.device) if ws.value else None
    _check(lib.fate_score_frontier(C.byref(packed.handle), C.byref(state.handle), C.byref(params),
                                   C.c_void_p(out.data_ptr()), int(out.numel()),
                                   C.c_void_p(wsbuf.data_ptr()) if wsbuf is not None else None, ws.value,
                                   C.c_void_p(_stream_ptr(stream))), "fate_score_frontier")
    return out


def fate_score_topk(packed: PackedDags, state: PackedState, params: Params, k: int, out=None, idx=None, val=None,
                    stream=None):
    """Scores and per-stage top-k in one launch; returns (scores, idx [F,k], val [F,k])."""
    import torch
    lib = load()
    nc, F = state.n_cand, state.n_frontier
    dev = packed.buf.device
    if out is None:
        out = torch.empty(max(1, nc), dtype=torch.float32, device=dev)
    if idx is None:
        idx = torch.empty((max(1, F), k), dtype=torch.int32, device=dev)
    if val is None:
        val = torch.empty((max(1, F), k), dtype=torch.float32, device=dev)
    ws = C.c_size_t(0)
    _check(lib.fate_score_ws_size(C.byref(packed.handle), C.byref(state.handle), C.byref(ws)), "fate_score_ws_size")
    wsbuf = torch.empty(max(1, ws.value), dtype=torch.uint8, device=dev) if ws.value else None
    _check(lib.fate_score_topk(C.byref(packed.handle), C.byref(state.handle), C.byref(params),
                               C.c_void_p(out.data_ptr()), int(out.numel()), int(k), C.c_void_p(idx.data_ptr()),
                               C.c_void_p(val.data_ptr()),
                               C.c_void_p(wsbuf.data_ptr()) if wsbuf is not None else None, ws.value,
                               C.c_void_p(_stream_ptr(stream))), "fate_score_topk")
    return out, idx[:F], val[:F]


def fate_topk(state: PackedState, scores, k: int, idx=None, val=None, stream=None):
    """Per-frontier-stage top-k; returns (int32 [F, k], float32 [F, k]) device tensors."""
    import torch
    lib = load()
    F = state.n_frontier
    dev = scores.device
    if idx is None:
        idx = torch.empty((max(1, F), k), dtype=torch.int32, device=dev)
    if val is None:
        val = torch.empty((max(1, F), k), dtype=torch.float32, device=dev)
    _check(lib.fate_topk(C.byref(state.handle), C.c_void_p(scores.data_ptr()), int(scores.numel()), int(k),
                         C.c_void_p(idx.data_ptr()), C.c_void_p(val.data_ptr()),
                         C.c_void_p(_stream_ptr(stream))), "fate_topk")
    return idx[:F], val[:F]


def fate_score_sweep(packed: PackedDags, state: PackedState, params, out=None, stride: Optional[int] = None,
                     stream=None):
    """Score every candidate under each of ``params`` (a list of Params, at
    most FATE_MAX_SWEEP) in one launch; returns a float32 device tensor
    [len(params), stride] (set p in row p)."""
    import torch
    lib = load()
    P = len(params)
    stride = int(stride if stride is not None else max(1, state.n_cand))
    if out is None:
        out = torch.empty((max(1, P), stride), dtype=torch.float32, device=packed.buf.device)
    arr = (Params * max(1, P))(*params)
    _check(lib.fate_score_sweep(C.byref(packed.handle), C.byref(state.handle), arr, int(P),
                                C.c_void_p(out.data_ptr()), int(out.numel()), stride, None, 0,
                                C.c_void_p(_stream_ptr(stream))), "fate_score_sweep")
    return out


def fate_topk_sweep(state: PackedState, scores, k: int, idx=None, val=None, stream=None):
    """Top-k of every row of a [P, stride] score tensor (the fate_score_sweep
    layout); returns (int32 [P, F, k], float32 [P, F, k]) device tensors, F the
    handle's frontier size (its capacity for a planning state)."""
    import torch
    lib = load()
    P, stride = int(scores.shape[0]), int(scores.shape[1])
    F = state.n_frontier
    dev = scores.device
    if idx is None:
        idx = torch.empty((P, max(1, F), k), dtype=torch.int32, device=dev)
    if val is None:
        val = torch.empty((P, max(1, F), k), dtype=torch.float32, device=dev)
    _check(lib.fate_topk_sweep(C.byref(state.handle), C.c_void_p(scores.data_ptr()), int(scores.numel()), stride,
                               P, int(k), C.c_void_p(idx.data_ptr()), C.c_void_p(val.data_ptr()),
                               C.c_void_p(_stream_ptr(stream))), "fate_topk_sweep")
    return idx[:, :F], val[:, :F]


def fate_plan_wave(state: PackedState, idx, val, sel=None, stream=None):
    """One frontier planning wave from per-stage choices ``idx`` / ``val``
    ([F, k] device tensors, the fate_topk layout); returns the int32 device
    tensor sel [F] (-1 = not placed in this wave)."""
    import torch
    lib = load()
    F = state.n_frontier
    k = int(idx.shape[1]) if idx.dim() == 2 else 1
    if sel is None:
        sel = torch.empty(max(1, F), dtype=torch.int32, device=idx.device)
    _check(lib.fate_plan_wave(C.byref(state.handle), C.c_void_p(idx.data_ptr()), C.c_void_p(val.data_ptr()), k,
                              C.c_void_p(sel.data_ptr()), C.c_void_p(_stream_ptr(stream))), "fate_plan_wave")
    return sel[:F]


def fate_simulate(w, devices, order, kappa_prefix: Optional[float] = None) -> dict:
    """Execute a placement (host arrays: devices [N] uint64 masks, order [N]
    int64 keys) on every instance of ``w``; returns per-instance numpy arrays
    tasks, makespan, p95, xdev_edges, cache_hits, model_cont."""
    lib = load()
    hi = HostInputs(w)
    kpf = float(w.params["kappa_prefix"] if kappa_prefix is None else kappa_prefix)
    dev = np.ascontiguousarray(devices, np.uint64)
    odr = np.ascontiguousarray(order, np.int64)
    out = (SimMetrics * max(1, w.B))()
    _check(lib.fate_simulate(C.byref(hi.cluster), C.byref(hi.batch), C.byref(hi.state), dev.ctypes.data,
                             odr.ctypes.data, kpf, out), "fate_simulate")
    res = {}
    for name, _ in SimMetrics._fields_:
        res[name] = np.array([getattr(out[b], name) for b in range(w.B)],
                             np.float64 if name in ("makespan", "p95") else np.int64)
    return res


def fate_place_baseline(w, policy: int, kappa_prefix: Optional[float] = None):
    """Round-robin or HEFT-style placement of ``w``'s pending stages:
    (devices [N] uint64, order [N] int64) host arrays."""
    lib = load()
    hi = HostInputs(w)
    kpf = float(w.params["kappa_prefix"] if kappa_prefix is None else kappa_prefix)
    dev = np.zeros(w.N, np.uint64)
    odr = np.zeros(w.N, np.int64)
    _check(lib.fate_place_baseline(C.byref(hi.cluster), C.byref(hi.batch), C.byref(hi.state), int(policy), kpf,
                                   dev.ctypes.data, odr.ctypes.data), "fate_place_baseline")
    return dev, odr


def fate_commit_ws_size(packed: PackedDags, state: PackedState) -> int:
    ws = C.c_size_t(0)
    _check(load().fate_commit_ws_size(C.byref(packed.handle), C.byref(state.handle), C.byref(ws)),
           "fate_commit_ws_size")
    return int(ws.value)


def fate_commit_advance(packed: PackedDags, state: PackedState, sel, ws=None, stream=None):
    """Commit the candidate chosen per frontier slot and advance the planning
    state on the device.  ``sel``: int32 device tensor [F] or [F, k] (a top-k
    array: its first column is used), -1 = leave pending.  Returns ``ws``."""
    import torch
    lib = load()
    if sel.dtype != torch.int32 or not sel.is_contiguous():
        raise ValueError("sel must be a contiguous int32 tensor")
    stride = int(sel.shape[1]) if sel.dim() == 2 else 1
    nbytes = fate_commit_ws_size(packed, state)
    if ws is None or ws.numel() < nbytes:
        ws = torch.empty(max(1, nbytes), dtype=torch.uint8, device=packed.buf.device)
    _check(lib.fate_commit_advance(C.byref(packed.handle), C.byref(state.handle), C.c_void_p(sel.data_ptr()),
                                   stride, C.c_void_p(ws.data_ptr()), nbytes, C.c_void_p(_stream_ptr(stream))),
           "fate_commit_advance")
    return ws


def fate_commit_advance_noalloc(packed: PackedDags, state: PackedState, sel, stream=None):
    """fate_commit_advance with the library-held workspace (no device
    allocation by the library or here).  ``sel`` as for fate_commit_advance."""
    import torch
    if sel.dtype != torch.int32 or not sel.is_contiguous():
        raise ValueError("sel must be a contiguous int32 tensor")
    stride = int(sel.shape[1]) if sel.dim() == 2 else 1
    _check(load().fate_commit_advance_noalloc(C.byref(packed.handle), C.byref(state.handle),
                                              C.c_void_p(sel.data_ptr()), stride, C.c_void_p(_stream_ptr(stream))),
           "fate_commit_advance_noalloc")


def fate_sim_ws_size(packed: PackedDags) -> int:
    n = C.c_size_t(0)
    _check(load().fate_sim_ws_size(C.byref(packed.handle), C.byref(n)), "fate_sim_ws_size")
    return int(n.value)


def _sim_status(status, what: str):
    bad = status.cpu().numpy()
    nz = np.nonzero(bad != FATE_OK)[0]
    if len(nz):
        raise FateError(int(bad[nz[0]]), "%s (instance %d)" % (what, int(nz[0])))


def fate_simulate_device(packed: PackedDags, state: PackedState, devices, order, kappa_prefix: float,
                         ws=None, stream=None) -> dict:
    """Execute a placement on the device: ``devices`` uint64 (as int64) and
    ``order`` int64 device tensors [N] over flat stage ids.  Returns the
    per-instance metrics as numpy arrays (tasks, makespan, p95, xdev_edges,
    cache_hits, model_cont); raises on a per-instance error status."""
    import torch
    lib = load()
    dev = packed.buf.device
    for t, nm in ((devices, "devices"), (order, "order")):
        if t.dtype != torch.int64 or not t.is_contiguous() or t.numel() < packed.handle.N:
            raise ValueError("%s must be a contiguous int64 tensor of N elements" % nm)
    nbytes = fate_sim_ws_size(packed)
    if ws is None or ws.numel() < nbytes:
        ws = torch.empty(max(1, nbytes), dtype=torch.uint8, device=dev)
    B = int(packed.handle.B)
    out = torch.empty((max(1, B), C.sizeof(SimMetrics)), dtype=torch.uint8, device=dev)
    status = torch.empty(max(1, B), dtype=torch.int32, device=dev)
    _check(lib.fate_simulate_device(C.byref(packed.handle), C.byref(state.handle), C.c_void_p(devices.data_ptr()),
                                    C.c_void_p(order.data_ptr()), float(kappa_prefix), C.c_void_p(out.data_ptr()),
                                    C.c_void_p(status.data_ptr()), C.c_void_p(ws.data_ptr()), nbytes,
                                    C.c_void_p(_stream_ptr(stream))), "fate_simulate_device")
    _sim_status(status[:B], "fate_simulate_device")
    raw = out[:B].cpu().numpy()
    rec = np.frombuffer(raw.tobytes(), dtype=np.dtype([(name, np.float64 if name in ("makespan", "p95") else np.int64)
                                                       for name, _ in SimMetrics._fields_]), count=B)
    return {name: np.array(rec[name]) for name, _ in SimMetrics._fields_}


def fate_place_baseline_device(packed: PackedDags, state: PackedState, policy: int, kappa_prefix: float,
                               ws=None, stream=None):
    """Round-robin or HEFT-style placement built on the device: (devices,
    order) int64 device tensors [N] (devices holds the uint64 masks)."""
    import torch
    lib = load()
    dev = packed.buf.device
    N, B = int(packed.handle.N), int(packed.handle.B)
    nbytes = fate_sim_ws_size(packed)
    if ws is None or ws.numel() < nbytes:
        ws = torch.empty(max(1, nbytes), dtype=torch.uint8, device=dev)
    devices = torch.empty(max(1, N), dtype=torch.int64, device=dev)
    order = torch.empty(max(1, N), dtype=torch.int64, device=dev)
    status = torch.empty(max(1, B), dtype=torch.int32, device=dev)
    _check(lib.fate_place_baseline_device(C.byref(packed.handle), C.byref(state.handle), int(policy),
                                          float(kappa_prefix), C.c_void_p(devices.data_ptr()),
                                          C.c_void_p(order.data_ptr()), C.c_void_p(status.data_ptr()),
                                          C.c_void_p(ws.data_ptr()), nbytes, C.c_void_p(_stream_ptr(stream))),
           "fate_place_baseline_device")
    _sim_status(status[:B], "fate_place_baseline_device")
    return devices[:N], order[:N]


def state_arrays(state: PackedState):
    """Host copies of the packed state arrays: resident [B, D], prefix slots
    [B, D, K], holders [N], free times [B, D], and (planning state) status [N]
    and planned finish [N]."""
    import torch
    h = state.handle
    base = state.buf.data_ptr()
    B, D, K, N = int(h.B), int(h.D), int(h.K), int(h.N)

    def take(ptr, n, dt):
        off = ptr - base
        nb = n * np.dtype(dt).itemsize
        if n == 0:
            return np.zeros(0, dt)
        return state.buf[off:off + nb].cpu().numpy().view(dt).copy()

    out = dict(resident=take(h.resident, B * D, np.uint64).reshape(B, D),
               prefix_cache=take(h.prefix_cache, B * D * K, np.uint64).reshape(B, D, K),
               holders=take(h.holders, N, np.uint64), tau_free=take(h.tau_free, B * D, np.float32).reshape(B, D))
    if h.advance:
        out["status"] = take(h.status, N, np.uint8)
        out["finish"] = take(h.finish, N, np.float32)
    return out


def frontier_table(state: PackedState):
    """Host copies of the packed frontier: (flat stage ids, instances, cand_off)."""
    import torch
    h = state.handle
    F = state.counts()[0]
    base = state.buf.data_ptr()
    off_f = h.frontier - base
    off_c = h.cand_off - base
    fr = state.buf[off_f:off_f + 8 * F].view(torch.int32).cpu().numpy().reshape(F, 2) if F else np.zeros((0, 2), np.int32)
    co = state.buf[off_c:off_c + 4 * (F + 1)].view(torch.int32).cpu().numpy()
    return fr[:, 0].astype(np.int64), fr[:, 1].astype(np.int64), co.astype(np.int64)


def desc_counts(packed: PackedDags):
    """Host copy of every stage's horizon-descendant count (from desc_off)."""
    import torch
    h = packed.handle
    N = int(h.N)
    off = h.desc_off - packed.buf.data_ptr()
    do = packed.buf[off:off + 4 * (N + 1)].view(torch.int32).cpu().numpy().astype(np.int64)
    return np.diff(do)


# ---- attention of a planned wave -------------------------------------------
# A serving step makes these calls tens of thousands of times a second and the
# small ones are over in a few microseconds, so the checks are written to be
# cheap: torch is looked up once, and each property of a tensor is asked for once.

_t = None  # the parts of torch that the calls use


class _Torch:
    def __init__(self):
        import torch
        self.types = {torch.bfloat16: FATE_BF16, torch.float16: FATE_F16}
        self.logit_types = {torch.bfloat16: FATE_BF16, torch.float16: FATE_F16, torch.float32: FATE_F32}
        self.int32, self.int64, self.float32, self.uint8 = torch.int32, torch.int64, torch.float32, torch.uint8
        self.empty, self.empty_like, self.Tensor = torch.empty, torch.empty_like, torch.Tensor
        self.device, self.stream = torch.cuda.device, torch.cuda.stream
        self.current_device = torch.cuda.current_device
        self.raw_stream = torch._C._cuda_getCurrentRawStream
        self.grad_enabled = torch.is_grad_enabled


def _here(device, stream) -> bool:
    """Whether a call's device and stream are the current ones (else :func:`_there`)."""
    global _t
    if _t is None:
        _t = _Torch()
    if stream is None and device.index is not None and device.index == _t.current_device():
        return True
    if device.type != "cuda":
        raise ValueError("attention takes tensors on a GPU, got %s" % device)
    if stream is not None and stream.device != device:
        raise ValueError("the stream is on %s, the tensors are on %s" % (stream.device, device))
    return False


def _there(device, stream, call, *args, **more):
    """A call made with the tensors' device and `stream` current: what it takes from the allocator then belongs to the
    stream its kernels run on, and is handed out again only behind them; so are the caller's tensors, of whatever stream."""
    with _t.device(device):
        if stream is None:
            return call(*args, **more)
        with _t.stream(stream):
            result = call(*args, **more)
        for x in args:
            for y in x if isinstance(x, tuple) else (x,):
                if isinstance(y, _t.Tensor):
                    y.record_stream(stream)
        return result


def _no_gradient():
    """The attention calls have no backward pass: what they return carries no graph."""
    return ValueError("the attention calls have no gradient: pass detached tensors or call them under torch.no_grad()")


def _rows(t, name, shape, dtype, device):
    """A [T, heads, head_dim] tensor of the call as packed rows."""
    if t.shape != shape or t.dtype is not dtype or t.device != device:
        raise ValueError("%s must be %s %s on %s, got %s %s on %s" % (
            name, list(shape), dtype, device, list(t.shape), t.dtype, t.device))
    token, head, one = t.stride()
    if one != 1:
        raise ValueError("%s: the elements of a head must be contiguous" % name)
    T, heads, d = shape
    # the stride of a dimension of one entry means nothing: any valid one will do
    return Rows(t.data_ptr(), token if T > 1 else heads * d, head if heads > 1 else d)


def _attn_heads(dtype, shape, hkv) -> Heads:
    kind = _t.types.get(dtype)
    if kind is None:
        raise ValueError("attention takes bfloat16 or float16, got %s" % dtype)
    return Heads(kind, shape[1], hkv, shape[2])


def _three(t, name):
    shape = t.shape
    if len(shape) != 3:
        raise ValueError("%s must be [tokens, heads, head_dim], got %s" % (name, list(shape)))
    return shape


def _attn_seqs(off, kv_len, pages, T, device) -> Seqs:
    int32 = _t.int32
    if off.dtype is not int32 or off.device != device or off.dim() != 1 or off.stride(0) != 1 or off.shape[0] < 1:
        raise ValueError("off must be a contiguous int32 tensor of B + 1 elements on %s" % device)
    B = off.shape[0] - 1
    if pages is None:
        return Seqs(B, 0, T, 0, off.data_ptr(), None, None)
    n, width = pages.shape if pages.dim() == 2 else (-1, 0)
    if n != B or kv_len.shape != (B,):
        raise ValueError("kv_len must be [%d] and pages [%d, max_pages], got %s and %s" % (
            B, B, list(kv_len.shape), list(pages.shape)))
    if kv_len.dtype is not int32 or pages.dtype is not int32 or kv_len.device != device or pages.device != device:
        raise ValueError("kv_len and pages must be int32 on %s" % device)
    row, one = pages.stride()
    if (one != 1 and width > 1) or (B > 1 and kv_len.stride(0) != 1):
        raise ValueError("kv_len, and each row of pages, must be contiguous")
    return Seqs(B, width, T, row if B > 1 else width, off.data_ptr(), kv_len.data_ptr(), pages.data_ptr())


def _attn_cache(k_cache, v_cache, heads, head_dim, dtype, device) -> KvCache:
    shape, strides = k_cache.shape, k_cache.stride()
    if len(shape) != 4 or shape[1] != heads or shape[3] != head_dim or v_cache.shape != shape or v_cache.stride() != strides:
        raise ValueError("k_cache and v_cache must be [pages, %d, page_size, %d] with the same strides, got %s and %s" % (
            heads, head_dim, list(shape), list(v_cache.shape)))
    if k_cache.dtype is not dtype or v_cache.dtype is not dtype or k_cache.device != device or v_cache.device != device:
        raise ValueError("k_cache and v_cache must be %s on %s" % (dtype, device))
    page, head, token, one = strides
    if one != 1:
        raise ValueError("the elements of a cached head must be contiguous")
    n, _, size, _ = shape
    return KvCache(k_cache.data_ptr(), v_cache.data_ptr(), page if n > 1 else heads * size * head_dim,
                   head if heads > 1 else size * head_dim, token if size > 1 else head_dim, n, size)


def _attn_status(status, B, device):
    if status is None:
        return None
    if status.dtype is not _t.int32 or status.device != device or not status.is_contiguous() or status.numel() < B:
        raise ValueError("status must be a contiguous int32 tensor of B elements on %s" % device)
    return status.data_ptr()


def fate_kv_append(q, k, v, k_cache, v_cache, off, kv_len, pages, table=None, interleaved: bool = False, q_out=None,
                   status=None, stream=None):
    """Store new keys, rotated to their positions, and values in a paged cache
    and rotate the queries.

    q [T, heads_q, head_dim] or None; k, v [T, heads_kv, head_dim] (bfloat16 or
    float16; any token and head strides that are multiples of 8); k_cache,
    v_cache [pages, heads_kv, page_size, head_dim]; off [B + 1], kv_len [B] and
    pages [B, max_pages] int32: sequence b has rows off[b] .. off[b + 1] and,
    these included, kv_len[b] keys.  table [positions, rot] float32 (see
    :func:`rotation_table`): cosines, then sines of the first rot dimensions,
    paired (j, j + rot / 2) or, interleaved, (2 j, 2 j + 1); None leaves all
    unrotated.  Returns q_out (None without q), which may be q itself.
    ``status`` (int32 [B], cleared by the caller) receives FATE_EINVAL for
    sequences whose device arrays are out of range.

    The attention calls have no backward pass: with gradients enabled, tensors
    that require one are refused (ValueError)."""
    dev, dtype = k.device, k.dtype
    if not _here(dev, stream):
        return _there(dev, stream, fate_kv_append, q, k, v, k_cache, v_cache, off, kv_len, pages, table, interleaved,
                      q_out, status)
    if _t.grad_enabled() and (k.requires_grad or v.requires_grad or k_cache.requires_grad or v_cache.requires_grad or
                              (q is not None and q.requires_grad) or (table is not None and table.requires_grad) or
                              (q_out is not None and q_out.requires_grad)):
        raise _no_gradient()
    return _append(q, k, v, k_cache, v_cache, off, kv_len, pages, table, None, interleaved, q_out, status)


def _append(q, k, v, k_cache, v_cache, off, kv_len, pages, table, axes, interleaved, q_out, status):
    """The call itself, on the current device and stream; axes: :class:`Axes` or None."""
    dev, dtype = k.device, k.dtype
    shape = _three(k, "k")
    T, hkv, d = shape
    c = _attn_cache(k_cache, v_cache, hkv, d, dtype, dev)
    s = _attn_seqs(off, kv_len, pages, T, dev)
    rk, rv = _rows(k, "k", shape, dtype, dev), _rows(v, "v", shape, dtype, dev)
    rq = ro = turns = None
    rot = positions = 0
    if table is not None:
        if table.dtype is not _t.float32 or table.dim() != 2 or table.device != dev or not table.is_contiguous():
            raise ValueError("table must be a contiguous float32 [positions, rot] tensor on %s" % dev)
        positions, rot = table.shape
        turns = table.data_ptr()
    if q is not None:
        shape = _three(q, "q")
        if shape[0] != T or shape[2] != d:
            raise ValueError("q must be [%d, heads_q, %d], got %s" % (T, d, list(shape)))
        rq = _rows(q, "q", shape, dtype, dev)
        if q_out is None:
            q_out = _t.empty_like(q)
        ro = _rows(q_out, "q_out", shape, dtype, dev)
    elif q_out is not None:
        raise ValueError("q_out without q")
    heads, state, stream = _attn_heads(dtype, shape, hkv), _attn_status(status, s.B, dev), _t.raw_stream(dev.index)
    if axes is None:
        st = load().fate_kv_append(heads, s, rq, rk, rv, turns, positions, rot, 1 if interleaved else 0, c, ro, state, stream)
    else:
        st = load().fate_kv_append_axes(heads, s, rq, rk, rv, turns, positions, rot, 1 if interleaved else 0, axes, c, ro,
                                        state, stream)
    if st != FATE_OK:
        raise FateError(st, "fate_kv_append" if axes is None else "fate_kv_append_axes")
    return q_out


def fate_kv_append_axes(q, k, v, k_cache, v_cache, off, kv_len, pages, table, positions, axis, interleaved: bool = False,
                        q_out=None, status=None, stream=None):
    """:func:`fate_kv_append` for tokens with positions on several axes, as the
    patches of images and videos have (time, height, width): pair j is rotated
    by the table's row of the token's position on axis axis[j].

    positions [axes, T] int32 on the device (each axis contiguous), up to four
    axes; axis: a tuple of rot / 2 axis numbers (see :func:`rotation_axes`).  A
    token's place in the cache follows from kv_len as before.  A position
    outside the table is an error of its sequence."""
    dev = k.device
    if not _here(dev, stream):
        return _there(dev, stream, fate_kv_append_axes, q, k, v, k_cache, v_cache, off, kv_len, pages, table, positions, axis,
                      interleaved, q_out, status)
    if _t.grad_enabled() and (k.requires_grad or v.requires_grad or k_cache.requires_grad or v_cache.requires_grad or
                              (q is not None and q.requires_grad) or table.requires_grad or
                              (q_out is not None and q_out.requires_grad)):
        raise _no_gradient()
    T = k.shape[0]
    if positions.dtype is not _t.int32 or positions.device != dev or positions.dim() != 2 or positions.shape[1] != T:
        raise ValueError("positions must be int32 [axes, %d] on %s, got %s %s on %s" % (
            T, dev, positions.dtype, list(positions.shape), positions.device))
    row, one = positions.stride()
    if one != 1 and T > 1:
        raise ValueError("each axis of positions must be contiguous")
    if 2 * len(axis) != table.shape[-1]:
        raise ValueError("axis must name one for each of the table's %d pairs, got %d" % (table.shape[-1] // 2, len(axis)))
    of_pairs = _pair_axis(tuple(axis))
    return _append(q, k, v, k_cache, v_cache, off, kv_len, pages, table,
                   Axes(positions.shape[0], C.addressof(of_pairs), positions.data_ptr(), row), interleaved, q_out, status)


@functools.lru_cache(maxsize=256)
def _pair_axis(axis):
    if not all(0 <= a < 256 for a in axis):
        raise ValueError("axes are numbered from 0, got %s" % (axis,))
    return (C.c_uint8 * max(1, len(axis)))(*axis)


def rotation_axes(sections, cyclic: bool = False):
    """Axes of the pairs for :func:`fate_kv_append_axes` from the number of
    pairs that each axis has: one section behind the other, or, cyclic, one
    pair of each in turn while it has any left."""
    if not cyclic:
        return tuple(a for a, n in enumerate(sections) for _ in range(n))
    return tuple(a for i in range(max(sections, default=0)) for a, n in enumerate(sections) if i < n)


def fate_attn_paged(q, k_cache, v_cache, off, kv_len, pages, max_new: Optional[int] = None, scale: Optional[float] = None,
                    lse: bool = False, out=None, status=None, ws=None, stream=None):
    """Causal attention of new tokens q [T, heads_q, head_dim] over their
    sequences' keys and values in a paged cache (append first); arguments as
    for :func:`fate_kv_append`.  ``max_new`` bounds the tokens per sequence
    (default T): a small bound picks the kernels for few tokens.  ``scale``
    defaults to 1 / sqrt(head_dim).  Returns (out, lse): lse [T, heads_q]
    float32 if asked for, else None.  ``ws`` (uint8, as large as
    :func:`fate_attn_paged_ws_size` says) is taken from the allocator if not
    given."""
    dev, dtype = q.device, q.dtype
    if not _here(dev, stream):
        return _there(dev, stream, fate_attn_paged, q, k_cache, v_cache, off, kv_len, pages, max_new, scale, lse, out,
                      status, ws)
    if _t.grad_enabled() and (q.requires_grad or k_cache.requires_grad or v_cache.requires_grad or
                              (out is not None and out.requires_grad)):
        raise _no_gradient()
    return _paged(q, k_cache, v_cache, off, kv_len, pages, max_new, scale, None, lse, out, status, ws)


def _paged(q, k_cache, v_cache, off, kv_len, pages, max_new, scale, shaping, lse, out, status, ws):
    """The call itself, on the current device and stream; shaping: cap, slopes, prefix and start, or None."""
    dev, dtype = q.device, q.dtype
    shape = _three(q, "q")
    T, hq, d = shape
    hkv = k_cache.shape[1] if k_cache.dim() == 4 else 0
    h = _attn_heads(dtype, shape, hkv)
    c = _attn_cache(k_cache, v_cache, hkv, d, dtype, dev)
    s = _attn_seqs(off, kv_len, pages, T, dev)
    most = T if max_new is None or max_new > T else int(max_new)
    rq = _rows(q, "q", shape, dtype, dev)
    if out is None:
        out = _t.empty_like(q)
    ro = _rows(out, "out", shape, dtype, dev)
    sums = _t.empty((T, hq), dtype=_t.float32, device=dev) if lse else None
    if ws is None:
        ws = _t.empty(_ws_bytes(h.dtype, hq, hkv, d, most), dtype=_t.uint8, device=dev)
    elif ws.device != dev or not ws.is_contiguous():
        raise ValueError("ws must be contiguous, on %s" % dev)
    scale = 1.0 / math.sqrt(d or 1) if scale is None else scale
    rest = (ro, sums.data_ptr() if lse else None, _attn_status(status, s.B, dev), ws.data_ptr(), ws.nbytes,
            _t.raw_stream(dev.index))
    if shaping is None:
        st = load().fate_attn_paged(h, s, rq, c, most, scale, *rest)
    else:
        st = load().fate_attn_paged_shaped(h, s, rq, c, most, scale, _scores(*shaping, hq, s.B, T, dev), *rest)
    if st != FATE_OK:
        raise FateError(st, "fate_attn_paged" if shaping is None else "fate_attn_paged_shaped")
    return out, sums


def _scores(cap, slopes, prefix, start, heads, B, T, device) -> Scores:
    def of(t, name, n, dtype):
        if t is None:
            return None
        if t.dtype is not dtype or t.device != device or t.shape != (n,) or (n > 1 and t.stride(0) != 1):
            raise ValueError("%s must be a contiguous %s tensor of %d elements on %s, got %s %s on %s" % (
                name, dtype, n, device, t.dtype, list(t.shape), t.device))
        return t.data_ptr()

    return Scores(cap, of(slopes, "slopes", heads, _t.float32), of(prefix, "prefix", B, _t.int32), of(start, "start", T, _t.int32))


def fate_attn_paged_shaped(q, k_cache, v_cache, off, kv_len, pages, max_new: Optional[int] = None,
                           scale: Optional[float] = None, cap: float = 0.0, slopes=None, prefix=None, start=None,
                           lse: bool = False, out=None, status=None, ws=None, stream=None):
    """:func:`fate_attn_paged` with shaped scores.  With s = scale q.k of the
    row at position p and the key at position j: s becomes cap tanh(s / cap)
    where cap is not 0, less slopes[head] |p - j| (float32 [heads_q]); the row
    sees j < prefix[b] (int32 [B]: a prefix that every row of the sequence sees)
    and start[t] <= j <= p (int32 [T], not falling within a sequence: the first
    key of the row's document, or p - w + 1 for a window of w keys)."""
    dev = q.device
    if not _here(dev, stream):
        return _there(dev, stream, fate_attn_paged_shaped, q, k_cache, v_cache, off, kv_len, pages, max_new, scale, cap, slopes,
                      prefix, start, lse, out, status, ws)
    if _t.grad_enabled() and (q.requires_grad or k_cache.requires_grad or v_cache.requires_grad or
                              (slopes is not None and slopes.requires_grad) or (out is not None and out.requires_grad)):
        raise _no_gradient()
    return _paged(q, k_cache, v_cache, off, kv_len, pages, max_new, scale, (cap, slopes, prefix, start), lse, out, status, ws)


@functools.lru_cache(maxsize=1024)
def _ws_bytes(dtype: int, heads_q: int, heads_kv: int, head_dim: int, max_new: int) -> int:
    """The library's workspace size, which depends on these alone (a call that is empty needs none)."""
    nbytes = C.c_size_t(0)
    st = load().fate_attn_paged_ws_size(Heads(dtype, heads_q, heads_kv, head_dim), Seqs(1, 0, max(1, max_new)),
                                        KvCache(page_size=1), max_new, nbytes)
    if st != FATE_OK:
        raise FateError(st, "fate_attn_paged_ws_size")
    return nbytes.value


def fate_attn_paged_ws_size(T: int, heads_q: int, k_cache, B: int, max_pages: int, max_new: int) -> int:
    """Workspace bytes of :func:`fate_attn_paged` for a call of these sizes."""
    if k_cache.dim() != 4:
        raise ValueError("k_cache must be [pages, heads_kv, page_size, head_dim]")
    hkv, d = k_cache.shape[1], k_cache.shape[3]
    _here(k_cache.device, None)
    if T == 0 or B == 0:
        return 0
    if max_new > T:
        raise ValueError("max_new is at most T")
    return _ws_bytes(_attn_heads(k_cache.dtype, (T, heads_q, d), hkv).dtype, heads_q, hkv, d, max_new)


def fate_attn_prompt(q, k, v, off, scale: Optional[float] = None, lse: bool = False, out=None, status=None,
                     stream=None):
    """Causal attention of whole prompts, packed: q [T, heads_q, head_dim]
    over k, v [T, heads_kv, head_dim] (views of one projection will do),
    sequence b in rows off[b] .. off[b + 1].  Returns (out, lse) as
    :func:`fate_attn_paged`."""
    dev, dtype = q.device, q.dtype
    if not _here(dev, stream):
        return _there(dev, stream, fate_attn_prompt, q, k, v, off, scale, lse, out, status)
    if _t.grad_enabled() and (q.requires_grad or k.requires_grad or v.requires_grad or
                              (out is not None and out.requires_grad)):
        raise _no_gradient()
    return _prompt(q, k, v, off, scale, None, lse, out, status)


def _prompt(q, k, v, off, scale, shaping, lse, out, status):
    """The call itself, on the current device and stream; shaping as for :func:`_paged`."""
    dev, dtype = q.device, q.dtype
    shape, kv_shape = _three(q, "q"), _three(k, "k")
    T, hq, d = shape
    if kv_shape[0] != T or kv_shape[2] != d:
        raise ValueError("k must be [%d, heads_kv, %d], got %s" % (T, d, list(kv_shape)))
    h = _attn_heads(dtype, shape, kv_shape[1])
    s = _attn_seqs(off, None, None, T, dev)
    rq = _rows(q, "q", shape, dtype, dev)
    rk, rv = _rows(k, "k", kv_shape, dtype, dev), _rows(v, "v", kv_shape, dtype, dev)
    if out is None:
        out = _t.empty_like(q)
    ro = _rows(out, "out", shape, dtype, dev)
    sums = _t.empty((T, hq), dtype=_t.float32, device=dev) if lse else None
    scale = 1.0 / math.sqrt(d or 1) if scale is None else scale
    rest = (ro, sums.data_ptr() if lse else None, _attn_status(status, s.B, dev), _t.raw_stream(dev.index))
    if shaping is None:
        st = load().fate_attn_prompt(h, s, rq, rk, rv, scale, *rest)
    else:
        st = load().fate_attn_prompt_shaped(h, s, rq, rk, rv, scale, _scores(*shaping, hq, s.B, T, dev), *rest)
    if st != FATE_OK:
        raise FateError(st, "fate_attn_prompt" if shaping is None else "fate_attn_prompt_shaped")
    return out, sums


def fate_attn_prompt_shaped(q, k, v, off, scale: Optional[float] = None, cap: float = 0.0, slopes=None, prefix=None,
                            start=None, lse: bool = False, out=None, status=None, stream=None):
    """:func:`fate_attn_prompt` with scores shaped as in
    :func:`fate_attn_paged_shaped`."""
    dev = q.device
    if not _here(dev, stream):
        return _there(dev, stream, fate_attn_prompt_shaped, q, k, v, off, scale, cap, slopes, prefix, start, lse, out, status)
    if _t.grad_enabled() and (q.requires_grad or k.requires_grad or v.requires_grad or
                              (slopes is not None and slopes.requires_grad) or (out is not None and out.requires_grad)):
        raise _no_gradient()
    return _prompt(q, k, v, off, scale, (cap, slopes, prefix, start), lse, out, status)


class Reserved(NamedTuple):
    """What :func:`fate_kv_reserve` returns, or writes to: off [B + 1], kv_len [B], n_free [1], taken [B + 1], slots [T]
    int64, positions [T]; the others int32."""

    off: object
    kv_len: object
    n_free: object
    taken: object
    slots: object
    positions: object


class Trimmed(NamedTuple):
    """What :func:`fate_kv_trim` returns, or writes to: kv_len [B], n_free [1], given [B + 1], int32."""

    kv_len: object
    n_free: object
    given: object


def _array(t, name, n, dtype, device):
    """A contiguous tensor of n numbers."""
    if t.dtype is not dtype or t.device != device or t.shape != (n,) or (n > 1 and t.stride(0) != 1):
        raise ValueError("%s must be a contiguous %s tensor of %d elements on %s, got %s %s on %s" % (
            name, dtype, n, device, t.dtype, list(t.shape), t.device))
    return t.data_ptr()


def _kv_tables(counts, name, kv_len, pages, free, n_free, page_size, device) -> KvTables:
    int32 = _t.int32
    if kv_len.dim() != 1 or pages.dim() != 2 or pages.shape[0] != kv_len.shape[0] or free.dim() != 1:
        raise ValueError("kv_len must be [B], pages [B, max_pages] and free [n_pages], got %s, %s and %s" % (
            list(kv_len.shape), list(pages.shape), list(free.shape)))
    B, width = pages.shape
    row, one = pages.stride()
    if pages.dtype is not int32 or pages.device != device or (one != 1 and width > 1):
        raise ValueError("pages must be int32 on %s, each row contiguous" % device)
    if not -(1 << 31) <= page_size < 1 << 31:  # (the field would take its low bits)
        raise ValueError("page_size must be a 32-bit number, got %d" % page_size)
    for t, its, n in ((counts, name, B), (kv_len, "kv_len", B), (free, "free", free.shape[0]), (n_free, "n_free", 1)):
        if t.dtype is not int32 or t.device != device or t.shape != (n,) or not t.is_contiguous():
            _array(t, its, n, int32, device)  # says what is wrong
    return KvTables(B, width, page_size, free.shape[0], row if B > 1 else width, pages.data_ptr(), free.data_ptr(), n_free.data_ptr(),
                    kv_len.data_ptr())


def fate_kv_reserve(new, kv_len, pages, free, n_free, page_size: int, T: int, out: Optional[Reserved] = None, status=None,
                    stream=None) -> Reserved:
    """Room for new[b] tokens behind each sequence's keys: pages off the stack
    free[:n_free], entered in ``pages``, and the arrays of the calls that follow.

    new, kv_len [B], pages [B, max_pages], free [n_pages] and n_free [1] int32 on
    the device; T, the rows of the call, is at least the sum of new.  Returns
    :class:`Reserved`: off and kv_len (the new tokens among them) as
    :func:`fate_kv_append` and the attention calls take them, what is left on
    the stack, the pages taken before each sequence, and each row's slot
    (page * page_size + place) and position, -1 behind the last row.  ``out``
    names tensors to write to; its kv_len and n_free may be the call's own, its
    slots and positions None.  ``status`` (int32 [B], cleared by the caller)
    receives FATE_ESIZE for sequences that found too few pages or rows, which
    get nothing, FATE_EINVAL for those in error."""
    dev = pages.device
    if not _here(dev, stream):
        return _there(dev, stream, fate_kv_reserve, new, kv_len, pages, free, n_free, page_size, T, out, status)
    int32, int64 = _t.int32, _t.int64
    t = _kv_tables(new, "new", kv_len, pages, free, n_free, page_size, dev)
    B = t.B
    if not 0 <= T < 1 << 63:
        raise ValueError("T must not be negative or past 64 bits, got %d" % T)
    if out is None:
        n, slots = _t.empty(3 * B + 3 + T, dtype=int32, device=dev), _t.empty(T, dtype=int64, device=dev)
        # (whole numbers: no gradient has to follow the views)
        off, kv, left, taken, positions = n.unsafe_split_with_sizes((B + 1, B, 1, B + 1, T))
        out = Reserved(off, kv, left, taken, slots, positions)
        at = n.data_ptr()
        where = (at, at + 4 * B + 4, at + 8 * B + 4, at + 8 * B + 8, slots.data_ptr(), at + 12 * B + 12)
    else:
        where = (_array(out.off, "out.off", B + 1, int32, dev), _array(out.kv_len, "out.kv_len", B, int32, dev),
                 _array(out.n_free, "out.n_free", 1, int32, dev), _array(out.taken, "out.taken", B + 1, int32, dev),
                 None if out.slots is None else _array(out.slots, "out.slots", T, int64, dev),
                 None if out.positions is None else _array(out.positions, "out.positions", T, int32, dev))
    st = load().fate_kv_reserve(t, new.data_ptr(), T, *where, _attn_status(status, B, dev), _t.raw_stream(dev.index))
    if st != FATE_OK:
        raise FateError(st, "fate_kv_reserve")
    return out


def fate_kv_trim(keep, kv_len, pages, free, n_free, page_size: int, out: Optional[Trimmed] = None, status=None,
                 stream=None) -> Trimmed:
    """Cut each sequence to its first keep[b] keys: pages that hold none of
    these go back on the stack ``free``, which is written behind n_free;
    ``pages`` is only read.  Arguments as for :func:`fate_kv_reserve`."""
    dev = pages.device
    if not _here(dev, stream):
        return _there(dev, stream, fate_kv_trim, keep, kv_len, pages, free, n_free, page_size, out, status)
    int32 = _t.int32
    t = _kv_tables(keep, "keep", kv_len, pages, free, n_free, page_size, dev)
    B = t.B
    if out is None:
        n = _t.empty(2 * B + 2, dtype=int32, device=dev)
        out, at = Trimmed(*n.unsafe_split_with_sizes((B, 1, B + 1))), n.data_ptr()
        where = (at, at + 4 * B, at + 4 * B + 4)
    else:
        where = (_array(out.kv_len, "out.kv_len", B, int32, dev), _array(out.n_free, "out.n_free", 1, int32, dev),
                 _array(out.given, "out.given", B + 1, int32, dev))
    st = load().fate_kv_trim(t, keep.data_ptr(), *where, _attn_status(status, B, dev), _t.raw_stream(dev.index))
    if st != FATE_OK:
        raise FateError(st, "fate_kv_trim")
    return out


def fate_sample(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, logprob: bool = False, out=None, status=None,
                ws=None, stream=None):
    """One token of each row of logits [rows, vocab] (bfloat16, float16 or
    float32, each row contiguous) from random numbers u [rows] in [0, 1).

    temperature, top_k, top_p and min_p are numbers, or tensors [rows] (top_k
    int32, the others float32): temperature 0 takes the largest logit (the lowest
    index of equal ones), top_k 0, top_p 1 and min_p 0 cut nothing.  Of the tokens
    by falling logit the first top_k are kept, of these those before which less
    than top_p of their sum lies, of these those whose weight is at least min_p
    times the largest.  The token is the lowest index at which the kept weights
    sum to more than u of their whole.  Returns (token, logprob): int32 [rows], and
    the logarithm of the token's share of what is kept, float32, if asked for,
    else None.  Rows with nothing to take get -1.  ``out`` and ``ws`` (uint8, as
    large as :func:`fate_sample_ws_size` says) are made if not given; ``status``
    (int32 [rows], cleared by the caller) receives FATE_EINVAL for rows whose
    settings or u are out of range.  There is no gradient."""
    dev = logits.device
    if not _here(dev, stream):
        return _there(dev, stream, fate_sample, logits, u, temperature, top_k, top_p, min_p, logprob, out, status, ws)
    if _t.grad_enabled() and logits.requires_grad:
        raise ValueError("sampling has no gradient: pass detached logits or call it under torch.no_grad()")
    s = _sampling(logits, dev)
    R = s.rows
    f32, i32 = _t.float32, _t.int32
    s.u = _array(u, "u", R, f32, dev)
    for name, value, dtype in (("temperature", temperature, f32), ("top_k", top_k, i32), ("top_p", top_p, f32), ("min_p", min_p, f32)):
        if isinstance(value, _t.Tensor):
            setattr(s, name, _array(value, name, R, dtype, dev))
        else:
            if name == "top_k":  # the field would take a larger number by its low bits; no row has so many tokens
                value = max(-1, min(value, 0x7fffffff))
            setattr(s, name + "_all", value)
    if out is None:
        out = _t.empty(R, dtype=i32, device=dev)
    shares = _t.empty(R, dtype=f32, device=dev) if logprob else None
    need = _sample_ws(s.dtype, R, s.vocab)
    if ws is None:
        ws = _t.empty(need, dtype=_t.uint8, device=dev) if need else None
    elif ws.device != dev or not ws.is_contiguous():
        raise ValueError("ws must be contiguous, on %s" % dev)
    st = load().fate_sample(s, _array(out, "out", R, i32, dev), shares.data_ptr() if logprob else None,
                            _attn_status(status, R, dev), None if ws is None else ws.data_ptr(), 0 if ws is None else ws.nbytes,
                            _t.raw_stream(dev.index))
    if st != FATE_OK:
        raise FateError(st, "fate_sample")
    return out, shares


def _sampling(logits, dev) -> Sampling:
    kind = _t.logit_types.get(logits.dtype)
    if kind is None or logits.dim() != 2:
        raise ValueError("logits must be bfloat16, float16 or float32 [rows, vocab], got %s %s" % (logits.dtype, list(logits.shape)))
    R, V = logits.shape
    row, one = logits.stride()
    if one != 1 and V > 1:
        raise ValueError("each row of logits must be contiguous")
    return Sampling(kind, R, V, row if R > 1 else V, logits.data_ptr(), temperature_all=1.0, top_p_all=1.0)


@functools.lru_cache(maxsize=1024)
def _sample_ws(dtype: int, rows: int, vocab: int) -> int:
    """The library's workspace size, which depends on these alone."""
    nbytes = C.c_size_t(0)
    st = load().fate_sample_ws_size(Sampling(dtype, rows, vocab, temperature_all=1.0, top_p_all=1.0), nbytes)
    if st != FATE_OK:
        raise FateError(st, "fate_sample_ws_size")
    return nbytes.value


def fate_sample_ws_size(logits) -> int:
    """Workspace bytes of :func:`fate_sample` for logits of this type and shape."""
    _here(logits.device, None)
    s = _sampling(logits, logits.device)
    return _sample_ws(s.dtype, s.rows, s.vocab)


def rotation_table(positions: int, rot: int, base: float = 10000.0, device="cuda"):
    """Cosines and sines for :func:`fate_kv_append`: float32 [positions, rot],
    angle p * base ** (-j / (rot / 2)) of pair j, computed in float64."""
    import torch
    half = rot // 2
    angle = torch.outer(torch.arange(positions, dtype=torch.float64),
                        base ** (-torch.arange(half, dtype=torch.float64) / max(1, half)))
    return torch.cat([angle.cos(), angle.sin()], 1).float().to(device)
