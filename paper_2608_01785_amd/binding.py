"""ctypes binding of ``libhorizon.so``: argument marshalling only.

Every function here has the name of the C entry point it calls and only
converts arguments (torch tensors -> device pointers, Python sequences ->
host arrays, status codes -> exceptions).  All computation happens in the
library's HIP kernels.  Importing this module fails loudly when the library
has not been built.
"""
from __future__ import annotations

import array
import ctypes
import os
from typing import Dict, List, Optional, Sequence, Tuple

import numpy as np

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libhorizon.so")

HS_OK, HS_ERR_INVALID_ARG, HS_ERR_UNSUPPORTED, HS_ERR_BUDGET, HS_ERR_WORKSPACE, HS_ERR_HIP, HS_ERR_INTERNAL = range(7)
HS_ROLE_SHARED, HS_ROLE_DOWN = 0, 1

SYMBOLS = (
    "hs_status_string", "hs_last_error", "hs_default_topology", "hs_cu_partition", "hs_plan_metadata",
    "hs_context_create", "hs_context_topology", "hs_context_stream", "hs_context_masks",
    "hs_context_destroy", "hs_workspace_size", "hs_workspace_size_paged", "hs_shared_stage_forward",
    "hs_shared_stage_forward_mrope", "hs_downstream_decode_step_mrope", "hs_downstream_decode_step",
    "hs_downstream_decode_step_noalloc", "hs_decode_graph_create", "hs_decode_graph_launch",
    "hs_decode_graph_destroy", "hs_dit_workspace_size", "hs_dit_forward",
    "hs_probe_hw_ids", "hs_timing_enable", "hs_timing_read", "hs_timing_read_clock", "hs_convert_weights_f16",
    "hs_controller_create", "hs_controller_step", "hs_controller_destroy", "hs_pressure_sample",
    "hs_temporal_create", "hs_temporal_step", "hs_temporal_destroy",
    "hs_quantize_rows", "hs_linear_i8", "hs_logprobs_workspace_size", "hs_logprobs",
    "hs_beam_select_workspace_size", "hs_beam_select", "hs_cache_copy", "hs_prefix_attention_workspace_size",
    "hs_prefix_attention", "hs_workspace_size_prefix", "hs_downstream_decode_step_prefix", "hs_pages_create", "hs_pages_destroy", "hs_pages_reserve", "hs_pages_fork",
    "hs_pages_compact", "hs_pages_table", "hs_pages_shared", "hs_pages_free_count",
)
HS_WEIGHTS_BF16, HS_WEIGHTS_F16 = 0, 1
HS_TYPE_F32, HS_TYPE_BF16, HS_TYPE_F16 = 0, 1, 2

KERNEL_KINDS = {"rmsnorm": 0, "qkv": 1, "attention": 2, "decode_attn": 3, "o_proj": 4, "gate_up": 5,
                "down": 6, "rope_table": 7, "modulation": 8, "ln_mod": 9, "mlp_up": 10, "mlp_down": 11,
                "quantize": 12, "linear_i8": 13, "logprobs": 14, "beam_select": 15, "cache_copy": 16,
                "prefix_attn": 17}


class LayerCfg(ctypes.Structure):
    _fields_ = [("hidden", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("ffn", ctypes.c_int32), ("rms_eps", ctypes.c_float),
                ("rope_base", ctypes.c_float), ("mrope_sections", ctypes.c_int32 * 3)]

    @classmethod
    def of(cls, s) -> "LayerCfg":
        sec = tuple(getattr(s, "mrope_sections", (0, 0, 0)))
        return cls(s.hidden, s.n_q_heads, s.n_kv_heads, s.head_dim, s.ffn, s.rms_eps, s.rope_base,
                   (ctypes.c_int32 * 3)(*sec))


MATRICES = ("w_qkv", "w_o", "w_gate_up", "w_down")
DIT_MATRICES = ("w_qkv", "w_o", "w_fc1", "w_fc2")   # the DiT projections fp16 preparation applies to
DIT_FIELDS = ("w_ada", "b_ada", "w_qkv", "b_qkv", "w_o", "b_o", "w_fc1", "b_fc1", "w_fc2", "b_fc2")


class DitCfg(ctypes.Structure):
    _fields_ = [("hidden", ctypes.c_int32), ("n_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("mlp", ctypes.c_int32), ("ln_eps", ctypes.c_float)]

    @classmethod
    def of(cls, s) -> "DitCfg":
        return cls(s.hidden, s.n_heads, s.head_dim, s.mlp, s.ln_eps)


class DitWeights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in DIT_FIELDS] + [("format", ctypes.c_int32)]


class LayerWeights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("ln1", "w_qkv", "w_o", "ln2", "w_gate_up", "w_down")] + \
               [("format", ctypes.c_int32), ("b_qkv", ctypes.c_void_p)]


class KvCache(ctypes.Structure):
    _fields_ = [("k", ctypes.POINTER(ctypes.c_void_p)), ("v", ctypes.POINTER(ctypes.c_void_p)),
                ("n_slots", ctypes.c_int32), ("max_ctx", ctypes.c_int32),
                ("block_table", ctypes.POINTER(ctypes.c_int32)), ("pages_per_seq", ctypes.c_int32)]


class Topology(ctypes.Structure):
    _fields_ = [("n_cus", ctypes.c_int32), ("n_xcc", ctypes.c_int32), ("xcc", ctypes.c_uint8 * 256),
                ("se", ctypes.c_uint8 * 256), ("cu", ctypes.c_uint8 * 256)]


class ControllerCfg(ctypes.Structure):
    _fields_ = [("total_cus", ctypes.c_int32), ("aggressive_cus", ctypes.c_int32),
                ("ladder", ctypes.POINTER(ctypes.c_int32)), ("n_ladder", ctypes.c_int32),
                ("ewma_weight", ctypes.c_double), ("saturation", ctypes.c_double),
                ("hysteresis_steps", ctypes.c_int32)]


HS_PATH_SHORT, HS_PATH_LONG = 0, 1
HS_WORK_PREFILL, HS_WORK_DECODE = 0, 1


class TemporalCfg(ctypes.Structure):
    _fields_ = [("n_min", ctypes.c_int32), ("n_max", ctypes.c_int32), ("m", ctypes.c_int32),
                ("u_guard", ctypes.c_double), ("long_cap", ctypes.c_int32)]


class RequestView(ctypes.Structure):
    _fields_ = [("path", ctypes.c_int32), ("work", ctypes.c_int32), ("deadline", ctypes.c_double),
                ("remaining", ctypes.c_double)]


class TemporalStepInfo(ctypes.Structure):
    _fields_ = [("step", ctypes.c_int64), ("n", ctypes.c_int32), ("phase", ctypes.c_int32),
                ("n_protected", ctypes.c_int32), ("n_hidden", ctypes.c_int32), ("n_capped", ctypes.c_int32)]


class Split(ctypes.Structure):
    _fields_ = [("shared_cus", ctypes.c_int32), ("down_cus", ctypes.c_int32), ("level", ctypes.c_int32),
                ("changed", ctypes.c_int32), ("pressure", ctypes.c_double), ("rho", ctypes.c_double)]


class HorizonError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{_status_name(status)}: {msg}")
        self.status = status


_lib = None


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise ImportError(f"{_LIB_PATH} is missing: build it with python -m paper_2608_01785_amd.build")
        L = ctypes.CDLL(_LIB_PATH)
        vp, i32, u32p, i32p = ctypes.c_void_p, ctypes.c_int32, ctypes.POINTER(ctypes.c_uint32), ctypes.POINTER(ctypes.c_int32)
        i64, f32 = ctypes.c_int64, ctypes.c_float
        L.hs_status_string.restype = ctypes.c_char_p
        L.hs_status_string.argtypes = [ctypes.c_int]
        L.hs_last_error.restype = ctypes.c_char_p
        L.hs_last_error.argtypes = []
        sigs = {
            "hs_default_topology": [i32, i32, ctypes.POINTER(Topology)],
            "hs_cu_partition": [ctypes.POINTER(Topology), i32, u32p, u32p],
            "hs_plan_metadata": [i32p, i32p, i32, i32p, i32p],
            "hs_context_create": [i32, i32p, i32, ctypes.POINTER(Topology), ctypes.POINTER(vp)],
            "hs_context_topology": [vp, ctypes.POINTER(Topology)],
            "hs_context_stream": [vp, i32, i32, ctypes.POINTER(vp)],
            "hs_context_masks": [vp, i32, u32p, u32p],
            "hs_context_destroy": [vp],
            "hs_workspace_size": [ctypes.POINTER(LayerCfg), i32, i32, i32, ctypes.POINTER(ctypes.c_size_t)],
            "hs_workspace_size_paged": [ctypes.POINTER(LayerCfg), i32, i32, i32, i32,
                                        ctypes.POINTER(ctypes.c_size_t)],
            "hs_shared_stage_forward": [vp, ctypes.POINTER(LayerCfg), ctypes.POINTER(LayerWeights), i32, vp, vp,
                                        i32p, i32p, i32, ctypes.POINTER(KvCache), i32, vp, vp, ctypes.c_size_t],
            "hs_shared_stage_forward_mrope": [vp, ctypes.POINTER(LayerCfg), ctypes.POINTER(LayerWeights), i32, vp,
                                              vp, i32p, i32p, i32, ctypes.POINTER(KvCache), i32p, i32, vp, vp,
                                              ctypes.c_size_t],
            "hs_downstream_decode_step_mrope": [vp, ctypes.POINTER(LayerCfg), ctypes.POINTER(LayerWeights), i32, vp,
                                                vp, ctypes.POINTER(KvCache), i32p, i32p, i32, i32, vp, vp,
                                                ctypes.c_size_t],
            "hs_downstream_decode_step": [vp, ctypes.POINTER(LayerCfg), ctypes.POINTER(LayerWeights), i32, vp, vp,
                                          ctypes.POINTER(KvCache), i32p, i32, i32, vp, vp, ctypes.c_size_t],
            "hs_downstream_decode_step_noalloc": [vp, ctypes.POINTER(LayerCfg), ctypes.POINTER(LayerWeights), i32,
                                                  vp, vp, ctypes.POINTER(KvCache), i32p, i32, i32, vp],
            "hs_decode_graph_create": [vp, ctypes.POINTER(LayerCfg), ctypes.POINTER(LayerWeights), i32, vp, vp,
                                       ctypes.POINTER(KvCache), i32, i32, vp, vp, ctypes.c_size_t,
                                       ctypes.POINTER(vp)],
            "hs_decode_graph_launch": [vp, i32p, i32p],
            "hs_dit_workspace_size": [ctypes.POINTER(DitCfg), i32, i32, ctypes.POINTER(ctypes.c_size_t)],
            "hs_dit_forward": [vp, ctypes.POINTER(DitCfg), ctypes.POINTER(DitWeights), i32, vp, vp, vp, i32p, i32,
                               i32, vp, vp, ctypes.c_size_t],
            "hs_decode_graph_destroy": [vp],
            "hs_probe_hw_ids": [vp, vp, i32, vp],
            "hs_timing_enable": [vp, i32],
            "hs_timing_read": [vp, i32, ctypes.POINTER(ctypes.c_double), i32p],
            "hs_timing_read_clock": [vp, i32, ctypes.POINTER(ctypes.c_double), i32p],
            "hs_convert_weights_f16": [vp, vp, vp, ctypes.c_int64, ctypes.c_int64, vp],
            "hs_controller_create": [ctypes.POINTER(ControllerCfg), ctypes.POINTER(vp)],
            "hs_controller_step": [vp, i32, ctypes.c_double, ctypes.POINTER(Split)],
            "hs_controller_destroy": [vp],
            "hs_pressure_sample": [i32, ctypes.POINTER(ctypes.c_double)],
            "hs_temporal_create": [ctypes.POINTER(TemporalCfg), ctypes.POINTER(vp)],
            "hs_temporal_step": [vp, ctypes.c_double, ctypes.POINTER(RequestView), i32,
                                 ctypes.POINTER(ctypes.c_uint8), ctypes.POINTER(TemporalStepInfo)],
            "hs_temporal_destroy": [vp],
            "hs_quantize_rows": [vp, vp, i32, i64, vp, f32, i32, i32, vp, i64, vp, i32, vp],
            "hs_linear_i8": [vp, vp, i64, vp, vp, i64, vp, vp, vp, i32, i64, i32, i32, i32, i32, vp],
            "hs_logprobs_workspace_size": [i32, i32, i32, ctypes.POINTER(ctypes.c_size_t)],
            "hs_logprobs": [vp, vp, i32, i64, i32, i32, vp, i32, vp, vp, i32, vp, vp, i32, vp, vp, ctypes.c_size_t],
            "hs_beam_select_workspace_size": [i32, i32, i32, i32, ctypes.POINTER(ctypes.c_size_t)],
            "hs_beam_select": [vp, vp, i32, i64, i32, i32, i32, vp, vp, i32, i32, vp, vp, vp, vp, i32, vp, vp,
                               ctypes.c_size_t],
            "hs_cache_copy": [vp, vp, i32, i32, i32, vp, vp, vp, i32, i32, vp],
            "hs_prefix_attention_workspace_size": [i32, i32, i32, i32, i32, i32, ctypes.POINTER(ctypes.c_size_t)],
            "hs_prefix_attention": [vp, vp, i32, i64, vp, i64, i32, i32, i32, vp, vp, i32, i32, vp, i32, vp, i32, vp,
                                    vp, i32, i32, i32, i32, vp, vp, ctypes.c_size_t],
            "hs_workspace_size_prefix": [ctypes.POINTER(LayerCfg), i32, i32, i32, i32, i32,
                                         ctypes.POINTER(ctypes.c_size_t)],
            "hs_downstream_decode_step_prefix": [vp, ctypes.POINTER(LayerCfg), ctypes.POINTER(LayerWeights), i32, vp,
                                                 vp, ctypes.POINTER(KvCache), i32p, i32, i32p, i32p, i32, i32, vp, vp,
                                                 ctypes.c_size_t],
            "hs_pages_create": [i32, i32, i32, i32, ctypes.POINTER(vp)],
            "hs_pages_destroy": [vp],
            "hs_pages_reserve": [vp, i32p, i32p, i32, i32p, i32p, i32p, i32p],
            "hs_pages_fork": [vp, i32p, i32p, i32],
            "hs_pages_compact": [vp, i32, i32p, i32p, i32p, i32p],
            "hs_pages_table": [vp, i32p, i32, i32p, i32p],
            "hs_pages_shared": [vp, i32p, i32, i32p],
            "hs_pages_free_count": [vp, i32p],
        }
        for name, args in sigs.items():
            fn = getattr(L, name)
            fn.restype = ctypes.c_int
            fn.argtypes = args
        _lib = L
    return _lib


def _status_name(s: int) -> str:
    try:
        return lib().hs_status_string(s).decode()
    except Exception:  # pragma: no cover - library missing
        return str(s)


def _check(status: int) -> None:
    if status != HS_OK:
        raise HorizonError(status, lib().hs_last_error().decode())


def hs_last_error() -> str:
    return lib().hs_last_error().decode()


def _as_i32(values, name: str = "a list") -> np.ndarray:
    """Host integers as a contiguous array of 32-bit words; others are refused, not cut to their lower bits."""
    if isinstance(values, (list, tuple)):
        try:
            return np.array(array.array("i", values), dtype=np.int32)
        except (OverflowError, TypeError):
            pass   # refused below, or a list of lists
    a = np.asarray(values)
    if a.dtype != np.int32 and a.size and (a.dtype.kind not in "iub" or a.min() < -2 ** 31 or a.max() > _INT32_MAX):
        raise ValueError(f"{name} holds no 32-bit numbers")
    return np.ascontiguousarray(a, dtype=np.int32)


def _i32_array(values) -> Optional[ctypes.Array]:
    if values is None:
        return None
    a = _as_i32(values)
    return (ctypes.c_int32 * len(a))(*a.tolist())


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


# --------------------------------------------------------------------------- host-only calls

def hs_default_topology(n_cus: int = 256, n_xcc: int = 8) -> Topology:
    t = Topology()
    _check(lib().hs_default_topology(n_cus, n_xcc, ctypes.byref(t)))
    return t


def topology_from_lists(xcc, se, cu, n_xcc: int) -> Topology:
    t = Topology()
    t.n_cus, t.n_xcc = len(xcc), n_xcc
    for i in range(len(xcc)):
        t.xcc[i], t.se[i], t.cu[i] = int(xcc[i]), int(se[i]), int(cu[i])
    return t


def hs_cu_partition(topo: Topology, shared_cus: int) -> Tuple[List[int], List[int]]:
    sh = (ctypes.c_uint32 * 8)()
    dn = (ctypes.c_uint32 * 8)()
    _check(lib().hs_cu_partition(ctypes.byref(topo), shared_cus, sh, dn))
    return list(sh), list(dn)


def hs_plan_metadata(seq_offsets, ctx_lens=None) -> Tuple[np.ndarray, np.ndarray]:
    off = _i32_array(seq_offsets)
    T = int(off[len(off) - 1]) if len(off) else 0
    pos = (ctypes.c_int32 * max(T, 1))()
    sid = (ctypes.c_int32 * max(T, 1))()
    _check(lib().hs_plan_metadata(off, _i32_array(ctx_lens), len(off) - 1, pos, sid))
    return np.frombuffer(pos, dtype=np.int32)[:T].copy(), np.frombuffer(sid, dtype=np.int32)[:T].copy()


def hs_workspace_size(cfg, max_tokens: int, max_seqs: int, max_pos: int) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().hs_workspace_size(ctypes.byref(LayerCfg.of(cfg)), max_tokens, max_seqs, max_pos, ctypes.byref(n)))
    return int(n.value)


def hs_workspace_size_paged(cfg, max_tokens: int, max_seqs: int, max_pos: int, page_positions: int) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().hs_workspace_size_paged(ctypes.byref(LayerCfg.of(cfg)), max_tokens, max_seqs, max_pos,
                                         page_positions, ctypes.byref(n)))
    return int(n.value)


# --------------------------------------------------------------------------- spatial controller

class Controller:
    """Owns an hs_controller handle (the C object copies the configuration)."""

    def __init__(self, total_cus: int, aggressive_cus: int, ladder: Sequence[int], ewma_weight: float,
                 saturation: float, hysteresis_steps: int = 1):
        self._ladder = _i32_array(ladder)
        cfg = ControllerCfg(total_cus, aggressive_cus, self._ladder, len(ladder), ewma_weight, saturation,
                            hysteresis_steps)
        h = ctypes.c_void_p()
        _check(lib().hs_controller_create(ctypes.byref(cfg), ctypes.byref(h)))
        self.handle = h

    def close(self):
        if self.handle:
            lib().hs_controller_destroy(self.handle)
            self.handle = None

    def __del__(self):  # pragma: no cover
        try:
            self.close()
        except Exception:
            pass


def hs_controller_step(ctrl: Controller, downstream_active: bool, sample: float) -> Split:
    out = Split()
    _check(lib().hs_controller_step(ctrl.handle, 1 if downstream_active else 0, float(sample), ctypes.byref(out)))
    return out


class Temporal:
    """Owns an hs_temporal handle (shared-stage path rotation)."""

    def __init__(self, n_min: int = 2, n_max: int = 8, m: int = 2, u_guard: float = 1.0, long_cap: int = -1):
        cfg = TemporalCfg(n_min, n_max, m, u_guard, long_cap)
        h = ctypes.c_void_p()
        _check(lib().hs_temporal_create(ctypes.byref(cfg), ctypes.byref(h)))
        self.handle = h

    def close(self):
        if self.handle:
            lib().hs_temporal_destroy(self.handle)
            self.handle = None

    def __del__(self):  # pragma: no cover
        try:
            self.close()
        except Exception:
            pass


def hs_temporal_step(sched: Temporal, now: float, requests) -> Tuple[np.ndarray, TemporalStepInfo]:
    """requests: sequence of (path, work, deadline, remaining); returns (visible bool array, step info)."""
    n = len(requests)
    arr = (RequestView * max(n, 1))(*[RequestView(int(p), int(w), float(d), float(r)) for p, w, d, r in requests])
    vis = np.zeros(max(n, 1), np.uint8)
    info = TemporalStepInfo()
    _check(lib().hs_temporal_step(sched.handle, float(now), arr, n, vis.ctypes.data_as(ctypes.POINTER(ctypes.c_uint8)),
                                  ctypes.byref(info)))
    return vis[:n].astype(bool), info


def hs_pressure_sample(device: int = 0) -> float:
    v = ctypes.c_double(0.0)
    _check(lib().hs_pressure_sample(device, ctypes.byref(v)))
    return float(v.value)


# --------------------------------------------------------------------------- context

class Context:
    """Owns an ``hs_context`` (CU-masked stream ladder)."""

    def __init__(self, device: int = 0, budgets: Sequence[int] = (64, 128, 192, 256),
                 topo: Optional[Topology] = None):
        h = ctypes.c_void_p()
        b = _i32_array(list(budgets))
        _check(lib().hs_context_create(device, b, len(budgets), ctypes.byref(topo) if topo else None,
                                       ctypes.byref(h)))
        self.handle = h
        self.device = device

    def close(self):
        if self.handle:
            lib().hs_context_destroy(self.handle)
            self.handle = None

    def __del__(self):  # pragma: no cover
        try:
            self.close()
        except Exception:
            pass


def hs_context_create(device: int = 0, budgets=(64, 128, 192, 256), topo=None) -> Context:
    return Context(device, budgets, topo)


def hs_context_stream(ctx: Context, cu_budget: int, role: int = HS_ROLE_SHARED) -> int:
    s = ctypes.c_void_p()
    _check(lib().hs_context_stream(ctx.handle, cu_budget, role, ctypes.byref(s)))
    return int(s.value)


def hs_context_masks(ctx: Context, cu_budget: int) -> Tuple[List[int], List[int]]:
    sh = (ctypes.c_uint32 * 8)()
    dn = (ctypes.c_uint32 * 8)()
    _check(lib().hs_context_masks(ctx.handle, cu_budget, sh, dn))
    return list(sh), list(dn)


def hs_context_topology(ctx: Context) -> Topology:
    t = Topology()
    _check(lib().hs_context_topology(ctx.handle, ctypes.byref(t)))
    return t


def hs_context_destroy(ctx: Context) -> None:
    ctx.close()


# --------------------------------------------------------------------------- compute calls

def _weights_array(weights: List[Dict[str, object]]):
    arr = (LayerWeights * len(weights))()
    for i, w in enumerate(weights):
        for name in ("ln1", "w_qkv", "w_o", "ln2", "w_gate_up", "w_down"):
            setattr(arr[i], name, _ptr(w[name]))
        arr[i].format = int(w.get("format", HS_WEIGHTS_BF16))
        arr[i].b_qkv = _ptr(w.get("b_qkv"))
    return arr


def _kv_struct(kv) -> Optional[KvCache]:
    """kv: None, (k_list, v_list, n_slots, max_ctx) of device tensors / pointers, or the same
    plus a host block table [n_seqs, pages_per_seq] of slot indices (a paged cache)."""
    if kv is None:
        return None
    k_list, v_list, n_slots, max_ctx = kv[:4]
    table = kv[4] if len(kv) > 4 else None
    kp = (ctypes.c_void_p * len(k_list))(*[_ptr(t) for t in k_list])
    vp = (ctypes.c_void_p * len(v_list))(*[_ptr(t) for t in v_list])
    tp, pps = None, 0
    if table is not None:
        table = np.ascontiguousarray(_as_i32(table, "the block table"))
        assert table.ndim == 2
        pps = table.shape[1]
        tp = table.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))
    s = KvCache(ctypes.cast(kp, ctypes.POINTER(ctypes.c_void_p)), ctypes.cast(vp, ctypes.POINTER(ctypes.c_void_p)),
                n_slots, max_ctx, tp, pps)
    s._keep = (kp, vp, table)
    return s


def hs_shared_stage_forward(ctx: Context, cfg, weights, x_in, x_out, seq_offsets, ctx_lens=None, kv=None,
                            cu_budget: int = 256, stream=None, workspace=None, ws_bytes: Optional[int] = None) -> None:
    warr = _weights_array(weights)
    off = _i32_array(seq_offsets)
    kvs = _kv_struct(kv)
    if ws_bytes is None:
        ws_bytes = workspace.numel() * workspace.element_size()
    _check(lib().hs_shared_stage_forward(
        ctx.handle, ctypes.byref(LayerCfg.of(cfg)), warr, len(weights), _ptr(x_in), _ptr(x_out), off,
        _i32_array(ctx_lens), len(off) - 1, ctypes.byref(kvs) if kvs is not None else None, cu_budget,
        _ptr(stream), _ptr(workspace), ws_bytes))


def hs_shared_stage_forward_mrope(ctx: Context, cfg, weights, x_in, x_out, seq_offsets, positions3, ctx_lens=None,
                                  kv=None, cu_budget: int = 256, stream=None, workspace=None,
                                  ws_bytes: Optional[int] = None) -> None:
    """positions3: host int array [3, T] (temporal, height, width position of every packed row)."""
    warr = _weights_array(weights)
    off = _i32_array(seq_offsets)
    kvs = _kv_struct(kv)
    pos = np.ascontiguousarray(positions3, dtype=np.int32)
    n_rows = int(off[len(off) - 1])
    if pos.shape != (3, n_rows):
        raise ValueError(f"positions3 has shape {pos.shape}, expected (3, {n_rows})")
    if ws_bytes is None:
        ws_bytes = workspace.numel() * workspace.element_size()
    _check(lib().hs_shared_stage_forward_mrope(
        ctx.handle, ctypes.byref(LayerCfg.of(cfg)), warr, len(weights), _ptr(x_in), _ptr(x_out), off,
        _i32_array(ctx_lens), len(off) - 1, ctypes.byref(kvs) if kvs is not None else None,
        pos.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), cu_budget, _ptr(stream), _ptr(workspace), ws_bytes))


def hs_downstream_decode_step_mrope(ctx: Context, cfg, weights, x_in, x_out, kv, kv_lens, positions3, cu_budget: int,
                                    stream=None, workspace=None, ws_bytes: Optional[int] = None) -> None:
    """positions3: host int array [3, batch] (the new rows' temporal, height and width positions)."""
    warr = _weights_array(weights)
    kvs = _kv_struct(kv)
    lens = _i32_array(kv_lens)
    pos = np.ascontiguousarray(positions3, dtype=np.int32)
    if pos.shape != (3, len(lens)):
        raise ValueError(f"positions3 has shape {pos.shape}, expected (3, {len(lens)})")
    if ws_bytes is None:
        ws_bytes = workspace.numel() * workspace.element_size()
    _check(lib().hs_downstream_decode_step_mrope(
        ctx.handle, ctypes.byref(LayerCfg.of(cfg)), warr, len(weights), _ptr(x_in), _ptr(x_out), ctypes.byref(kvs),
        lens, pos.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), len(lens), cu_budget, _ptr(stream),
        _ptr(workspace), ws_bytes))


def hs_downstream_decode_step(ctx: Context, cfg, weights, x_in, x_out, kv, kv_lens, cu_budget: int,
                              stream=None, workspace=None, ws_bytes: Optional[int] = None) -> None:
    warr = _weights_array(weights)
    kvs = _kv_struct(kv)
    lens = _i32_array(kv_lens)
    if ws_bytes is None:
        ws_bytes = workspace.numel() * workspace.element_size()
    _check(lib().hs_downstream_decode_step(
        ctx.handle, ctypes.byref(LayerCfg.of(cfg)), warr, len(weights), _ptr(x_in), _ptr(x_out),
        ctypes.byref(kvs), lens, len(lens), cu_budget, _ptr(stream), _ptr(workspace), ws_bytes))


def hs_downstream_decode_step_noalloc(ctx: Context, cfg, weights, x_in, x_out, kv, kv_lens, cu_budget: int,
                                      stream=None) -> None:
    """The decode step on the library's static scratch (no workspace argument)."""
    warr = _weights_array(weights)
    kvs = _kv_struct(kv)
    lens = _i32_array(kv_lens)
    _check(lib().hs_downstream_decode_step_noalloc(
        ctx.handle, ctypes.byref(LayerCfg.of(cfg)), warr, len(weights), _ptr(x_in), _ptr(x_out),
        ctypes.byref(kvs) if kvs is not None else None, lens, len(lens), cu_budget, _ptr(stream)))


def hs_workspace_size_prefix(cfg, batch: int, max_pos: int, page_positions: int, max_prefix: int,
                             max_rest: int) -> int:
    n = ctypes.c_size_t(0)
    args = (min(v, _INT32_MAX) for v in (batch, max_pos, page_positions, max_prefix, max_rest))
    _check(lib().hs_workspace_size_prefix(ctypes.byref(LayerCfg.of(cfg)), *args, ctypes.byref(n)))
    return int(n.value)


def hs_downstream_decode_step_prefix(ctx: Context, cfg, weights, x_in, x_out, kv, kv_lens, group_offsets, prefix_lens,
                                     cu_budget: int, stream=None, workspace=None,
                                     ws_bytes: Optional[int] = None) -> None:
    """The decode step on a paged cache whose rows share prefixes; group_offsets, prefix_lens: host lists."""
    warr = _weights_array(weights)
    kvs = _kv_struct(kv)
    lens = _i32_array(kv_lens)
    if len(group_offsets) != len(prefix_lens) + 1:
        raise ValueError(f"{len(group_offsets)} offsets, {len(prefix_lens)} prefixes")
    if len(kv) > 4 and kv[4] is not None and len(kv[4]) != len(lens):
        raise ValueError(f"the block table has {len(kv[4])} rows, the batch {len(lens)}")
    if ws_bytes is None:
        ws_bytes = workspace.numel() * workspace.element_size()
    _check(lib().hs_downstream_decode_step_prefix(
        ctx.handle, ctypes.byref(LayerCfg.of(cfg)), warr, len(weights), _ptr(x_in), _ptr(x_out),
        ctypes.byref(kvs), lens, len(lens), _i32_array(group_offsets), _i32_array(prefix_lens), len(prefix_lens),
        cu_budget, _ptr(stream), _ptr(workspace), ws_bytes))


class DecodeGraph:
    """A captured decode step (hs_decode_graph_create); launch(kv_lens[, block_table]) replays it.

    kv as for hs_downstream_decode_step; with a block table there (any contents of the right
    shape [batch, pages_per_seq]) the graph addresses a paged cache and every launch takes
    that step's table."""

    def __init__(self, ctx: Context, cfg, weights, x_in, x_out, kv, batch: int, cu_budget: int,
                 stream=None, workspace=None, ws_bytes: Optional[int] = None):
        self.handle = None
        self._ctx = ctx
        warr = _weights_array(weights)
        kvs = _kv_struct(kv)
        if ws_bytes is None:
            ws_bytes = workspace.numel() * workspace.element_size()
        h = ctypes.c_void_p()
        _check(lib().hs_decode_graph_create(
            ctx.handle, ctypes.byref(LayerCfg.of(cfg)), warr, len(weights), _ptr(x_in), _ptr(x_out),
            ctypes.byref(kvs), batch, cu_budget, _ptr(stream), _ptr(workspace), ws_bytes, ctypes.byref(h)))
        self.handle = h
        self.batch = batch

    def launch(self, kv_lens, block_table=None) -> None:
        lens = _i32_array(kv_lens)
        assert len(lens) == self.batch, (len(lens), self.batch)
        tp = None
        if block_table is not None:
            table = np.ascontiguousarray(block_table, dtype=np.int32)
            assert table.ndim == 2 and table.shape[0] == self.batch
            tp = table.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))
        _check(lib().hs_decode_graph_launch(self.handle, lens, tp))

    def close(self) -> None:
        if self.handle is not None:
            _check(lib().hs_decode_graph_destroy(self.handle))
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def hs_dit_workspace_size(cfg, max_tokens: int, max_seqs: int) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().hs_dit_workspace_size(ctypes.byref(DitCfg.of(cfg)), max_tokens, max_seqs, ctypes.byref(n)))
    return int(n.value)


def _dit_weights_array(weights):
    arr = (DitWeights * len(weights))()
    for i, w in enumerate(weights):
        for name in DIT_FIELDS:
            setattr(arr[i], name, _ptr(w[name]))
        arr[i].format = int(w.get("format", HS_WEIGHTS_BF16))
    return arr


def hs_dit_forward(ctx: Context, cfg, weights, x_in, x_out, cond, seq_offsets, cu_budget: int, stream=None,
                   workspace=None, ws_bytes: Optional[int] = None) -> None:
    """DiT blocks over a packed ragged batch on the downstream side (cu_budget = its CUs)."""
    warr = _dit_weights_array(weights)
    off = _i32_array(seq_offsets)
    if ws_bytes is None:
        ws_bytes = workspace.numel() * workspace.element_size()
    _check(lib().hs_dit_forward(ctx.handle, ctypes.byref(DitCfg.of(cfg)), warr, len(weights), _ptr(x_in),
                                _ptr(x_out), _ptr(cond), off, len(off) - 1, cu_budget, _ptr(stream),
                                _ptr(workspace), ws_bytes))


# The calls below take torch tensors and read types, sizes and strides off them, so a
# tensor that does not fit is a ValueError here, before the library sees a pointer.
# A decode step makes them per token: what they read is read once, and the message
# is put together only for a refusal.

class _Kinds:
    """torch dtype -> HS_TYPE_* (or 0) of what an argument accepts; filled on first use."""
    rows: Dict[object, int] = {}
    f32: Dict[object, int] = {}
    bf16: Dict[object, int] = {}
    i8: Dict[object, int] = {}
    i32: Dict[object, int] = {}
    u8: Dict[object, int] = {}
    halves: Dict[object, int] = {}
    f16: Dict[object, int] = {}

    @classmethod
    def fill(cls) -> None:
        import torch
        cls.rows.update({torch.float32: HS_TYPE_F32, torch.bfloat16: HS_TYPE_BF16, torch.float16: HS_TYPE_F16})
        for kinds, t in ((cls.f32, torch.float32), (cls.bf16, torch.bfloat16), (cls.i8, torch.int8),
                         (cls.i32, torch.int32), (cls.u8, torch.uint8), (cls.f16, torch.float16)):
            kinds[t] = 0
        cls.halves.update({torch.bfloat16: HS_TYPE_BF16, torch.float16: HS_TYPE_F16})


def _refuse(ctx: Context, t, name: str, kinds, ndim: int) -> None:
    if t.dtype not in kinds:
        raise ValueError(f"{name} has type {t.dtype}, expected {' or '.join(str(k) for k in kinds)}")
    if t.dim() != ndim:
        raise ValueError(f"{name} has {t.dim()} dimensions, expected {ndim}")
    raise ValueError(f"{name} is on {t.device}, the context on cuda:{ctx.device}")


# Counts are 32 bits wide in the ABI.  Larger ones are passed as the largest, which every call refuses, and not
# without their upper bits.
_INT32_MAX = 2 ** 31 - 1


def _matrix(ctx: Context, t, name: str, kinds) -> Tuple[int, int, int, int]:
    """(pointer, row stride, rows, columns) of a 2-d tensor whose rows are contiguous."""
    shape = t.shape
    if t.dtype not in kinds or len(shape) != 2 or t.get_device() != ctx.device:
        _refuse(ctx, t, name, kinds, 2)
    rows, cols = shape
    ld, step = t.stride()
    if step != 1 and cols > 1 and rows > 0:
        raise ValueError(f"the rows of {name} are not contiguous (stride {step})")
    if (rows | cols) >> 31:
        rows, cols = min(rows, _INT32_MAX), min(cols, _INT32_MAX)
    return t.data_ptr(), (ld if rows > 1 else max(cols, 1)), rows, cols


def _dense(ctx: Context, t, name: str, kinds, *shape) -> Optional[int]:
    """Pointer of a contiguous tensor of exactly this shape (None stays None)."""
    if t is None:
        return None
    size = t.shape
    if t.dtype not in kinds or len(size) != len(shape) or t.get_device() != ctx.device:
        _refuse(ctx, t, name, kinds, len(shape))
    if size != shape and tuple(min(n, _INT32_MAX) for n in size) != shape:
        raise ValueError(f"{name} has shape {tuple(size)}, expected {shape}")
    if not t.is_contiguous():
        raise ValueError(f"{name} is not contiguous")
    return t.data_ptr()


def _workspace(ctx: Context, t, n_bytes: Optional[int]) -> Tuple[Optional[int], int]:
    """(pointer, bytes) of a workspace: a contiguous tensor of any type (its bytes, or fewer where n_bytes says so), a
    device address with n_bytes, or None."""
    if t is None:
        return None, n_bytes or 0
    if type(t) is int:
        if n_bytes is None:
            raise ValueError("a workspace address needs ws_bytes")
        return t, n_bytes
    if t.get_device() != ctx.device:
        raise ValueError(f"workspace is on {t.device}, the context on cuda:{ctx.device}")
    if not t.is_contiguous():
        raise ValueError("workspace is not contiguous")
    size = t.nbytes
    if n_bytes is not None:
        if n_bytes > size:
            raise ValueError(f"workspace has {size} bytes, ws_bytes is {n_bytes}")
        size = n_bytes
    return t.data_ptr(), size


def hs_quantize_rows(ctx: Context, x, q, scale, gain=None, eps: float = 1e-6, cu_budget: int = 256,
                     stream=None) -> None:
    """x [rows, d] (fp32, bf16 or fp16) -> q int8 [rows, d] and scale fp32 [rows]; gain: bf16 [d] (RMSNorm) or None."""
    if not _Kinds.rows:
        _Kinds.fill()
    px, ldx, rows, d = _matrix(ctx, x, "x", _Kinds.rows)
    pq, ldq, *q_shape = _matrix(ctx, q, "q", _Kinds.i8)
    if q_shape != [rows, d]:
        raise ValueError(f"q has shape {tuple(q_shape)}, x ({rows}, {d})")
    status = lib().hs_quantize_rows(ctx.handle, px, _Kinds.rows[x.dtype], ldx,
                                    _dense(ctx, gain, "gain", _Kinds.bf16, d), eps, rows, d, pq, ldq,
                                    _dense(ctx, scale, "scale", _Kinds.f32, rows), cu_budget, _ptr(stream))
    if status:
        _check(status)


def hs_linear_i8(ctx: Context, a, a_scale, w, w_scale, out, bias=None, cu_budget: int = 256, stream=None) -> None:
    """out [m, n] = (a int8 [m, k] * a_scale fp32 [m]) (w int8 [n, k] * w_scale fp32 [n])^T + bias bf16 [n]."""
    if not _Kinds.rows:
        _Kinds.fill()
    pa, lda, m, k = _matrix(ctx, a, "a", _Kinds.i8)
    pw, ldw, n, wk = _matrix(ctx, w, "w", _Kinds.i8)
    po, ldo, om, on = _matrix(ctx, out, "out", _Kinds.rows)
    if wk != k or om != m or on != n:
        raise ValueError(f"a ({m}, {k}), w ({n}, {wk}) and out ({om}, {on}) do not fit")
    status = lib().hs_linear_i8(ctx.handle, pa, lda, _dense(ctx, a_scale, "a_scale", _Kinds.f32, m), pw, ldw,
                                _dense(ctx, w_scale, "w_scale", _Kinds.f32, n),
                                _dense(ctx, bias, "bias", _Kinds.bf16, n), po, _Kinds.rows[out.dtype], ldo, m, n, k,
                                cu_budget, _ptr(stream))
    if status:
        _check(status)


def hs_logprobs_workspace_size(max_rows: int, vocab: int, top_k: int = 0) -> int:
    n = ctypes.c_size_t(0)
    max_rows, vocab, top_k = (min(v, _INT32_MAX) for v in (max_rows, vocab, top_k))
    _check(lib().hs_logprobs_workspace_size(max_rows, vocab, top_k, ctypes.byref(n)))
    return int(n.value)


def hs_logprobs(ctx: Context, logits, tokens=None, token_logprobs=None, entropy=None, top_logprobs=None,
                top_tokens=None, cu_budget: int = 256, stream=None, workspace=None,
                ws_bytes: Optional[int] = None) -> None:
    """logits [rows, vocab]; tokens int32 and token_logprobs fp32 [rows, n]; entropy fp32 [rows]; top_logprobs fp32 and
    top_tokens int32 [rows, k].  What is None is not computed."""
    if not _Kinds.rows:
        _Kinds.fill()
    pz, ld, rows, vocab = _matrix(ctx, logits, "logits", _Kinds.rows)
    if (tokens is None) != (token_logprobs is None) or (top_logprobs is None) != (top_tokens is None):
        raise ValueError("tokens and token_logprobs, top_logprobs and top_tokens go together")
    n = k = 0
    try:
        if tokens is not None:
            n = tokens.shape[-1]
        if top_tokens is not None:
            k = top_tokens.shape[-1]
    except IndexError:   # no dimensions: refused with the others below
        pass
    if (n | k) >> 31:
        n, k = min(n, _INT32_MAX), min(k, _INT32_MAX)
    ws, ws_bytes = _workspace(ctx, workspace, ws_bytes)
    f32, i32 = _Kinds.f32, _Kinds.i32
    status = lib().hs_logprobs(
        ctx.handle, pz, _Kinds.rows[logits.dtype], ld, rows, vocab, _dense(ctx, tokens, "tokens", i32, rows, n), n,
        _dense(ctx, token_logprobs, "token_logprobs", f32, rows, n), _dense(ctx, entropy, "entropy", f32, rows), k,
        _dense(ctx, top_logprobs, "top_logprobs", f32, rows, k), _dense(ctx, top_tokens, "top_tokens", i32, rows, k),
        cu_budget, stream and _ptr(stream), ws, ws_bytes)
    if status:
        _check(status)


def hs_beam_select_workspace_size(max_groups: int, beams: int, vocab: int, n_select: int) -> int:
    n = ctypes.c_size_t(0)
    args = (min(v, _INT32_MAX) for v in (max_groups, beams, vocab, n_select))
    _check(lib().hs_beam_select_workspace_size(*args, ctypes.byref(n)))
    return int(n.value)


def hs_beam_select(ctx: Context, logits, scores, out_scores, out_parents, out_tokens, finished=None, out_finished=None,
                   end_token: int = -1, cu_budget: int = 256, stream=None, workspace=None,
                   ws_bytes: Optional[int] = None) -> None:
    """logits [groups * beams, vocab], scores fp32 and finished uint8 [groups, beams] -> out_scores fp32, out_parents and
    out_tokens int32, out_finished uint8 [groups, n_select]; what is None is not used."""
    if not _Kinds.rows:
        _Kinds.fill()
    pz, ld, rows, vocab = _matrix(ctx, logits, "logits", _Kinds.rows)
    for t, name, kinds in ((scores, "scores", _Kinds.f32), (out_scores, "out_scores", _Kinds.f32)):
        if t.dim() != 2:
            _refuse(ctx, t, name, kinds, 2)
    groups, beams = scores.shape
    if groups * beams != rows:
        raise ValueError(f"logits has {rows} rows, scores {groups} x {beams}")
    select = min(out_scores.shape[1], _INT32_MAX)
    f32, i32, u8 = _Kinds.f32, _Kinds.i32, _Kinds.u8
    ws, ws_bytes = _workspace(ctx, workspace, ws_bytes)
    status = lib().hs_beam_select(
        ctx.handle, pz, _Kinds.rows[logits.dtype], ld, groups, beams, vocab,
        _dense(ctx, scores, "scores", f32, groups, beams), _dense(ctx, finished, "finished", u8, groups, beams),
        max(-2, min(end_token, _INT32_MAX)), select, _dense(ctx, out_scores, "out_scores", f32, groups, select),
        _dense(ctx, out_parents, "out_parents", i32, groups, select),
        _dense(ctx, out_tokens, "out_tokens", i32, groups, select),
        _dense(ctx, out_finished, "out_finished", u8, groups, select), cu_budget, stream and _ptr(stream), ws, ws_bytes)
    if status:
        _check(status)


def _cache_layers(ctx: Context, k, v, n_slots: int, max_ctx: int) -> Tuple[int, int]:
    """(key/value heads, head size) of a cache's layers: k[l] fp16 [n_slots, hkv, max_ctx, dh], v[l] the same in value
    tiles [n_slots, hkv, max_ctx / 32, dh, 32]."""
    if len(k) != len(v) or not k:
        raise ValueError(f"{len(k)} layers of keys, {len(v)} of values")
    if k[0].dim() != 4:
        _refuse(ctx, k[0], "k", _Kinds.f16, 4)
    _, hkv, _, dh = k[0].shape
    f16, device = _Kinds.f16, ctx.device
    for layers, name, shape in ((k, "k", (n_slots, hkv, max_ctx, dh)), (v, "v", (n_slots, hkv, max_ctx // 32, dh, 32))):
        for t in layers:
            if t.shape != shape or t.dtype not in f16 or t.get_device() != device or not t.is_contiguous():
                _dense(ctx, t, name, f16, *shape)   # the message of what does not fit
    return hkv, dh


def _host_ints(values, name: str):
    """(keeper, address) of host integers as 32-bit words."""
    if values is None:
        return None, None
    if isinstance(values, np.ndarray):
        if values.ndim != 1:
            raise ValueError(f"{name} holds no list of 32-bit numbers")
        a = _as_i32(values, name)
        return a, a.ctypes.data
    try:
        a = array.array("i", values)
    except (OverflowError, TypeError) as e:
        raise ValueError(f"{name} holds no list of 32-bit numbers: {e}") from None
    return a, a.buffer_info()[0]


class _KvAddresses(ctypes.Structure):
    """KvCache with plain addresses, which cost less to fill in."""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("n_slots", ctypes.c_int32), ("max_ctx", ctypes.c_int32),
                ("block_table", ctypes.c_void_p), ("pages_per_seq", ctypes.c_int32)]


def hs_cache_copy(ctx: Context, kv, src, dst, positions=None, cu_budget: int = 256, stream=None) -> None:
    """kv: (k, v, n_slots, max_ctx[, block table]) as for the decode step, of tensors; src, dst, positions: host lists,
    positions None for whole slots."""
    if not _Kinds.rows:
        _Kinds.fill()
    k, v, n_slots, max_ctx = kv[:4]
    hkv, dh = _cache_layers(ctx, k, v, n_slots, max_ctx)
    n = len(src)
    if len(dst) != n or (positions is not None and len(positions) != n):
        raise ValueError(f"{n} sources, {len(dst)} destinations"
                         + ("" if positions is None else f", {len(positions)} numbers of positions"))
    ks, vs = array.array("Q", [t.data_ptr() for t in k]), array.array("Q", [t.data_ptr() for t in v])
    arg = _KvAddresses(ks.buffer_info()[0], vs.buffer_info()[0], n_slots, max_ctx, None, 0)
    (s, ps), (d, pd), (p, pp) = _host_ints(src, "src"), _host_ints(dst, "dst"), _host_ints(positions, "positions")
    status = lib().hs_cache_copy(ctx.handle, ctypes.byref(arg), len(k), hkv, dh, ps, pd, pp, n, cu_budget, _ptr(stream))
    if status:
        _check(status)


def hs_prefix_attention_workspace_size(n_q_heads: int, n_kv_heads: int, head_dim: int, n_seqs: int, max_prefix: int,
                                       max_rest: int) -> int:
    n = ctypes.c_size_t(0)
    args = (min(v, _INT32_MAX) for v in (n_q_heads, n_kv_heads, head_dim, n_seqs, max_prefix, max_rest))
    _check(lib().hs_prefix_attention_workspace_size(*args, ctypes.byref(n)))
    return int(n.value)


def hs_prefix_attention(ctx: Context, q, out, k, v, block_table, lens, group_offsets, prefix_lens, max_prefix: int,
                        max_rest: int, cu_budget: int = 256, stream=None, workspace=None,
                        ws_bytes: Optional[int] = None) -> None:
    """q and out (fp16 or bf16) [n_seqs, n_q_heads * head_dim]; k and v: one layer of a cache; block_table int32
    [n_seqs, pages_per_seq], lens int32 [n_seqs], group_offsets int32 [n_groups + 1], prefix_lens int32 [n_groups],
    all on the device (group_offsets and prefix_lens None: no prefixes)."""
    if not _Kinds.rows:
        _Kinds.fill()
    halves = _Kinds.halves
    pq, ldq, n, cols = _matrix(ctx, q, "q", halves)
    po, ldo, o_rows, o_cols = _matrix(ctx, out, "out", halves)
    if out.dtype is not q.dtype or o_rows != n or o_cols != cols:
        raise ValueError(f"out has type {out.dtype} and shape {tuple(out.shape)}, q {q.dtype} and {tuple(q.shape)}")
    if len(k.shape) != 4:
        _refuse(ctx, k, "k", _Kinds.f16, 4)
    n_slots, hkv, page, dh = k.shape
    pk = _dense(ctx, k, "k", _Kinds.f16, n_slots, hkv, page, dh)
    pv = _dense(ctx, v, "v", _Kinds.f16, n_slots, hkv, page // 32, dh, 32)
    if dh < 1 or cols % dh:
        raise ValueError(f"q has {cols} columns, the cache heads of {dh}")
    if len(block_table.shape) != 2:
        _refuse(ctx, block_table, "block_table", _Kinds.i32, 2)
    per_seq = block_table.shape[1]
    groups = 0
    if prefix_lens is not None and group_offsets is not None:
        if len(prefix_lens.shape) != 1:
            _refuse(ctx, prefix_lens, "prefix_lens", _Kinds.i32, 1)
        groups = prefix_lens.shape[0]
    elif prefix_lens is not group_offsets:
        raise ValueError("group_offsets and prefix_lens go together")
    i32 = _Kinds.i32
    ws, ws_bytes = _workspace(ctx, workspace, ws_bytes)
    status = lib().hs_prefix_attention(
        ctx.handle, pq, halves[q.dtype], ldq, po, ldo, cols // dh, hkv, dh, pk, pv, n_slots, page,
        _dense(ctx, block_table, "block_table", i32, n, per_seq), per_seq, _dense(ctx, lens, "lens", i32, n), n,
        _dense(ctx, group_offsets, "group_offsets", i32, groups + 1),
        _dense(ctx, prefix_lens, "prefix_lens", i32, groups), groups, min(max_prefix, _INT32_MAX),
        min(max_rest, _INT32_MAX), cu_budget, stream and _ptr(stream), ws, ws_bytes)
    if status:
        _check(status)


class Pages:
    """Owns an ``hs_pages`` handle: which pages of a cache the sequences list (host only).

    Calls that move data return (src, dst, positions) for ``hs_cache_copy``."""

    def __init__(self, n_pages: int, page_positions: int, max_seqs: int, pages_per_seq: int):
        self.handle = None
        h = ctypes.c_void_p()
        args = (min(v, _INT32_MAX) for v in (n_pages, page_positions, max_seqs, pages_per_seq))
        _check(lib().hs_pages_create(*args, ctypes.byref(h)))
        self.handle = h
        self.n_pages, self.pages_per_seq = n_pages, pages_per_seq

    def _copies(self, room: int, call) -> Tuple[List[int], List[int], List[int]]:
        lists = [(ctypes.c_int32 * max(room, 1))() for _ in range(3)]
        n = ctypes.c_int32(0)
        _check(call(*lists, ctypes.byref(n)))
        return tuple(list(x[:n.value]) for x in lists)

    def reserve(self, seqs, add):
        if len(seqs) != len(add):
            raise ValueError(f"{len(seqs)} sequences, {len(add)} numbers of positions")
        return self._copies(len(seqs), lambda *out: lib().hs_pages_reserve(
            self.handle, _i32_array(seqs), _i32_array(add), len(seqs), *out))

    def fork(self, seqs, parents) -> None:
        if len(seqs) != len(parents):
            raise ValueError(f"{len(seqs)} sequences, {len(parents)} parents")
        _check(lib().hs_pages_fork(self.handle, _i32_array(seqs), _i32_array(parents), len(seqs)))

    def release(self, seqs) -> None:
        self.fork(seqs, [-1] * len(seqs))

    def compact(self, room: int):
        room = min(room, self.n_pages)   # no more can move
        return self._copies(room, lambda *out: lib().hs_pages_compact(self.handle, room, *out))

    def table(self, seqs) -> Tuple[np.ndarray, np.ndarray]:
        """(block table [n, pages_per_seq], lengths [n])."""
        table = np.zeros((len(seqs), self.pages_per_seq), np.int32)
        lens = np.zeros(len(seqs), np.int32)
        as_i32 = ctypes.POINTER(ctypes.c_int32)
        _check(lib().hs_pages_table(self.handle, _i32_array(seqs), len(seqs), table.ctypes.data_as(as_i32),
                                    lens.ctypes.data_as(as_i32)))
        return table, lens

    def shared(self, seqs) -> int:
        n = ctypes.c_int32(0)
        _check(lib().hs_pages_shared(self.handle, _i32_array(seqs), len(seqs), ctypes.byref(n)))
        return int(n.value)

    def free_count(self) -> int:
        n = ctypes.c_int32(0)
        _check(lib().hs_pages_free_count(self.handle, ctypes.byref(n)))
        return int(n.value)

    def close(self) -> None:
        if self.handle is not None:
            lib().hs_pages_destroy(self.handle)
            self.handle = None

    def __del__(self):  # pragma: no cover
        try:
            self.close()
        except Exception:
            pass


def hs_probe_hw_ids(ctx: Context, stream, n_groups: int, out_ids) -> None:
    _check(lib().hs_probe_hw_ids(ctx.handle, _ptr(stream), n_groups, _ptr(out_ids)))


def hs_timing_enable(ctx: Context, enable: bool = True) -> None:
    _check(lib().hs_timing_enable(ctx.handle, 1 if enable else 0))


def hs_timing_read_clock(ctx: Context, kind) -> Tuple[float, int]:
    """(average shader clock in MHz, launches with clock records) of one kernel kind."""
    k = KERNEL_KINDS[kind] if isinstance(kind, str) else int(kind)
    mhz = ctypes.c_double(0)
    n = ctypes.c_int32(0)
    _check(lib().hs_timing_read_clock(ctx.handle, k, ctypes.byref(mhz), ctypes.byref(n)))
    return float(mhz.value), int(n.value)


def hs_timing_read(ctx: Context, kind) -> Tuple[float, int]:
    """(summed milliseconds, launches) of one kernel kind since timing was enabled."""
    k = KERNEL_KINDS[kind] if isinstance(kind, str) else int(kind)
    ms = ctypes.c_double(0)
    n = ctypes.c_int32(0)
    _check(lib().hs_timing_read(ctx.handle, k, ctypes.byref(ms), ctypes.byref(n)))
    return float(ms.value), int(n.value)


def hs_convert_weights_f16(ctx: Context, src, dst, rows: Optional[int] = None, cols: Optional[int] = None,
                           stream=None) -> None:
    """bf16 [rows, cols] -> fp16 panel-major [cols / 32][rows][32] (shape taken from src if not given)."""
    if rows is None or cols is None:
        rows, cols = int(src.shape[0]), int(src.shape[1])
    _check(lib().hs_convert_weights_f16(ctx.handle, _ptr(src), _ptr(dst), int(rows), int(cols), _ptr(stream)))
