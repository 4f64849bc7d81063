"""ctypes binding of libpsrl.so: same names as the C ABI, argument marshalling only.

Every step of the path runs inside the library's kernels.  The binding raises
if the library has not been built; there is no fallback of any kind.  Calls
whose kernels take a few microseconds have their plain case in csrc/torch_calls.cpp.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from typing import Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpsrl.so")

PSRL_OK = 0
STATUS_NAMES = [
    "PSRL_OK", "PSRL_ERR_INVALID_ARG", "PSRL_ERR_BAD_TREE", "PSRL_ERR_BAD_BLOCK_SIZE", "PSRL_ERR_SHAPE",
    "PSRL_ERR_UNSUPPORTED", "PSRL_ERR_POOL_FULL", "PSRL_ERR_WORKSPACE", "PSRL_ERR_HOST_OOM", "PSRL_ERR_CUDA",
    "PSRL_ERR_TIMEOUT", "PSRL_ERR_INTERNAL",
]
PSRL_F32, PSRL_BF16, PSRL_E4M3 = 0, 1, 2
BWD_STATIC_SCRATCH_BYTES = 16 * 1024 * 1024 + 256   # PSRL_BWD_STATIC_SCRATCH_BYTES of include/psrl.h
SEG_HAS_Q, SEG_SAMPLE_END = 1, 2

EXPORTS = [
    "psrl_plan_build", "psrl_plan_view", "psrl_plan_device_bytes", "psrl_plan_upload",
    "psrl_fwd_workspace_bytes", "psrl_bwd_workspace_bytes", "psrl_tree_attn_fwd", "psrl_tree_attn_bwd",
    "psrl_device_status", "psrl_last_cuda_error", "psrl_plan_destroy", "psrl_status_string",
    "psrl_bench_bwd_phases", "psrl_tree_attn_bwd_static", "psrl_launch_count", "psrl_plan_schedule",
    "psrl_cache_create", "psrl_cache_begin", "psrl_cache_end", "psrl_cache_stats", "psrl_cache_refcounts",
    "psrl_cache_destroy",
    "psrl_kv_scatter", "psrl_kv_gather",
    "psrl_rope_create", "psrl_rope_frequencies", "psrl_rope_destroy", "psrl_rope_qkv_fwd", "psrl_rope_qkv_bwd",
    "psrl_rope_rows",
    "psrl_rope_create_axes", "psrl_rope_axes_qkv_fwd", "psrl_rope_axes_qkv_bwd", "psrl_rope_axes_rows",
    "psrl_rms_norm_fwd", "psrl_rms_norm_bwd", "psrl_rms_norm_workspace_bytes", "psrl_quantize_rows",
    "psrl_linear_fwd", "psrl_linear_bwd", "psrl_linear_workspace_bytes",
    "psrl_plan_next_tokens", "psrl_token_logprob_workspace_bytes", "psrl_token_logprob_fwd", "psrl_token_logprob_bwd",
    "psrl_cache_compact", "psrl_kv_copy", "psrl_kv_move",
    "psrl_cost_sequence", "psrl_group_workloads", "psrl_place_groups", "psrl_microbatch_tokens",
]

_I32P = C.POINTER(C.c_int32)


class TreeDesc(C.Structure):
    _fields_ = [
        ("n_segments", C.c_int32), ("parent", _I32P), ("seg_len", _I32P), ("seg_flags", C.POINTER(C.c_uint8)),
        ("group_block_size", _I32P), ("n_groups", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
        ("head_dim", C.c_int32), ("dtype", C.c_int), ("free_extents", _I32P), ("n_free", C.c_int32),
        ("seg_slot_base", _I32P),
    ]


class CostModel(C.Structure):
    _fields_ = [("a1", C.c_double), ("a2", C.c_double), ("a3", C.c_double)]


class CacheDesc(C.Structure):
    _fields_ = [
        ("n_segments", C.c_int32), ("parent", _I32P), ("seg_len", _I32P), ("seg_flags", C.POINTER(C.c_uint8)),
        ("group_block_size", _I32P), ("n_groups", C.c_int32), ("n_microbatches", C.c_int32), ("mb_of_seg", _I32P),
        ("capacity_slots", C.c_int64),
    ]


class CacheStep(C.Structure):
    _fields_ = [
        ("n_segments", C.c_int32), ("seg_id", _I32P), ("parent", _I32P), ("seg_len", _I32P),
        ("seg_flags", C.POINTER(C.c_uint8)), ("group_block_size", _I32P), ("n_groups", C.c_int32),
        ("seg_slot_base", _I32P), ("n_new", C.c_int32), ("n_reload", C.c_int32), ("n_evict", C.c_int32),
        ("new_seg", _I32P), ("reload_seg", _I32P), ("evict_seg", _I32P), ("evict_base", _I32P),
        ("live_slots", C.c_int64), ("pool_slots", C.c_int64),
    ]


class CacheStats(C.Structure):
    _fields_ = [("peak_slots", C.c_int64), ("evicted_slots", C.c_int64), ("reloaded_slots", C.c_int64),
                ("pool_high_water", C.c_int64), ("total_slots", C.c_int64)]


class RopeDesc(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("rotary_dim", C.c_int32), ("layout", C.c_int32), ("scaling", C.c_int32),
                ("base", C.c_double), ("factor", C.c_double), ("original_positions", C.c_int32), ("low", C.c_double),
                ("high", C.c_double), ("attention_scale", C.c_double)]


_VIEW_SCALARS32 = ["n_seg", "n_groups", "n_pages", "n_samples", "max_depth", "T", "T_q", "pool_slots"]
_VIEW_SCALARS64 = ["flat_tokens", "tree_pairs", "flat_pairs"]
_VIEW_ARRAYS = [
    "canon_of_input", "input_of_canon", "seg_group", "seg_bs", "seg_parent", "seg_len", "seg_flags", "seg_depth",
    "seg_anc_tokens", "seg_sub_end", "seg_tok_off", "seg_q_off", "seg_refcount", "anc_off", "anc_list",
    "seg_first_page", "seg_n_pages", "page_seg", "page_bs", "page_valid", "page_pos", "page_refcount", "page_slot",
    "bt_off", "bt_pages", "tok_slot", "sample_end_seg", "sample_len",
]


class PlanView(C.Structure):
    _fields_ = (
        [(n, C.c_int32) for n in _VIEW_SCALARS32]
        + [(n, C.c_int64) for n in _VIEW_SCALARS64]
        + [("n_anc", C.c_int32), ("n_bt", C.c_int32)]
        + [(n, _I32P) for n in _VIEW_ARRAYS]
    )


class PsrlError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str = ""):
        name = STATUS_NAMES[status] if 0 <= status < len(STATUS_NAMES) else str(status)
        super().__init__(f"{where}: {name}{(' (' + detail + ')') if detail else ''}")
        self.status = status
        self.name = name


_lib = None


def lib() -> C.CDLL:
    """Load libpsrl.so (once).  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2608_25683_b200.build` "
            "(there is no fallback path)")
    L = C.CDLL(LIB_PATH)
    L.psrl_plan_build.argtypes = [C.POINTER(TreeDesc), C.POINTER(C.c_void_p)]
    L.psrl_plan_build.restype = C.c_int
    L.psrl_plan_view.argtypes = [C.c_void_p, C.POINTER(PlanView)]
    L.psrl_plan_view.restype = C.c_int
    L.psrl_plan_device_bytes.argtypes = [C.c_void_p]
    L.psrl_plan_device_bytes.restype = C.c_size_t
    L.psrl_plan_upload.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    L.psrl_plan_upload.restype = C.c_int
    for f in (L.psrl_fwd_workspace_bytes, L.psrl_bwd_workspace_bytes):
        f.argtypes = [C.c_void_p]
        f.restype = C.c_size_t
    L.psrl_tree_attn_fwd.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p,
                                     C.c_void_p, C.c_float, C.c_void_p, C.c_size_t, C.c_void_p]
    L.psrl_tree_attn_fwd.restype = C.c_int
    L.psrl_tree_attn_bwd.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p,
                                     C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_float,
                                     C.c_void_p, C.c_size_t, C.c_void_p]
    L.psrl_tree_attn_bwd.restype = C.c_int
    L.psrl_device_status.argtypes = [C.c_void_p, C.c_void_p]
    L.psrl_device_status.restype = C.c_int
    L.psrl_tree_attn_bwd_static.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p,
                                            C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_float,
                                            C.POINTER(C.c_void_p), C.c_void_p]
    L.psrl_tree_attn_bwd_static.restype = C.c_int
    L.psrl_bench_bwd_phases.argtypes = L.psrl_tree_attn_bwd.argtypes + [C.c_int]
    L.psrl_bench_bwd_phases.restype = C.c_int
    L.psrl_plan_schedule.argtypes = [C.c_void_p, C.POINTER(_I32P), C.POINTER(C.c_size_t)]
    L.psrl_plan_schedule.restype = C.c_int
    _F64P = C.POINTER(C.c_double)
    _U8P = C.POINTER(C.c_uint8)
    L.psrl_cost_sequence.argtypes = [C.POINTER(CostModel), C.c_int64, C.c_int64]
    L.psrl_cost_sequence.restype = C.c_double
    L.psrl_group_workloads.argtypes = [C.c_int32, _I32P, _I32P, _U8P, C.POINTER(CostModel), C.c_int32, _F64P]
    L.psrl_group_workloads.restype = C.c_int
    L.psrl_place_groups.argtypes = [C.c_int32, _F64P, C.c_int32, _I32P, _F64P]
    L.psrl_place_groups.restype = C.c_int
    L.psrl_microbatch_tokens.argtypes = [C.c_int32, _I32P, _I32P, _U8P, C.POINTER(CostModel), C.c_int32, C.c_int32,
                                         _I32P, _I32P, _I32P, _I32P, _I32P, _I32P, _F64P]
    L.psrl_microbatch_tokens.restype = C.c_int
    L.psrl_kv_scatter.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p]
    L.psrl_kv_scatter.restype = C.c_int
    L.psrl_kv_gather.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p]
    L.psrl_kv_gather.restype = C.c_int
    L.psrl_cache_create.argtypes = [C.POINTER(CacheDesc), C.POINTER(C.c_void_p)]
    L.psrl_cache_create.restype = C.c_int
    L.psrl_cache_begin.argtypes = [C.c_void_p, C.c_int32, C.POINTER(CacheStep)]
    L.psrl_cache_begin.restype = C.c_int
    L.psrl_cache_end.argtypes = [C.c_void_p, C.c_int32, C.POINTER(C.c_int32), C.POINTER(_I32P), C.POINTER(C.c_int64)]
    L.psrl_cache_end.restype = C.c_int
    L.psrl_cache_stats.argtypes = [C.c_void_p, C.POINTER(CacheStats)]
    L.psrl_cache_stats.restype = C.c_int
    L.psrl_cache_refcounts.argtypes = [C.c_void_p, C.POINTER(_I32P)]
    L.psrl_cache_refcounts.restype = C.c_int
    L.psrl_cache_destroy.argtypes = [C.c_void_p]
    L.psrl_cache_destroy.restype = None
    L.psrl_cache_compact.argtypes = [C.c_void_p, C.POINTER(C.c_int32), C.POINTER(_I32P), C.POINTER(C.c_int64)]
    L.psrl_cache_compact.restype = C.c_int
    L.psrl_kv_copy.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_int64,
                               C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p]
    L.psrl_kv_copy.restype = C.c_int
    L.psrl_kv_move.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_int64,
                               C.c_void_p, C.c_size_t, C.c_void_p]
    L.psrl_kv_move.restype = C.c_int
    L.psrl_rope_create.argtypes = [C.POINTER(RopeDesc), C.POINTER(C.c_void_p)]
    L.psrl_rope_create.restype = C.c_int
    L.psrl_rope_frequencies.argtypes = [C.c_void_p, C.POINTER(_F64P), C.POINTER(C.c_int32), C.POINTER(C.c_double)]
    L.psrl_rope_frequencies.restype = C.c_int
    L.psrl_rope_destroy.argtypes = [C.c_void_p]
    L.psrl_rope_destroy.restype = None
    _VP, _I64 = C.c_void_p, C.c_int64
    L.psrl_rope_qkv_fwd.argtypes = [_VP, _VP, _VP, _I64, _VP, _I64, _VP, _I64, _VP, _VP, _VP, _I64, _VP]
    L.psrl_rope_qkv_fwd.restype = C.c_int
    L.psrl_rope_qkv_bwd.argtypes = [_VP, _VP, _VP, _VP, _VP, _I64, _VP, _I64, _VP, _I64, _VP, _I64, _VP]
    L.psrl_rope_qkv_bwd.restype = C.c_int
    L.psrl_rope_rows.argtypes = [_VP, C.c_int, _VP, _I64, _VP, _I64, C.c_int32, _VP, _I64, C.c_int, _VP]
    L.psrl_rope_rows.restype = C.c_int
    L.psrl_rope_create_axes.argtypes = [C.POINTER(RopeDesc), C.c_int32, _I32P, C.c_int, C.POINTER(C.c_void_p)]
    L.psrl_rope_create_axes.restype = C.c_int
    L.psrl_rope_axes_qkv_fwd.argtypes = [_VP, _VP, _VP, _I64, _VP, _I64, _VP, _I64, _VP, _I64, _VP, _VP, _VP, _I64, _VP]
    L.psrl_rope_axes_qkv_fwd.restype = C.c_int
    L.psrl_rope_axes_qkv_bwd.argtypes = [_VP, _VP, _VP, _I64, _VP, _VP, _VP, _I64, _VP, _I64, _VP, _I64, _VP, _I64, _VP]
    L.psrl_rope_axes_qkv_bwd.restype = C.c_int
    L.psrl_rope_axes_rows.argtypes = [_VP, C.c_int, _VP, _I64, _VP, _I64, _I64, C.c_int32, _VP, _I64, C.c_int, _VP]
    L.psrl_rope_axes_rows.restype = C.c_int
    L.psrl_rms_norm_fwd.argtypes = [C.c_int, _I64, C.c_int32, C.c_int32, _VP, _I64, _VP, _I64, _VP, C.c_float, _VP, _I64, _VP, _I64, _VP,
                                    _I64, _VP, _VP]
    L.psrl_rms_norm_fwd.restype = C.c_int
    L.psrl_rms_norm_workspace_bytes.argtypes = [C.c_int, _I64, C.c_int32, C.c_int32]
    L.psrl_rms_norm_workspace_bytes.restype = C.c_size_t
    L.psrl_rms_norm_bwd.argtypes = [C.c_int, _I64, C.c_int32, C.c_int32, _VP, _I64, _VP, C.c_float, _VP, _I64, _VP, _I64, _VP, _I64, _VP, _VP,
                                    C.c_size_t, _VP]
    L.psrl_rms_norm_bwd.restype = C.c_int
    L.psrl_quantize_rows.argtypes = [C.c_int, _I64, C.c_int32, _VP, _I64, _VP, _I64, _VP, _VP]
    L.psrl_quantize_rows.restype = C.c_int
    L.psrl_linear_workspace_bytes.argtypes = [C.c_int, _I64, C.c_int32, C.c_int32, C.c_int]
    L.psrl_linear_workspace_bytes.restype = C.c_size_t
    L.psrl_linear_fwd.argtypes = [C.c_int, _I64, C.c_int32, C.c_int32, _VP, _I64, _VP, _VP, _I64, _VP, _VP, C.c_int, _VP, _I64, _VP, _I64, _VP, _I64,
                                  _VP, _I64, _VP, C.c_size_t, _VP]
    L.psrl_linear_fwd.restype = C.c_int
    L.psrl_linear_bwd.argtypes = [C.c_int, _I64, C.c_int32, C.c_int32, _VP, _I64, _VP, _I64, _VP, _I64, C.c_int, _VP, _I64, _VP, _I64, _VP, _I64, _VP, _I64,
                                  _VP, _VP, _I64, _VP, C.c_size_t, _VP]
    L.psrl_linear_bwd.restype = C.c_int
    L.psrl_plan_next_tokens.argtypes = [_VP, C.POINTER(_I32P), C.POINTER(_I32P)]
    L.psrl_plan_next_tokens.restype = C.c_int
    L.psrl_token_logprob_workspace_bytes.argtypes = [C.c_int, _I64, C.c_int32, C.c_int32, _I64, C.c_int]
    L.psrl_token_logprob_workspace_bytes.restype = C.c_size_t
    lp = [C.c_int, _I64, C.c_int32, C.c_int32, _VP, _I64, _VP, _I64, _VP, _I64, _VP, C.c_float, _VP, _VP]
    L.psrl_token_logprob_fwd.argtypes = lp + [_VP, C.c_size_t, _VP]
    L.psrl_token_logprob_fwd.restype = C.c_int
    L.psrl_token_logprob_bwd.argtypes = lp + [_VP, _VP, _I64, _VP, _I64, _VP, C.c_size_t, _VP]
    L.psrl_token_logprob_bwd.restype = C.c_int
    L.psrl_launch_count.argtypes = [C.c_void_p, C.c_int]
    L.psrl_launch_count.restype = C.c_int
    L.psrl_last_cuda_error.restype = C.c_char_p
    L.psrl_plan_destroy.argtypes = [C.c_void_p]
    L.psrl_plan_destroy.restype = None
    L.psrl_status_string.argtypes = [C.c_int]
    L.psrl_status_string.restype = C.c_char_p
    _lib = L
    return L


def _check(status: int, where: str):
    if status != PSRL_OK:
        detail = ""
        if status == 9:
            detail = lib().psrl_last_cuda_error().decode()
        raise PsrlError(status, where, detail)


def _i32(a) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a, dtype=np.int32))


class Plan:
    """Owner of a psrl_plan_t.  `view` holds numpy copies of the canonical arrays."""

    def __init__(self, parent: Sequence[int], seg_len: Sequence[int], group_block_size: Sequence[int],
                 n_q_heads: int, n_kv_heads: int, head_dim: int, dtype: str,
                 seg_flags: Optional[Sequence[int]] = None, free_extents=None, seg_slot_base=None):
        self._h = C.c_void_p()
        self._dev = None
        self._ws = {}
        L = lib()
        p, l, g = _i32(parent), _i32(seg_len), _i32(group_block_size)
        d = TreeDesc()
        d.n_segments = len(p)
        d.parent = p.ctypes.data_as(_I32P)
        d.seg_len = l.ctypes.data_as(_I32P)
        fl = None
        if seg_flags is not None:
            fl = np.ascontiguousarray(np.asarray(seg_flags, dtype=np.uint8))
            d.seg_flags = fl.ctypes.data_as(C.POINTER(C.c_uint8))
        d.group_block_size = g.ctypes.data_as(_I32P)
        d.n_groups = len(g)
        d.n_q_heads, d.n_kv_heads, d.head_dim = int(n_q_heads), int(n_kv_heads), int(head_dim)
        d.dtype = {"f32": PSRL_F32, "bf16": PSRL_BF16}.get(dtype, 99)
        fe = None
        if free_extents is not None:
            fe = _i32(np.asarray(free_extents, dtype=np.int64).reshape(-1))
            d.free_extents = fe.ctypes.data_as(_I32P)
            d.n_free = len(fe) // 2
        sb = None
        if seg_slot_base is not None:
            sb = _i32(seg_slot_base)
            if len(sb) != len(p):
                raise ValueError("seg_slot_base needs one entry per segment")
            d.seg_slot_base = sb.ctypes.data_as(_I32P)
        _check(L.psrl_plan_build(C.byref(d), C.byref(self._h)), "psrl_plan_build")
        self.n_q_heads, self.n_kv_heads, self.head_dim, self.dtype = int(n_q_heads), int(n_kv_heads), int(head_dim), dtype
        v = PlanView()
        _check(L.psrl_plan_view(self._h, C.byref(v)), "psrl_plan_view")
        self.view = self._copy_view(v)

    @staticmethod
    def _copy_view(v: PlanView) -> dict:
        out = {n: int(getattr(v, n)) for n in _VIEW_SCALARS32 + _VIEW_SCALARS64}
        n_seg, n_pages = out["n_seg"], out["n_pages"]
        sizes = {n: n_seg for n in _VIEW_ARRAYS}
        sizes.update(anc_off=n_seg + 1, anc_list=int(v.n_anc), bt_off=n_seg + 1, bt_pages=int(v.n_bt),
                     tok_slot=out["T"], sample_end_seg=out["n_samples"], sample_len=out["n_samples"])
        for n in ("page_seg", "page_bs", "page_valid", "page_pos", "page_refcount", "page_slot"):
            sizes[n] = n_pages
        for n in _VIEW_ARRAYS:
            sz = sizes[n]
            ptr = getattr(v, n)
            out[n] = np.ctypeslib.as_array(ptr, shape=(sz,)).copy() if sz > 0 else np.zeros(0, dtype=np.int32)
        return out

    @property
    def handle(self):
        return self._h

    def schedule(self) -> np.ndarray:
        """Copy of the device work schedule (int32 words) for host-side checks."""
        words, n = _I32P(), C.c_size_t()
        _check(lib().psrl_plan_schedule(self._h, C.byref(words), C.byref(n)), "psrl_plan_schedule")
        return np.ctypeslib.as_array(words, shape=(n.value,)).copy()

    def next_tokens(self):
        """What every query row predicts: (off [T_q + 1], tokens), indices into the tree's tokens in canonical order."""
        off, nxt = _I32P(), _I32P()
        _check(lib().psrl_plan_next_tokens(self._h, C.byref(off), C.byref(nxt)), "psrl_plan_next_tokens")
        o = np.ctypeslib.as_array(off, shape=(self.view["T_q"] + 1,)).copy()
        return o, np.ctypeslib.as_array(nxt, shape=(int(o[-1]),)).copy() if o[-1] else np.zeros(0, dtype=np.int32)

    def device_bytes(self) -> int:
        return int(lib().psrl_plan_device_bytes(self._h))

    def fwd_workspace_bytes(self) -> int:
        return int(lib().psrl_fwd_workspace_bytes(self._h))

    def bwd_workspace_bytes(self) -> int:
        return int(lib().psrl_bwd_workspace_bytes(self._h))

    def upload(self, device="cuda", stream=None):
        """Allocate the device mirror with torch and upload the schedule."""
        import torch

        buf = torch.empty(self.device_bytes() + 256, dtype=torch.uint8, device=device)
        ptr = (buf.data_ptr() + 255) // 256 * 256
        s = _stream_ptr(stream)
        _check(lib().psrl_plan_upload(self._h, C.c_void_p(ptr), self.device_bytes(), s), "psrl_plan_upload")
        self._dev = buf
        return self

    def workspace(self, kind: str, device="cuda"):
        """A cached torch workspace of the right size ('fwd' | 'bwd'); returns (ptr, bytes)."""
        import torch

        need = self.fwd_workspace_bytes() if kind == "fwd" else self.bwd_workspace_bytes()
        key = (kind, str(torch.device(device if self._dev is None else self._dev.device)))
        if key not in self._ws:
            self._ws[key] = torch.empty(need + 256, dtype=torch.uint8, device=device)
        buf = self._ws[key]
        return (buf.data_ptr() + 255) // 256 * 256, need

    def close(self):
        if self._h:
            lib().psrl_plan_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _stream_ptr(stream) -> C.c_void_p:
    if stream is None:
        import torch

        if torch.cuda.is_available():
            return C.c_void_p(torch.cuda.current_stream().cuda_stream)
        return C.c_void_p(0)
    if hasattr(stream, "cuda_stream"):
        return C.c_void_p(stream.cuda_stream)
    return C.c_void_p(int(stream))


def psrl_tree_attn_fwd(plan: Plan, q, k_pool, v_pool, softmax_scale: float, o=None, lse=None, stream=None,
                       workspace=None):
    """Forward.  q [T_q,Hq,d], pools [Hkv,capacity,d] torch CUDA tensors of the
    plan's dtype.  Returns (o, lse); both are allocated with torch if not given."""
    import torch

    V = plan.view
    assert q.is_contiguous() and k_pool.is_contiguous() and v_pool.is_contiguous()
    assert tuple(q.shape) == (V["T_q"], plan.n_q_heads, plan.head_dim), q.shape
    assert k_pool.shape == v_pool.shape and k_pool.shape[0] == plan.n_kv_heads and k_pool.shape[2] == plan.head_dim
    _check_dtype(plan, q, k_pool, v_pool)
    if o is None:
        o = torch.empty_like(q)
    if lse is None:
        lse = torch.empty((plan.n_q_heads, V["T_q"]), dtype=torch.float32, device=q.device)
    ws, wsb = workspace if workspace is not None else plan.workspace("fwd", q.device)
    st = lib().psrl_tree_attn_fwd(plan.handle, q.data_ptr(), k_pool.data_ptr(), v_pool.data_ptr(),
                                  int(k_pool.shape[1]), o.data_ptr(), lse.data_ptr(), float(softmax_scale),
                                  C.c_void_p(ws), wsb, _stream_ptr(stream))
    _check(st, "psrl_tree_attn_fwd")
    return o, lse


def psrl_tree_attn_bwd(plan: Plan, q, k_pool, v_pool, o, lse, d_o, softmax_scale: float, d_q=None, dk_pool=None,
                       dv_pool=None, stream=None, workspace=None):
    """Backward.  Returns (d_q, dk_pool, dv_pool).  dk/dv pools are allocated
    zero-filled if not given (the library itself only writes the plan's pages)."""
    import torch

    _check_dtype(plan, q, k_pool, v_pool, o, d_o)
    assert d_o.is_contiguous() and o.is_contiguous() and lse.is_contiguous()
    if d_q is None:
        d_q = torch.empty_like(q)
    if dk_pool is None:
        dk_pool = torch.zeros_like(k_pool)
    if dv_pool is None:
        dv_pool = torch.zeros_like(v_pool)
    ws, wsb = workspace if workspace is not None else plan.workspace("bwd", q.device)
    st = lib().psrl_tree_attn_bwd(plan.handle, q.data_ptr(), k_pool.data_ptr(), v_pool.data_ptr(),
                                  int(k_pool.shape[1]), o.data_ptr(), lse.data_ptr(), d_o.data_ptr(), d_q.data_ptr(),
                                  dk_pool.data_ptr(), dv_pool.data_ptr(), float(softmax_scale), C.c_void_p(ws), wsb,
                                  _stream_ptr(stream))
    _check(st, "psrl_tree_attn_bwd")
    return d_q, dk_pool, dv_pool


class Workspace:
    """Device memory for a call's temporaries and its status word, for psrl_kv_move, the token log-probabilities, products and the norms'
    gradients (`workspace=`).  status() tells whether a wait inside the kernels gave up; without a workspace of one's own the
    log-probabilities, products and norms make one that is gone when the call returns (or need none), and its status with it.  Calls that
    may overlap on the GPU need workspaces of their own."""

    __slots__ = ("ptr", "nbytes", "_buf", "_home", "_raw")

    def __init__(self, nbytes: int, device="cuda", stream=None, _raw=None):
        """On `stream` of the device (a torch stream), or its current one."""
        import torch

        self.nbytes = nbytes = nbytes if nbytes > 256 else 256
        if stream is None:
            buf = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
        else:
            buf = _new(stream, nbytes + 256, torch.uint8, device)
        self._buf = buf
        self.ptr = (buf.data_ptr() + 255) // 256 * 256
        self._raw = _raw     # stream of the last call
        # the stream that the memory belongs to
        if _raw is None:
            _raw = _cuda()._cuda_getCurrentRawStream(buf.get_device()) if stream is None else stream.cuda_stream
        self._home = _raw

    def __iter__(self):
        return iter((self.ptr, self.nbytes))

    def status(self, stream=None) -> int:
        """PSRL_OK, or PSRL_ERR_TIMEOUT where the last call's results are not to be used (psrl_kv_move: nor its pools).  Waits
        for the stream of that call, or for `stream`: the one that a graph with the call was replayed on."""
        if self._raw is None:
            raise RuntimeError("no call has used this workspace")
        import torch

        with torch.cuda.device(self._buf.device):
            return int(lib().psrl_device_status(self.ptr, self._raw if stream is None else _stream_ptr(stream)))


def _use_workspace(workspace, raw: int, keep, dev: int):
    """(pointer, bytes) of what the caller passed, a Workspace or such a pair, for a call on a stream."""
    if isinstance(workspace, Workspace):
        if workspace._buf.get_device() != dev:
            raise ValueError(f"workspace on {workspace._buf.device}, tensors on cuda:{dev}")
        workspace._raw = raw
        if raw != workspace._home:   # its memory must outlive this call, too
            import torch

            workspace._buf.record_stream(keep or torch.cuda.current_stream(dev))
    ptr, nbytes = workspace
    return ptr, nbytes


def psrl_device_status(plan, kind: str = "fwd", stream=None, device="cuda") -> int:
    """Status of the last attention call of `plan`, or of the last call with a Workspace."""
    if isinstance(plan, Workspace):
        return plan.status(stream)
    ws, _ = plan.workspace(kind, device)
    return int(lib().psrl_device_status(C.c_void_p(ws), _stream_ptr(stream)))


def psrl_tree_attn_bwd_static(plan: Plan, q, k_pool, v_pool, o, lse, d_o, softmax_scale: float, d_q, dk_pool,
                              dv_pool, stream=None) -> int:
    """Backward without any device allocation: for callers that may not touch
    the CUDA allocator (see include/psrl.h).  Unlike psrl_tree_attn_bwd this
    wrapper allocates nothing either, so every output tensor must be passed in.
    The library's built-in scratch array serves as workspace; it is shared by
    all calls on the device, so calls must not overlap on the GPU, and its size
    caps the problem: plan.bwd_workspace_bytes() (header + D, one float per query
    row and head, + slabs of split KV tiles + partial dQ rows) must not exceed
    BWD_STATIC_SCRATCH_BYTES = 16 MiB + 256 (PSRL_ERR_WORKSPACE beyond).
    Returns the device address of the status header (for psrl_device_status)."""
    _check_dtype(plan, q, k_pool, v_pool, o, d_o, d_q, dk_pool, dv_pool)
    ws = C.c_void_p()
    st = lib().psrl_tree_attn_bwd_static(plan.handle, q.data_ptr(), k_pool.data_ptr(), v_pool.data_ptr(),
                                         int(k_pool.shape[1]), o.data_ptr(), lse.data_ptr(), d_o.data_ptr(),
                                         d_q.data_ptr(), dk_pool.data_ptr(), dv_pool.data_ptr(),
                                         float(softmax_scale), C.byref(ws), _stream_ptr(stream))
    _check(st, "psrl_tree_attn_bwd_static")
    return int(ws.value or 0)


def psrl_bench_bwd_phases(plan: Plan, q, k_pool, v_pool, o, lse, d_o, softmax_scale: float, d_q, dk_pool, dv_pool,
                          phases: int, stream=None, workspace=None):
    """Benchmark aid: the backward with a mask of the kernels to launch (bit 0 D pre-pass, bit 1 dQ,
    bit 2 dK/dV), so that each can be timed on its own.  Outputs must be passed in."""
    _check_dtype(plan, q, k_pool, v_pool, o, d_o, d_q, dk_pool, dv_pool)
    ws, wsb = workspace if workspace is not None else plan.workspace("bwd", q.device)
    st = lib().psrl_bench_bwd_phases(plan.handle, q.data_ptr(), k_pool.data_ptr(), v_pool.data_ptr(),
                                     int(k_pool.shape[1]), o.data_ptr(), lse.data_ptr(), d_o.data_ptr(),
                                     d_q.data_ptr(), dk_pool.data_ptr(), dv_pool.data_ptr(), float(softmax_scale),
                                     C.c_void_p(ws), wsb, _stream_ptr(stream), int(phases))
    _check(st, "psrl_bench_bwd_phases")


def psrl_kv_scatter(plan: Plan, k_tok, v_tok, k_pool, v_pool, stream=None):
    """Token-major K, V [T, Hkv, d] -> slots tok_slot[t] of the pools [Hkv, capacity, d] (in place)."""
    _check_dtype(plan, k_tok, v_tok, k_pool, v_pool)
    T, Hkv, d = plan.view["T"], plan.n_kv_heads, plan.head_dim
    for t in (k_tok, v_tok):
        if tuple(t.shape) != (T, Hkv, d) or not t.is_contiguous():
            raise ValueError("k_tok / v_tok must be contiguous [T, Hkv, d]")
    if k_pool.shape != v_pool.shape or k_pool.shape[0] != Hkv or k_pool.shape[2] != d or not k_pool.is_contiguous():
        raise ValueError("pools must be contiguous [Hkv, capacity, d]")
    _check(lib().psrl_kv_scatter(plan._h, k_tok.data_ptr(), v_tok.data_ptr(), k_pool.data_ptr(), v_pool.data_ptr(),
                                 int(k_pool.shape[1]), _stream_ptr(stream)), "psrl_kv_scatter")


def psrl_kv_gather(plan: Plan, k_pool, v_pool, k_tok=None, v_tok=None, stream=None):
    """The inverse read: pools -> token-major [T, Hkv, d] (e.g. dK, dV back to the projections)."""
    import torch

    _check_dtype(plan, k_pool, v_pool)
    T, Hkv, d = plan.view["T"], plan.n_kv_heads, plan.head_dim
    if k_tok is None:
        k_tok = torch.empty((T, Hkv, d), dtype=k_pool.dtype, device=k_pool.device)
    if v_tok is None:
        v_tok = torch.empty((T, Hkv, d), dtype=v_pool.dtype, device=v_pool.device)
    _check(lib().psrl_kv_gather(plan._h, k_pool.data_ptr(), v_pool.data_ptr(), int(k_pool.shape[1]), k_tok.data_ptr(),
                                v_tok.data_ptr(), _stream_ptr(stream)), "psrl_kv_gather")
    return k_tok, v_tok


def _device_of(*tensors) -> int:
    """The CUDA device that all the tensors of a call live on."""
    dev = tensors[0].get_device()
    if dev < 0:
        raise RuntimeError("tensors must live on a CUDA device: this library has no CPU path")
    for t in tensors:
        if t.get_device() != dev:
            raise ValueError(f"tensors on {t.device} and {tensors[0].device}: one call works on one device")
    return dev


_torch_c = None


def _cuda():
    """torch's C module, looked up once: small calls are bound by the host's time."""
    global _torch_c
    if _torch_c is None:
        import torch

        _torch_c = torch._C
    return _torch_c


_torch_calls = None


def _calls():
    """The module of csrc/torch_calls.cpp: the plain case of the calls below in one step (checks, outputs, C call).  It answers None
    for any other case, which then takes the way through this file, and a status where the library refuses."""
    global _torch_calls
    if _torch_calls is None:
        lib()
        import torch  # noqa: F401  (its libraries)

        try:
            from . import _torch_calls as m
        except ImportError as e:
            raise RuntimeError(f"{_HERE}/_torch_calls.so cannot be loaded ({e}): build it with `python -m paper_2608_25683_b200.build`") from e
        _torch_calls = m
    return _torch_calls


def _answer(r, name: str):
    """The outputs, or the library's refusal."""
    if type(r) is not tuple:
        _check(r, name)
    return r


_torch_module = None


def _torch():
    """torch, looked up once."""
    global _torch_module
    if _torch_module is None:
        import torch

        _torch_module = torch
    return _torch_module


def _scratch(nbytes: int, keep, like):
    """(address, bytes, tensor that holds them until the call is on its stream) of a call's own workspace."""
    if keep is None:
        buf = like.new_empty(((nbytes + 256) // like.element_size() + 1,))
    else:
        buf = _new(keep, nbytes + 256, _torch().uint8, like.device)
    return (buf.data_ptr() + 255) // 256 * 256, nbytes, buf


@functools.lru_cache(maxsize=4096)
def _workspace_bytes(name: str, dev: int, *args) -> int:
    """What the library asks for a call of these sizes on device `dev`, asked once with that device as the current one: some sizes go by its
    number of SMs."""
    fn = getattr(lib(), name)
    if dev == _cuda()._cuda_getDevice():
        return int(fn(*args))
    with _torch().cuda.device(dev):
        return int(fn(*args))


_type_codes = None


def _type_code(t):
    """PSRL_F32, PSRL_BF16 or None."""
    global _type_codes
    codes = _type_codes
    if codes is None:
        import torch

        codes = _type_codes = {torch.float32: PSRL_F32, torch.bfloat16: PSRL_BF16}
    return codes.get(t.dtype)


def _stream_on(stream, dev: int):
    """(raw stream handle of a call on device `dev`, torch stream to keep temporaries for or None).  Without a stream it is
    torch's current one of that device; the raw handle skips a Stream object, a third of a small call's host time."""
    if stream is None:
        return (_torch_c or _cuda())._cuda_getCurrentRawStream(dev), None
    import torch

    if not hasattr(stream, "cuda_stream"):
        stream = torch.cuda.ExternalStream(int(stream), device=dev)
    elif stream.device.index != dev:
        raise ValueError(f"stream of {stream.device} for tensors on cuda:{dev}")
    return stream.cuda_stream, stream


def _new(stream, shape, dtype, device):
    """A tensor made for a call.  With a stream of its own the call's tensors come from that stream's memory: memory that
    the current stream gave back may still be in use there."""
    import torch

    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _launch(name: str, dev: int, *args):
    """One C call with the tensors' device as the current one: the library launches there."""
    fn = getattr(_lib or lib(), name)
    if dev == (_torch_c or _cuda())._cuda_getDevice():
        st = fn(*args)
    else:
        import torch

        with torch.cuda.device(dev):
            st = fn(*args)
    if st != PSRL_OK:
        _check(st, name)


_ROPE_LAYOUTS = {"half": 0, "interleaved": 1}
_ROPE_ORDERS = {"blocks": 0, "cyclic": 1}
_ROPE_SCALINGS = {None: 0, "none": 0, "linear": 1, "ntk": 2, "yarn": 3, "banded": 4}


class Rope:
    """Owner of a psrl_rope_t: a rotary position embedding (include/psrl.h has the formulas).  `freq` holds the radians
    per position of each pair, `scale` the factor on cos and sin.  low / high / attention_scale 0: the defaults.
    `sections` = [pairs of axis 0, of axis 1, ...]: several axes (time, height, width), with the pairs of an axis in "blocks" or
    going round them in turn ("cyclic")."""

    def __init__(self, head_dim: int, rotary_dim: int = 0, base: float = 10000.0, layout: str = "half",
                 scaling: Optional[str] = None, factor: float = 1.0, original_positions: int = 0, low: float = 0.0,
                 high: float = 0.0, attention_scale: float = 0.0, sections: Optional[Sequence[int]] = None, order: str = "blocks"):
        self._h = C.c_void_p()
        self._destroy = lib().psrl_rope_destroy
        if layout not in _ROPE_LAYOUTS or scaling not in _ROPE_SCALINGS or order not in _ROPE_ORDERS:
            raise ValueError(f"layout {layout!r}, scaling {scaling!r} or order {order!r} unknown")
        d = RopeDesc(int(head_dim), int(rotary_dim or head_dim), _ROPE_LAYOUTS[layout], _ROPE_SCALINGS[scaling], float(base),
                     float(factor), int(original_positions), float(low), float(high), float(attention_scale))
        if sections is None:
            _check(lib().psrl_rope_create(C.byref(d), C.byref(self._h)), "psrl_rope_create")
        else:
            parts = _i32(sections)
            _check(lib().psrl_rope_create_axes(C.byref(d), len(parts), parts.ctypes.data_as(_I32P), _ROPE_ORDERS[order],
                                               C.byref(self._h)), "psrl_rope_create_axes")
        self.n_axes = 1 if sections is None else len(parts)
        f, n, sc = C.POINTER(C.c_double)(), C.c_int32(), C.c_double()
        _check(lib().psrl_rope_frequencies(self._h, C.byref(f), C.byref(n), C.byref(sc)), "psrl_rope_frequencies")
        self.head_dim, self.rotary_dim = d.head_dim, d.rotary_dim
        self.freq, self.scale = np.ctypeslib.as_array(f, shape=(n.value,)).copy(), float(sc.value)

    def __del__(self):
        if getattr(self, "_h", None) and self._h.value:
            self._destroy(self._h)      # held by the object: at the interpreter's end this module's names may be gone
            self._h.value = None


def _rows_pitch(t, rows: int, heads: int, d: int, name: str) -> int:
    """Row pitch in elements of a [rows, heads, d] tensor whose rows may be slices of a wider matrix."""
    if t.shape != (rows, heads, d):
        raise ValueError(f"{name} must be [{rows}, {heads}, {d}], got {tuple(t.shape)}")
    if t.is_contiguous():
        return heads * d
    s = t.stride()
    if (s[2] != 1 and d > 1) or (s[1] != d and heads > 1):
        raise ValueError(f"{name}: the heads of a row must be contiguous")
    return s[0] if rows > 1 else heads * d


def _plan_device(plan, dev: int):
    if plan._dev is not None and plan._dev.get_device() != dev:
        raise ValueError(f"the plan was uploaded to {plan._dev.device}, the tensors live on cuda:{dev}")


def _rope_pools(plan, *pools):
    shape = pools[0].shape
    if len(shape) == 3 and shape[0] == plan.n_kv_heads and shape[2] == plan.head_dim:
        for p in pools:
            if p.shape != shape or not p.is_contiguous():
                break
        else:
            return shape[1]
    raise ValueError("pools must be contiguous [Hkv, capacity, d]")


def psrl_rope_qkv_fwd(plan: Plan, rope: Rope, q, k, v, k_pool, v_pool, q_out=None, stream=None):
    """Rotates the query rows' Q [T_q, Hq, d] into q_out and their K, V [T_q, Hkv, d] into the pools (K rotated), in one
    launch.  q, k, v may be slices of one projection output (rows at any pitch).  Returns q_out."""
    return _rope_qkv_fwd("psrl_rope_qkv_fwd", plan, rope, None, q, k, v, k_pool, v_pool, q_out, stream)


def psrl_rope_axes_qkv_fwd(plan: Plan, rope: Rope, positions, q, k, v, k_pool, v_pool, q_out=None, stream=None):
    """The same with int32 `positions` [axes, T_q] of the caller's own, a row for each axis of the rope."""
    if stream is None and plan._dev is not None and plan._dev.get_device() == q.get_device():
        r = (_torch_calls or _calls()).rope_axes_qkv_fwd(*_tree_args(plan, rope), positions, q, k, v, k_pool, v_pool, q_out)
        if r is not None:
            _answer(r, "psrl_rope_axes_qkv_fwd")
            return r[0] if q_out is None else q_out
    return _rope_qkv_fwd("psrl_rope_axes_qkv_fwd", plan, rope, positions, q, k, v, k_pool, v_pool, q_out, stream)


def psrl_rope_qkv_bwd(plan: Plan, rope: Rope, d_q, dk_pool, dv_pool, dq_out=None, dk_out=None, dv_out=None, stream=None):
    """The way back: inverse rotation of d_q and of the query rows' slots of dk_pool, and the rows' slots of dv_pool, to
    dq_out [T_q, Hq, d], dk_out, dv_out [T_q, Hkv, d] (which may be slices of one gradient matrix).  Returns the three."""
    return _rope_qkv_bwd("psrl_rope_qkv_bwd", plan, rope, None, d_q, dk_pool, dv_pool, dq_out, dk_out, dv_out, stream)


def psrl_rope_axes_qkv_bwd(plan: Plan, rope: Rope, positions, d_q, dk_pool, dv_pool, dq_out=None, dk_out=None, dv_out=None, stream=None):
    """The same with int32 `positions` [axes, T_q], as in the forward."""
    if stream is None and plan._dev is not None and plan._dev.get_device() == d_q.get_device():
        r = (_torch_calls or _calls()).rope_axes_qkv_bwd(*_tree_args(plan, rope), positions, d_q, dk_pool, dv_pool, dq_out, dk_out, dv_out)
        if r is not None:
            return _answer(r, "psrl_rope_axes_qkv_bwd")
    return _rope_qkv_bwd("psrl_rope_axes_qkv_bwd", plan, rope, positions, d_q, dk_pool, dv_pool, dq_out, dk_out, dv_out, stream)


def _tree_args(plan: Plan, rope: Rope):
    """Handles and sizes as rope calls of csrc/torch_calls.cpp take them; None where there is no handle any more."""
    return (plan._h.value, rope._h.value, rope.n_axes, PSRL_F32 if plan.dtype == "f32" else PSRL_BF16, plan.view["T_q"], plan.n_q_heads, plan.n_kv_heads,
            plan.head_dim)


def _axis_pitch(rope: Rope, positions, rows: int) -> int:
    """Elements between two axes' positions."""
    if positions.dtype is _torch().int32 and positions.shape == (rope.n_axes, rows):
        if positions.is_contiguous():
            return rows
        if rows <= 1 or positions.stride(1) == 1:
            return positions.stride(0) if rope.n_axes > 1 else rows
    raise ValueError(f"positions must be int32 [{rope.n_axes}, {rows}], the rows of an axis contiguous")


def _rope_qkv_fwd(name, plan, rope, positions, q, k, v, k_pool, v_pool, q_out, stream):
    V, d, hkv = plan.view, plan.head_dim, plan.n_kv_heads
    _check_dtype(plan, q, k, v, k_pool, v_pool)
    pq = _rows_pitch(q, V["T_q"], plan.n_q_heads, d, "q")
    pk, pv = _rows_pitch(k, V["T_q"], hkv, d, "k"), _rows_pitch(v, V["T_q"], hkv, d, "v")
    cap = _rope_pools(plan, k_pool, v_pool)
    at = () if positions is None else (positions.data_ptr(), _axis_pitch(rope, positions, V["T_q"]))
    dev = _device_of(q, k, v, k_pool, v_pool, *(() if positions is None else (positions,)))
    _plan_device(plan, dev)
    raw, keep = _stream_on(stream, dev)
    if q_out is None:
        q_out = _new(keep, (V["T_q"], plan.n_q_heads, d), q.dtype, q.device)
    else:
        _check_dtype(plan, q_out)
        if q_out.shape != q.shape or not q_out.is_contiguous() or q_out.device != q.device:
            raise ValueError("q_out must be contiguous [T_q, Hq, d] on the same device")
    _launch(name, dev, plan._h, rope._h, *at, q.data_ptr(), pq, k.data_ptr(), pk, v.data_ptr(), pv,
            q_out.data_ptr(), k_pool.data_ptr(), v_pool.data_ptr(), cap, raw)
    return q_out


def _rope_qkv_bwd(name, plan, rope, positions, d_q, dk_pool, dv_pool, dq_out, dk_out, dv_out, stream):
    V, d = plan.view, plan.head_dim
    _check_dtype(plan, d_q, dk_pool, dv_pool)
    if d_q.shape != (V["T_q"], plan.n_q_heads, d) or not d_q.is_contiguous():
        raise ValueError("d_q must be contiguous [T_q, Hq, d]")
    cap = _rope_pools(plan, dk_pool, dv_pool)
    at = () if positions is None else (positions.data_ptr(), _axis_pitch(rope, positions, V["T_q"]))
    dev = _device_of(d_q, dk_pool, dv_pool, *(() if positions is None else (positions,)))
    _plan_device(plan, dev)
    raw, keep = _stream_on(stream, dev)
    outs, pitch = [], []
    for t, heads, which in ((dq_out, plan.n_q_heads, "dq_out"), (dk_out, plan.n_kv_heads, "dk_out"), (dv_out, plan.n_kv_heads, "dv_out")):
        if t is None:
            t = _new(keep, (V["T_q"], heads, d), d_q.dtype, d_q.device)
        else:
            _check_dtype(plan, t)
            if t.device != d_q.device:
                raise ValueError(f"{which} lives on another device")
        outs.append(t)
        pitch.append(_rows_pitch(t, V["T_q"], heads, d, which))
    _launch(name, dev, plan._h, rope._h, *at, d_q.data_ptr(), dk_pool.data_ptr(), dv_pool.data_ptr(), cap,
            outs[0].data_ptr(), pitch[0], outs[1].data_ptr(), pitch[1], outs[2].data_ptr(),
            pitch[2], raw)
    return tuple(outs)


def psrl_rope_rows(rope: Rope, x, positions, y=None, inverse: bool = False, stream=None):
    """Rotates x [rows, heads, head_dim] (f32 or bf16, rows at any pitch) at int32 `positions` [rows].  Returns y (y may be x)."""
    if positions.dtype is not _torch().int32 or positions.shape != x.shape[:1] or not positions.is_contiguous():
        raise ValueError("positions must be contiguous int32 [rows]")
    return _rope_rows("psrl_rope_rows", rope, x, positions, (), y, inverse, stream)


def psrl_rope_axes_rows(rope: Rope, x, positions, y=None, inverse: bool = False, stream=None):
    """The same at `positions` [axes, rows], a row for each axis of the rope."""
    if stream is None and y is None:
        r = (_torch_calls or _calls()).rope_axes_rows(rope._h.value, rope.n_axes, rope.head_dim, x, positions, inverse)
        if r is not None:
            return _answer(r, "psrl_rope_axes_rows")[0]
    return _rope_rows("psrl_rope_axes_rows", rope, x, positions, (_axis_pitch(rope, positions, x.shape[0]),), y, inverse, stream)


def _rope_rows(name, rope, x, positions, axis_pitch, y, inverse, stream):
    dt = _type_code(x)
    if dt is None:
        raise TypeError(f"dtype {x.dtype} is neither float32 nor bfloat16")
    shape = x.shape
    if len(shape) != 3:
        raise ValueError("x must be [rows, heads, head_dim]")
    rows, heads, _ = shape
    _int32(heads)
    px = _rows_pitch(x, rows, heads, rope.head_dim, "x")
    dev = _device_of(x, positions)
    raw, keep = _stream_on(stream, dev)
    if y is None:
        y, py = _like(x, keep), heads * rope.head_dim
    elif y.dtype is not x.dtype or y.get_device() != dev:
        raise ValueError("y must have x's type and device")
    else:
        py = px if y is x else _rows_pitch(y, rows, heads, rope.head_dim, "y")
    _launch(name, dev, rope._h, dt, x.data_ptr(), px, positions.data_ptr(), *axis_pitch, rows, heads, y.data_ptr(), py, 1 if inverse else 0, raw)
    return y


def _extents(extents):
    """[n, 3] int32 (source slot, destination slot, slots), kept alive by the caller, and its address."""
    e = np.asarray(extents)
    if e.dtype != np.int32:
        if e.size and (e.dtype.kind not in "iu" or int(e.min()) < -2 ** 31 or int(e.max()) >= 2 ** 31):
            raise ValueError("extents must be 32-bit integers")
        e = e.astype(np.int32)
    e = np.ascontiguousarray(e)
    if e.size == 0:
        return e, 0, None
    if e.ndim != 2 or e.shape[1] != 3:
        raise ValueError("extents must be [n, 3]: source slot, destination slot, slots")
    return e, len(e), e.__array_interface__["data"][0]


def _pair_of_pools(k, v, what: str):
    """(heads, capacity, bytes of a slot and head) of two pools of one shape."""
    shape, size = k.shape, k.element_size()
    if _type_code(k) is None or v.dtype is not k.dtype:
        raise TypeError(f"{what} must both be float32 or both bfloat16")
    if len(shape) != 3 or shape != v.shape or not k.is_contiguous() or not v.is_contiguous():
        raise ValueError(f"{what} must be contiguous [Hkv, capacity, d] of one shape")
    return shape[0], shape[1], shape[2] * size


def psrl_kv_copy(extents, k_src, v_src, k_dst, v_dst, stream=None):
    """Copies extents [n, 3] (source slot, destination slot, slots) of all heads from the pools k_src, v_src
    [Hkv, capacity, d] to k_dst, v_dst (another capacity is fine).  Destinations must not overlap one another, nor, inside
    one pool, any source."""
    heads, cap, row = _pair_of_pools(k_src, v_src, "source pools")
    heads2, cap2, row2 = _pair_of_pools(k_dst, v_dst, "destination pools")
    if heads != heads2 or row != row2 or k_src.dtype != k_dst.dtype:
        raise ValueError("source and destination pools differ in heads, head dimension or type")
    e, n, at = _extents(extents)
    dev = _device_of(k_src, v_src, k_dst, v_dst)
    raw, keep = _stream_on(stream, dev)
    _launch("psrl_kv_copy", dev, at, n, heads, row, k_src.data_ptr(), v_src.data_ptr(), cap, k_dst.data_ptr(),
            v_dst.data_ptr(), cap2, raw)


def psrl_kv_move(moves, k_pool, v_pool, stream=None, workspace=None):
    """Performs the moves of a compaction ([n, 3], ascending, downwards: Cache.compact()) inside the pools, as if every
    source were read first.  `workspace`: a Workspace, or (pointer, bytes) of 256 bytes of device memory; made if not given.
    Returns the workspace; its status() tells whether the move came to its end (a wait that gave up leaves the pools half
    moved)."""
    heads, cap, row = _pair_of_pools(k_pool, v_pool, "pools")
    e, n, at = _extents(moves)
    dev = _device_of(k_pool, v_pool)
    raw, keep = _stream_on(stream, dev)
    if workspace is None:
        workspace = Workspace(256, k_pool.device, keep, raw)
        ws, wsb = workspace.ptr, 256
    else:
        ws, wsb = _use_workspace(workspace, raw, keep, dev)
    _launch("psrl_kv_move", dev, at, n, heads, row, k_pool.data_ptr(), v_pool.data_ptr(), cap, ws, wsb, raw)
    return workspace


def psrl_token_logprob_workspace_bytes(n_rows: int, hidden_dim: int, vocab: int, n_targets: int, backward: bool,
                                       dtype: str = "bf16") -> int:
    return int(lib().psrl_token_logprob_workspace_bytes(PSRL_F32 if dtype == "f32" else PSRL_BF16, int(n_rows), int(hidden_dim), int(vocab), int(n_targets),
                                                        int(bool(backward))))


def _logprob_args(hidden, weight, targets, target_off, floats):
    """Checks shared by the two directions; the shape arguments of the C call."""
    import torch

    dt = _type_code(hidden)
    if dt is None or weight.dtype is not hidden.dtype:
        raise TypeError("hidden and weight must both be bfloat16 or both float32")
    if hidden.dim() != 2 or weight.dim() != 2 or hidden.shape[1] != weight.shape[1]:
        raise ValueError("hidden must be [rows, hidden_dim], weight [vocab, hidden_dim]")
    n, h = hidden.shape
    _int32(h, weight.shape[0])
    for name, t, count in [("targets", targets, None), ("target_off", target_off, n + 1)]:
        if t is not None and (t.dtype != torch.int32 or t.dim() != 1 or not t.is_contiguous() or (count and t.shape[0] != count)):
            raise ValueError(f"{name} must be a contiguous int32 vector" + (f" of {count}" if count else ""))
    for name, t, count in floats:
        if t is not None and (t.dtype != torch.float32 or tuple(t.shape) != (count,) or not t.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous float32 vector of {count}")
    return dt, n, h, weight.shape[0], targets.shape[0]


def _matrix_pitch(t, name: str) -> int:
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{name}: the elements of a row must be contiguous")
    return t.stride(0) if t.shape[0] > 1 else -(-t.shape[1] // 8) * 8   # one row: any pitch will do


def _logprob_workspace(workspace, raw, keep, dt, n, h, v, m, backward, device):
    """(pointer, bytes, what holds the memory until the call is on its stream)"""
    if workspace is None:
        workspace = Workspace(_workspace_bytes("psrl_token_logprob_workspace_bytes", device.index, dt, n, h, v, m, int(backward)), device, keep, raw)
        return workspace.ptr, workspace.nbytes, workspace
    return (*_use_workspace(workspace, raw, keep, device.index), workspace)


def psrl_token_logprob_fwd(hidden, weight, targets, target_off=None, scale: float = 1.0, logprob=None, lse=None, stream=None,
                           workspace=None):
    """Log-probabilities of `targets` (int32) under softmax(scale * hidden weight^T), without storing the logits.  hidden
    [rows, H], weight [vocab, H], both bf16 or both f32; row r's targets are targets[target_off[r] : target_off[r + 1]], or targets[r] without
    target_off.  `workspace`: a Workspace of psrl_token_logprob_workspace_bytes(), whose status() tells whether a wait inside
    the kernels gave up; made if not given.  Returns (logprob [targets], lse [rows]), fp32."""
    import torch

    dt, n, h, v, m = _logprob_args(hidden, weight, targets, target_off, [])
    _logprob_args(hidden, weight, targets, target_off, [("logprob", logprob, m), ("lse", lse, n)])
    given = [t for t in (target_off, logprob, lse) if t is not None]
    dev = _device_of(hidden, weight, targets, *given)
    raw, keep = _stream_on(stream, dev)
    if logprob is None:
        logprob = _new(keep, m, torch.float32, hidden.device)
    if lse is None:
        lse = _new(keep, n, torch.float32, hidden.device)
    ws, wsb, held = _logprob_workspace(workspace, raw, keep, dt, n, h, v, m, False, hidden.device)
    _launch("psrl_token_logprob_fwd", dev, dt, n, h, v, hidden.data_ptr(), _matrix_pitch(hidden, "hidden"), weight.data_ptr(),
            _matrix_pitch(weight, "weight"), targets.data_ptr(), m,
            None if target_off is None else target_off.data_ptr(), float(scale), logprob.data_ptr(),
            lse.data_ptr(), ws, wsb, raw)
    return logprob, lse


def psrl_token_logprob_bwd(hidden, weight, targets, logprob, lse, d_logprob, target_off=None, scale: float = 1.0, d_hidden=None,
                           d_weight=None, want_hidden: bool = True, want_weight: bool = True, stream=None, workspace=None):
    """Gradients of the above: (d_hidden, d_weight), of hidden's type, given d_logprob [targets] and the forward's logprob and lse.
    want_hidden / want_weight False: that one is None and not computed.  `workspace` as above (backward True)."""
    m = targets.shape[0]
    dt, n, h, v, m = _logprob_args(hidden, weight, targets, target_off,
                                   [("logprob", logprob, m), ("lse", lse, hidden.shape[0]), ("d_logprob", d_logprob, m)])
    for name, t, like in (("d_hidden", d_hidden, hidden), ("d_weight", d_weight, weight)):
        if t is not None and (t.dtype is not hidden.dtype or t.shape != like.shape):
            raise ValueError(f"{name} must be {hidden.dtype} {tuple(like.shape)}")
    given = [t for t in (target_off, d_hidden, d_weight) if t is not None]
    dev = _device_of(hidden, weight, targets, logprob, lse, d_logprob, *given)
    raw, keep = _stream_on(stream, dev)
    if d_hidden is None and want_hidden:
        d_hidden = _new(keep, (n, h), hidden.dtype, hidden.device)
    if d_weight is None and want_weight:
        d_weight = _new(keep, (v, h), hidden.dtype, hidden.device)
    out = [t if w else None for t, w in ((d_hidden, want_hidden), (d_weight, want_weight))]
    ws, wsb, held = _logprob_workspace(workspace, raw, keep, dt, n, h, v, m, True, hidden.device)
    args = [x for t, name in zip(out, ("d_hidden", "d_weight"))
            for x in ((None, 0) if t is None else (t.data_ptr(), _matrix_pitch(t, name)))]
    _launch("psrl_token_logprob_bwd", dev, dt, n, h, v, hidden.data_ptr(), _matrix_pitch(hidden, "hidden"), weight.data_ptr(),
            _matrix_pitch(weight, "weight"), targets.data_ptr(), m,
            None if target_off is None else target_off.data_ptr(), float(scale), logprob.data_ptr(),
            lse.data_ptr(), d_logprob.data_ptr(), *args, ws, wsb, raw)
    return tuple(out)


def _int32(*sizes):
    """Sizes that the library takes in 32 bits; ctypes would cut larger ones off without a word."""
    for n in sizes:
        if n > 0x7fffffff:
            raise ValueError(f"{n} is beyond the library's dimensions")


def _stream_rows(t, shape, name: str, like=None) -> int:
    """Row pitch of a [rows, dim] or [rows, heads, dim] tensor of `shape`, of the type and on the device of `like`."""
    if t.shape != shape or (like is not None and (t.dtype is not like.dtype or t.get_device() != like.get_device())):
        raise ValueError(f"{name} must be {tuple(shape)}" + (f" of {like.dtype} on {like.device}" if like is not None else ""))
    if t.is_contiguous():
        return shape[1] if len(shape) == 2 else shape[1] * shape[2]
    if len(shape) == 2:
        return _matrix_pitch(t, name)
    return _rows_pitch(t, shape[0], shape[1], shape[2], name)


def _like(t, keep):
    """A contiguous tensor of t's shape, type and device, made for a call."""
    if keep is not None:
        return _new(keep, t.shape, t.dtype, t.device)
    return _torch().empty_like(t) if t.is_contiguous() else t.new_empty(t.shape)


def _norm_args(x, weight):
    """(type, rows, heads, dim, device) of the rows to be normed; weight fits them."""
    dt, shape = _type_code(x), x.shape
    if dt is None:
        raise TypeError(f"dtype {x.dtype} is neither float32 nor bfloat16")
    if len(shape) == 2:
        (rows, dim), heads = shape, 1
    elif len(shape) == 3:
        rows, heads, dim = shape
    else:
        raise ValueError("rows must be [rows, dim] or [rows, heads, dim]")
    _int32(heads, dim)
    dev = x.get_device()
    if dev < 0:
        raise RuntimeError("tensors must live on a CUDA device: this library has no CPU path")
    if weight is not None:
        if weight.dtype is not x.dtype:
            raise TypeError(f"weight is {weight.dtype}, the rows are {x.dtype}")
        if weight.shape != (dim,) or weight.get_device() != dev or not weight.is_contiguous():
            raise ValueError(f"weight must be a contiguous vector of {dim} on {x.device}")
    return dt, rows, heads, dim, dev


def _codes_rows(codes, shape, keep, like, name="codes"):
    """(tensor of 8-bit codes of `shape`, row pitch), made if not given: rows 16 bytes or a multiple apart."""
    rows, least = shape[0], shape[1] if len(shape) == 2 else shape[1] * shape[2]
    pitch = -(-least // 16) * 16
    if codes is None:
        if pitch == least:
            if keep is None and like.is_contiguous():
                t = _torch()
                return t.empty_like(like, dtype=t.float8_e4m3fn), pitch
            return _new(keep, shape, _torch().float8_e4m3fn, like.device), pitch
        codes = _new(keep, (rows, pitch), _torch().float8_e4m3fn, like.device)[:, :least]
        return codes.unflatten(1, shape[1:]) if len(shape) == 3 else codes, pitch
    if codes.dtype is not _torch().float8_e4m3fn or codes.get_device() != like.get_device():
        raise ValueError(f"{name} must be float8_e4m3fn on {like.device}")
    at = _stream_rows(codes, shape, name)
    return codes, at if rows > 1 else pitch


def _floats(t, shape, keep, device, name):
    """A contiguous float32 tensor of `shape`, made if not given."""
    if t is None:
        return _new(keep, shape, _torch().float32, device)
    if t.dtype is not _torch().float32 or t.shape != shape or not t.is_contiguous() or t.device != device:
        raise ValueError(f"{name} must be contiguous float32 {tuple(shape)} on {device}")
    return t


def psrl_rms_norm_fwd(x, weight, eps: float = 1e-6, residual=None, y=None, summed=None, codes=None, scales=None, want_y: bool = True,
                      want_codes: bool = False, stream=None):
    """Root-mean-square norm of h = x + residual: x [rows, dim], or [rows, heads, dim] with a norm for each head (f32 or bf16, rows
    at any pitch), weight [dim] or None.  Returns (y, summed, codes, scales): summed = h where there is a residual, codes and scales
    the rows in 8 bits (float8_e4m3fn, a float32 scale for each) with want_codes; what is not wanted is None.  Outputs may be inputs."""
    if stream is None and y is None and summed is None and codes is None and scales is None:
        r = (_torch_calls or _calls()).rms_norm_fwd(x, weight, eps, residual, want_y, want_codes)
        if r is not None:
            return _answer(r, "psrl_rms_norm_fwd")
    dt, rows, heads, dim, dev = _norm_args(x, weight)
    shape, least = x.shape, heads * dim
    raw, keep = _stream_on(stream, dev)
    px = _stream_rows(x, shape, "x")
    a_res, p_res, a_sum, p_sum, a_y, p_y, a_c, p_c, a_s = None, 0, None, 0, None, 0, None, 0, None
    if residual is not None:
        a_res, p_res = residual.data_ptr(), _stream_rows(residual, shape, "residual", x)
        if summed is None:
            summed, p_sum = _like(x, keep), least
        else:
            p_sum = _stream_rows(summed, shape, "summed", x)
        a_sum = summed.data_ptr()
    elif summed is not None:
        raise ValueError("summed without a residual: x itself is the stream")
    if not want_y:
        y = None
    else:
        if y is None:
            y, p_y = _like(x, keep), least
        else:
            p_y = _stream_rows(y, shape, "y", x)
        a_y = y.data_ptr()
    if want_codes:
        codes, p_c = _codes_rows(codes, shape, keep, x)
        scales = _floats(scales, shape[:-1], keep, x.device, "scales")
        a_c, a_s = codes.data_ptr(), scales.data_ptr()
    else:
        codes = scales = None
    _launch("psrl_rms_norm_fwd", dev, dt, rows, heads, dim, x.data_ptr(), px, a_res, p_res, None if weight is None else weight.data_ptr(),
            eps, a_sum, p_sum, a_y, p_y, a_c, p_c, a_s, raw)
    return y, summed, codes, scales


def psrl_rms_norm_workspace_bytes(n_rows: int, n_heads: int, dim: int, dtype: str = "bf16") -> int:
    return int(lib().psrl_rms_norm_workspace_bytes(PSRL_F32 if dtype == "f32" else PSRL_BF16, int(n_rows), int(n_heads), int(dim)))


def psrl_rms_norm_bwd(summed, weight, d_y, eps: float = 1e-6, d_summed=None, d_x=None, d_weight=None, want_x: bool = True,
                      want_weight: bool = True, stream=None, workspace=None):
    """Gradients of the above: (d_x, d_weight) given the rows h that were normed (the forward's `summed`, or its x), d_y and, with a
    residual, the gradient d_summed that the stream brings back; d_x is the gradient of x and of residual.  d_x may be d_y or
    d_summed.  `workspace`: a Workspace of psrl_rms_norm_workspace_bytes(); made if not given."""
    if stream is None and d_x is None and d_weight is None and workspace is None:
        r = (_torch_calls or _calls()).rms_norm_bwd(summed, weight, d_y, eps, d_summed, want_x, want_weight)
        if r is not None:
            return _answer(r, "psrl_rms_norm_bwd")
    dt, rows, heads, dim, dev = _norm_args(summed, weight)
    shape = summed.shape
    raw, keep = _stream_on(stream, dev)
    ph, pd = _stream_rows(summed, shape, "summed"), _stream_rows(d_y, shape, "d_y", summed)
    a_s, p_s, a_x, p_x = None, 0, None, 0
    if d_summed is not None:
        a_s, p_s = d_summed.data_ptr(), _stream_rows(d_summed, shape, "d_summed", summed)
    if not want_x:
        d_x = None
    else:
        if d_x is None:
            d_x, p_x = _like(d_y, keep), heads * dim
        else:
            p_x = _stream_rows(d_x, shape, "d_x", summed)
        a_x = d_x.data_ptr()
    if not want_weight or weight is None:
        d_weight = None
    elif d_weight is None:
        d_weight = _like(weight, keep)
    elif d_weight.dtype is not weight.dtype or d_weight.shape != weight.shape or not d_weight.is_contiguous() or d_weight.get_device() != dev:
        raise ValueError(f"d_weight must be a contiguous vector of {dim}, {weight.dtype} on {weight.device}")
    if workspace is None:
        ws, wsb, held = None, 0, None
        if d_weight is not None:
            ws, wsb, held = _scratch(_workspace_bytes("psrl_rms_norm_workspace_bytes", dev, dt, rows, heads, dim), keep, summed)
    else:
        ws, wsb = _use_workspace(workspace, raw, keep, dev)
    _launch("psrl_rms_norm_bwd", dev, dt, rows, heads, dim, summed.data_ptr(), ph, None if weight is None else weight.data_ptr(), eps,
            d_y.data_ptr(), pd, a_s, p_s, a_x, p_x, None if d_weight is None else d_weight.data_ptr(), ws, wsb, raw)
    return d_x, d_weight


def psrl_quantize_rows(x, codes=None, scales=None, stream=None):
    """Rows x [rows, dim] (f32 or bf16) in 8 bits: (codes float8_e4m3fn [rows, dim], scales float32 [rows])."""
    dt, rows, heads, dim, dev = _norm_args(x, None)
    if x.dim() != 2:
        raise ValueError("x must be [rows, dim]")
    raw, keep = _stream_on(stream, dev)
    px = _matrix_pitch(x, "x")
    codes, pc = _codes_rows(codes, x.shape, keep, x)
    scales = _floats(scales, x.shape[:1], keep, x.device, "scales")
    _launch("psrl_quantize_rows", dev, dt, rows, dim, x.data_ptr(), px, codes.data_ptr(), pc, scales.data_ptr(), raw)
    return codes, scales


_ACTIVATIONS = {None: 0, "none": 0, "relu": 1, "silu": 2, "gelu": 3, "gelu_tanh": 4}


def _linear_args(x, weight, activation):
    """(type, rows, in_dim, out_dim, device, the outputs' type) with what the two directions check alike."""
    dt, out = _type_code(x), x.dtype
    if dt is None:
        if out is not _torch().float8_e4m3fn:
            raise TypeError(f"dtype {x.dtype} is none of float32, bfloat16, float8_e4m3fn")
        dt, out = PSRL_E4M3, _torch().bfloat16
    if weight.dtype is not x.dtype:
        raise TypeError(f"weight is {weight.dtype}, x is {x.dtype}")
    xs, ws = x.shape, weight.shape
    if len(xs) != 2 or len(ws) != 2 or xs[1] != ws[1]:
        raise ValueError("x must be [rows, in_dim], weight [out_dim, in_dim]")
    if activation not in _ACTIVATIONS:
        raise ValueError(f"activation {activation!r} unknown")
    _int32(xs[1], ws[0])
    return dt, xs[0], xs[1], ws[0], _device_of(x, weight), out


def _operand_pitch(t, name: str) -> int:
    """Row pitch of a matrix operand; a lone row has any that will do."""
    rows, cols = t.shape
    pitch, step = t.stride()
    if step != 1 and cols != 1:
        raise ValueError(f"{name}: the elements of a row must be contiguous")
    return pitch if rows > 1 else -(-cols // 16) * 16


def _beside(t, rows: int, cols: int, dtype, dev: int, name: str):
    """(address, row pitch) of a [rows, cols] matrix beside the operands, (None, 0) without one."""
    if t is None:
        return None, 0
    if t.dtype is not dtype or t.get_device() != dev or t.shape != (rows, cols):
        raise ValueError(f"{name} must be {dtype} {(rows, cols)} on cuda:{dev}")
    return t.data_ptr(), _operand_pitch(t, name)


def _beside_vector(t, count: int, dtype, dev: int, name: str):
    if t is None:
        return None
    if t.dtype is not dtype or t.get_device() != dev or t.shape != (count,) or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous {dtype} {(count,)} on cuda:{dev}")
    return t.data_ptr()


def _result(t, rows: int, cols: int, dtype, keep, like, name: str):
    """A [rows, cols] output, made if not given with rows that are whole 16-byte vectors apart, its address and row pitch."""
    if t is not None:
        return (t, *_beside(t, rows, cols, dtype, like.get_device(), name))
    pitch = -(-cols // 8) * 8
    if keep is None and pitch == cols and like.shape == (rows, cols) and dtype is like.dtype and like.is_contiguous():
        t = _torch().empty_like(like)
        return t, t.data_ptr(), cols
    if keep is None and dtype is like.dtype:
        t = like.new_empty((rows, pitch))
    else:
        t = _new(keep, (rows, pitch), dtype, like.device)
    return (t if pitch == cols else t[:, :cols]), t.data_ptr(), pitch


def psrl_linear_workspace_bytes(n_rows: int, in_dim: int, out_dim: int, backward: bool, dtype: str = "bf16") -> int:
    return int(lib().psrl_linear_workspace_bytes({"f32": PSRL_F32, "e4m3": PSRL_E4M3}.get(dtype, PSRL_BF16), int(n_rows), int(in_dim), int(out_dim),
                                                 int(bool(backward))))


def psrl_linear_fwd(x, weight, bias=None, activation=None, mul=None, residual=None, x_scale=None, weight_scale=None, y=None, z=None,
                    want_z: bool = False, stream=None, workspace=None):
    """y = act(x weight^T + bias) * mul + residual: x [rows, in_dim], weight [out_dim, in_dim], both f32, both bf16, or both 8-bit codes
    (float8_e4m3fn) with float32 x_scale [rows] and weight_scale [out_dim], the rest then bf16.  activation: None, "relu", "silu",
    "gelu", "gelu_tanh".  Returns (y, z), z = x weight^T + bias with want_z (for the backward), else None.  y and z may be mul or
    residual.  `workspace`: a Workspace of psrl_linear_workspace_bytes(), whose status() tells whether a wait inside the kernel gave
    up; without one it cannot be asked."""
    if stream is None and y is None and z is None and workspace is None and activation in _ACTIVATIONS:
        r = (_torch_calls or _calls()).linear_fwd(x, weight, bias, _ACTIVATIONS[activation], mul, residual, x_scale, weight_scale, want_z)
        if r is not None:
            return _answer(r, "psrl_linear_fwd")
    dt, m, k, n, dev, out = _linear_args(x, weight, activation)
    if dt == PSRL_E4M3:
        if x_scale is None or weight_scale is None:
            raise ValueError("8-bit operands come with x_scale and weight_scale")
        a_xs = _beside_vector(x_scale, m, _torch().float32, dev, "x_scale")
        a_ws = _beside_vector(weight_scale, n, _torch().float32, dev, "weight_scale")
    elif x_scale is not None or weight_scale is not None:
        raise ValueError("x_scale and weight_scale belong to 8-bit operands")
    else:
        a_xs = a_ws = None
    raw, keep = _stream_on(stream, dev)
    a_mul, p_mul = _beside(mul, m, n, out, dev, "mul")
    a_res, p_res = _beside(residual, m, n, out, dev, "residual")
    a_bias = _beside_vector(bias, n, out, dev, "bias")
    px, pw = _operand_pitch(x, "x"), _operand_pitch(weight, "weight")
    y, a_y, p_y = _result(y, m, n, out, keep, x, "y")
    z, a_z, p_z = _result(z, m, n, out, keep, x, "z") if want_z else (None, None, 0)
    if workspace is not None:
        ws, wsb = _use_workspace(workspace, raw, keep, dev)
    elif dt == PSRL_F32:
        ws, wsb, held = _scratch(_workspace_bytes("psrl_linear_workspace_bytes", dev, dt, m, k, n, 0), keep, x)
    else:
        ws, wsb = None, 0
    _launch("psrl_linear_fwd", dev, dt, m, k, n, x.data_ptr(), px, a_xs, weight.data_ptr(), pw, a_ws, a_bias, _ACTIVATIONS[activation],
            a_mul, p_mul, a_res, p_res, a_y, p_y, a_z, p_z, ws, wsb, raw)
    return y, z


def psrl_linear_bwd(x, weight, d_y, z=None, activation=None, mul=None, d_x=None, d_weight=None, d_bias=None, d_mul=None, want_x: bool = True,
                    want_weight: bool = True, want_bias: bool = False, want_mul: Optional[bool] = None, stream=None, workspace=None):
    """Gradients of the above, f32 or bf16: (d_x, d_weight, d_bias, d_mul) given d_y and the forward's z (which may be None without an
    activation where d_mul is not wanted); what is not wanted is None, d_mul is wanted where there is a mul.  The gradient of residual
    is d_y.  `workspace` as above (backward True)."""
    if want_mul is None:
        want_mul = mul is not None
    if (stream is None and d_x is None and d_weight is None and d_bias is None and d_mul is None and workspace is None and activation in _ACTIVATIONS
            and (mul is not None or not want_mul)):
        r = (_torch_calls or _calls()).linear_bwd(x, weight, d_y, z, _ACTIVATIONS[activation], mul, want_x, want_weight, want_bias, want_mul)
        if r is not None:
            return _answer(r, "psrl_linear_bwd")
    dt, m, k, n, dev, out = _linear_args(x, weight, activation)
    if dt == PSRL_E4M3:
        raise TypeError("8-bit operands have no backward")
    if want_mul and mul is None:
        raise ValueError("d_mul without a mul")
    raw, keep = _stream_on(stream, dev)
    a_d, p_d = _beside(d_y, m, n, out, dev, "d_y")
    a_z, p_z = _beside(z, m, n, out, dev, "z")
    a_mul, p_mul = _beside(mul, m, n, out, dev, "mul")
    px, pw = _operand_pitch(x, "x"), _operand_pitch(weight, "weight")
    d_x, a_x, p_x = _result(d_x, m, k, out, keep, x, "d_x") if want_x else (None, None, 0)
    d_weight, a_w, p_w = _result(d_weight, n, k, out, keep, weight, "d_weight") if want_weight else (None, None, 0)
    d_mul, a_m, p_m = _result(d_mul, m, n, out, keep, d_y, "d_mul") if want_mul else (None, None, 0)
    if not want_bias:
        d_bias = None
    elif d_bias is None:
        d_bias = d_y.new_empty((n,)) if keep is None else _new(keep, (n,), out, x.device)
    a_bias = _beside_vector(d_bias, n, out, dev, "d_bias")
    if workspace is not None:
        ws, wsb = _use_workspace(workspace, raw, keep, dev)
    elif activation not in (None, "none") or mul is not None or want_bias or dt == PSRL_F32:
        ws, wsb, held = _scratch(_workspace_bytes("psrl_linear_workspace_bytes", dev, dt, m, k, n, 1), keep, x)
    else:
        ws, wsb = None, 0
    _launch("psrl_linear_bwd", dev, dt, m, k, n, x.data_ptr(), px, weight.data_ptr(), pw, a_z, p_z, _ACTIVATIONS[activation], a_mul, p_mul,
            a_d, p_d, a_x, p_x, a_w, p_w, a_bias, a_m, p_m, ws, wsb, raw)
    return d_x, d_weight, d_bias, d_mul


def _flags_ptr(seg_flags):
    if seg_flags is None:
        return None, None
    fl = np.ascontiguousarray(np.asarray(seg_flags, dtype=np.uint8))
    return fl, fl.ctypes.data_as(C.POINTER(C.c_uint8))


def psrl_cost_sequence(alpha, l: int, h: int) -> float:
    """Eq. 1 for one sequence of length l with a cached prefix of h tokens."""
    m = CostModel(*[float(a) for a in alpha])
    return float(lib().psrl_cost_sequence(C.byref(m), int(l), int(h)))


def psrl_group_workloads(parent, seg_len, alpha, seg_flags=None):
    """Workload of every prefix group (sum of Eq. 1 over its samples)."""
    p, l = _i32(parent), _i32(seg_len)
    n_groups = int((p == -1).sum())
    out = np.zeros(n_groups, dtype=np.float64)
    m = CostModel(*[float(a) for a in alpha])
    keep, fp = _flags_ptr(seg_flags)
    _check(lib().psrl_group_workloads(len(p), p.ctypes.data_as(_I32P), l.ctypes.data_as(_I32P), fp, C.byref(m), n_groups,
                                      out.ctypes.data_as(C.POINTER(C.c_double))), "psrl_group_workloads")
    return out


def psrl_place_groups(workload, n_workers: int):
    """Longest-processing-time-first placement: (worker of every group, load of every worker)."""
    w = np.ascontiguousarray(np.asarray(workload, dtype=np.float64))
    worker = np.zeros(len(w), dtype=np.int32)
    load = np.zeros(int(n_workers), dtype=np.float64)
    _check(lib().psrl_place_groups(len(w), w.ctypes.data_as(C.POINTER(C.c_double)), int(n_workers),
                                   worker.ctypes.data_as(_I32P), load.ctypes.data_as(C.POINTER(C.c_double))),
           "psrl_place_groups")
    return worker, load


def psrl_microbatch_tokens(parent, seg_len, alpha, n_microbatches: int, seg_flags=None):
    """Token-wise micro-batching: the forest of pieces as a dict of arrays (parent, seg_len, mb, seg, begin)
    plus the per-micro-batch budget."""
    p, l = _i32(parent), _i32(seg_len)
    cap = len(p) + int(n_microbatches)
    outs = [np.zeros(cap, dtype=np.int32) for _ in range(5)]
    n, budget = C.c_int32(), C.c_double()
    m = CostModel(*[float(a) for a in alpha])
    keep, fp = _flags_ptr(seg_flags)
    _check(lib().psrl_microbatch_tokens(len(p), p.ctypes.data_as(_I32P), l.ctypes.data_as(_I32P), fp, C.byref(m),
                                        int(n_microbatches), cap, C.byref(n), *[o.ctypes.data_as(_I32P) for o in outs],
                                        C.byref(budget)), "psrl_microbatch_tokens")
    k = n.value
    return dict(parent=outs[0][:k].copy(), seg_len=outs[1][:k].copy(), mb=outs[2][:k].copy(), seg=outs[3][:k].copy(),
                begin=outs[4][:k].copy(), budget=float(budget.value))


class Cache:
    """Owner of a psrl_cache_t (Dynamic Block Caching over an ordered list of micro-batches).
    begin(m) returns the micro-batch's tree as plain lists, ready for Plan(..., seg_slot_base=...)."""

    def __init__(self, parent, seg_len, group_block_size, mb_of_seg, n_microbatches: int, seg_flags=None,
                 capacity_slots: int = 0):
        self._h = C.c_void_p()
        self._destroy = lib().psrl_cache_destroy
        p, l, g, mb = _i32(parent), _i32(seg_len), _i32(group_block_size), _i32(mb_of_seg)
        d = CacheDesc()
        d.n_segments = len(p)
        d.parent, d.seg_len = p.ctypes.data_as(_I32P), l.ctypes.data_as(_I32P)
        fl = None
        if seg_flags is not None:
            fl = np.ascontiguousarray(np.asarray(seg_flags, dtype=np.uint8))
            d.seg_flags = fl.ctypes.data_as(C.POINTER(C.c_uint8))
        d.group_block_size, d.n_groups = g.ctypes.data_as(_I32P), len(g)
        d.n_microbatches = int(n_microbatches)
        if len(mb) != len(p) or len(l) != len(p):
            raise ValueError("parent, seg_len and mb_of_seg need one entry per segment")
        d.mb_of_seg = mb.ctypes.data_as(_I32P)
        d.capacity_slots = int(capacity_slots)
        self.n_segments = len(p)
        _check(lib().psrl_cache_create(C.byref(d), C.byref(self._h)), "psrl_cache_create")

    def begin(self, m: int) -> dict:
        st = CacheStep()
        _check(lib().psrl_cache_begin(self._h, int(m), C.byref(st)), "psrl_cache_begin")
        arr = lambda ptr, k: [int(ptr[i]) for i in range(k)]
        k = st.n_segments
        return dict(seg_id=arr(st.seg_id, k), parent=arr(st.parent, k), seg_len=arr(st.seg_len, k),
                    seg_flags=arr(st.seg_flags, k), group_block_size=arr(st.group_block_size, st.n_groups),
                    seg_slot_base=arr(st.seg_slot_base, k), new=arr(st.new_seg, st.n_new),
                    reload=arr(st.reload_seg, st.n_reload),
                    evict=list(zip(arr(st.evict_seg, st.n_evict), arr(st.evict_base, st.n_evict))),
                    live_slots=int(st.live_slots), pool_slots=int(st.pool_slots))

    def end(self, m: int) -> dict:
        nf, ptr, live = C.c_int32(), _I32P(), C.c_int64()
        _check(lib().psrl_cache_end(self._h, int(m), C.byref(nf), C.byref(ptr), C.byref(live)), "psrl_cache_end")
        return dict(freed=[int(ptr[i]) for i in range(nf.value)], live_slots=int(live.value))

    def compact(self):
        """Slides the resident blocks together (between end and the next begin).  Returns the moves for psrl_kv_move,
        [n, 3] int32, and the slot behind the last resident block."""
        n, ptr, top = C.c_int32(), _I32P(), C.c_int64()
        _check(lib().psrl_cache_compact(self._h, C.byref(n), C.byref(ptr), C.byref(top)), "psrl_cache_compact")
        k = n.value
        moves = np.ctypeslib.as_array(ptr, shape=(k, 3)).copy() if k else np.zeros((0, 3), dtype=np.int32)
        return moves, int(top.value)

    def stats(self) -> dict:
        s = CacheStats()
        _check(lib().psrl_cache_stats(self._h, C.byref(s)), "psrl_cache_stats")
        return {n: int(getattr(s, n)) for n, _ in CacheStats._fields_}

    def refcounts(self):
        ptr = _I32P()
        _check(lib().psrl_cache_refcounts(self._h, C.byref(ptr)), "psrl_cache_refcounts")
        return [int(ptr[i]) for i in range(self.n_segments)]

    def __del__(self):
        if getattr(self, "_h", None) and self._h.value:
            self._destroy(self._h)      # held by the object: at the interpreter's end this module's names may be gone
            self._h.value = None


def psrl_launch_count(plan: Plan, backward: bool) -> int:
    """Kernels one forward (backward=False) or backward call launches for this plan."""
    return int(lib().psrl_launch_count(plan._h, int(bool(backward))))


def _check_dtype(plan: Plan, *tensors):
    want = _torch().float32 if plan.dtype == "f32" else _torch().bfloat16
    for t in tensors:
        if t.dtype is not want:
            raise TypeError(f"tensor dtype {t.dtype} does not match the plan's {want}")
        if not t.is_cuda:
            raise RuntimeError("tensors must live on a CUDA device: this library has no CPU path")
