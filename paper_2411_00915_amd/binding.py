"""Thin binding over the C-ABI library (include/lora_abi.h): ctypes, and for the compute calls, which are made per layer,
the extension module _calls.

Argument marshalling only: every step of the operator runs in the HIP kernels
of liblora_amd.so.  There is no CPU fallback; if the library has not been built
the import of this module fails.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
# LORA_AMD_LIBRARY names another build of the same library (instrumented or experimental builds); unset, the
# library built in-tree is the one that runs
LIB_PATH = os.environ.get("LORA_AMD_LIBRARY") or os.path.join(_HERE, "liblora_amd.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it with `python -m paper_2411_00915_amd.build` "
        "(there is no fallback path)")

_lib = ctypes.CDLL(LIB_PATH)

try:
    from . import _calls
except ImportError as e:
    if not os.environ.get("LORA_AMD_LIBRARY"):
        raise ImportError(f"the extension module _calls is missing or cannot be loaded ({e}): build it with "
                          "`python -m paper_2411_00915_amd.build`") from e
    from . import calls_ctypes as _calls               # a library built elsewhere, in a tree that has not been built

LORA_OK, LORA_ERR_INVALID_ARG, LORA_ERR_UNSUPPORTED, LORA_ERR_NOMEM, LORA_ERR_WORKSPACE, LORA_ERR_DEVICE = range(6)
LORA_F32, LORA_BF16 = 0, 1
LORA_VARIANT_AUTO, LORA_VARIANT_GENERAL, LORA_VARIANT_TILED = 0, 1, 2
LORA_MAX_RANK = 256
LORA_TUNING_COUNT = 17
LORA_EXPAND_BY_ROUNDS = 1 << 30
LORA_STATIC_V_BYTES = 16 << 20
LORA_STATIC_MAX_GROUPS = 4096
LORA_MAX_HEAD_DIM = 256
LORA_MAX_BEAMS = 64

_i32p = ctypes.POINTER(ctypes.c_int32)
_f32p = ctypes.POINTER(ctypes.c_float)


class BatchDesc(ctypes.Structure):
    _fields_ = [("num_tokens", ctypes.c_int32), ("num_segments", ctypes.c_int32),
                ("seg_indptr", _i32p), ("seg_adapter", _i32p),
                ("num_adapters", ctypes.c_int32), ("adapter_rank", _i32p), ("adapter_scale", _f32p),
                ("k", ctypes.c_int32), ("n", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("variant", ctypes.c_int32), ("tuning", _i32p), ("tuning_count", ctypes.c_int32),
                ("merged_adapter_plus1", ctypes.c_int32)]


class Tile(ctypes.Structure):
    _fields_ = [("adapter", ctypes.c_int32), ("row0", ctypes.c_int32), ("nrows", ctypes.c_int32),
                ("c0", ctypes.c_int32), ("cn", ctypes.c_int32), ("shape", ctypes.c_int32),
                ("reserved0", ctypes.c_int32), ("reserved1", ctypes.c_int32)]


class PlanView(ctypes.Structure):
    _fields_ = [("num_tokens", ctypes.c_int32), ("num_active", ctypes.c_int32),
                ("num_groups", ctypes.c_int32), ("v_row_stride", ctypes.c_int32),
                ("kernel_family", ctypes.c_int32), ("shrink_waves", ctypes.c_int32),
                ("v_parts", ctypes.c_int32), ("tuning_source", ctypes.c_int32),
                ("tuning", ctypes.c_int32 * LORA_TUNING_COUNT), ("shrink_kernel_family", ctypes.c_int32),
                ("token_adapter", _i32p), ("perm", _i32p), ("group_adapter", _i32p), ("group_offset", _i32p),
                ("shrink_tiles", ctypes.POINTER(Tile)), ("num_shrink_tiles", ctypes.c_int32),
                ("expand_tiles", ctypes.POINTER(Tile)), ("num_expand_tiles", ctypes.c_int32),
                ("num_gemm_rows", ctypes.c_int32), ("num_gemm_tiles", ctypes.c_int32),
                ("gemm_order", _i32p), ("gemm_stage_offset", _i32p), ("gemm_stage", _i32p),
                ("merged_adapter", ctypes.c_int32), ("num_unmerge", ctypes.c_int32),
                ("unmerge_v_row_stride", ctypes.c_int32), ("unmerge_v_parts", ctypes.c_int32),
                ("unmerge_v_offset", ctypes.c_size_t), ("unmerge_perm", _i32p),
                ("unmerge_shrink_tiles", ctypes.POINTER(Tile)), ("num_unmerge_shrink_tiles", ctypes.c_int32),
                ("unmerge_expand_tiles", ctypes.POINTER(Tile)), ("num_unmerge_expand_tiles", ctypes.c_int32)]


class AttentionDesc(ctypes.Structure):
    _fields_ = [("num_seqs", ctypes.c_int32), ("q_indptr", _i32p), ("kv_indptr", _i32p), ("num_heads", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("causal", ctypes.c_int32)]


class CacheDesc(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_void_p), ("weight", ctypes.c_void_p), ("page_table", ctypes.c_void_p), ("length", ctypes.c_void_p),
                ("num_pages", ctypes.c_int64), ("num_seqs", ctypes.c_int32), ("table_stride", ctypes.c_int32), ("max_length", ctypes.c_int32),
                ("page_tokens", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32)]


class PagesDesc(ctypes.Structure):
    _fields_ = [("page_table", ctypes.c_void_p), ("length", ctypes.c_void_p), ("users", ctypes.c_void_p), ("num_pages", ctypes.c_int64),
                ("num_seqs", ctypes.c_int32), ("table_stride", ctypes.c_int32), ("max_length", ctypes.c_int32), ("page_tokens", ctypes.c_int32)]


_vp = ctypes.c_void_p
_lib.lora_plan_create.restype = ctypes.c_int
_lib.lora_plan_create.argtypes = [ctypes.POINTER(BatchDesc), ctypes.POINTER(_vp)]
_lib.lora_plan_destroy.restype = None
_lib.lora_plan_destroy.argtypes = [_vp]
_lib.lora_plan_query.restype = ctypes.c_int
_lib.lora_plan_query.argtypes = [_vp, _i32p, ctypes.POINTER(ctypes.c_size_t), ctypes.POINTER(ctypes.c_size_t)]
_lib.lora_plan_export.restype = ctypes.c_int
_lib.lora_plan_export.argtypes = [_vp, ctypes.POINTER(PlanView)]
_lib.lora_plan_upload.restype = ctypes.c_int
_lib.lora_plan_upload.argtypes = [_vp, _vp]
_lib.lora_shrink.restype = ctypes.c_int
_lib.lora_shrink.argtypes = [_vp, _vp, ctypes.c_int64, _vp, _vp, _vp]
_lib.lora_expand.restype = ctypes.c_int
_lib.lora_expand.argtypes = [_vp, _vp, _vp, _vp, ctypes.c_int64, ctypes.c_float, _vp]
_lib.lora_delta.restype = ctypes.c_int
_lib.lora_delta.argtypes = [_vp, _vp, ctypes.c_int64, _vp, _vp, _vp, _vp, ctypes.c_int64, ctypes.c_float, _vp]
_lib.lora_delta_static.restype = ctypes.c_int
_lib.lora_delta_static.argtypes = [_vp, _vp, ctypes.c_int64, _vp, _vp, _vp, ctypes.c_int64, ctypes.c_float, _vp]
_lib.lora_base_gemm.restype = ctypes.c_int
_lib.lora_base_gemm.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                _vp, ctypes.c_int64, _vp, ctypes.c_int64, _vp, ctypes.c_int64, _vp]
_lib.lora_fused_forward.restype = ctypes.c_int
_lib.lora_fused_forward.argtypes = [_vp, _vp, ctypes.c_int64, _vp, ctypes.c_int64, _vp, _vp,
                                    _vp, ctypes.c_int64, _vp, ctypes.c_size_t, _vp]
_lib.lora_merge.restype = ctypes.c_int
_lib.lora_merge.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_float, ctypes.c_int32,
                            ctypes.c_int32, _vp, ctypes.c_int64, _vp, _vp, _vp]
_lib.lora_attention_plan_create.restype = ctypes.c_int
_lib.lora_attention_plan_create.argtypes = [ctypes.POINTER(AttentionDesc), ctypes.POINTER(_vp)]
_lib.lora_attention_plan_destroy.restype = None
_lib.lora_attention_plan_destroy.argtypes = [_vp]
_lib.lora_attention_plan_items.restype = ctypes.c_int32
_lib.lora_attention_plan_items.argtypes = [_vp, ctypes.POINTER(_i32p)]
_lib.lora_attention_plan_instance.restype = None
_lib.lora_attention_plan_instance.argtypes = [_vp, ctypes.c_int32, ctypes.c_int64, _i32p]
_lib.lora_cache_page_bytes.restype = ctypes.c_size_t
_lib.lora_cache_page_bytes.argtypes = [ctypes.c_int32, ctypes.c_int32]
_lib.lora_cache_workspace.restype = ctypes.c_int
_lib.lora_cache_workspace.argtypes = [_vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.POINTER(ctypes.c_size_t)]
_lib.lora_pages_workspace.restype = ctypes.c_int
_lib.lora_pages_workspace.argtypes = [_vp, ctypes.POINTER(ctypes.c_size_t)]
_lib.lora_beam_workspace.restype = ctypes.c_int
_lib.lora_beam_workspace.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.POINTER(ctypes.c_size_t)]
_lib.lora_cache_choose_workspace.restype = ctypes.c_int
_lib.lora_cache_choose_workspace.argtypes = [_vp, ctypes.c_int32, ctypes.c_int32, ctypes.POINTER(ctypes.c_size_t)]
_lib.lora_cache_chosen_workspace.restype = ctypes.c_int
_lib.lora_cache_chosen_workspace.argtypes = [_vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.POINTER(ctypes.c_size_t)]
_lib.lora_status_str.restype = ctypes.c_char_p
_lib.lora_status_str.argtypes = [ctypes.c_int]
_lib.lora_tuning_set.restype = None
_lib.lora_tuning_set.argtypes = [_i32p, ctypes.c_int32]
_lib.lora_tuning_get.restype = None
_lib.lora_tuning_get.argtypes = [_i32p, ctypes.c_int32]



class TuningEntry(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int32), ("k", ctypes.c_int32), ("n", ctypes.c_int32), ("max_rank", ctypes.c_int32),
                ("group_class", ctypes.c_int32), ("values", ctypes.c_int32 * LORA_TUNING_COUNT)]


_lib.lora_tuning_table_set.restype = ctypes.c_int
_lib.lora_tuning_table_set.argtypes = [ctypes.POINTER(TuningEntry), ctypes.c_int32]
_lib.lora_tuning_table_get.restype = ctypes.c_int32
_lib.lora_tuning_table_get.argtypes = [ctypes.POINTER(TuningEntry), ctypes.c_int32]
_lib.lora_probe.restype = ctypes.c_int
_lib.lora_probe.argtypes = [ctypes.c_int32, _vp, ctypes.c_size_t, ctypes.c_int32, _vp]
_lib.lora_trace_tick_khz.restype = ctypes.c_int32
_lib.lora_trace_set.restype = ctypes.c_int
_lib.lora_trace_set.argtypes = [_vp, ctypes.c_size_t]
_lib.lora_timing_begin.restype = ctypes.c_int
_lib.lora_timing_end.restype = ctypes.c_int
_lib.lora_timing_read.restype = ctypes.c_int
_lib.lora_timing_read.argtypes = [ctypes.c_int32, ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_double),
                                  ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double)]
_lib.lora_kernel_name.restype = ctypes.c_char_p
_lib.lora_kernel_name.argtypes = [ctypes.c_int32]
_lib.lora_layer_shrink_tiles.restype = ctypes.c_int32
_lib.lora_layer_shrink_tiles.argtypes = [_vp, ctypes.c_int32, ctypes.c_int32, ctypes.POINTER(ctypes.POINTER(Tile))]
_lib.lora_kernel_count.restype = ctypes.c_int32

EXPORTED = ["lora_timing_begin", "lora_timing_end", "lora_timing_read", "lora_kernel_name", "lora_kernel_count",
            "lora_plan_create", "lora_plan_destroy", "lora_plan_query", "lora_plan_export",
            "lora_plan_upload", "lora_shrink", "lora_expand", "lora_delta", "lora_delta_static", "lora_base_gemm",
            "lora_fused_forward", "lora_merge", "lora_status_str", "lora_tuning_set", "lora_tuning_get",
            "lora_attention_plan_create", "lora_attention_plan_destroy", "lora_attention_plan_upload", "lora_attention",
            "lora_cache_page_bytes", "lora_cache_append", "lora_cache_read", "lora_cache_workspace", "lora_cache_attention", "lora_cache_evict",
            "lora_pages_workspace", "lora_pages_resize", "lora_pages_fork", "lora_cache_copy", "lora_beam_workspace", "lora_beam_select",
            "lora_cache_digest", "lora_cache_choose_workspace", "lora_cache_choose", "lora_cache_chosen_workspace", "lora_cache_attention_chosen",
            "lora_tuning_table_set", "lora_tuning_table_get", "lora_probe", "lora_trace_set", "lora_trace_tick_khz"]

TUNING_FIELDS = ["shrink_waves", "shrink_tb2_min_rows", "shrink_max_jb", "expand_wave_bytes",
                 "expand_tb2_min_rows", "expand_tb4_min_rows", "tiled_min_tokens",
                 "shrink_small_waves", "shrink_small_jb", "shrink_target_wgs", "fused_wait_us", "fused_delay", "expand_wave_bytes_big", "shrink_tb4_min_rows",
                 "shrink_stream_min_tokens", "shrink_stream_wgs", "expand_stream_stages"]


class LoraError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {lora_status_str(status)} (status {status})")


def lora_status_str(status: int) -> str:
    return _lib.lora_status_str(int(status)).decode()


def _check(status: int, where: str):
    if status != LORA_OK:
        raise LoraError(status, where)


def _ptr(obj) -> Optional[int]:
    """Device/host address of a torch tensor, or an int address, or None."""
    if obj is None:
        return None
    if isinstance(obj, int):
        return obj
    return int(obj.data_ptr())


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch
        return int(torch.cuda.current_stream().cuda_stream) or None
    if isinstance(stream, int):
        return stream or None
    return int(stream.cuda_stream) or None


def lora_tuning_get() -> dict:
    buf = (ctypes.c_int32 * len(TUNING_FIELDS))()
    _lib.lora_tuning_get(buf, len(TUNING_FIELDS))
    return dict(zip(TUNING_FIELDS, list(buf)))


def lora_tuning_set(**kw) -> None:
    """Set the process's default tunables (values <= 0 or missing keep the current value)."""
    vals = _tuning_values(kw)
    buf = (ctypes.c_int32 * len(vals))(*vals)
    _lib.lora_tuning_set(buf, len(vals))


def _tuning_values(tunables: dict):
    unknown = set(tunables) - set(TUNING_FIELDS)
    if unknown:
        raise KeyError(f"unknown tuning fields: {sorted(unknown)}")
    return [int(tunables.get(f, 0)) for f in TUNING_FIELDS]


def lora_tuning_table_set(entries) -> None:
    """Replace the process's shape table.  entries: iterable of dicts with the key fields tokens, k, n, max_rank,
    group_class and `tunables` (name -> value); None or empty restores the table the library ships with."""
    entries = list(entries or [])
    arr = (TuningEntry * max(len(entries), 1))()
    for i, e in enumerate(entries):
        arr[i].tokens, arr[i].k, arr[i].n = int(e["tokens"]), int(e["k"]), int(e["n"])
        arr[i].max_rank, arr[i].group_class = int(e["max_rank"]), int(e["group_class"])
        for j, val in enumerate(_tuning_values(e["tunables"])):
            arr[i].values[j] = val
    _check(_lib.lora_tuning_table_set(arr if entries else None, len(entries)), "lora_tuning_table_set")


def lora_tuning_table_get() -> list:
    n = _lib.lora_tuning_table_get(None, 0)
    arr = (TuningEntry * max(n, 1))()
    n = min(n, _lib.lora_tuning_table_get(arr, n))
    return [dict(tokens=arr[i].tokens, k=arr[i].k, n=arr[i].n, max_rank=arr[i].max_rank, group_class=arr[i].group_class,
                 tunables={f: int(arr[i].values[j]) for j, f in enumerate(TUNING_FIELDS) if arr[i].values[j] > 0})
            for i in range(n)]


def lora_gemm_choice(tokens: int, k: int, n: int, dtype: int, delta: bool):
    """(kernel, feature blocks, token blocks): what an aligned product takes; kernel 1 small; 6, 2, 3 and 7 medium,
    of 64, 128, 192 and 256 features; 4 ring (or register-staged), 5 register-staged 128 x 128; the blocks of 16 are the small
    kernel's tile."""
    c = int(_lib.lora_gemm_choice(int(tokens), int(k), int(n), int(dtype), int(delta)))
    return c >> 16, c >> 8 & 255, c & 255


def lora_layer_shrink_tiles(plan: "Plan", removal: bool = False, own: bool = False):
    """Shrink tiles that the plan (removal: its removal's) has only for lora_fused_forward's launch of shrink and product;
    own: those that the launch takes, which may be the plan's own; none where there are two launches"""
    p = ctypes.POINTER(Tile)()
    n = _lib.lora_layer_shrink_tiles(plan.handle, int(removal), int(own), ctypes.byref(p))
    return np.ctypeslib.as_array(ctypes.cast(p, _i32p), shape=(n * 8,)).copy().reshape(n, 8) if n else np.zeros((0, 8), np.int32)


LORA_PROBE_EMPTY, LORA_PROBE_READ, LORA_PROBE_MFMA = 0, 1, 2


def lora_probe(kind: int, buffer, nbytes: int, iters: int = 1, stream=None):
    _check(_lib.lora_probe(int(kind), _ptr(buffer), int(nbytes), int(iters), _stream(stream)), "lora_probe")


def lora_trace_set(buffer=None):
    """buffer: an int64 device tensor with 8 entries per tile of the plans used while it is set; None switches off"""
    if buffer is None:
        _check(_lib.lora_trace_set(None, 0), "lora_trace_set")
    else:
        _check(_lib.lora_trace_set(_ptr(buffer), buffer.numel() * buffer.element_size()), "lora_trace_set")


def lora_trace_tick_khz() -> int:
    return int(_lib.lora_trace_tick_khz())


def lora_timing_begin():
    _check(_lib.lora_timing_begin(), "lora_timing_begin")


def lora_timing_end() -> dict:
    """Stop timing; returns {kernel name: dict(count, avg_us, min_us, max_us)} for kernels that ran."""
    _check(_lib.lora_timing_end(), "lora_timing_end")
    out = {}
    for kid in range(_lib.lora_kernel_count()):
        c, tot, mn, mx = ctypes.c_int64(), ctypes.c_double(), ctypes.c_double(), ctypes.c_double()
        _check(_lib.lora_timing_read(kid, ctypes.byref(c), ctypes.byref(tot), ctypes.byref(mn), ctypes.byref(mx)),
               "lora_timing_read")
        if c.value:
            out[_lib.lora_kernel_name(kid).decode()] = dict(count=int(c.value), avg_us=tot.value / c.value,
                                                            min_us=mn.value, max_us=mx.value)
    return out


class Plan:
    """Owner of a lora_plan handle."""

    def __init__(self, handle: int, keepalive):
        self._h = handle
        self._keep = keepalive

    @property
    def handle(self) -> int:
        return self._h

    def destroy(self):
        if self._h:
            _lib.lora_plan_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def lora_plan(num_tokens, seg_indptr, seg_adapter, adapter_rank, adapter_scale, k, n, dtype,
              variant=LORA_VARIANT_AUTO, tuning: Optional[dict] = None, merged_adapter: Optional[int] = None) -> Plan:
    """lora_plan_create; tables are host arrays (numpy or sequences).  tuning: tunables for this plan only
    (name -> value), on top of the shape table's entry and the process defaults.  merged_adapter: mixture mode,
    the adapter that is folded into the base weight the batch runs on (None: no adapter is)."""
    indptr = np.ascontiguousarray(seg_indptr, dtype=np.int32)
    seg_ad = np.ascontiguousarray(seg_adapter, dtype=np.int32)
    rank = np.ascontiguousarray(adapter_rank, dtype=np.int32)
    scale = np.ascontiguousarray(adapter_scale, dtype=np.float32)
    desc = BatchDesc(int(num_tokens), int(seg_ad.shape[0]),
                     indptr.ctypes.data_as(_i32p), seg_ad.ctypes.data_as(_i32p),
                     int(rank.shape[0]), rank.ctypes.data_as(_i32p), scale.ctypes.data_as(_f32p),
                     int(k), int(n), int(dtype), int(variant), None, 0,
                     0 if merged_adapter is None else int(merged_adapter) + 1)
    if tuning:
        vals = (ctypes.c_int32 * LORA_TUNING_COUNT)(*_tuning_values(tuning))
        desc.tuning = ctypes.cast(vals, _i32p)
        desc.tuning_count = LORA_TUNING_COUNT
    out = _vp()
    _check(_lib.lora_plan_create(ctypes.byref(desc), ctypes.byref(out)), "lora_plan_create")
    return Plan(out.value, None)


def lora_plan_create_raw(desc: Optional[BatchDesc]):
    """Direct call for error-path tests: returns (status, handle)."""
    out = _vp()
    st = _lib.lora_plan_create(ctypes.byref(desc) if desc is not None else None, ctypes.byref(out))
    return st, out.value


def lora_plan_destroy(plan: Plan):
    plan.destroy()


def lora_plan_query(plan: Plan):
    r = ctypes.c_int32()
    vb = ctypes.c_size_t()
    ws = ctypes.c_size_t()
    _check(_lib.lora_plan_query(plan.handle, ctypes.byref(r), ctypes.byref(vb), ctypes.byref(ws)), "lora_plan_query")
    return int(r.value), int(vb.value), int(ws.value)


def lora_plan_export(plan: Plan) -> dict:
    """Copy of the plan's host tables as numpy arrays."""
    v = PlanView()
    _check(_lib.lora_plan_export(plan.handle, ctypes.byref(v)), "lora_plan_export")

    def arr(p, n):
        return np.ctypeslib.as_array(p, shape=(n,)).copy() if n > 0 else np.zeros(0, np.int32)

    def tiles(p, n):
        if n == 0:
            return np.zeros((0, 8), np.int32)
        raw = np.ctypeslib.as_array(ctypes.cast(p, _i32p), shape=(n * 8,)).copy()
        return raw.reshape(n, 8)

    return dict(num_tokens=v.num_tokens, num_active=v.num_active, num_groups=v.num_groups,
                v_row_stride=v.v_row_stride, kernel_family=v.kernel_family, shrink_kernel_family=v.shrink_kernel_family,
                shrink_waves=v.shrink_waves,
                v_parts=v.v_parts, tuning_source=v.tuning_source,
                tuning={f: int(v.tuning[j]) for j, f in enumerate(TUNING_FIELDS)},
                token_adapter=arr(v.token_adapter, v.num_tokens), perm=arr(v.perm, v.num_active),
                group_adapter=arr(v.group_adapter, v.num_groups),
                group_offset=arr(v.group_offset, v.num_groups + 1),
                shrink_tiles=tiles(v.shrink_tiles, v.num_shrink_tiles),
                expand_tiles=tiles(v.expand_tiles, v.num_expand_tiles),
                gemm_order=arr(v.gemm_order, v.num_gemm_rows),
                gemm_stage_offset=arr(v.gemm_stage_offset, v.num_gemm_tiles + 1 if v.num_gemm_tiles else 0),
                gemm_stage=(arr(v.gemm_stage, int(v.gemm_stage_offset[v.num_gemm_tiles])) if v.num_gemm_tiles
                            else np.zeros(0, np.int32)),
                merged_adapter=v.merged_adapter, num_unmerge=v.num_unmerge,
                unmerge_v_row_stride=v.unmerge_v_row_stride, unmerge_v_parts=v.unmerge_v_parts,
                unmerge_v_offset=int(v.unmerge_v_offset), unmerge_perm=arr(v.unmerge_perm, v.num_unmerge),
                unmerge_shrink_tiles=tiles(v.unmerge_shrink_tiles, v.num_unmerge_shrink_tiles),
                unmerge_expand_tiles=tiles(v.unmerge_expand_tiles, v.num_unmerge_expand_tiles))


class AttentionPlan:
    """Owner of a lora_attention_plan handle."""

    def __init__(self, handle: int):
        self._h = handle

    @property
    def handle(self) -> int:
        return self._h

    def destroy(self):
        if self._h:
            _lib.lora_attention_plan_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def lora_attention_plan(q_indptr, kv_indptr, num_heads, num_kv_heads, head_dim, dtype, causal=True) -> AttentionPlan:
    """lora_attention_plan_create; offsets are host arrays (numpy or sequences).  kv_indptr None: as q_indptr."""
    qi = np.ascontiguousarray(q_indptr, dtype=np.int32)
    ki = qi if kv_indptr is None else np.ascontiguousarray(kv_indptr, dtype=np.int32)
    if qi.ndim != 1 or qi.shape != ki.shape or qi.shape[0] < 1:
        raise ValueError("q_indptr and kv_indptr: one offset for every sequence and one behind the last")
    desc = AttentionDesc(qi.shape[0] - 1, qi.ctypes.data_as(_i32p), ki.ctypes.data_as(_i32p), int(num_heads), int(num_kv_heads), int(head_dim),
                         int(dtype), int(causal))
    out = _vp()
    _check(_lib.lora_attention_plan_create(ctypes.byref(desc), ctypes.byref(out)), "lora_attention_plan_create")
    return AttentionPlan(out.value)


def lora_attention_plan_create_raw(desc: Optional[AttentionDesc]):
    """Direct call for error-path tests: returns (status, handle)."""
    out = _vp()
    st = _lib.lora_attention_plan_create(ctypes.byref(desc) if desc is not None else None, ctypes.byref(out))
    return st, out.value


def lora_attention_plan_items(plan: AttentionPlan) -> np.ndarray:
    """The plan's work by workgroup, [items, 8]: first query row, queries, first key row, keys of the sequence, keys that the query before
    the first sees, keys that the last sees, heads (0: nothing to do), first head"""
    p = _i32p()
    n = _lib.lora_attention_plan_items(plan.handle, ctypes.byref(p))
    return np.ctypeslib.as_array(p, shape=(n * 8,)).copy().reshape(n, 8) if n else np.zeros((0, 8), np.int32)


def lora_attention_plan_instance(plan: AttentionPlan, aligned, pitch) -> tuple:
    """The kernel that a call with this plan takes where its rows are (not) aligned to 16 bytes and those of keys and values at most
    `pitch` bytes apart: dims it is made for, keys of a tile, wavefronts that share them, whether they go straight to LDS"""
    n = (ctypes.c_int32 * 4)()
    _lib.lora_attention_plan_instance(plan.handle, int(bool(aligned)), int(pitch), n)
    return n[0], n[1], n[2], bool(n[3])


def lora_cache_page_bytes(page_tokens: int, head_dim: int) -> int:
    return int(_lib.lora_cache_page_bytes(int(page_tokens), int(head_dim)))


class Cache:
    """A lora_cache descriptor and the device tensors that it names (kept alive by it)."""

    def __init__(self, desc: CacheDesc, pages=None, weight=None, page_table=None, length=None):
        self.desc = desc
        self.handle = ctypes.addressof(desc)
        self.pages, self.weight, self.page_table, self.length = pages, weight, page_table, length


def lora_cache(pages, page_table, length, page_tokens, num_kv_heads, head_dim, max_length, weight=None) -> Cache:
    """Descriptor over device tensors: pages (uint8, [num_pages][num_kv_heads][lora_cache_page_bytes]), page_table (int32, [num_seqs,
    table_stride]), length (int32, [num_seqs]), weight (float32, [num_pages, num_kv_heads, page_tokens], or None)."""
    import torch
    page_bytes = lora_cache_page_bytes(page_tokens, head_dim) * int(num_kv_heads)
    if page_bytes <= 0:
        raise ValueError(f"no cache has pages of {page_tokens} tokens, {num_kv_heads} heads of {head_dim}")
    for name, x, dtype in (("pages", pages, torch.uint8), ("page_table", page_table, torch.int32), ("length", length, torch.int32),
                           ("weight", weight, torch.float32)):
        if x is not None and (x.dtype != dtype or not x.is_contiguous()):
            raise ValueError(f"{name}: a contiguous tensor of {dtype}")
    num_pages = pages.numel() // page_bytes
    if page_table.dim() != 2 or length.dim() != 1 or page_table.shape[0] != length.shape[0] or pages.numel() != num_pages * page_bytes:
        raise ValueError("page_table [num_seqs, table_stride], length [num_seqs], whole pages")
    if weight is not None and weight.numel() != num_pages * num_kv_heads * page_tokens:
        raise ValueError("weight: one for every slot of every page and head")
    desc = CacheDesc(_ptr(pages), _ptr(weight), _ptr(page_table), _ptr(length), num_pages, int(length.shape[0]), int(page_table.shape[1]),
                     int(max_length), int(page_tokens), int(num_kv_heads), int(head_dim))
    return Cache(desc, pages, weight, page_table, length)


def lora_cache_workspace(cache: Cache, num_heads, num_tokens, max_new, weights=False) -> int:
    """Bytes that lora_cache_attention needs with these arguments"""
    n = ctypes.c_size_t()
    _check(_lib.lora_cache_workspace(cache.handle, int(num_heads), int(num_tokens), int(max_new), int(bool(weights)), ctypes.byref(n)),
           "lora_cache_workspace")
    return int(n.value)


class Pages:
    """A lora_pages descriptor and the device tensors that it names (kept alive by it)."""

    def __init__(self, desc: PagesDesc, page_table=None, length=None, users=None):
        self.desc = desc
        self.handle = ctypes.addressof(desc)
        self.page_table, self.length, self.users = page_table, length, users


def lora_pages(page_table, length, users, page_tokens, max_length) -> Pages:
    """Descriptor over device tensors of int32: page_table [num_seqs, table_stride], length [num_seqs], users [num_pages]."""
    import torch
    for name, x in (("page_table", page_table), ("length", length), ("users", users)):
        if x.dtype != torch.int32 or not x.is_contiguous():
            raise ValueError(f"{name}: a contiguous tensor of int32")
    if page_table.dim() != 2 or length.dim() != 1 or users.dim() != 1 or page_table.shape[0] != length.shape[0]:
        raise ValueError("page_table [num_seqs, table_stride], length [num_seqs], users [num_pages]")
    desc = PagesDesc(_ptr(page_table), _ptr(length), _ptr(users), int(users.shape[0]), int(length.shape[0]), int(page_table.shape[1]), int(max_length),
                     int(page_tokens))
    return Pages(desc, page_table, length, users)


def _workspace(function, *arguments) -> int:
    n = ctypes.c_size_t()
    _check(getattr(_lib, function)(*arguments, ctypes.byref(n)), function)
    return int(n.value)


def lora_pages_workspace(pages: Pages) -> int:
    """Bytes that lora_pages_resize and lora_pages_fork need"""
    return _workspace("lora_pages_workspace", pages.handle)


def lora_beam_workspace(num_groups, beams, vocab, num_out) -> int:
    """Bytes that lora_beam_select needs with these arguments"""
    return _workspace("lora_beam_workspace", int(num_groups), int(beams), int(vocab), int(num_out))


def lora_cache_choose_workspace(cache: Cache, num_tokens, max_new) -> int:
    """Bytes that lora_cache_choose needs with these arguments"""
    return _workspace("lora_cache_choose_workspace", cache.handle, int(num_tokens), int(max_new))


def lora_cache_chosen_workspace(cache: Cache, num_heads, num_tokens, max_new, budget) -> int:
    """Bytes that lora_cache_attention_chosen needs with these arguments"""
    return _workspace("lora_cache_chosen_workspace", cache.handle, int(num_heads), int(num_tokens), int(max_new), int(budget))


def _first_stream():
    """torch's current stream, and the functions that give the current device and a device's current stream once torch is
    initialised"""
    import torch
    # (torch's own, below its Python layer; the public functions where a torch has them under no such name)
    return (_stream(None) or 0, getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device),
            getattr(torch._C, "_cuda_getCurrentRawStream", lambda device: torch.cuda.current_stream(device).cuda_stream))


def _address(function) -> int:
    return ctypes.cast(function, ctypes.c_void_p).value


_calls.bind(_check, _first_stream, *(_address(f) for f in (
    _lib.lora_plan_upload, _lib.lora_shrink, _lib.lora_expand, _lib.lora_delta, _lib.lora_delta_static, _lib.lora_base_gemm,
    _lib.lora_fused_forward, _lib.lora_merge)))

# lora_plan_upload(plan, stream=None), lora_shrink(plan, x, ldx, d_At_ptrs, v, stream=None),
# lora_expand(plan, v, d_Bt_ptrs, y, ldy, beta=1.0, stream=None),
# lora_delta(plan, x, ldx, d_At_ptrs, d_Bt_ptrs, v, y, ldy, beta=1.0, stream=None),
# lora_delta_static(plan, x, ldx, d_At_ptrs, d_Bt_ptrs, y, ldy, beta=1.0, stream=None),
# lora_base_gemm(num_tokens, k, n, dtype, x, ldx, Wt, ldw, y, ldy, stream=None),
# lora_merge(num_layers, n, k, rank, scale, dtype, d_Wt_ptrs, ldw, d_At_ptrs, d_Bt_ptrs, variant=LORA_VARIANT_AUTO, stream=None),
# lora_fused_forward(plan, x, ldx, Wt, ldw, d_At_ptrs, d_Bt_ptrs, y, ldy, workspace, workspace_bytes, stream=None)
(lora_plan_upload, lora_shrink, lora_expand, lora_delta, lora_delta_static, lora_base_gemm, lora_fused_forward, lora_merge) = (
    _calls.lora_plan_upload, _calls.lora_shrink, _calls.lora_expand, _calls.lora_delta, _calls.lora_delta_static,
    _calls.lora_base_gemm, _calls.lora_fused_forward, _calls.lora_merge)

_calls.bind_attention(*(_address(f) for f in (_lib.lora_attention_plan_upload, _lib.lora_attention, _lib.lora_cache_append, _lib.lora_cache_read,
                                              _lib.lora_cache_attention, _lib.lora_cache_evict)))

# lora_attention_plan_upload(plan, stream=None),
# lora_attention(plan, q, ldq, k, ldk, v, ldv, o, ldo, scale, stream=None),
# lora_cache_append(cache, dtype, num_tokens, max_new, d_indptr, k, ldk, v, ldv, stream=None),
# lora_cache_read(cache, dtype, num_tokens, max_new, d_indptr, k, ldk, v, ldv, stream=None),
# lora_cache_attention(cache, dtype, num_heads, num_tokens, max_new, d_indptr, q, ldq, o, ldo, scale, decay, workspace, workspace_bytes, stream=None),
# lora_cache_evict(cache, target, budget, recent, d_kept, stream=None)
(lora_attention_plan_upload, lora_attention, lora_cache_append, lora_cache_read, lora_cache_attention, lora_cache_evict) = (
    _calls.lora_attention_plan_upload, _calls.lora_attention, _calls.lora_cache_append, _calls.lora_cache_read, _calls.lora_cache_attention,
    _calls.lora_cache_evict)

_calls.bind_sequences(*(_address(f) for f in (_lib.lora_pages_resize, _lib.lora_pages_fork, _lib.lora_cache_copy, _lib.lora_beam_select, _lib.lora_cache_digest,
                                              _lib.lora_cache_choose, _lib.lora_cache_attention_chosen)))

# lora_pages_resize(pages, d_wanted, num_tokens, d_granted, d_indptr, d_token_seq, d_token_position, d_token_slot, d_copies, workspace,
#     workspace_bytes, stream=None),
# lora_pages_fork(pages, d_parent, workspace, workspace_bytes, stream=None),
# lora_cache_copy(cache, num_copies, d_copies, stream=None),
# lora_beam_select(dtype, num_groups, beams, vocab, logits, ld, d_score, d_last_token, end_token, num_out, d_out_score, d_out_parent, d_out_token,
#     workspace, workspace_bytes, stream=None),
# lora_cache_digest(cache, num_tokens, max_new, d_indptr, d_bounds, d_steps, stream=None),
# lora_cache_choose(cache, dtype, num_heads, num_tokens, max_new, d_indptr, q, ldq, d_bounds, d_steps, budget, first, recent, d_chosen, workspace,
#     workspace_bytes, stream=None),
# lora_cache_attention_chosen(cache, dtype, num_heads, num_tokens, max_new, d_indptr, q, ldq, o, ldo, scale, budget, d_chosen, workspace,
#     workspace_bytes, stream=None)
(lora_pages_resize, lora_pages_fork, lora_cache_copy, lora_beam_select, lora_cache_digest, lora_cache_choose, lora_cache_attention_chosen) = (
    _calls.lora_pages_resize, _calls.lora_pages_fork, _calls.lora_cache_copy, _calls.lora_beam_select, _calls.lora_cache_digest, _calls.lora_cache_choose,
    _calls.lora_cache_attention_chosen)
