"""ctypes binding of include/*.h: same names, argument marshalling only.

Device buffers come from the caller (torch tensors, or raw integer addresses); every step of the
path runs in the library's kernels.  A non-OK status raises ``LoraError`` carrying the status name
and the library's detail line.  Loading fails loudly when the shared library has not been built.
"""
from __future__ import annotations

import ctypes
import os
from operator import index
from typing import Optional, Sequence

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
# LORA_GFX950_LIB selects another build of the same library (the measurement build with device clocks)
LIB_PATH = os.environ.get("LORA_GFX950_LIB") or os.path.join(_PKG, "liblora_gfx950.so")

LORA_MAX_RANK = 256
LORA_BF16 = 1
STATUS = ("LORA_OK", "LORA_ERR_INVALID_ARG", "LORA_ERR_SHAPE", "LORA_ERR_OOM", "LORA_ERR_NOT_RESIDENT",
          "LORA_ERR_STALE_SEGMENTS", "LORA_ERR_WORKSPACE", "LORA_ERR_DEVICE")

# include/lora_experts.h.  Builds of the host source alone do not have these; a call then ends in an AttributeError.
_EXPERTS = (
    "lora_rows_quantize", "lora_experts_packed_bytes", "lora_experts_pack_weight", "lora_linear_scaled", "lora_experts_group_workspace_bytes",
    "lora_experts_group", "lora_experts_linear", "lora_experts_linear_scaled", "lora_experts_combine",
)
# include/lora_attention.h, on the same terms.
_ATTENTION = ("lora_rotary_turns", "lora_rotary", "lora_cache_append", "lora_attention_workspace_bytes", "lora_attention")
# every symbol include/*.h declare
EXPORTS = (
    "lora_pool_bytes", "lora_pool_create", "lora_pool_create_live", "lora_pool_load", "lora_pool_evict",
    "lora_pool_reserve", "lora_pool_mark_resident", "lora_pool_space", "lora_pool_compact", "lora_pool_adapter_info",
    "lora_pool_destroy", "lora_pool_load_staging_bytes", "lora_pool_load_staged", "lora_segments_plan",
    "lora_segments_plan_opts", "lora_segments_set_options", "lora_segments_table_bytes", "lora_segments_upload_to",
    "lora_segments_build_opts", "lora_segments_plan_multi_opts", "lora_segments_build_multi_opts", "lora_segments_plan_ranges", "lora_segments_upload",
    "lora_segments_build", "lora_segments_build_ranges", "lora_segments_rebuild", "lora_segments_info",
    "lora_segments_export", "lora_segments_export_units", "lora_segments_export_launch_units", "lora_segments_destroy", "lora_workspace_bytes",
    "lora_shrink", "lora_expand", "lora_apply_workspace_bytes", "lora_apply", "lora_apply_static", "lora_linear_pack_weight", "lora_linear",
    "lora_profile_next_apply",
    "lora_segments_plan_multi", "lora_segments_build_multi", "lora_apply_multi",
    "lora_set_fused_apply", "lora_set_decode_single_launch", "lora_set_whole_k_limit", "lora_segments_check", "lora_set_side_stream", "lora_set_merged_launches", "lora_set_fused_wait_limit",
    "lora_status_string",
    "lora_last_error",
    "lora_place_extrapolate", "lora_place_assign",
) + _EXPERTS + _ATTENTION


class LoraError(RuntimeError):
    def __init__(self, status: int, detail: str):
        self.status = status
        self.status_name = STATUS[status] if 0 <= status < len(STATUS) else f"status {status}"
        self.detail = detail
        super().__init__(f"{self.status_name}: {detail}")


class _Desc(ctypes.Structure):
    _fields_ = [("in_features", ctypes.c_int32), ("out_features", ctypes.c_int32), ("n_adapters", ctypes.c_int32),
                ("ranks", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("dtype", ctypes.c_int32)]


class _AdapterInfo(ctypes.Structure):
    _fields_ = [("a_offset", ctypes.c_uint64), ("b_offset", ctypes.c_uint64), ("rank", ctypes.c_int32),
                ("rank_padded", ctypes.c_int32), ("scale", ctypes.c_float), ("resident", ctypes.c_int32)]


class _SegInfo(ctypes.Structure):
    _fields_ = [("n_tokens", ctypes.c_int32), ("n_active", ctypes.c_int32), ("n_segments", ctypes.c_int32),
                ("n_shrink_units", ctypes.c_int32), ("n_expand_units", ctypes.c_int32),
                ("n_k_slices", ctypes.c_int32), ("v_floats", ctypes.c_int64), ("weight_bytes", ctypes.c_int64),
                ("single_launch", ctypes.c_int32), ("launch_work_groups", ctypes.c_int32)]


class _PlanOptions(ctypes.Structure):
    _fields_ = [("whole_k_limit", ctypes.c_int32), ("merged_launches", ctypes.c_int32), ("side_stream", ctypes.c_int32),
                ("fused_apply", ctypes.c_int32), ("decode_single_launch", ctypes.c_int32),
                ("fused_wait_limit", ctypes.c_uint32), ("whole_k_max_in", ctypes.c_int32),
                ("heavy_min_tokens", ctypes.c_int32), ("heavy_min_batch", ctypes.c_int32),
                ("heavy_k_cut_max_units", ctypes.c_int32), ("big_runs_max_units", ctypes.c_int32)]


def plan_options(whole_k_limit: int = -1, merged_launches: int = -1, side_stream: int = -1, fused_apply: int = -1,
                 decode_single_launch: int = -1, fused_wait_limit: int = 0, whole_k_max_in: int = -1,
                 heavy_min_tokens: int = -1, heavy_min_batch: int = -1, heavy_k_cut_max_units: int = -1,
                 big_runs_max_units: int = -1) -> _PlanOptions:
    """lora_plan_options_t; -1 (0 for the wait limit) = the process-wide default or the built-in threshold."""
    return _PlanOptions(int(whole_k_limit), int(merged_launches), int(side_stream), int(fused_apply),
                        int(decode_single_launch), int(fused_wait_limit), int(whole_k_max_in), int(heavy_min_tokens),
                        int(heavy_min_batch), int(heavy_k_cut_max_units), int(big_runs_max_units))


def _opts(options):
    return ctypes.byref(options) if options is not None else None


_lib = None

# Argument types of the calls a serving loop makes for every projection or adapter: ctypes then converts plain
# ints itself, without an object per argument made here (a decode step of one token waits for the host:
# lora_apply of one token 9.8 -> 8.9 us a call, its launches included).
_P, _I32, _I64, _SZ, _F64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_double
_ARGTYPES = {
    "lora_pool_load": (_P, _I32, _P, _P, ctypes.c_int, _P),
    "lora_pool_load_staged": (_P, _I32, _P, _P, _P, _SZ, _P),
    "lora_segments_rebuild": (_P, _P, _I32, _P),
    "lora_shrink": (_P, _P, _P, _I64, _P, _P, _SZ, _P),
    "lora_expand": (_P, _P, _P, _P, _I64, _P),
    "lora_apply": (_P, _P, _P, _I64, _P, _I64, _P, _SZ, _P),
    "lora_apply_static": (_P, _P, _P, _I64, _P, _I64, _P),
    "lora_apply_multi": (_P, _I32, _P, _P, _I64, _P, _I64, _P, _SZ, _P),
    "lora_linear": (_P, _P, _P, _I64, _P, _P, _I64, _P, _SZ, _P),
    "lora_rows_quantize": (_P, _I64, _I64, _I32, _P, _I64, _P, _I64, _P),
    "lora_experts_packed_bytes": (_I32, _I32, _I32, _I32, _P),
    "lora_experts_pack_weight": (_P, _I32, _I32, _I32, _I32, _P, _SZ, _P),
    "lora_linear_scaled": (_P, _I64, _P, _I64, _I32, _I32, _P, _P, _I32, _P, _I64, _P),
    "lora_experts_group_workspace_bytes": (_I64, _I32, _P),
    "lora_experts_group": (_P, _I64, _I32, _I32, _I32, _P, _P, _P, _P, _SZ, _P),
    "lora_experts_linear": (_P, _I64, _I32, _P, _P, _I32, _I32, _I32, _I32, _P, _I32, _P, _I64, _P),
    "lora_experts_linear_scaled": (_P, _I64, _P, _I64, _I32, _P, _P, _I32, _I32, _I32, _I32, _P, _P, _I32, _P, _I64, _P),
    "lora_experts_combine": (_P, _I64, _I32, _P, _P, _I32, _I32, _I32, _P, _I64, _P),
    "lora_rotary_turns": (_I32, _F64, _I32, _F64, _F64, _F64, _F64, _P, _P),
    "lora_rotary": (_P, _I64, _I64, _I32, _I32, _I32, _P, _P, _I32, _P, _I64, _I64, _P),
    "lora_cache_append": (_P, _I64, _I64, _P, _I64, _I64, _I32, _P, _P, _P, _P, _P, _I64, _I64, _I32, _P, _I64, _I64, _P),
    "lora_attention_workspace_bytes": (_I32, _I32, _I32, _I32, _P, _P),
    "lora_attention": (_P, _I64, _I64, _I32, _I32, _P, _P, _I32, _P, _I64, _I32, _P, _I32, _P, ctypes.c_float, _P, _I64, _I64, _P, _SZ, _P),
}


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: run `python -m paper_2511_22880_amd.build` "
                              "(there is no fallback path)")
        L = ctypes.CDLL(LIB_PATH)
        for name in EXPORTS:
            if name in _EXPERTS + _ATTENTION and not hasattr(L, name):
                continue
            fn = getattr(L, name)
            fn.restype = ctypes.c_char_p if name in ("lora_status_string", "lora_last_error") else ctypes.c_int
            if name in _ARGTYPES:
                fn.argtypes = _ARGTYPES[name]
        _lib = L
    return _lib


def _check(status: int) -> None:
    if status != 0:
        raise LoraError(status, lib().lora_last_error().decode("utf-8", "replace"))


def _ptr(obj) -> ctypes.c_void_p:
    """Address of a torch tensor, a numpy array, or an integer address; None -> NULL."""
    if obj is None:
        return ctypes.c_void_p(None)
    if isinstance(obj, ctypes.c_void_p):
        return obj
    if isinstance(obj, int):
        return ctypes.c_void_p(obj)
    if isinstance(obj, np.ndarray):
        return ctypes.c_void_p(obj.ctypes.data)
    if hasattr(obj, "data_ptr"):
        return ctypes.c_void_p(obj.data_ptr())
    raise TypeError(f"cannot take the address of {type(obj)}")


def _addr(obj):
    """_ptr for the calls of _ARGTYPES: a plain int (or None, or a c_void_p)."""
    if hasattr(obj, "data_ptr"):
        return obj.data_ptr()
    return obj if obj is None or isinstance(obj, int) else _ptr(obj)


def _queue(stream):
    """_stream for the calls of _ARGTYPES."""
    if stream is None:
        return None
    return int(stream.cuda_stream if hasattr(stream, "cuda_stream") else stream)


def _stream(stream) -> ctypes.c_void_p:
    return ctypes.c_void_p(_queue(stream) or None)


def _i32(a) -> np.ndarray:
    return np.ascontiguousarray(a, dtype=np.int32)


class Pool:
    """Handle of a lora_pool_t plus the objects that must outlive it (arena tensor, desc arrays)."""

    def __init__(self, handle, in_features, out_features, ranks, scales, arena):
        self.handle = handle
        self.in_features, self.out_features = in_features, out_features
        self.ranks, self.scales = ranks, scales
        self.arena = arena

    @property
    def n_adapters(self) -> int:
        return int(self.ranks.shape[0])


class Segments:
    def __init__(self, handle, pool: Pool):
        self.handle = handle
        self.pool = pool


def _desc(in_features, out_features, ranks, scales):
    ranks = _i32(ranks)
    scales = np.ascontiguousarray(scales, dtype=np.float32)
    if ranks.shape != scales.shape:
        raise ValueError("ranks and scales differ in length")
    d = _Desc(int(in_features), int(out_features), int(ranks.shape[0]), ranks.ctypes.data, scales.ctypes.data,
              LORA_BF16)
    return d, ranks, scales


def lora_pool_bytes(in_features: int, out_features: int, ranks, scales) -> int:
    d, _r, _s = _desc(in_features, out_features, ranks, scales)
    n = ctypes.c_size_t(0)
    _check(lib().lora_pool_bytes(ctypes.byref(d), ctypes.byref(n)))
    return int(n.value)


def lora_pool_create(in_features: int, out_features: int, ranks, scales, dev_arena, arena_bytes: Optional[int] = None) -> Pool:
    """dev_arena: a torch device tensor (uint8/any dtype) or an integer device address."""
    d, r, s = _desc(in_features, out_features, ranks, scales)
    if arena_bytes is None:
        arena_bytes = dev_arena.numel() * dev_arena.element_size()
    h = ctypes.c_void_p(None)
    _check(lib().lora_pool_create(ctypes.byref(d), _ptr(dev_arena), ctypes.c_size_t(arena_bytes), ctypes.byref(h)))
    return Pool(h, int(in_features), int(out_features), r, s, dev_arena)


def lora_pool_create_live(in_features: int, out_features: int, ranks, scales, dev_arena,
                          arena_bytes: Optional[int] = None) -> Pool:
    """A pool over an arena of any size: adapters get their place when loaded (see include/lora.h)."""
    d, r, s = _desc(in_features, out_features, ranks, scales)
    if arena_bytes is None:
        arena_bytes = dev_arena.numel() * dev_arena.element_size()
    h = ctypes.c_void_p(None)
    _check(lib().lora_pool_create_live(ctypes.byref(d), _ptr(dev_arena), ctypes.c_size_t(arena_bytes), ctypes.byref(h)))
    return Pool(h, int(in_features), int(out_features), r, s, dev_arena)


def lora_pool_reserve(pool: Pool, adapter: int) -> None:
    _check(lib().lora_pool_reserve(pool.handle, ctypes.c_int32(adapter)))


def lora_pool_space(pool: Pool) -> dict:
    fr, lg = ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check(lib().lora_pool_space(pool.handle, ctypes.byref(fr), ctypes.byref(lg)))
    return {"free_bytes": int(fr.value), "largest_free_bytes": int(lg.value)}


def lora_pool_compact(pool: Pool, scratch=None, stream=None, scratch_bytes: Optional[int] = None) -> int:
    """Returns the number of adapters that were moved."""
    moved = ctypes.c_int32(0)
    nbytes = (_nbytes(scratch) if scratch is not None else 0) if scratch_bytes is None else scratch_bytes
    _check(lib().lora_pool_compact(pool.handle, _ptr(scratch), ctypes.c_size_t(nbytes), _stream(stream),
                                   ctypes.byref(moved)))
    return int(moved.value)


def lora_pool_load(pool: Pool, adapter: int, A, B, src_is_device: Optional[bool] = None, stream=None) -> None:
    """A [in][rank], B [rank][out] bf16: numpy uint16 arrays (host) or torch device tensors."""
    host = isinstance(A, np.ndarray)
    if src_is_device is None:
        src_is_device = not host
    if host:
        A, B = np.ascontiguousarray(A), np.ascontiguousarray(B)
        r = int(pool.ranks[adapter]) if 0 <= adapter < pool.n_adapters else -1
        if r >= 0 and (A.shape != (pool.in_features, r) or B.shape != (r, pool.out_features) or A.itemsize != 2
                       or B.itemsize != 2):
            raise ValueError(f"adapter {adapter}: A {A.shape} / B {B.shape} do not match rank {r}")
    try:
        a, b = A.data_ptr(), B.data_ptr()
    except AttributeError:
        a, b = _addr(A), _addr(B)
    status = (_lib or lib()).lora_pool_load(pool.handle, index(adapter), a, b, 1 if src_is_device else 0,
                                            None if stream is None else _queue(stream))
    if status:
        _check(status)


def lora_pool_evict(pool: Pool, adapter: int) -> None:
    _check(lib().lora_pool_evict(pool.handle, ctypes.c_int32(adapter)))


def lora_pool_mark_resident(pool: Pool, adapter: int) -> None:
    _check(lib().lora_pool_mark_resident(pool.handle, ctypes.c_int32(adapter)))


def lora_pool_adapter_info(pool: Pool, adapter: int) -> dict:
    info = _AdapterInfo()
    _check(lib().lora_pool_adapter_info(pool.handle, ctypes.c_int32(adapter), ctypes.byref(info)))
    return {k: getattr(info, k) for k, _ in _AdapterInfo._fields_}


def lora_pool_destroy(pool: Pool) -> None:
    if pool.handle:
        _check(lib().lora_pool_destroy(pool.handle))
        pool.handle = ctypes.c_void_p(None)


def lora_segments_plan(pool: Pool, token_adapter, options=None) -> Segments:
    ta = _i32(token_adapter)
    h = ctypes.c_void_p(None)
    _check(lib().lora_segments_plan_opts(pool.handle, _ptr(ta), ctypes.c_int32(ta.shape[0]), _opts(options),
                                         ctypes.byref(h)))
    return Segments(h, pool)


def lora_segments_set_options(seg: Segments, options=None) -> None:
    _check(lib().lora_segments_set_options(seg.handle, _opts(options)))


def lora_segments_table_bytes(seg: Segments) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().lora_segments_table_bytes(seg.handle, ctypes.byref(n)))
    return int(n.value)


def lora_segments_upload_to(seg: Segments, dev_table, host_staging, stream=None) -> None:
    """dev_table: device tensor; host_staging: pinned host tensor; both at least lora_segments_table_bytes long."""
    _check(lib().lora_segments_upload_to(seg.handle, _ptr(dev_table), ctypes.c_size_t(_nbytes(dev_table)),
                                         _ptr(host_staging), ctypes.c_size_t(_nbytes(host_staging)), _stream(stream)))
    seg.keepalive = (dev_table, host_staging)


def lora_pool_load_staging_bytes(pool: Pool, adapter: int) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().lora_pool_load_staging_bytes(pool.handle, ctypes.c_int32(adapter), ctypes.byref(n)))
    return int(n.value)


def lora_pool_load_staged(pool: Pool, adapter: int, A, B, dev_staging, stream=None) -> None:
    """A, B: host arrays (numpy uint16 or pinned torch tensors); dev_staging: device tensor of the caller's."""
    n = ctypes.c_int32(adapter).value
    if 0 <= n < pool.n_adapters:
        r = int(pool.ranks[n])
        for name, obj, features in (("A", A, pool.in_features), ("B", B, pool.out_features)):
            have = getattr(obj, "nbytes", None)  # (an address states no size)
            if have is not None and have < 2 * r * features:
                raise ValueError(f"adapter {n}: {name} of {have} bytes is shorter than rank {r} x {features} bf16 values")
    _check(lib().lora_pool_load_staged(pool.handle, ctypes.c_int32(adapter), _addr(A), _addr(B), _addr(dev_staging), _nbytes(dev_staging),
                                       _queue(stream)))


def lora_segments_plan_ranges(pool: Pool, seg_start, seg_adapter) -> Segments:
    st, ad = _i32(seg_start), _i32(seg_adapter)
    if st.shape[0] != ad.shape[0] + 1:
        raise ValueError("seg_start has one more entry than seg_adapter")
    h = ctypes.c_void_p(None)
    _check(lib().lora_segments_plan_ranges(pool.handle, _ptr(st), _ptr(ad), ctypes.c_int32(ad.shape[0]), ctypes.byref(h)))
    return Segments(h, pool)


def lora_segments_upload(seg: Segments, stream=None) -> None:
    _check(lib().lora_segments_upload(seg.handle, _stream(stream)))


def lora_segments_build(pool: Pool, token_adapter, stream=None, options=None) -> Segments:
    ta = _i32(token_adapter)
    h = ctypes.c_void_p(None)
    _check(lib().lora_segments_build_opts(pool.handle, _ptr(ta), ctypes.c_int32(ta.shape[0]), _opts(options),
                                          _stream(stream), ctypes.byref(h)))
    return Segments(h, pool)


def lora_segments_build_ranges(pool: Pool, seg_start, seg_adapter, stream=None) -> Segments:
    st, ad = _i32(seg_start), _i32(seg_adapter)
    if st.shape[0] != ad.shape[0] + 1:
        raise ValueError("seg_start has one more entry than seg_adapter")
    h = ctypes.c_void_p(None)
    _check(lib().lora_segments_build_ranges(pool.handle, _ptr(st), _ptr(ad), ctypes.c_int32(ad.shape[0]),
                                            _stream(stream), ctypes.byref(h)))
    return Segments(h, pool)


def lora_segments_rebuild(seg: Segments, token_adapter, stream=None) -> None:
    ta = _i32(token_adapter)
    _check(lib().lora_segments_rebuild(seg.handle, _addr(ta), ta.shape[0], _queue(stream)))


def lora_segments_info(seg: Segments) -> dict:
    info = _SegInfo()
    _check(lib().lora_segments_info(seg.handle, ctypes.byref(info)))
    return {k: getattr(info, k) for k, _ in _SegInfo._fields_}


def lora_segments_export(seg: Segments) -> dict:
    i = lora_segments_info(seg)
    perm = np.zeros(i["n_active"], dtype=np.int32)
    start = np.zeros(i["n_segments"] + 1, dtype=np.int32)
    adapter = np.zeros(i["n_segments"], dtype=np.int32)
    voff = np.zeros(i["n_tokens"], dtype=np.int64)
    _check(lib().lora_segments_export(seg.handle, _ptr(perm), _ptr(start), _ptr(adapter), _ptr(voff)))
    return {"perm": perm, "seg_start": start, "seg_adapter": adapter, "v_offset": voff}


def lora_segments_export_units(seg: Segments) -> dict:
    i = lora_segments_info(seg)
    su = np.zeros((i["n_shrink_units"], 6), dtype=np.int32)
    eu = np.zeros((i["n_expand_units"], 6), dtype=np.int32)
    _check(lib().lora_segments_export_units(seg.handle, _ptr(su), _ptr(eu)))
    return {"shrink": su, "expand": eu}


def lora_segments_export_launch_units(seg: Segments) -> dict:
    """The one-launch decode form's lists by place in the launch, 7 int32 per place."""
    g = lora_segments_info(seg)["launch_work_groups"]
    su = np.zeros((g, 7), dtype=np.int32)
    eu = np.zeros((4 * g, 7), dtype=np.int32)
    _check(lib().lora_segments_export_launch_units(seg.handle, _ptr(su), _ptr(eu)))
    return {"shrink": su, "expand": eu}


def lora_segments_destroy(seg: Segments) -> None:
    if seg.handle:
        _check(lib().lora_segments_destroy(seg.handle))
        seg.handle = ctypes.c_void_p(None)


def lora_workspace_bytes(pool: Pool, seg: Segments) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().lora_workspace_bytes(pool.handle, seg.handle, ctypes.byref(n)))
    return int(n.value)


def lora_apply_workspace_bytes(pool: Pool, seg: Segments) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().lora_apply_workspace_bytes(pool.handle, seg.handle, ctypes.byref(n)))
    return int(n.value)


def _ld(t, ld):
    if ld is not None:
        return int(ld)
    return int(t.stride(0)) if hasattr(t, "stride") else 0


def _nbytes(ws) -> int:
    return 0 if ws is None else ws.numel() * ws.element_size()


def _ws_bytes(workspace, ws_bytes):
    return _nbytes(workspace) if ws_bytes is None else ctypes.c_size_t(ws_bytes)


# The calls of a serving loop take their common arguments, tensors that state their own strides and sizes, without the helpers above;
# anything else (an address, an array, None) has no such attributes and goes through them.
def lora_shrink(pool: Pool, seg: Segments, x, v, workspace=None, stream=None, ldx: Optional[int] = None,
                ws_bytes: Optional[int] = None) -> None:
    """x: bf16 device tensor [T][in]; v: fp32 device tensor of info['v_floats'] elements."""
    try:
        px, pv, pw = x.data_ptr(), v.data_ptr(), workspace.data_ptr()
        lx = x.stride(0) if ldx is None else int(ldx)
        nw = workspace.nbytes if ws_bytes is None else ctypes.c_size_t(ws_bytes)
    except AttributeError:
        px, pv, pw, lx, nw = _addr(x), _addr(v), _addr(workspace), _ld(x, ldx), _ws_bytes(workspace, ws_bytes)
    status = (_lib or lib()).lora_shrink(pool.handle, seg.handle, px, lx, pv, pw, nw, None if stream is None else _queue(stream))
    if status:
        _check(status)


def lora_expand(pool: Pool, seg: Segments, v, y, stream=None, ldy: Optional[int] = None) -> None:
    """y: bf16 device tensor [T][out], updated in place."""
    try:
        pv, py = v.data_ptr(), y.data_ptr()
        ly = y.stride(0) if ldy is None else int(ldy)
    except AttributeError:
        pv, py, ly = _addr(v), _addr(y), _ld(y, ldy)
    status = (_lib or lib()).lora_expand(pool.handle, seg.handle, pv, py, ly, None if stream is None else _queue(stream))
    if status:
        _check(status)


def lora_apply(pool: Pool, seg: Segments, x, y, workspace, stream=None, ldx: Optional[int] = None,
               ldy: Optional[int] = None, ws_bytes: Optional[int] = None) -> None:
    try:
        px, py, pw = x.data_ptr(), y.data_ptr(), workspace.data_ptr()
        lx = x.stride(0) if ldx is None else int(ldx)
        ly = y.stride(0) if ldy is None else int(ldy)
        nw = workspace.nbytes if ws_bytes is None else ctypes.c_size_t(ws_bytes)
    except AttributeError:
        px, py, pw, lx, ly, nw = _addr(x), _addr(y), _addr(workspace), _ld(x, ldx), _ld(y, ldy), _ws_bytes(workspace, ws_bytes)
    status = (_lib or lib()).lora_apply(pool.handle, seg.handle, px, lx, py, ly, pw, nw, None if stream is None else _queue(stream))
    if status:
        _check(status)


def lora_linear_pack_weight(wt, in_features: int, out_features: int, dev_packed, stream=None) -> None:
    """wt: device tensor W^T [out][in] bf16; dev_packed: device tensor of in * out * 2 bytes."""
    _check(lib().lora_linear_pack_weight(_ptr(wt), ctypes.c_int32(in_features), ctypes.c_int32(out_features),
                                         _ptr(dev_packed), _stream(stream)))


def lora_linear(pool: Pool, seg: Segments, x, w_packed, y, workspace, stream=None, ldx: Optional[int] = None,
                ldy: Optional[int] = None, ws_bytes: Optional[int] = None) -> None:
    """y = bf16(x W + delta) for every token, y written once."""
    try:
        px, pp, py, pw = x.data_ptr(), w_packed.data_ptr(), y.data_ptr(), workspace.data_ptr()
        lx = x.stride(0) if ldx is None else int(ldx)
        ly = y.stride(0) if ldy is None else int(ldy)
        nw = workspace.nbytes if ws_bytes is None else ctypes.c_size_t(ws_bytes)
    except AttributeError:
        px, pp, py, pw = _addr(x), _addr(w_packed), _addr(y), _addr(workspace)
        lx, ly, nw = _ld(x, ldx), _ld(y, ldy), _ws_bytes(workspace, ws_bytes)
    status = (_lib or lib()).lora_linear(pool.handle, seg.handle, px, lx, pp, py, ly, pw, nw,
                                         None if stream is None else _queue(stream))
    if status:
        _check(status)


LORA_STATIC_WORKSPACE_BYTES = 32 << 20


def lora_apply_static(pool: Pool, seg: Segments, x, y, stream=None, ldx: Optional[int] = None,
                      ldy: Optional[int] = None) -> None:
    """lora_apply on the library's own static workspace: allocates nothing."""
    _check(lib().lora_apply_static(pool.handle, seg.handle, _addr(x), _ld(x, ldx), _addr(y), _ld(y, ldy), _queue(stream)))


def _pool_array(pools):
    arr = (ctypes.c_void_p * len(pools))(*[p.handle.value for p in pools])
    return arr


def lora_segments_plan_multi(pools, token_adapter, options=None) -> Segments:
    ta = _i32(token_adapter)
    h = ctypes.c_void_p(None)
    _check(lib().lora_segments_plan_multi_opts(_pool_array(pools), ctypes.c_int32(len(pools)), _ptr(ta),
                                               ctypes.c_int32(ta.shape[0]), _opts(options), ctypes.byref(h)))
    return Segments(h, pools[0])


def lora_segments_build_multi(pools, token_adapter, stream=None, options=None) -> Segments:
    ta = _i32(token_adapter)
    h = ctypes.c_void_p(None)
    _check(lib().lora_segments_build_multi_opts(_pool_array(pools), ctypes.c_int32(len(pools)), _ptr(ta),
                                                ctypes.c_int32(ta.shape[0]), _opts(options), _stream(stream),
                                                ctypes.byref(h)))
    return Segments(h, pools[0])


def lora_apply_multi(pools, seg: Segments, x, y, workspace, stream=None, ldx: Optional[int] = None,
                     ldy: Optional[int] = None, ws_bytes: Optional[int] = None) -> None:
    """y: bf16 device tensor [T][sum of the pools' out_features], updated in place."""
    try:
        px, py, pw = x.data_ptr(), y.data_ptr(), workspace.data_ptr()
        lx = x.stride(0) if ldx is None else int(ldx)
        ly = y.stride(0) if ldy is None else int(ldy)
        nw = workspace.nbytes if ws_bytes is None else ctypes.c_size_t(ws_bytes)
    except AttributeError:
        px, py, pw, lx, ly, nw = _addr(x), _addr(y), _addr(workspace), _ld(x, ldx), _ld(y, ldy), _ws_bytes(workspace, ws_bytes)
    status = (_lib or lib()).lora_apply_multi(_pool_array(pools), len(pools), seg.handle, px, lx, py, ly, pw, nw,
                                              None if stream is None else _queue(stream))
    if status:
        _check(status)


def _switch(enabled) -> ctypes.c_int:
    return ctypes.c_int(-1 if enabled == -1 else 1 if enabled else 0)


def lora_set_fused_apply(enabled) -> None:
    """True, False, or -1: the library's own choice, as before the first call."""
    _check(lib().lora_set_fused_apply(_switch(enabled)))


def lora_set_decode_single_launch(enabled) -> None:
    """True, False, or -1: the library's own choice, as before the first call."""
    _check(lib().lora_set_decode_single_launch(_switch(enabled)))


def lora_set_side_stream(enabled: bool) -> None:
    _check(lib().lora_set_side_stream(ctypes.c_int(1 if enabled else 0)))


def lora_set_merged_launches(enabled: bool) -> None:
    _check(lib().lora_set_merged_launches(ctypes.c_int(1 if enabled else 0)))


def lora_set_fused_wait_limit(polls: int) -> None:
    _check(lib().lora_set_fused_wait_limit(ctypes.c_uint32(polls)))


def lora_set_whole_k_limit(max_units: int) -> None:
    _check(lib().lora_set_whole_k_limit(ctypes.c_int32(int(max_units))))


def lora_segments_check(seg: Segments, stream=None) -> None:
    _check(lib().lora_segments_check(seg.handle, _stream(stream)))


def lora_profile_next_apply(before=None, between=None, after=None) -> None:
    """hipEvent_t handles (integers) recorded around the two launches of the next lora_apply."""
    _check(lib().lora_profile_next_apply(_ptr(before), _ptr(between), _ptr(after)))


def lora_debug_clock_buffer(dev_buf, n_work_groups: int) -> None:
    """Measurement build only: 8 uint64 clock values (100 MHz) per work group of the launches that follow."""
    fn = getattr(lib(), "lora_debug_clock_buffer", None)
    if fn is None:
        raise RuntimeError("this build of the library has no device clocks: build with `python -m "
                           "paper_2511_22880_amd.build --clocks` and set LORA_GFX950_LIB to it")
    rc = fn(_ptr(dev_buf), ctypes.c_uint(int(n_work_groups)))
    if rc != 0:
        raise RuntimeError(f"lora_debug_clock_buffer: hip error {rc}")


def lora_status_string(status: int) -> str:
    return lib().lora_status_string(ctypes.c_int(status)).decode()


def lora_last_error() -> str:
    return lib().lora_last_error().decode("utf-8", "replace")


# ---- adapter placement and routing (include/lora_placement.h; host only) ----------------------------
class _PlaceProblem(ctypes.Structure):
    _fields_ = [("n_servers", ctypes.c_int32), ("n_adapters", ctypes.c_int32), ("ranks", ctypes.c_void_p),
                ("demand_tps", ctypes.c_void_p), ("n_ops", ctypes.c_int32), ("op_ranks", ctypes.c_void_p),
                ("op_tps", ctypes.c_void_p), ("prev_phi", ctypes.c_void_p)]


def lora_place_extrapolate(history, current: float) -> float:
    h = np.ascontiguousarray(history, dtype=np.float64)
    out = ctypes.c_double(0.0)
    _check(lib().lora_place_extrapolate(_ptr(h) if h.size else ctypes.c_void_p(None), ctypes.c_int32(h.size),
                                        ctypes.c_double(float(current)), ctypes.byref(out)))
    return float(out.value)


def lora_place_assign(n_servers: int, ranks, demand_tps, operating_points: dict, prev_phi=None) -> dict:
    """operating_points: {rank: tokens/s}.  Returns phi [n_adapters][n_servers], server_util,
    server_max_rank, budget {rank: servers} and target."""
    ranks = _i32(ranks)
    demand = np.ascontiguousarray(demand_tps, dtype=np.float64)
    op_r = _i32(sorted(operating_points))
    op_t = np.ascontiguousarray([operating_points[int(r)] for r in op_r], dtype=np.float64)
    prev = None if prev_phi is None else np.ascontiguousarray(prev_phi, dtype=np.float64)
    n = int(ranks.shape[0])
    phi = np.zeros((n, n_servers), dtype=np.float64)
    util = np.zeros(n_servers, dtype=np.float64)
    maxr = np.zeros(n_servers, dtype=np.int32)
    budget = np.zeros(op_r.shape[0], dtype=np.int32)
    target = ctypes.c_double(0.0)
    pr = _PlaceProblem(int(n_servers), n, ranks.ctypes.data, demand.ctypes.data, int(op_r.shape[0]), op_r.ctypes.data,
                       op_t.ctypes.data, None if prev is None else prev.ctypes.data)
    _check(lib().lora_place_assign(ctypes.byref(pr), _ptr(phi), _ptr(util), _ptr(maxr), _ptr(budget),
                                   ctypes.byref(target)))
    return {"phi": phi, "server_util": util, "server_max_rank": maxr,
            "budget": {int(r): int(b) for r, b in zip(op_r, budget)}, "target": float(target.value)}


# ---- frozen layers beside an adapter, in block-scaled 8 bits and grouped by expert (include/lora_experts.h) ----------------
# The arguments are torch device tensors, whose shapes and strides say what the C calls are told; a tensor of another type, one that is not on a GPU, or one that
# cannot hold what a call writes or reads there, is refused here, since the library sees addresses only.
# Element types, filled in when the first tensor comes (this module does not import torch).  bf16 and 8-bit values may also come as their bits.
_BF16, _F32, _INT32, _E4M3 = set(), set(), set(), set()


def _know_types() -> None:
    import torch
    _BF16.update((torch.bfloat16, torch.uint16))
    _F32.add(torch.float32)
    _INT32.add(torch.int32)
    _E4M3.update((torch.float8_e4m3fn, torch.uint8))


def _blocks(n: int) -> int:
    return (n + 127) >> 7


# What a tensor is asked for costs 0.1 us each time, and so does a call of Python's: the calls below, which a decode step waits for, ask for shape and
# strides once, in line, and compare; where anything is unusual _usable, _whole and _packed look closer.
def _names(types) -> str:
    return " or ".join(sorted(str(t).replace("torch.", "") for t in types))


def _on_gpu(name: str, t) -> None:
    if not t.is_cuda:
        raise ValueError(f"{name}: a tensor on {t.device} does not do: one on the GPU is meant")


def _usable(name: str, t, rows: int, columns: int, types: set) -> None:
    """Refuses a tensor that does not hold so many rows of so many elements of one of these types, side by side within a row."""
    if not types:
        _know_types()
    if t.dtype not in types:
        raise ValueError(f"{name}: {t.dtype} does not do: {_names(types)} is meant")
    if t.dim() != 2 or t.shape[0] < rows or t.shape[1] < columns or (t.stride(1) != 1 and t.shape[1] > 1):
        raise ValueError(f"{name}: {tuple(t.shape)} with strides {t.stride()} does not do: {rows} rows of {columns} elements side by side are meant")
    _on_gpu(name, t)


def _whole(name: str, t, n: int, types: set) -> None:
    """Refuses a tensor that is not n contiguous elements, or more, of one of these types."""
    if not types:
        _know_types()
    if t.dtype not in types:
        raise ValueError(f"{name}: {t.dtype} does not do: {_names(types)} is meant")
    if t.numel() < n or not t.is_contiguous():
        raise ValueError(f"{name}: {tuple(t.shape)} with strides {t.stride()} does not do: {n} contiguous elements are meant")
    _on_gpu(name, t)


def _packed(t, n: int) -> None:
    """Refuses packed weights that are not n contiguous bytes, of whatever type, or more."""
    if t.nbytes < n or not t.is_contiguous():
        raise ValueError(f"w_packed: {tuple(t.shape)} of {t.dtype} does not do: {n} contiguous bytes are meant")
    _on_gpu("w_packed", t)


def _two(t, name: str):
    """Shape and strides of a tensor of rows."""
    if t.dim() != 2:
        raise ValueError(f"{name}: {tuple(t.shape)} does not do: rows are meant")
    return t.shape, t.stride()


def _last_block(q, rows: int, ldq: int, row: int) -> None:
    """The products read a row's last block of 128 whole, so memory goes on that far behind columns that end inside it."""
    if q.storage_offset() + (rows - 1) * ldq + row > q.untyped_storage().nbytes():
        raise ValueError(f"q: the last row's block of 128 that column {q.shape[1]} ends in is not all there")


def lora_rows_quantize(x, q, scales, stream=None) -> None:
    """x: bf16 [rows][in]; q: 8-bit [rows][128 * blocks]; scales: fp32 [rows][blocks]."""
    try:
        (rows, in_f), (ldx, x1) = x.shape, x.stride()
        (qr, qc), (ldq, q1) = q.shape, q.stride()
        (sr, sc), (lds, s1) = scales.shape, scales.stride()
    except ValueError:
        (rows, in_f), (ldx, x1), (qr, qc), (ldq, q1), (sr, sc), (lds, s1) = _two(x, "x") + _two(q, "q") + _two(scales, "scales")
    blocks = (in_f + 127) >> 7
    if x1 != 1 or x.dtype not in _BF16 or not x.is_cuda:
        _usable("x", x, rows, in_f, _BF16)
    if qr < rows or qc < blocks << 7 or q1 != 1 or q.dtype not in _E4M3 or not q.is_cuda:
        _usable("q", q, rows, blocks << 7, _E4M3)
    if sr < rows or sc < blocks or s1 != 1 or scales.dtype not in _F32 or not scales.is_cuda:
        _usable("scales", scales, rows, blocks, _F32)
    if rows == 1:  # (of a single row torch states any stride)
        ldx = in_f
    if qr == 1:
        ldq = blocks << 7
    if sr == 1:
        lds = sc
    status = (_lib or lib()).lora_rows_quantize(x.data_ptr(), ldx, rows, in_f, q.data_ptr(), ldq, scales.data_ptr(), lds,
                                                None if stream is None else _queue(stream))
    if status:
        _check(status)


def lora_experts_packed_bytes(n_experts: int, in_features: int, out_features: int, bits: int) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().lora_experts_packed_bytes(n_experts, in_features, out_features, bits, ctypes.addressof(n)))
    return int(n.value)


def lora_experts_pack_weight(w, dev_packed, stream=None, in_features: Optional[int] = None) -> None:
    """w: [experts][out][in] bf16, or 8-bit with rows of 128 * blocks; dev_packed: lora_experts_packed_bytes long."""
    e, out_f, row = w.shape
    bits = 8 * w.itemsize
    in_f = row if in_features is None else int(in_features)
    if row != (in_f if bits == 16 else _blocks(in_f) << 7):
        raise ValueError(f"w: rows of {row} elements are not those of {in_f} input features")
    _on_gpu("dev_packed", dev_packed)
    _whole("w", w, 0, _BF16 if bits == 16 else _E4M3)
    _check(lib().lora_experts_pack_weight(w.data_ptr(), e, in_f, out_f, bits, dev_packed.data_ptr(), _nbytes(dev_packed), _queue(stream)))


def lora_linear_scaled(q, scales, w_packed, w_scales, y, stream=None) -> None:
    """q, scales: of lora_rows_quantize, q's columns all or the first in_features; w_packed: uint8; w_scales: fp32 [out / 128][blocks]; y: bf16 [rows][out]."""
    try:
        (rows, in_f), (ldq, q1) = q.shape, q.stride()
        (sr, sc), (lds, s1) = scales.shape, scales.stride()
        (yr, out_f), (ldy, y1) = y.shape, y.stride()
    except ValueError:
        (rows, in_f), (ldq, q1), (sr, sc), (lds, s1), (yr, out_f), (ldy, y1) = _two(q, "q") + _two(scales, "scales") + _two(y, "y")
    blocks = (in_f + 127) >> 7
    if q1 != 1 or q.dtype not in _E4M3 or not q.is_cuda:
        _usable("q", q, rows, in_f, _E4M3)
    if sr < rows or sc < blocks or s1 != 1 or scales.dtype not in _F32 or not scales.is_cuda:
        _usable("scales", scales, rows, blocks, _F32)
    if yr < rows or y1 != 1 or y.dtype not in _BF16 or not y.is_cuda:
        _usable("y", y, rows, out_f, _BF16)
    if rows == 1:
        ldq = blocks << 7
    if in_f & 127:
        _last_block(q, rows, ldq, blocks << 7)
    if sr == 1:
        lds = sc
    if yr == 1:
        ldy = out_f
    if w_packed.nbytes < out_f * blocks << 7 or not w_packed.is_contiguous() or not w_packed.is_cuda:
        _packed(w_packed, out_f * blocks << 7)
    if w_scales.dtype not in _F32 or w_scales.numel() < (out_f >> 7) * blocks or not w_scales.is_contiguous() or not w_scales.is_cuda:
        _whole("w_scales", w_scales, (out_f >> 7) * blocks, _F32)
    status = (_lib or lib()).lora_linear_scaled(q.data_ptr(), ldq, scales.data_ptr(), lds, rows, in_f, w_packed.data_ptr(), w_scales.data_ptr(), out_f,
                                                y.data_ptr(), ldy,
                                                None if stream is None else _queue(stream))
    if status:
        _check(status)


def lora_experts_group_workspace_bytes(n_picks: int, n_experts: int) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().lora_experts_group_workspace_bytes(n_picks, n_experts, ctypes.addressof(n)))
    return int(n.value)


def lora_experts_group(ids, starts, order, place, workspace=None, stream=None) -> None:
    """ids: int32 [tokens][picks]; written: starts [experts + 1], order and place [tokens * picks], int32."""
    try:
        (tokens, picks), (ldi, i1) = ids.shape, ids.stride()
    except ValueError:
        (tokens, picks), (ldi, i1) = _two(ids, "ids")
    n_experts, n = starts.numel() - 1, tokens * picks
    if n > 0x7FFFFFFF:  # (ctypes passes on the low 32 bits of the tokens)
        raise ValueError(f"ids: {tokens} tokens x {picks} picks do not fit 32 bits")
    if i1 != 1 or ids.dtype not in _INT32 or not ids.is_cuda:
        _usable("ids", ids, tokens, picks, _INT32)
    if workspace is None:
        pw, nw = None, 0
    else:
        if not workspace.is_cuda or not workspace.is_contiguous():
            _on_gpu("workspace", workspace)
            raise ValueError(f"workspace: strides {workspace.stride()} do not do: contiguous bytes are meant")
        pw, nw = workspace.data_ptr(), workspace.nbytes
    if starts.dtype not in _INT32 or n_experts < 0 or not starts.is_contiguous() or not starts.is_cuda:
        _whole("starts", starts, 1, _INT32)
    if order.dtype not in _INT32 or order.numel() < n or not order.is_contiguous() or not order.is_cuda:
        _whole("order", order, n, _INT32)
    if place.dtype not in _INT32 or place.numel() < n or not place.is_contiguous() or not place.is_cuda:
        _whole("place", place, n, _INT32)
    status = (_lib or lib()).lora_experts_group(ids.data_ptr(), ldi if tokens > 1 else picks, tokens, picks, n_experts, starts.data_ptr(), order.data_ptr(),
                                                place.data_ptr(), pw, nw,
                                                None if stream is None else _queue(stream))
    if status:
        _check(status)


def lora_experts_linear(x, starts, order, picks: int, w_packed, y, stream=None) -> None:
    """x: bf16 [tokens][in]; starts, order: of lora_experts_group (order None: x is in expert order); y: bf16 [tokens * picks][out]."""
    try:
        (tokens, in_f), (ldx, x1) = x.shape, x.stride()
        (yr, out_f), (ldy, y1) = y.shape, y.stride()
    except ValueError:
        (tokens, in_f), (ldx, x1), (yr, out_f), (ldy, y1) = _two(x, "x") + _two(y, "y")
    n_experts, n_rows = starts.numel() - 1, tokens if order is None else tokens * picks
    if x1 != 1 or x.dtype not in _BF16 or not x.is_cuda:
        _usable("x", x, tokens, in_f, _BF16)
    if yr < n_rows or y1 != 1 or y.dtype not in _BF16 or not y.is_cuda:
        _usable("y", y, n_rows, out_f, _BF16)
    if tokens == 1:
        ldx = in_f
    if yr == 1:
        ldy = out_f
    if starts.dtype not in _INT32 or n_experts < 0 or not starts.is_contiguous() or not starts.is_cuda:
        _whole("starts", starts, 1, _INT32)
    if order is not None and (order.dtype not in _INT32 or order.numel() < n_rows or not order.is_contiguous() or not order.is_cuda):
        _whole("order", order, n_rows, _INT32)
    if w_packed.nbytes < n_experts * out_f * in_f << 1 or not w_packed.is_contiguous() or not w_packed.is_cuda:
        _packed(w_packed, n_experts * out_f * in_f << 1)
    status = (_lib or lib()).lora_experts_linear(x.data_ptr(), ldx, tokens, starts.data_ptr(), None if order is None else order.data_ptr(), picks, n_rows,
                                                 n_experts, in_f, w_packed.data_ptr(), out_f, y.data_ptr(), ldy,
                                                 None if stream is None else _queue(stream))
    if status:
        _check(status)


def lora_experts_linear_scaled(q, scales, starts, order, picks: int, w_packed, w_scales, y, stream=None) -> None:
    """The same in 8 bits: q, scales of lora_rows_quantize, w_scales fp32 [experts][out / 128][blocks]."""
    try:
        (tokens, in_f), (ldq, q1) = q.shape, q.stride()
        (sr, sc), (lds, s1) = scales.shape, scales.stride()
        (yr, out_f), (ldy, y1) = y.shape, y.stride()
    except ValueError:
        (tokens, in_f), (ldq, q1), (sr, sc), (lds, s1), (yr, out_f), (ldy, y1) = _two(q, "q") + _two(scales, "scales") + _two(y, "y")
    n_experts, n_rows, blocks = starts.numel() - 1, tokens if order is None else tokens * picks, (in_f + 127) >> 7
    if q1 != 1 or q.dtype not in _E4M3 or not q.is_cuda:
        _usable("q", q, tokens, in_f, _E4M3)
    if sr < tokens or sc < blocks or s1 != 1 or scales.dtype not in _F32 or not scales.is_cuda:
        _usable("scales", scales, tokens, blocks, _F32)
    if yr < n_rows or y1 != 1 or y.dtype not in _BF16 or not y.is_cuda:
        _usable("y", y, n_rows, out_f, _BF16)
    if tokens == 1:
        ldq = blocks << 7
    if in_f & 127:
        _last_block(q, tokens, ldq, blocks << 7)
    if sr == 1:
        lds = sc
    if yr == 1:
        ldy = out_f
    if starts.dtype not in _INT32 or n_experts < 0 or not starts.is_contiguous() or not starts.is_cuda:
        _whole("starts", starts, 1, _INT32)
    if order is not None and (order.dtype not in _INT32 or order.numel() < n_rows or not order.is_contiguous() or not order.is_cuda):
        _whole("order", order, n_rows, _INT32)
    if w_packed.nbytes < n_experts * out_f * blocks << 7 or not w_packed.is_contiguous() or not w_packed.is_cuda:
        _packed(w_packed, n_experts * out_f * blocks << 7)
    if w_scales.dtype not in _F32 or w_scales.numel() < n_experts * (out_f >> 7) * blocks or not w_scales.is_contiguous() or not w_scales.is_cuda:
        _whole("w_scales", w_scales, n_experts * (out_f >> 7) * blocks, _F32)
    status = (_lib or lib()).lora_experts_linear_scaled(q.data_ptr(), ldq, scales.data_ptr(), lds, tokens, starts.data_ptr(),
                                                        None if order is None else order.data_ptr(), picks, n_rows, n_experts, in_f, w_packed.data_ptr(),
                                                        w_scales.data_ptr(), out_f, y.data_ptr(), ldy,
                                                        None if stream is None else _queue(stream))
    if status:
        _check(status)


def lora_experts_combine(y, place, weights, z, stream=None) -> None:
    """y: bf16 [rows][out]; place, weights: int32 and fp32 [tokens][picks]; z: bf16 [tokens][out]."""
    try:
        (yr, yc), (ldy, y1) = y.shape, y.stride()
        (zr, out_f), (ldz, z1) = z.shape, z.stride()
        tokens, picks = weights.shape
    except ValueError:
        (yr, yc), (ldy, y1), (zr, out_f), (ldz, z1), (tokens, picks), _ = _two(y, "y") + _two(z, "z") + _two(weights, "weights")
    n = tokens * picks
    if yc < out_f or y1 != 1 or y.dtype not in _BF16 or not y.is_cuda:
        _usable("y", y, 0, out_f, _BF16)
    if zr < tokens or z1 != 1 or z.dtype not in _BF16 or not z.is_cuda:
        _usable("z", z, tokens, out_f, _BF16)
    if yr == 1:
        ldy = out_f
    if zr == 1:
        ldz = out_f
    if place.dtype not in _INT32 or place.numel() < n or not place.is_contiguous() or not place.is_cuda:
        _whole("place", place, n, _INT32)
    if weights.dtype not in _F32 or weights.numel() < n or not weights.is_contiguous() or not weights.is_cuda:
        _whole("weights", weights, n, _F32)
    status = (_lib or lib()).lora_experts_combine(y.data_ptr(), ldy, yr, place.data_ptr(), weights.data_ptr(), tokens, picks, out_f,
                                                  z.data_ptr(), ldz, None if stream is None else _queue(stream))
    if status:
        _check(status)


# ---- between the projections: rotary positions, the paged cache, attention (include/lora_attention.h) ----------------------
# A call's tensors are all on one GPU, the current one: a launch goes there whatever the tensors' own device is.
ROTARY_SCALING = ("none", "linear", "wavelength", "dimension")  # LORA_ROTARY_*, in that order


class _RotaryArgs(ctypes.Structure):
    _fields_ = [("turns", ctypes.c_void_p), ("dims", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("magnitude", ctypes.c_float)]


class _CacheArgs(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scales", ctypes.c_void_p), ("v_scales", ctypes.c_void_p),
                ("pages", ctypes.c_int32), ("page_size", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("bits", ctypes.c_int32)]


def lora_rotary_turns(dims: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0, low: float = 1.0, high: float = 4.0,
                      length: float = 8192.0):
    """(uint64 [dims / 2], magnitude): the part of a turn, in units of 2^-64, that every pair makes in a position."""
    turns, magnitude = np.zeros(max(0, dims // 2), dtype=np.uint64), ctypes.c_float(1.0)
    if scaling not in ROTARY_SCALING:
        raise ValueError(f"scaling: {scaling!r} is none of {', '.join(ROTARY_SCALING)}")
    _check(lib().lora_rotary_turns(dims, base, ROTARY_SCALING.index(scaling), factor, low, high, length, turns.ctypes.data, ctypes.addressof(magnitude)))
    return turns, float(magnitude.value)


class Rotary:
    """lora_rotary_t: the frequencies on the GPU (int64, the bits of lora_rotary_turns), and how a head's elements pair up."""

    def __init__(self, dims: int, base: float = 10000.0, *, interleaved: bool = False, scaling: str = "none", factor: float = 1.0, low: float = 1.0,
                 high: float = 4.0, length: float = 8192.0, device="cuda"):
        import torch
        turns, magnitude = lora_rotary_turns(dims, base, scaling, factor, low, high, length)
        self.turns, self.dims, self.interleaved, self.magnitude = torch.from_numpy(turns.view(np.int64)).to(device), dims, interleaved, magnitude
        self.args = _RotaryArgs(self.turns.data_ptr(), dims, 1 if interleaved else 0, magnitude)
        self.address, self.device = ctypes.addressof(self.args), self.turns.get_device()


class Cache:
    """lora_cache_t over the caller's tensors: k, v [pages][kv_heads][page_size][head_dim], bf16, or 8-bit with fp32 scales [pages][kv_heads][page_size]."""

    def __init__(self, k, v, k_scales=None, v_scales=None):
        if not _BF16:
            _know_types()
        if k.dim() != 4 or k.shape != v.shape or k.dtype != v.dtype or not k.is_contiguous() or not v.is_contiguous():
            raise ValueError(f"k, v: {tuple(k.shape)} of {k.dtype} and {tuple(v.shape)} of {v.dtype} do not do: contiguous [pages][heads][slots][dim] alike are meant")
        if k.dtype not in _BF16 and k.dtype not in _E4M3:
            raise ValueError(f"k: {k.dtype} does not do: {_names(_BF16 | _E4M3)} is meant")
        bits = 16 if k.dtype in _BF16 else 8
        _on_gpu("k", k)
        self.k, self.v, self.k_scales, self.v_scales = k, v, k_scales, v_scales
        self.pages, self.kv_heads, self.page_size, self.head_dim = k.shape
        if (k_scales is None) != (bits == 16) or (v_scales is None) != (bits == 16):
            raise ValueError(f"k_scales, v_scales: a cache in {bits} bits has {'none' if bits == 16 else 'both'}")
        for name, t in (("v", v), ("k_scales", k_scales), ("v_scales", v_scales)):
            if t is None:
                continue
            if name != "v":
                if t.shape != k.shape[:3]:
                    raise ValueError(f"{name}: {tuple(t.shape)} does not do: {tuple(k.shape[:3])} is meant")
                _whole(name, t, 0, _F32)
            if t.get_device() != k.get_device():
                raise ValueError(f"{name}: on another device than k")
        self.args = _CacheArgs(k.data_ptr(), v.data_ptr(), *(None if t is None else t.data_ptr() for t in (k_scales, v_scales)),
                               *(int(n) for n in (self.pages, self.page_size, self.kv_heads, self.head_dim)), bits)
        self.address, self.device = ctypes.addressof(self.args), k.get_device()


_current_device = None


def _here(device: int, stream) -> None:
    """Refuses tensors of another GPU than the one that the launch goes to."""
    global _current_device
    if _current_device is None:
        import torch
        _current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)  # (the latter asks first whether torch is at work there)
    if device < 0:
        raise ValueError("a tensor on the CPU does not do: ones on the GPU are meant")
    at = _current_device()
    if device != at or getattr(stream, "device_index", at) != at:
        raise ValueError(f"tensors on device {device}, stream {stream}: the current device is {at}")


def _heads(name: str, t, device: int) -> None:
    """Refuses a tensor that is not bf16 [tokens][heads][dim] on that device, a head's elements side by side."""
    if not _BF16:
        _know_types()
    if t.dtype not in _BF16:
        raise ValueError(f"{name}: {t.dtype} does not do: {_names(_BF16)} is meant")
    if t.dim() != 3 or t.get_device() != device:
        raise ValueError(f"{name}: {tuple(t.shape)} on {t.device} does not do: [tokens][heads][dim] on the other tensors' GPU is meant")
    if t.stride(2) != 1 and t.shape[2] > 1:
        raise ValueError(f"{name}: strides {t.stride()} do not do: a head's elements lie side by side")


def _three(t, name: str):
    """Shape and strides of a tensor of heads."""
    if t.dim() != 3:
        raise ValueError(f"{name}: {tuple(t.shape)} does not do: [tokens][heads][dim] is meant")
    return t.shape, t.stride()


def _ints(name: str, t, n: int, device: int) -> None:
    _whole(name, t, n, _INT32)
    if t.get_device() != device:
        raise ValueError(f"{name}: on another device than the other tensors")


# (these calls too ask their tensors in line, and look closer where anything is unusual; of a dimension of one torch states any stride)
def lora_rotary(x, positions, rotary: Rotary, y=None, inverse: bool = False, stream=None) -> None:
    """x, y: bf16 [tokens][heads][dim] (y None: x, in place); positions: int32 [tokens]; inverse: the gradient's way."""
    if y is None:
        y = x
    try:
        (n, heads, dim), (xt, xh, x1) = x.shape, x.stride()
        (yn, yheads, ydim), (yt, yh, y1) = y.shape, y.stride()
    except ValueError:
        (n, heads, dim), (xt, xh, x1), (yn, yheads, ydim), (yt, yh, y1) = _three(x, "x") + _three(y, "y")
    device = x.get_device()
    if x1 != 1 or x.dtype not in _BF16:
        _heads("x", x, device)
    if y1 != 1 or y.dtype not in _BF16 or y.get_device() != device:
        _heads("y", y, device)
    if yn != n or yheads != heads or ydim != dim:
        raise ValueError(f"y: {tuple(y.shape)} does not do: {tuple(x.shape)} is meant")
    if positions.dtype not in _INT32 or positions.numel() < n or not positions.is_contiguous() or positions.get_device() != device:
        _ints("positions", positions, n, device)
    _here(device, stream)
    if rotary.device != device:
        raise ValueError("rotary: on another device than x")
    if heads == 1:
        xh = yh = dim
    if n == 1:
        xt, yt = heads * xh, heads * yh
    status = (_lib or lib()).lora_rotary(x.data_ptr(), xt, xh, n, heads, dim, positions.data_ptr(), rotary.address, 1 if inverse else 0, y.data_ptr(), yt, yh,
                                         None if stream is None else _queue(stream))
    if status:
        _check(status)


def lora_cache_append(k, v, slots, cache: Cache, rotary: Optional[Rotary] = None, positions=None, q=None, y=None, stream=None) -> None:
    """k, v: bf16 [tokens][kv_heads][dim]; slots, positions: int32 [tokens]; q: bf16 [tokens][q_heads][dim], turned into y (None: q, in place)."""
    try:
        (n, heads, dim), (kt, kh, k1) = k.shape, k.stride()
        (vn, vheads, vdim), (vt, vh, v1) = v.shape, v.stride()
    except ValueError:
        (n, heads, dim), (kt, kh, k1), (vn, vheads, vdim), (vt, vh, v1) = _three(k, "k") + _three(v, "v")
    device = k.get_device()
    if k1 != 1 or k.dtype not in _BF16:
        _heads("k", k, device)
    if v1 != 1 or v.dtype not in _BF16 or v.get_device() != device:
        _heads("v", v, device)
    if heads != cache.kv_heads or dim != cache.head_dim or vn != n or vheads != heads or vdim != dim:
        raise ValueError(f"k, v: {tuple(k.shape)} and {tuple(v.shape)} do not do: tokens x {cache.kv_heads} x {cache.head_dim} is meant")
    if heads == 1:
        kh = vh = dim
    if n == 1:
        kt, vt = heads * kh, heads * vh
    pq = py = pp = pr = None
    qt = qh = q_heads = yt = yh = 0
    if q is not None:
        if y is None:
            y = q
        try:
            (qn, q_heads, qdim), (qt, qh, q1) = q.shape, q.stride()
            (yn, yheads, ydim), (yt, yh, y1) = y.shape, y.stride()
        except ValueError:
            (qn, q_heads, qdim), (qt, qh, q1), (yn, yheads, ydim), (yt, yh, y1) = _three(q, "q") + _three(y, "y")
        if q1 != 1 or q.dtype not in _BF16 or q.get_device() != device:
            _heads("q", q, device)
        if y1 != 1 or y.dtype not in _BF16 or y.get_device() != device:
            _heads("y", y, device)
        if qn != n or qdim != dim or yn != n or yheads != q_heads or ydim != dim:
            raise ValueError(f"q, y: {tuple(q.shape)} and {tuple(y.shape)} do not do: {n} tokens of heads of {dim}, alike, are meant")
        if q_heads == 1:
            qh = yh = dim
        if n == 1:
            qt, yt = q_heads * qh, q_heads * yh
        pq, py = q.data_ptr(), y.data_ptr()
    elif y is not None:
        raise ValueError("y: without q there is nothing for it")
    if slots.dtype not in _INT32 or slots.numel() < n or not slots.is_contiguous() or slots.get_device() != device:
        _ints("slots", slots, n, device)
    if positions is not None:
        if positions.dtype not in _INT32 or positions.numel() < n or not positions.is_contiguous() or positions.get_device() != device:
            _ints("positions", positions, n, device)
        pp = positions.data_ptr()
    if rotary is not None:
        if rotary.device != device:
            raise ValueError("rotary: on another device than k")
        pr = rotary.address
    _here(device, stream)
    if cache.device != device:
        raise ValueError("cache: on another device than k")
    status = (_lib or lib()).lora_cache_append(k.data_ptr(), kt, kh, v.data_ptr(), vt, vh, n, slots.data_ptr(), pp, pr, cache.address, pq, qt, qh, q_heads, py, yt,
                                               yh, None if stream is None else _queue(stream))
    if status:
        _check(status)


def lora_attention_workspace_bytes(tokens: int, q_heads: int, requests: int, width: int, cache: Cache) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().lora_attention_workspace_bytes(tokens, q_heads, requests, width, cache.address, ctypes.addressof(n)))
    return int(n.value)


def lora_attention(q, starts, lengths, page_table, cache: Cache, y, workspace=None, scale: Optional[float] = None, tree=None, most: int = 0,
                   stream=None) -> None:
    """q, y: bf16 [tokens][q_heads][dim]; starts [requests + 1], lengths [requests], page_table [requests][width]: int32; tree: int64 [tokens], one
    word of 64 bits a row (None: rows see their request's own keys up to themselves); scale None: 1 / sqrt(dim); most: the most rows of a request, 0 if unknown.
    page_table's width stands for the longest request's keys: a view of the columns that the batch needs (page_table[:, :n]) takes short ones faster.
    starts must not descend: where they do (nothing says so, they are on the GPU), any row of y may stay as it was."""
    try:
        (n, heads, dim), (qt, qh, q1) = q.shape, q.stride()
        (yn, yheads, ydim), (yt, yh, y1) = y.shape, y.stride()
        (rows, width), (ld, t1) = page_table.shape, page_table.stride()
    except ValueError:
        (n, heads, dim), (qt, qh, q1), (yn, yheads, ydim), (yt, yh, y1), (rows, width), (ld, t1) = _three(q, "q") + _three(y, "y") + _two(page_table, "page_table")
    device = q.get_device()
    if q1 != 1 or q.dtype not in _BF16:
        _heads("q", q, device)
    if y1 != 1 or y.dtype not in _BF16 or y.get_device() != device:
        _heads("y", y, device)
    if dim != cache.head_dim or yn != n or yheads != heads or ydim != dim:
        raise ValueError(f"q, y: {tuple(q.shape)} and {tuple(y.shape)} do not do: alike, of heads of {cache.head_dim}, is meant")
    if heads == 1:
        qh = yh = dim
    if n == 1:
        qt, yt = heads * qh, heads * yh
    requests = lengths.numel()
    if page_table.dtype not in _INT32 or rows < requests or page_table.get_device() != device or (t1 != 1 and width > 1):
        _usable("page_table", page_table, requests, width, _INT32)
        raise ValueError("page_table: on another device than q")
    if requests <= 1 or width == 0:
        ld = width
    elif ld < width:
        raise ValueError(f"page_table: strides {page_table.stride()} do not do: rows overlap")
    if starts.dtype not in _INT32 or starts.numel() <= requests or not starts.is_contiguous() or starts.get_device() != device:
        _ints("starts", starts, requests + 1, device)
    if lengths.dtype not in _INT32 or not lengths.is_contiguous() or lengths.get_device() != device:
        _ints("lengths", lengths, requests, device)
    pt = None
    if tree is not None:
        if tree.element_size() != 8 or tree.is_floating_point() or tree.is_complex() or tree.numel() < n or not tree.is_contiguous() or tree.get_device() != device:
            raise ValueError(f"tree: {tuple(tree.shape)} of {tree.dtype} on {tree.device} does not do: {n} contiguous words of 64 bits are meant")
        pt = tree.data_ptr()
    if workspace is None:
        pw, nw = None, 0
    else:
        if workspace.get_device() != device or not workspace.is_contiguous():
            raise ValueError("workspace: contiguous bytes on the other tensors' GPU are meant")
        pw, nw = workspace.data_ptr(), workspace.nbytes
    _here(device, stream)
    if cache.device != device:
        raise ValueError("cache: on another device than q")
    status = (_lib or lib()).lora_attention(q.data_ptr(), qt, qh, n, heads, starts.data_ptr(), lengths.data_ptr(), requests, page_table.data_ptr(), ld, width, pt,
                                            most, cache.address, dim ** -0.5 if scale is None else scale, y.data_ptr(), yt, yh, pw, nw,
                                            None if stream is None else _queue(stream))
    if status:
        _check(status)
