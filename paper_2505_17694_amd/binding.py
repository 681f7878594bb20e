"""ctypes binding of libcodec.so: the C ABI of include/codec.h under the same names.

Argument marshalling only.  Every step of the decode path runs inside the
library; PyTorch is used by callers for device memory and streams.  If the
library has not been built, importing this module raises.
"""
from __future__ import annotations

import ctypes
import os
import struct
from ctypes import (POINTER, Structure, c_char_p, c_double, c_float, c_int, c_int32, c_int64, c_size_t,
                    c_void_p, byref)

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libcodec.so")

CODEC_OK = 0
CODEC_ERR_INVALID_ARGUMENT = -1
CODEC_ERR_INVALID_TREE = -2
CODEC_ERR_UNSUPPORTED = -3
CODEC_ERR_WORKSPACE_TOO_SMALL = -4
CODEC_ERR_HIP = -5
CODEC_ERR_NOT_UPLOADED = -6
CODEC_ERR_OUT_OF_MEMORY = -7
CODEC_ERR_NO_PAGES = -8
CODEC_DTYPE_FP16 = 0
CODEC_DTYPE_BF16 = 1
CODEC_DTYPE_FP32 = 2
CODEC_ROTARY_HALF = 0
CODEC_ROTARY_INTERLEAVED = 1
CODEC_ROTARY_UNSCALED = 0
CODEC_ROTARY_LINEAR = 1
CODEC_ROTARY_NTK = 2
CODEC_ROTARY_WAVELENGTH = 3
CODEC_ROTARY_YARN = 4
CODEC_PLAN_EXT_SLACK = 1
CODEC_PLAN_EXT_DIAGONAL = 2

# every symbol include/codec.h declares
EXPORTED_SYMBOLS = [
    "codec_plan_create", "codec_plan_destroy", "codec_plan_export", "codec_cost_estimate",
    "codec_default_cost_table", "codec_plan_device_bytes", "codec_plan_upload",
    "codec_plan_workspace_bytes", "codec_decode_attention", "codec_partial_attention",
    "codec_partial_reduction", "codec_status_string", "codec_last_error_message",
    "codec_plan_refresh_lengths", "codec_decode_attention_static", "codec_static_scratch_bytes",
    "codec_stream_read_probe", "codec_rotary_turns", "codec_rotary", "codec_append",
    "codec_pages_create", "codec_pages_destroy", "codec_pages_free", "codec_pages_take", "codec_pages_hold",
    "codec_pages_release", "codec_pages_fork", "codec_pages_compact", "codec_cache_copy",
    "codec_beam_workspace_bytes", "codec_beam_select", "codec_beam_reorder",
    "codec_rotary_by_axes", "codec_append_by_axes",
    "codec_block_table", "codec_slot_workspace_bytes", "codec_slot_map",
    "codec_differential_attention",
]

_i32p = POINTER(c_int32)
_i64p = POINTER(c_int64)


class codec_head_config(Structure):
    _fields_ = [("num_q_heads", c_int32), ("num_kv_heads", c_int32), ("head_dim", c_int32),
                ("dtype", c_int32), ("page_size", c_int32), ("scale", c_float)]


class codec_tree(Structure):
    _fields_ = [("num_nodes", c_int32), ("parent", _i32p), ("node_len", _i32p),
                ("num_requests", c_int32), ("req_node", _i32p),
                ("node_page_off", _i32p), ("page_ids", _i32p),
                ("req_mask_off", _i32p), ("req_mask", POINTER(ctypes.c_uint32))]


class codec_cost_table(Structure):
    _fields_ = [("num_row_points", c_int32), ("num_len_points", c_int32),
                ("row_grid", _i32p), ("len_grid", _i32p), ("cost", _i64p)]


class codec_plan_options(Structure):
    _fields_ = [("num_slots", c_int32), ("split_align", c_int32), ("max_rows", c_int32),
                ("share", c_int32), ("cost", POINTER(codec_cost_table)), ("fixed_slices", c_int32),
                ("schedule", c_int32), ("fused", c_int32), ("extensions", c_int32)]


class codec_item(Structure):
    _fields_ = [("node", c_int32), ("q_off", c_int32), ("n_req", c_int32), ("rows", c_int32),
                ("len", c_int32), ("ub", c_int32), ("b", c_int32), ("reserved", c_int32),
                ("cost", c_int64)]


class codec_task(Structure):
    _fields_ = [("item", c_int32), ("node", c_int32), ("kv_begin", c_int32), ("kv_len", c_int32),
                ("q_off", c_int32), ("n_req", c_int32), ("part_row_base", c_int32),
                ("slot", c_int32), ("cost", c_int64)]


class codec_plan_view(Structure):
    _fields_ = [("num_items", c_int32), ("items", POINTER(codec_item)),
                ("num_tasks", c_int32), ("tasks", POINTER(codec_task)),
                ("num_slots", c_int32), ("slot_off", _i32p), ("slot_tasks", _i32p),
                ("num_nodes", c_int32), ("node_q_off", _i32p), ("node_q", _i32p),
                ("num_requests", c_int32), ("req_part_off", _i32p), ("req_part", _i32p),
                ("cost_l", c_int64), ("makespan", c_int64), ("part_rows", c_int32),
                ("split_align", c_int32), ("max_rows", c_int32), ("share", c_int32),
                ("schedule", c_int32), ("fused", c_int32), ("num_entries", c_int32), ("queue_off", _i32p), ("queue_tasks", _i32p)]


class codec_kv_layout(Structure):
    _fields_ = [("num_pages", c_int64), ("page_stride", c_int64), ("token_stride", c_int64),
                ("head_stride", c_int64)]


class codec_differential(Structure):
    _fields_ = [("lambda_", c_void_p), ("lambda_request_stride", c_int64), ("lambda_head_stride", c_int64), ("norm", c_int32),
                ("weight_dtype", c_int32), ("weight", c_void_p), ("eps", c_float), ("gain", c_float)]


class codec_rotary_scaling(Structure):
    _fields_ = [("kind", c_int32), ("original_length", c_int32), ("factor", c_double),
                ("low", c_double), ("high", c_double), ("fast", c_double), ("slow", c_double)]


class codec_rotary_config(Structure):
    _fields_ = [("rotary_dim", c_int32), ("layout", c_int32), ("inverse", c_int32), ("magnitude", c_float),
                ("turns", c_void_p)]


class codec_rotary_axes(Structure):
    _fields_ = [("rotary", codec_rotary_config), ("block_dim", c_int32), ("num_axes", c_int32), ("axes", c_void_p),
                ("axis_stride", c_int64)]


class codec_rows(Structure):
    _fields_ = [("data", c_void_p), ("token_stride", c_int64), ("head_stride", c_int64)]


class codec_run(Structure):
    _fields_ = [("src_page", c_int32), ("src_token", c_int32), ("dst_page", c_int32), ("dst_token", c_int32),
                ("tokens", c_int32)]


class codec_slot_config(Structure):
    _fields_ = [("num_seq", c_int32), ("page_size", c_int32), ("width", c_int32), ("num_tokens", c_int32), ("num_spare", c_int32),
                ("num_pages", c_int64), ("table_stride", c_int64)]


class codec_beam_config(Structure):
    _fields_ = [("batch", c_int32), ("beams", c_int32), ("vocab", c_int32), ("k", c_int32), ("dtype", c_int32),
                ("eos", c_int32)]


class codec_state(Structure):
    _fields_ = [("src", c_void_p), ("dst", c_void_p), ("row_bytes", c_int64),
                ("src_batch_stride", c_int64), ("src_beam_stride", c_int64),
                ("dst_batch_stride", c_int64), ("dst_beam_stride", c_int64)]


# PyTorch wheels carry their own copy of the HIP runtime.  Device pointers and streams handed to the
# library come from PyTorch, so both must use the same runtime instance: load PyTorch's first, and
# libcodec.so's dependency on libamdhip64 then resolves to the copy already in the process.
try:
    import torch  # noqa: F401
except ImportError:
    pass

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2505_17694_amd.build` "
                      "(there is no CPU fallback)")
_lib = ctypes.CDLL(LIB_PATH)

_lib.codec_plan_create.restype = c_int
_lib.codec_plan_create.argtypes = [POINTER(codec_tree), POINTER(codec_head_config),
                                   POINTER(codec_plan_options), POINTER(c_void_p)]
_lib.codec_plan_destroy.restype = c_int
_lib.codec_plan_destroy.argtypes = [c_void_p]
_lib.codec_plan_export.restype = c_int
_lib.codec_plan_export.argtypes = [c_void_p, POINTER(codec_plan_view)]
_lib.codec_plan_refresh_lengths.restype = c_int
_lib.codec_plan_refresh_lengths.argtypes = [c_void_p, _i32p, _i32p, _i32p]
_lib.codec_cost_estimate.restype = c_int64
_lib.codec_cost_estimate.argtypes = [POINTER(codec_cost_table), c_int32, c_int32]
_lib.codec_default_cost_table.restype = POINTER(codec_cost_table)
_lib.codec_default_cost_table.argtypes = [c_int32]
_lib.codec_plan_device_bytes.restype = c_size_t
_lib.codec_plan_device_bytes.argtypes = [c_void_p]
_lib.codec_plan_upload.restype = c_int
_lib.codec_plan_upload.argtypes = [c_void_p, c_void_p, c_size_t, c_void_p]
_lib.codec_plan_workspace_bytes.restype = c_size_t
_lib.codec_plan_workspace_bytes.argtypes = [c_void_p]
_lib.codec_decode_attention.restype = c_int
_lib.codec_decode_attention.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p,
                                        POINTER(codec_kv_layout), c_void_p, c_void_p, c_size_t,
                                        c_void_p]
_lib.codec_partial_attention.restype = c_int
_lib.codec_partial_attention.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p,
                                         POINTER(codec_kv_layout), c_void_p, c_size_t, c_void_p]
_lib.codec_partial_reduction.restype = c_int
_lib.codec_partial_reduction.argtypes = [c_void_p, c_void_p, c_size_t, c_void_p, c_void_p]
_lib.codec_decode_attention_static.restype = c_int
_lib.codec_decode_attention_static.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p,
                                               POINTER(codec_kv_layout), c_void_p, c_void_p]
_lib.codec_static_scratch_bytes.restype = c_size_t
_lib.codec_static_scratch_bytes.argtypes = []
_lib.codec_differential_attention.restype = c_int
_lib.codec_differential_attention.argtypes = [c_void_p] * 8 + [c_size_t, c_void_p]
_lib.codec_stream_read_probe.restype = c_int
_lib.codec_stream_read_probe.argtypes = [c_void_p, c_size_t, c_int32, c_int32, c_int32, c_void_p, c_void_p]
_lib.codec_rotary_turns.restype = c_int
_lib.codec_rotary_turns.argtypes = [c_int32, c_double, POINTER(codec_rotary_scaling), POINTER(c_double), POINTER(c_float)]
_lib.codec_rotary.restype = c_int
_lib.codec_rotary.argtypes = [POINTER(codec_rotary_config), c_int32, c_int32, c_int32, POINTER(codec_rows), POINTER(codec_rows),
                              c_void_p, c_int32, c_void_p]
_lib.codec_append.restype = c_int
_lib.codec_append.argtypes = [POINTER(codec_head_config), POINTER(codec_rotary_config)] + [POINTER(codec_rows)] * 4 + [
    c_void_p, c_void_p, c_int32, c_void_p, c_void_p, POINTER(codec_kv_layout), c_void_p]
_lib.codec_rotary_by_axes.restype = c_int
_lib.codec_rotary_by_axes.argtypes = [c_void_p] + _lib.codec_rotary.argtypes[1:]
_lib.codec_append_by_axes.restype = c_int
_lib.codec_append_by_axes.argtypes = [POINTER(codec_head_config), c_void_p] + _lib.codec_append.argtypes[2:]
_lib.codec_pages_create.restype = c_int
_lib.codec_pages_create.argtypes = [c_int32, POINTER(c_void_p)]
_lib.codec_pages_destroy.restype = c_int
_lib.codec_pages_destroy.argtypes = [c_void_p]
_lib.codec_pages_free.restype = c_int32
_lib.codec_pages_free.argtypes = [c_void_p]
_lib.codec_pages_take.restype = c_int
_lib.codec_pages_take.argtypes = [c_void_p, c_int32, c_void_p]
_lib.codec_pages_hold.restype = c_int
_lib.codec_pages_hold.argtypes = [c_void_p, c_void_p, c_int32]
_lib.codec_pages_release.restype = c_int
_lib.codec_pages_release.argtypes = [c_void_p, c_void_p, c_int32]
_lib.codec_pages_fork.restype = c_int
_lib.codec_pages_fork.argtypes = [c_void_p, c_int32, c_int32, c_void_p, c_void_p, c_void_p, c_int32, c_void_p, c_void_p, c_void_p,
                                  c_int32, c_void_p, _i32p]
_lib.codec_pages_compact.restype = c_int
_lib.codec_pages_compact.argtypes = [c_void_p, c_int32, c_void_p, c_int32, _i32p]
_lib.codec_cache_copy.restype = c_int
_lib.codec_cache_copy.argtypes = [POINTER(codec_head_config), POINTER(codec_kv_layout), c_int32, c_void_p, c_void_p, c_void_p, c_int32,
                                  c_void_p]
_lib.codec_block_table.restype = c_int
_lib.codec_block_table.argtypes = [c_int32, c_int32, c_void_p, c_void_p, c_int32, c_void_p, c_void_p, c_int64, c_int32, c_void_p]
_lib.codec_slot_workspace_bytes.restype = c_size_t
_lib.codec_slot_workspace_bytes.argtypes = [c_void_p]
_lib.codec_slot_map.restype = c_int
_lib.codec_slot_map.argtypes = [c_void_p] * 13 + [c_size_t, c_void_p]
_lib.codec_beam_workspace_bytes.restype = c_size_t
_lib.codec_beam_workspace_bytes.argtypes = [POINTER(codec_beam_config)]
_lib.codec_beam_select.restype = c_int
_lib.codec_beam_select.argtypes = [POINTER(codec_beam_config), c_void_p, c_int64, c_int64, c_void_p, c_void_p, c_void_p, c_void_p,
                                   c_void_p, c_void_p, c_size_t, c_void_p]
_lib.codec_beam_reorder.restype = c_int
_lib.codec_beam_reorder.argtypes = [c_void_p, c_int32, c_void_p, c_int32, c_int32, c_int32, c_void_p]
_lib.codec_status_string.restype = c_char_p
_lib.codec_status_string.argtypes = [c_int]
_lib.codec_last_error_message.restype = c_char_p
_lib.codec_last_error_message.argtypes = []


class CodecError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        detail = codec_last_error_message() if status == CODEC_ERR_HIP else ""
        super().__init__(f"{where}: {codec_status_string(status)} ({status})" + (f": {detail}" if detail else ""))


def _is_int32(n) -> bool:
    """Whether n passes as an int32: ctypes would take its low bits."""
    return -0x80000000 <= n <= 0x7fffffff


def _i32(a):
    return np.ascontiguousarray(a, dtype=np.int32)


def _ids(a):
    """A list of pages, tokens or sequences as int32; None if one of them is no whole number of 32 bits (a cast would take
    its low bits, or another page)."""
    a = np.asarray(a)
    if a.dtype.kind not in "iu" and a.size:
        return None
    ids = _i32(a)
    return None if a.dtype.char != "i" and np.count_nonzero(ids != a) else ids


def _in(a):
    """Read-only argument of a short call: the array's bytes (a fifth of the time its pointer takes to get), if they are few."""
    return a.tobytes() if a.nbytes <= 1 << 16 else a.ctypes.data


# Structures of short calls as bytes, in a third of the time that their classes take.
pack_slot_config = struct.Struct("5i4x2q").pack             # fields of codec_slot_config
pack_differential = struct.Struct("P2q2iP2f").pack          # codec_differential
pack_kv_layout = struct.Struct("4q").pack                   # codec_kv_layout
pack_rotary_axes = struct.Struct("3ifP2iPq").pack           # codec_rotary_axes
assert [len(p(*[0] * n)) for p, n in ((pack_slot_config, 7), (pack_differential, 8), (pack_kv_layout, 4), (pack_rotary_axes, 9))] == [
    ctypes.sizeof(c) for c in (codec_slot_config, codec_differential, codec_kv_layout, codec_rotary_axes)]


def _struct(s):
    """Argument of a structure: as it is where it came as bytes (or None)."""
    return byref(s) if isinstance(s, Structure) else s


def _ptr(a, ct=c_int32):
    return a.ctypes.data_as(POINTER(ct)) if a is not None and a.size else None


def make_cost_table(row_grid, len_grid, cost):
    """Marshal a cost table; returns (struct, keepalive) - keep both alive while the struct is used."""
    rg, lg = _i32(row_grid), _i32(len_grid)
    c = np.ascontiguousarray(cost, dtype=np.int64).reshape(-1)
    t = codec_cost_table(len(rg), len(lg), _ptr(rg), _ptr(lg), _ptr(c, c_int64))
    return t, (rg, lg, c)


def codec_status_string(status: int) -> str:
    return _lib.codec_status_string(int(status)).decode()


def codec_last_error_message() -> str:
    return _lib.codec_last_error_message().decode()


def codec_plan_create(parent, node_len, req_node, node_page_off, page_ids,
                      num_q_heads, num_kv_heads, head_dim, dtype, page_size, scale,
                      num_slots=0, split_align=0, max_rows=0, share=1, cost_table=None, fixed_slices=0,
                      schedule=0, extensions=0, fused=0, req_mask_off=None, req_mask=None):
    """Returns (status, plan handle or None).  ``cost_table``: (row_grid, len_grid, cost) or None;
    ``req_mask_off`` / ``req_mask``: per-request visibility masks (see codec_tree) or None."""
    parent, node_len, req_node = _i32(parent), _i32(node_len), _i32(req_node)
    node_page_off, page_ids = _i32(node_page_off), _i32(page_ids)
    mask_off = mask_words = None
    if req_mask_off is not None:
        mask_off = _i32(req_mask_off)
        mask_words = np.ascontiguousarray(req_mask if req_mask is not None else [], dtype=np.uint32)
    tree = codec_tree(len(parent), _ptr(parent), _ptr(node_len), len(req_node), _ptr(req_node),
                      _ptr(node_page_off), _ptr(page_ids),
                      _ptr(mask_off) if mask_off is not None else None,
                      _ptr(mask_words, ctypes.c_uint32) if mask_words is not None else None)
    head = codec_head_config(num_q_heads, num_kv_heads, head_dim, dtype, page_size, scale)
    keep = None
    ct_ptr = None
    if cost_table is not None:
        ct, keep = make_cost_table(*cost_table)
        ct_ptr = ctypes.pointer(ct)
    opt = codec_plan_options(num_slots, split_align, max_rows, share, ct_ptr, fixed_slices, schedule,
                             fused, extensions)
    handle = c_void_p()
    st = _lib.codec_plan_create(byref(tree), byref(head), byref(opt), byref(handle))
    del keep
    return st, (handle if st == CODEC_OK else None)


def codec_plan_destroy(plan) -> int:
    return _lib.codec_plan_destroy(plan)


def _arr(ptr, n, dtype=np.int32):
    if n == 0:
        return np.zeros(0, dtype=dtype)
    return np.ctypeslib.as_array(ptr, shape=(n,)).copy()


def codec_plan_export(plan):
    """Returns (status, dict of numpy copies of the plan view)."""
    v = codec_plan_view()
    st = _lib.codec_plan_export(plan, byref(v))
    if st != CODEC_OK:
        return st, None
    items = [{f: getattr(v.items[i], f) for f, _ in codec_item._fields_ if f != "reserved"}
             for i in range(v.num_items)]
    tasks = [{f: getattr(v.tasks[i], f) for f, _ in codec_task._fields_} for i in range(v.num_tasks)]
    out = {
        "items": items, "tasks": tasks, "num_slots": v.num_slots,
        "slot_off": _arr(v.slot_off, v.num_slots + 1), "slot_tasks": _arr(v.slot_tasks, v.num_tasks),
        "node_q_off": _arr(v.node_q_off, v.num_nodes + 1),
        "req_part_off": _arr(v.req_part_off, v.num_requests + 1),
        "cost_l": v.cost_l, "makespan": v.makespan, "part_rows": v.part_rows,
        "split_align": v.split_align, "max_rows": v.max_rows, "share": v.share,
        "schedule": v.schedule, "fused": v.fused, "queue_off": _arr(v.queue_off, v.num_entries + 1),
        "queue_tasks": _arr(v.queue_tasks, v.num_tasks),
    }
    out["node_q"] = _arr(v.node_q, int(out["node_q_off"][-1]) if v.num_nodes else 0)
    out["req_part"] = _arr(v.req_part, int(out["req_part_off"][-1]))
    return st, out


def codec_plan_refresh_lengths(plan, node_len, node_page_off, page_ids) -> int:
    node_len, node_page_off, page_ids = _i32(node_len), _i32(node_page_off), _i32(page_ids)
    return _lib.codec_plan_refresh_lengths(plan, _ptr(node_len), _ptr(node_page_off), _ptr(page_ids))


def codec_cost_estimate(cost_table, rows: int, length: int) -> int:
    if cost_table is None:
        return int(_lib.codec_cost_estimate(None, rows, length))
    ct, keep = make_cost_table(*cost_table)
    r = int(_lib.codec_cost_estimate(byref(ct), rows, length))
    del keep
    return r


def codec_default_cost_table(wide: int):
    """Returns (row_grid, len_grid, cost[rows][lens]) of a built-in table as Python lists."""
    t = _lib.codec_default_cost_table(int(wide)).contents
    rg = [t.row_grid[i] for i in range(t.num_row_points)]
    lg = [t.len_grid[i] for i in range(t.num_len_points)]
    cost = [[t.cost[i * t.num_len_points + j] for j in range(t.num_len_points)]
            for i in range(t.num_row_points)]
    return rg, lg, cost


def codec_plan_device_bytes(plan) -> int:
    return int(_lib.codec_plan_device_bytes(plan))


def codec_plan_upload(plan, device_meta_ptr: int, device_meta_bytes: int, stream: int = 0) -> int:
    return _lib.codec_plan_upload(plan, c_void_p(device_meta_ptr), device_meta_bytes, c_void_p(stream))


def codec_plan_workspace_bytes(plan) -> int:
    return int(_lib.codec_plan_workspace_bytes(plan))


def codec_decode_attention(plan, q_ptr: int, k_ptr: int, v_ptr: int, num_pages: int,
                           page_stride: int, token_stride: int, head_stride: int, out_ptr: int,
                           workspace_ptr: int, workspace_bytes: int, stream: int = 0) -> int:
    lay = codec_kv_layout(num_pages, page_stride, token_stride, head_stride)
    # integers as they are: the declared argument types convert them
    return _lib.codec_decode_attention(plan, q_ptr, k_ptr, v_ptr, lay, out_ptr, workspace_ptr, workspace_bytes, stream)


def codec_partial_attention(plan, q_ptr: int, k_ptr: int, v_ptr: int, num_pages: int,
                            page_stride: int, token_stride: int, head_stride: int,
                            workspace_ptr: int, workspace_bytes: int, stream: int = 0) -> int:
    lay = codec_kv_layout(num_pages, page_stride, token_stride, head_stride)
    return _lib.codec_partial_attention(plan, c_void_p(q_ptr), c_void_p(k_ptr), c_void_p(v_ptr),
                                        byref(lay), c_void_p(workspace_ptr), workspace_bytes,
                                        c_void_p(stream))


def codec_partial_reduction(plan, workspace_ptr: int, workspace_bytes: int, out_ptr: int,
                            stream: int = 0) -> int:
    return _lib.codec_partial_reduction(plan, c_void_p(workspace_ptr), workspace_bytes,
                                        c_void_p(out_ptr), c_void_p(stream))


def codec_decode_attention_static(plan, q_ptr: int, k_ptr: int, v_ptr: int, num_pages: int,
                                  page_stride: int, token_stride: int, head_stride: int, out_ptr: int,
                                  stream: int = 0) -> int:
    lay = codec_kv_layout(num_pages, page_stride, token_stride, head_stride)
    return _lib.codec_decode_attention_static(plan, c_void_p(q_ptr), c_void_p(k_ptr), c_void_p(v_ptr),
                                              byref(lay), c_void_p(out_ptr), c_void_p(stream))


def codec_differential_attention(plan, differential, q_ptr: int, k_ptr: int, v_ptr: int, layout, out_ptr: int, workspace_ptr: int,
                                 workspace_bytes: int, stream: int = 0) -> int:
    """``differential``: codec_differential; ``layout``: codec_kv_layout; or their bytes."""
    return _lib.codec_differential_attention(plan, _struct(differential), q_ptr, k_ptr, v_ptr, _struct(layout), out_ptr, workspace_ptr, workspace_bytes, stream)


def codec_static_scratch_bytes() -> int:
    return int(_lib.codec_static_scratch_bytes())


def codec_stream_read_probe(buffer_ptr: int, nbytes: int, pattern: int, nontemporal: int, workgroups: int,
                            sink_ptr: int, stream: int = 0) -> int:
    return _lib.codec_stream_read_probe(c_void_p(buffer_ptr), nbytes, pattern, nontemporal, workgroups,
                                        c_void_p(sink_ptr), c_void_p(stream))


def codec_rotary_turns(rotary_dim: int, theta: float, scaling=None):
    """Returns (status, turns of the pairs as float64 array or None, magnitude).  ``scaling``: codec_rotary_scaling or None."""
    if not _is_int32(rotary_dim):
        return CODEC_ERR_INVALID_ARGUMENT, None, 0.0
    turns = np.zeros(max(1, rotary_dim // 2), np.float64)
    magnitude = c_float(0.0)
    st = _lib.codec_rotary_turns(rotary_dim, theta, byref(scaling) if scaling is not None else None, _ptr(turns, c_double),
                                 byref(magnitude))
    return st, (turns if st == CODEC_OK else None), magnitude.value


def codec_rotary(rotary, num_heads: int, head_dim: int, dtype: int, x, out, positions_ptr: int, num_tokens: int,
                 stream: int = 0) -> int:
    """``rotary``: codec_rotary_config; ``x`` and ``out``: codec_rows."""
    return _lib.codec_rotary(rotary, num_heads, head_dim, dtype, x, out, positions_ptr, num_tokens, stream)


def codec_append(head, rotary, q, q_out, k, v, positions_ptr: int, slots_ptr: int, num_tokens: int, k_ptr: int, v_ptr: int,
                 layout, stream: int = 0) -> int:
    """``head``: codec_head_config; ``rotary``: codec_rotary_config or None; ``q``, ``q_out``: codec_rows or None; ``k``,
    ``v``: codec_rows; ``layout``: codec_kv_layout."""
    return _lib.codec_append(head, rotary, q, q_out, k, v, positions_ptr, slots_ptr, num_tokens, k_ptr, v_ptr, layout, stream)


def codec_rotary_by_axes(rotary, num_heads: int, head_dim: int, dtype: int, x, out, positions_ptr: int, num_tokens: int,
                         stream: int = 0) -> int:
    """``rotary``: codec_rotary_axes, or its bytes; ``x`` and ``out``: codec_rows."""
    return _lib.codec_rotary_by_axes(_struct(rotary), num_heads, head_dim, dtype, x, out, positions_ptr, num_tokens, stream)


def codec_append_by_axes(head, rotary, q, q_out, k, v, positions_ptr: int, slots_ptr: int, num_tokens: int, k_ptr: int, v_ptr: int,
                         layout, stream: int = 0) -> int:
    """codec_append with a codec_rotary_axes, or its bytes."""
    return _lib.codec_append_by_axes(head, _struct(rotary), q, q_out, k, v, positions_ptr, slots_ptr, num_tokens, k_ptr, v_ptr, layout, stream)


def codec_pages_create(num_pages: int):
    """Returns (status, handle or None)."""
    if not _is_int32(num_pages):
        return CODEC_ERR_INVALID_ARGUMENT, None
    handle = c_void_p()
    st = _lib.codec_pages_create(num_pages, byref(handle))
    return st, (handle if st == CODEC_OK else None)


def codec_pages_destroy(pages) -> int:
    return _lib.codec_pages_destroy(pages)


def codec_pages_free(pages) -> int:
    return int(_lib.codec_pages_free(pages))


def codec_pages_take(pages, n: int):
    """Returns (status, ids or None)."""
    if not _is_int32(n):
        return CODEC_ERR_INVALID_ARGUMENT, None
    ids = np.empty(max(0, min(n, codec_pages_free(pages))), np.int32)           # (the call writes all of n or nothing)
    st = _lib.codec_pages_take(pages, n, ids.ctypes.data)
    return st, (ids if st == CODEC_OK else None)


def codec_pages_hold(pages, ids) -> int:
    ids = _ids(ids)
    if ids is None:
        return CODEC_ERR_INVALID_ARGUMENT
    return _lib.codec_pages_hold(pages, _in(ids), ids.size)


def codec_pages_release(pages, ids) -> int:
    ids = _ids(ids)
    if ids is None:
        return CODEC_ERR_INVALID_ARGUMENT
    return _lib.codec_pages_release(pages, _in(ids), ids.size)


def codec_pages_fork(pages, page_size: int, page_off, page_ids, tokens, parents):
    """Returns (status, page_off, page_ids, runs [n, 5]) of the sequences that go on, or (status, None, None, None)."""
    off, ids, tokens, parents = _ids(page_off), _ids(page_ids), _ids(tokens), _ids(parents)
    if off is None or ids is None or tokens is None or parents is None or not _is_int32(page_size):
        return CODEC_ERR_INVALID_ARGUMENT, None, None, None
    num_seq, num_out = tokens.size, parents.size
    if off.ndim != 1 or off.size != num_seq + 1 or off[0] != 0 or off[-1] != ids.size:      # the C call reads by these lengths
        return CODEC_ERR_INVALID_ARGUMENT, None, None, None
    # room for lists of the longest of the old ones' length, and for a run each, in one array
    longest = int(np.maximum.reduce(off[1:] - off[:-1], initial=0))
    capacity = min(longest * num_out, 0x7fffffff)
    room, n = np.empty(num_out + 1 + capacity + 5 * num_out, np.int32), c_int32(0)
    at = room.ctypes.data
    st = _lib.codec_pages_fork(pages, page_size, num_seq, _in(off), _in(ids), _in(tokens), num_out, _in(parents), at,
                               at + 4 * (num_out + 1), capacity, at + 4 * (num_out + 1 + capacity), byref(n))
    if st != CODEC_OK:
        return st, None, None, None
    out_off = room[:num_out + 1].copy()                     # (the lists that live on do not keep the room)
    out_ids = room[num_out + 1:num_out + 1 + out_off[-1]].copy()
    runs = room[num_out + 1 + capacity:num_out + 1 + capacity + 5 * n.value].reshape(-1, 5)
    return st, out_off, out_ids, runs


def codec_pages_compact(pages, page_size: int, capacity: int):
    """Returns (status, runs [n, 5] or None)."""
    if not (_is_int32(page_size) and _is_int32(capacity)):
        return CODEC_ERR_INVALID_ARGUMENT, None
    runs, n = np.empty((max(0, capacity), 5), np.int32), c_int32(0)
    st = _lib.codec_pages_compact(pages, page_size, runs.ctypes.data, capacity, byref(n))
    return st, (runs[:n.value] if st == CODEC_OK else None)


def codec_cache_copy(head, layout, k_ptrs, v_ptrs, runs, stream: int = 0) -> int:
    """``head``: codec_head_config; ``layout``: codec_kv_layout; ``k_ptrs``, ``v_ptrs``: the layers' pools; ``runs``: [n, 5]."""
    runs = _ids(runs)
    if runs is None or len(k_ptrs) != len(v_ptrs) or runs.ndim != 2 or runs.shape[1] != 5:
        return CODEC_ERR_INVALID_ARGUMENT
    pools = f"{len(k_ptrs)}P"                           # bytes as an array of pointers
    return _lib.codec_cache_copy(head, layout, len(k_ptrs), struct.pack(pools, *k_ptrs), struct.pack(pools, *v_ptrs), _in(runs), len(runs),
                                 stream)


def codec_block_table(page_size: int, num_seq: int, page_off_ptr: int, page_ids_ptr: int, num_ids: int, tokens_ptr: int, table_ptr: int,
                      table_stride: int, width: int, stream: int = 0) -> int:
    return _lib.codec_block_table(page_size, num_seq, page_off_ptr, page_ids_ptr, num_ids, tokens_ptr, table_ptr, table_stride, width, stream)


def codec_slot_workspace_bytes(config) -> int:
    """``config``: codec_slot_config, or its bytes."""
    return _lib.codec_slot_workspace_bytes(_struct(config))


def codec_slot_map(config, table_ptr: int, tokens_ptr: int, new_tokens_ptr: int, before_ptr: int, spare_ptr: int, positions_ptr: int,
                   slots_ptr: int, sequences_ptr: int, offsets_ptr: int, tokens_out_ptr: int, taken_ptr: int, workspace_ptr: int = 0,
                   workspace_bytes: int = 0, stream: int = 0) -> int:
    """``config``: codec_slot_config, or its bytes."""
    return _lib.codec_slot_map(_struct(config), table_ptr, tokens_ptr, new_tokens_ptr, before_ptr, spare_ptr, positions_ptr, slots_ptr, sequences_ptr,
                               offsets_ptr, tokens_out_ptr, taken_ptr, workspace_ptr, workspace_bytes, stream)


def codec_beam_workspace_bytes(config) -> int:
    return int(_lib.codec_beam_workspace_bytes(config))


def codec_beam_select(config, logits_ptr: int, batch_stride: int, beam_stride: int, scores_ptr: int, finished_ptr: int,
                      out_scores_ptr: int, out_beams_ptr: int, out_tokens_ptr: int, workspace_ptr: int, workspace_bytes: int,
                      stream: int = 0) -> int:
    """``config``: codec_beam_config."""
    return _lib.codec_beam_select(config, logits_ptr, batch_stride, beam_stride, scores_ptr, finished_ptr, out_scores_ptr,
                                  out_beams_ptr, out_tokens_ptr, workspace_ptr, workspace_bytes, stream)


def codec_beam_reorder(states, beams_ptr: int, batch: int, beams_in: int, beams_out: int, stream: int = 0) -> int:
    """``states``: the fields of every codec_state in a row (src, dst, row_bytes, src_batch_stride, src_beam_stride,
    dst_batch_stride, dst_beam_stride)."""
    n = len(states) // 7
    if len(states) != 7 * n:
        return CODEC_ERR_INVALID_ARGUMENT
    packed = struct.pack(f"{7 * n}q", *states)          # the layout of codec_state, several times faster than its class
    return _lib.codec_beam_reorder(packed, n, beams_ptr, batch, beams_in, beams_out, stream)
