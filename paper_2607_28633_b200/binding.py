"""ctypes binding of the TopKV C-ABI library (``include/topkv.h``).

Argument marshalling only: every function below has the name and the argument order of the
C entry point it calls, accepts torch tensors (their ``data_ptr()`` is passed) or raw integer
addresses, and returns the C status code unchanged. ``check()`` turns a negative status into
an exception. The library is loaded on first use; if it has not been built this module
raises — there is no fallback implementation.
"""
from __future__ import annotations

import ctypes
import os
from ctypes import c_double, c_float, c_int, c_int32, c_int64, c_uint32, c_void_p

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtopkv.so")

TOPKV_OK = 0
TOPKV_ERR_INVALID_ARG = -1
TOPKV_ERR_LAYER_RANGE = -2
TOPKV_ERR_ALIGNMENT = -3
TOPKV_ERR_CAPACITY = -4
TOPKV_ERR_UNSUPPORTED_LAYOUT = -5
TOPKV_ERR_CUDA = -6
TOPKV_ERR_CHECKSUM = -7

TOPKV_KIND_GQA, TOPKV_KIND_MLA = 0, 1
TOPKV_WIRE_TOKEN_KV, TOPKV_WIRE_PLANAR = 0, 1
TOPKV_MAX_INLINE_R = 1024
TOPKV_FLAG_OVERLAP_PREVIOUS = 1
TOPKV_FLAG_TABLES_SETTLED = 2
TOPKV_LINK_WAIT_PREVIOUS = 1
TOPKV_NOALLOC_STAGING_BYTES = 8 * 1024 * 1024
TOPKV_TYPE_BF16, TOPKV_TYPE_FP16, TOPKV_TYPE_E4M3 = 1, 2, 3

# every symbol include/topkv.h declares
EXPORTS = (
    "topkv_append_layer", "topkv_rotary_frequencies", "topkv_rotary_turns", "topkv_plan_prefixes",
    "topkv_attend_shared_workspace_bytes", "topkv_attend_shared_layer", "topkv_set_sharing_bytes", "topkv_bound_pages_layer",
    "topkv_page_choice_workspace_bytes", "topkv_choose_pages_layer", "topkv_attend_pages_layer",
    "topkv_pack_layer", "topkv_unpack_layer", "topkv_pack_layer_to_host",
    "topkv_unpack_layer_from_host", "topkv_build_plan", "topkv_validate_batch_host",
    "topkv_layout_default_strides", "topkv_wire_layer_bytes", "topkv_kv_bytes",
    "topkv_model_transfer_s", "topkv_model_t_eff_s", "topkv_model_hidden_fraction",
    "topkv_strerror", "topkv_version", "topkv_last_cuda_error", "topkv_kernel_launch_count",
    "topkv_set_kernel_variant", "topkv_pack_layer_to_host_noalloc", "topkv_device_error_flags",
    "topkv_reset_device_error_flags", "topkv_repage_layer", "topkv_kv_bytes_layered",
    "topkv_header_fill", "topkv_header_check", "topkv_crc64", "topkv_crc_workspace_bytes",
    "topkv_crc_begin", "topkv_pack_layer_crc", "topkv_unpack_layer_crc", "topkv_crc_finish",
    "topkv_retry", "topkv_pack_layer_to_host_crc", "topkv_unpack_layer_from_host_crc",
    "topkv_set_host_leg_ctas", "topkv_pack_layers_to_host_pipelined",
    "topkv_unpack_layers_from_host_pipelined", "topkv_pack_layers", "topkv_unpack_layers",
    "topkv_copy_vector_bytes", "topkv_copy_grid_ctas", "topkv_select_transport", "topkv_planning_rate",
    "topkv_transport_name", "topkv_layer_table_offsets", "topkv_pack_model_layers",
    "topkv_unpack_model_layers", "topkv_pack_model_layers_to_host_pipelined",
    "topkv_unpack_model_layers_from_host_pipelined", "topkv_span_link_words",
    "topkv_pack_layer_linked", "topkv_unpack_layer_linked",
    "topkv_pack_layers_to_host_two_lanes", "topkv_unpack_layers_from_host_two_lanes",
    "topkv_relay_layers_linked", "topkv_attend_workspace_bytes", "topkv_attend_layer",
    "topkv_page_workspace_bytes", "topkv_extend_requests", "topkv_fork_requests",
    "topkv_free_requests", "topkv_compact_pages", "topkv_copy_pages",
)


class topkv_layout(ctypes.Structure):
    _fields_ = [
        ("struct_size", c_uint32), ("kind", c_uint32), ("num_layers", c_uint32),
        ("kv_factor", c_uint32), ("num_kv_heads", c_uint32), ("head_dim", c_uint32),
        ("elem_bytes", c_uint32), ("page_tokens", c_uint32), ("wire_order", c_uint32),
        ("reserved", c_uint32), ("num_pool_pages", c_int64), ("pool_layer_stride", c_int64),
        ("pool_page_stride", c_int64), ("pool_kv_stride", c_int64),
        ("pool_token_stride", c_int64), ("pool_head_stride", c_int64),
        ("wire_layer_stride", c_int64), ("wire_plane_stride", c_int64),
    ]


class topkv_batch(ctypes.Structure):
    _fields_ = [
        ("struct_size", c_uint32), ("num_requests", c_int32), ("max_pages_per_req", c_int32),
        ("flags", c_uint32), ("block_table", c_void_p), ("seq_lens", c_void_p),
        ("cu_seq_lens", c_void_p), ("total_tokens", c_int64), ("window_tokens", c_int32),
        ("reserved", c_int32),
    ]


class topkv_layer_spec(ctypes.Structure):
    _fields_ = [("kind", c_uint32), ("reserved", c_uint32), ("param", c_int64)]


TOPKV_LAYER_FULL, TOPKV_LAYER_WINDOW, TOPKV_LAYER_STATE = 0, 1, 2


class topkv_span_link(ctypes.Structure):
    _fields_ = [("struct_size", c_uint32), ("await_epoch", c_uint32), ("signal_epoch", c_uint32),
                ("flags", c_uint32), ("d_await", c_void_p), ("d_signal", c_void_p)]


def make_span_link(d_await=None, await_epoch=0, d_signal=None, signal_epoch=0,
                   flags: int = 0) -> topkv_span_link:
    k = topkv_span_link()
    k.struct_size = ctypes.sizeof(topkv_span_link)
    k.await_epoch, k.signal_epoch, k.flags = await_epoch, signal_epoch, flags
    k.d_await, k.d_signal = _ptr(d_await), _ptr(d_signal)
    k._keepalive = (d_await, d_signal)
    return k


class topkv_layer_table(ctypes.Structure):
    _fields_ = [("struct_size", c_uint32), ("num_layers", c_uint32), ("specs", c_void_p),
                ("h_seq_lens", c_void_p), ("state_pool", c_void_p), ("state_slots", c_void_p),
                ("state_layer_stride", c_int64), ("state_slot_stride", c_int64),
                ("num_state_slots", c_int64)]


def make_layer_table(specs, h_seq_lens, state_pool=None, state_slots=None, state_layer_stride=0,
                     state_slot_stride=0, num_state_slots=0) -> topkv_layer_table:
    """specs: sequence of (kind, param) per model layer; h_seq_lens: numpy int32 [R] on the host;
    state_pool / state_slots: device tensors (or None). The table keeps what it points to alive."""
    import numpy as np
    arr = (topkv_layer_spec * len(specs))()
    for i, (kind, param) in enumerate(specs):
        arr[i].kind, arr[i].param = kind, param
    lens = np.ascontiguousarray(h_seq_lens, dtype=np.int32)
    t = topkv_layer_table()
    t.struct_size = ctypes.sizeof(topkv_layer_table)
    t.num_layers = len(specs)
    t.specs = ctypes.addressof(arr)
    t.h_seq_lens = lens.ctypes.data
    t.state_pool = _ptr(state_pool)
    t.state_slots = _ptr(state_slots)
    t.state_layer_stride, t.state_slot_stride = state_layer_stride, state_slot_stride
    t.num_state_slots = num_state_slots
    t._keepalive = (arr, lens, state_pool, state_slots)
    return t


class topkv_attention(ctypes.Structure):
    _fields_ = [
        ("struct_size", c_uint32), ("cache_type", c_uint32), ("io_type", c_uint32),
        ("num_q_heads", c_uint32), ("value_dim", c_uint32), ("sink_tokens", c_uint32),
        ("scale", c_float), ("k_scale", c_float), ("v_scale", c_float), ("reserved", c_uint32),
        ("q_request_stride", c_int64), ("q_head_stride", c_int64),
        ("out_request_stride", c_int64), ("out_head_stride", c_int64), ("lse", c_void_p),
    ]


def make_attention(q, out, cache_type: int, io_type: int, scale: float, value_dim: int = 0,
                   sink_tokens: int = 0, k_scale: float = 1.0, v_scale: float = 1.0,
                   lse=None) -> topkv_attention:
    """q [R][num_q_heads][head_dim] and out [R][num_q_heads][value_dim or head_dim]: device tensors
    of 16-bit elements, whose strides the descriptor takes (the last axis must be contiguous)."""
    for t in (q, out):
        if t.ndim != 3 or t.element_size() != 2 or (t.shape[2] > 1 and t.stride(2) != 1):
            raise ValueError("q and out are [requests][heads][elements] of 16-bit elements, the last axis contiguous")
    if q.shape[:2] != out.shape[:2]:
        raise ValueError("q and out differ in requests or heads")
    if q.dtype != out.dtype or q.device != out.device or (lse is not None and lse.device != q.device):
        raise ValueError("q and out differ in type, or the tensors in device")
    if out.shape[2] < (value_dim or q.shape[2]):
        raise ValueError("out has room for value_dim elements per head, or as many as q")
    if lse is not None and (tuple(lse.shape) != tuple(q.shape[:2]) or lse.element_size() != 4 or not lse.is_contiguous()):
        raise ValueError("lse is a contiguous float32 [requests][heads]")
    a = topkv_attention()
    a.struct_size = ctypes.sizeof(topkv_attention)
    a.cache_type, a.io_type, a.num_q_heads, a.value_dim = cache_type, io_type, q.shape[1], value_dim
    a.sink_tokens, a.scale, a.k_scale, a.v_scale = sink_tokens, scale, k_scale, v_scale
    a.q_request_stride, a.q_head_stride = 2 * q.stride(0), 2 * q.stride(1)
    a.out_request_stride, a.out_head_stride = 2 * out.stride(0), 2 * out.stride(1)
    a.lse = _ptr(lse)
    a._keepalive = lse
    return a


TOPKV_ROTARY_HALVES, TOPKV_ROTARY_PAIRS = 1, 2
TOPKV_STRETCH_NONE, TOPKV_STRETCH_LINEAR, TOPKV_STRETCH_BASE, TOPKV_STRETCH_RAMP = 0, 1, 2, 3
TOPKV_PLAN_ROWS = 6
TOPKV_DEFAULT_SHARING_BYTES = 8 * 1024 * 1024
(TOPKV_PLAN_LEADER, TOPKV_PLAN_COMMON, TOPKV_PLAN_SHARED, TOPKV_PLAN_MEMBERS, TOPKV_PLAN_ORDER,
 TOPKV_PLAN_PLACE) = range(TOPKV_PLAN_ROWS)


class topkv_rotary(ctypes.Structure):
    _fields_ = [("struct_size", c_uint32), ("style", c_uint32), ("first", c_uint32), ("count", c_uint32),
                ("scale", c_float), ("reserved", c_uint32), ("turns", c_void_p)]


class topkv_rotary_stretch(ctypes.Structure):
    _fields_ = [("struct_size", c_uint32), ("kind", c_uint32), ("base", c_double), ("factor", c_double),
                ("original_tokens", c_double), ("slow", c_double), ("fast", c_double)]


class topkv_new_tokens(ctypes.Structure):
    _fields_ = [("struct_size", c_uint32), ("cache_type", c_uint32), ("io_type", c_uint32), ("num_q_heads", c_uint32),
                ("num_rows", c_int64), ("k_scale", c_float), ("v_scale", c_float), ("cu_tokens", c_void_p),
                ("positions", c_void_p), ("rotary", ctypes.POINTER(topkv_rotary)),
                ("k_row_stride", c_int64), ("k_head_stride", c_int64), ("v_row_stride", c_int64), ("v_head_stride", c_int64),
                ("q_row_stride", c_int64), ("q_head_stride", c_int64), ("q_out_row_stride", c_int64), ("q_out_head_stride", c_int64)]


class topkv_page_choice(ctypes.Structure):
    _fields_ = [("struct_size", c_uint32), ("budget", c_uint32), ("first_pages", c_uint32), ("last_pages", c_uint32),
                ("bounds", c_void_p), ("steps", c_void_p), ("chosen", c_void_p)]


def make_rotary(turns, style: int = TOPKV_ROTARY_HALVES, first: int = 0, scale: float = 1.0) -> topkv_rotary:
    """turns: contiguous device tensor of 64-bit integers, one per pair, from topkv_rotary_turns."""
    if turns.ndim != 1 or turns.element_size() != 8 or turns.is_floating_point() or not turns.is_contiguous():
        raise ValueError("turns is a contiguous vector of 64-bit integers")
    t = topkv_rotary()
    t.struct_size = ctypes.sizeof(topkv_rotary)
    t.style, t.first, t.count, t.scale, t.turns = style, first, 2 * turns.numel(), scale, _ptr(turns)
    t._keepalive = turns
    return t


def make_new_tokens(k, v, cache_type: int, io_type: int, q=None, q_out=None, rotary: topkv_rotary | None = None,
                    cu_tokens=None, positions=None, k_scale: float = 1.0, v_scale: float = 1.0) -> topkv_new_tokens:
    """k, v [rows][kv heads][head_dim] and q, q_out [rows][q heads][head_dim]: device tensors of 16-bit
    elements (v None for latent rows, q and q_out None for keys alone), whose strides the descriptor takes (the
    last axis must be contiguous). cu_tokens: device int64 [R + 1] or None; positions: device int32 [rows] or None."""
    tensors = [t for t in (k, v, q, q_out) if t is not None]
    for t in tensors:
        if t.ndim != 3 or t.element_size() != 2 or (t.shape[2] > 1 and t.stride(2) != 1):
            raise ValueError("k, v, q and q_out are [rows][heads][elements] of 16-bit elements, the last axis contiguous")
        if t.dtype != k.dtype or t.device != k.device or t.shape[0] != k.shape[0] or t.shape[2] != k.shape[2]:
            raise ValueError("k, v, q and q_out differ in type, device, rows or elements")
    if (v is not None and v.shape != k.shape) or (q is None) != (q_out is None) or (q is not None and q.shape != q_out.shape):
        raise ValueError("v is shaped as k, q_out as q")
    for t, size in ((cu_tokens, 8), (positions, 4)):
        if t is not None and (t.ndim != 1 or t.element_size() != size or t.is_floating_point() or not t.is_contiguous() or t.device != k.device):
            raise ValueError("cu_tokens and positions are contiguous vectors of 64- and 32-bit integers on the tensors' device")
    if rotary is not None and getattr(rotary, "_keepalive", None) is not None and rotary._keepalive.device != k.device:
        raise ValueError("the rotary turns are on another device than the tensors")
    if positions is not None and positions.numel() < k.shape[0]:
        raise ValueError("a position for every row")
    stride = lambda t, i: 2 * t.stride(i) if t.shape[i] > 1 else 0
    n = topkv_new_tokens()
    n.struct_size = ctypes.sizeof(topkv_new_tokens)
    n.cache_type, n.io_type, n.num_q_heads, n.num_rows = cache_type, io_type, q.shape[1] if q is not None else 0, k.shape[0]
    n.k_scale, n.v_scale, n.cu_tokens, n.positions = k_scale, v_scale, _ptr(cu_tokens), _ptr(positions)
    if rotary is not None:
        n.rotary = ctypes.pointer(rotary)
    n.k_row_stride, n.k_head_stride = stride(k, 0), stride(k, 1)
    if v is not None:
        n.v_row_stride, n.v_head_stride = stride(v, 0), stride(v, 1)
    if q is not None:
        n.q_row_stride, n.q_head_stride = stride(q, 0), stride(q, 1)
        n.q_out_row_stride, n.q_out_head_stride = stride(q_out, 0), stride(q_out, 1)
    n._keepalive = (rotary, cu_tokens, positions)
    return n


def make_page_choice(budget: int, first_pages: int, last_pages: int, bounds, steps, chosen) -> topkv_page_choice:
    """bounds int8 [pages][kv heads][2][head_dim], steps float32 [pages][kv heads], chosen int32 [requests][kv
    heads][budget]: contiguous device tensors."""
    if bounds.ndim != 4 or bounds.element_size() != 1 or bounds.shape[2] != 2 or not bounds.is_contiguous():
        raise ValueError("bounds is a contiguous int8 [pages][kv heads][2][head_dim]")
    if tuple(steps.shape) != tuple(bounds.shape[:2]) or steps.element_size() != 4 or not steps.is_contiguous():
        raise ValueError("steps is a contiguous float32 [pages][kv heads]")
    if chosen.ndim != 3 or tuple(chosen.shape[1:]) != (bounds.shape[1], budget) or chosen.element_size() != 4 or not chosen.is_contiguous():
        raise ValueError("chosen is a contiguous int32 [requests][kv heads][budget]")
    if not (bounds.device == steps.device == chosen.device):
        raise ValueError("the tensors differ in device")
    c = topkv_page_choice()
    c.struct_size = ctypes.sizeof(topkv_page_choice)
    c.budget, c.first_pages, c.last_pages = budget, first_pages, last_pages
    c.bounds, c.steps, c.chosen = _ptr(bounds), _ptr(steps), _ptr(chosen)
    c._keepalive = (bounds, steps, chosen)
    return c


class topkv_page_tables(ctypes.Structure):
    _fields_ = [("struct_size", c_uint32), ("reserved", c_uint32), ("ref_counts", c_void_p),
                ("block_table_out", c_void_p), ("seq_lens_out", c_void_p), ("ref_counts_out", c_void_p)]


def make_page_tables(ref_counts, block_table_out, seq_lens_out, ref_counts_out) -> topkv_page_tables:
    """Device int32 tensors; an out tensor may be the one it is read from (in place)."""
    t = topkv_page_tables()
    t.struct_size = ctypes.sizeof(topkv_page_tables)
    t.ref_counts, t.block_table_out = _ptr(ref_counts), _ptr(block_table_out)
    t.seq_lens_out, t.ref_counts_out = _ptr(seq_lens_out), _ptr(ref_counts_out)
    t._keepalive = (ref_counts, block_table_out, seq_lens_out, ref_counts_out)
    return t


TOPKV_TRANSPORT_NVLINK, TOPKV_TRANSPORT_PCIE, TOPKV_TRANSPORT_RDMA, TOPKV_TRANSPORT_TCP = 1, 2, 3, 4


class topkv_endpoint(ctypes.Structure):
    _fields_ = [("struct_size", c_uint32), ("has_nvlink", c_uint32),
                ("nvlink_domain", ctypes.c_char_p), ("node_ip", ctypes.c_char_p)]


def make_endpoint(nvlink_domain, has_nvlink, node_ip) -> topkv_endpoint:
    e = topkv_endpoint()
    e.struct_size = ctypes.sizeof(topkv_endpoint)
    e.has_nvlink = 1 if has_nvlink else 0
    e.nvlink_domain = None if nvlink_domain is None else nvlink_domain.encode()
    e.node_ip = None if node_ip is None else node_ip.encode()
    return e


class topkv_wire_header(ctypes.Structure):
    _fields_ = [
        ("magic", ctypes.c_char * 8), ("request_id", ctypes.c_uint64), ("model_id", ctypes.c_uint64),
        ("seq_len", c_uint32), ("num_layers", c_uint32), ("num_kv_heads", c_uint32),
        ("head_dim", c_uint32), ("elem_bytes", c_uint32), ("kv_factor", c_uint32),
        ("k_bytes", ctypes.c_uint64), ("v_bytes", ctypes.c_uint64), ("crc_k", ctypes.c_uint64),
        ("crc_v", ctypes.c_uint64), ("reserved", ctypes.c_uint8 * 48),
    ]


RETRY_ATTEMPT = ctypes.CFUNCTYPE(c_int, c_void_p)


class TopkvError(RuntimeError):
    def __init__(self, status: int):
        self.status = status
        super().__init__(f"topkv status {status}: {topkv_strerror(status)}")


_lib = None


def lib() -> ctypes.CDLL:
    """Loads libtopkv.so (built by ``__graft_entry__.build()``); raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(
                f"{LIB_PATH} not found: build the CUDA library first "
                "(python -c 'import __graft_entry__ as g; g.build()'); there is no CPU fallback")
        L = ctypes.CDLL(LIB_PATH)
        lp, bp = ctypes.POINTER(topkv_layout), ctypes.POINTER(topkv_batch)
        L.topkv_pack_layer.argtypes = [c_int, c_void_p, lp, bp, c_void_p, c_int64, c_void_p]
        L.topkv_unpack_layer.argtypes = [c_int, c_void_p, lp, bp, c_void_p, c_int64, c_void_p]
        L.topkv_pack_layer_to_host.argtypes = [c_int, c_void_p, lp, bp, c_void_p, c_int64,
                                               c_void_p, c_int64, c_void_p]
        L.topkv_unpack_layer_from_host.argtypes = [c_int, c_void_p, lp, bp, c_void_p, c_int64,
                                                   c_void_p, c_int64, c_void_p]
        L.topkv_build_plan.argtypes = [bp, c_void_p, c_void_p]
        u64 = ctypes.c_uint64
        hp = ctypes.POINTER(topkv_wire_header)
        L.topkv_header_fill.argtypes = [hp, u64, u64, lp, c_int64, u64, u64]
        L.topkv_header_check.argtypes = [hp, lp, c_int64, u64, u64]
        L.topkv_crc64.argtypes = [c_void_p, c_int64]
        L.topkv_crc64.restype = u64
        L.topkv_crc_workspace_bytes.argtypes = [lp, c_int32, c_int32]
        L.topkv_crc_workspace_bytes.restype = c_int64
        L.topkv_crc_begin.argtypes = [lp, bp, c_void_p, c_int64, c_void_p]
        L.topkv_pack_layer_crc.argtypes = [c_int, c_void_p, lp, bp, c_void_p, c_int64, c_void_p,
                                           c_int64, c_void_p]
        L.topkv_unpack_layer_crc.argtypes = [c_int, c_void_p, lp, bp, c_void_p, c_int64, c_void_p,
                                             c_int64, c_void_p]
        L.topkv_crc_finish.argtypes = [lp, bp, c_void_p, c_int64, c_void_p, c_void_p]
        for fn in (L.topkv_pack_layer_to_host_crc, L.topkv_unpack_layer_from_host_crc):
            fn.argtypes = [c_int, c_void_p, lp, bp, c_void_p, c_int64, c_void_p, c_int64, c_void_p,
                           c_int64, c_void_p]
        L.topkv_retry.argtypes = [RETRY_ATTEMPT, c_void_p, c_int, c_int]
        L.topkv_repage_layer.argtypes = [c_int, c_void_p, lp, bp, c_void_p, lp, bp, c_void_p]
        L.topkv_pack_layer_to_host_noalloc.argtypes = [c_int, c_void_p, lp, bp, c_void_p, c_int64,
                                                       c_void_p]
        L.topkv_validate_batch_host.argtypes = [lp, c_int32, c_int32, c_void_p, c_void_p, c_int]
        L.topkv_layout_default_strides.argtypes = [lp]
        L.topkv_wire_layer_bytes.argtypes = [lp, c_int64]
        L.topkv_wire_layer_bytes.restype = c_int64
        L.topkv_kv_bytes.argtypes = [lp, c_int64]
        L.topkv_kv_bytes.restype = c_int64
        L.topkv_kv_bytes_layered.argtypes = [lp, c_void_p, c_int64]
        L.topkv_kv_bytes_layered.restype = c_int64
        L.topkv_model_transfer_s.argtypes = [c_double] * 3
        L.topkv_model_transfer_s.restype = c_double
        L.topkv_model_t_eff_s.argtypes = [c_double] * 3
        L.topkv_model_t_eff_s.restype = c_double
        L.topkv_model_hidden_fraction.argtypes = [c_int, c_double, c_double]
        L.topkv_model_hidden_fraction.restype = c_double
        L.topkv_strerror.argtypes = [c_int]
        L.topkv_strerror.restype = ctypes.c_char_p
        L.topkv_kernel_launch_count.restype = c_int64
        L.topkv_set_kernel_variant.argtypes = [c_int]
        L.topkv_set_host_leg_ctas.argtypes = [c_int]
        L.topkv_pack_layers.argtypes = [c_int, c_int, c_void_p, lp, bp, c_void_p, c_int64, c_void_p]
        L.topkv_unpack_layers.argtypes = [c_int, c_int, c_void_p, lp, bp, c_void_p, c_int64, c_void_p]
        for fn in (L.topkv_pack_layers_to_host_two_lanes, L.topkv_unpack_layers_from_host_two_lanes):
            fn.argtypes = [c_int, c_int, c_void_p, lp, bp, c_void_p, c_int64, c_void_p, c_int64,
                           c_void_p, c_void_p, c_void_p]
        kp_ = ctypes.POINTER(topkv_span_link)
        L.topkv_span_link_words.argtypes = [lp, bp]
        L.topkv_span_link_words.restype = c_int64
        L.topkv_pack_layer_linked.argtypes = [c_int, c_void_p, lp, bp, c_void_p, c_int64, kp_, c_void_p]
        L.topkv_unpack_layer_linked.argtypes = [c_int, c_void_p, lp, bp, c_void_p, c_int64, kp_, c_void_p]
        L.topkv_relay_layers_linked.argtypes = [c_int, c_int, c_void_p, lp, bp, c_void_p, lp, bp, c_void_p,
                                                c_int64, c_void_p, c_int64, c_uint32, c_void_p]
        tp = ctypes.POINTER(topkv_layer_table)
        L.topkv_layer_table_offsets.argtypes = [lp, tp, c_int32, c_void_p]
        L.topkv_pack_model_layers.argtypes = [c_int, c_int, c_void_p, lp, bp, tp, c_void_p, c_int64, c_void_p]
        L.topkv_unpack_model_layers.argtypes = [c_int, c_int, c_void_p, lp, bp, tp, c_void_p, c_int64, c_void_p]
        for fn in (L.topkv_pack_model_layers_to_host_pipelined,
                   L.topkv_unpack_model_layers_from_host_pipelined):
            fn.argtypes = [c_int, c_int, c_void_p, lp, bp, tp, c_void_p, c_int64, c_void_p, c_int64,
                           c_void_p, c_void_p, c_void_p]
        ap, pp = ctypes.POINTER(topkv_attention), ctypes.POINTER(topkv_page_tables)
        L.topkv_attend_workspace_bytes.argtypes = [lp, bp, ap]
        L.topkv_attend_workspace_bytes.restype = c_int64
        L.topkv_attend_layer.argtypes = [c_int, c_void_p, lp, bp, ap, c_void_p, c_void_p, c_void_p, c_int64,
                                         c_void_p]
        L.topkv_page_workspace_bytes.argtypes = [lp, bp, c_int32]
        L.topkv_page_workspace_bytes.restype = c_int64
        L.topkv_extend_requests.argtypes = [lp, bp, pp, c_void_p, c_void_p, c_int64, c_void_p]
        L.topkv_fork_requests.argtypes = [c_void_p, lp, bp, pp, c_void_p, c_void_p, c_int32, c_void_p, c_int64,
                                          c_void_p]
        L.topkv_free_requests.argtypes = [lp, bp, pp, c_void_p, c_int32, c_void_p]
        L.topkv_compact_pages.argtypes = [c_void_p, lp, bp, pp, c_void_p, c_void_p, c_void_p, c_int64, c_void_p]
        L.topkv_copy_pages.argtypes = [c_int, c_int, c_void_p, lp, c_void_p, c_void_p, c_int32, c_void_p]
        np_, cp = ctypes.POINTER(topkv_new_tokens), ctypes.POINTER(topkv_page_choice)
        L.topkv_append_layer.argtypes = [c_int, c_void_p, lp, bp, np_, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]
        L.topkv_rotary_frequencies.argtypes = [ctypes.POINTER(topkv_rotary_stretch), c_uint32, c_void_p]
        L.topkv_rotary_turns.argtypes = [c_void_p, c_uint32, c_void_p]
        L.topkv_plan_prefixes.argtypes = [lp, bp, c_int32, c_void_p, c_void_p]
        L.topkv_set_sharing_bytes.argtypes = [c_int64]
        L.topkv_set_sharing_bytes.restype = c_int64
        L.topkv_attend_shared_workspace_bytes.argtypes = [lp, bp, ap]
        L.topkv_attend_shared_workspace_bytes.restype = c_int64
        L.topkv_attend_shared_layer.argtypes = [c_int, c_void_p, lp, bp, ap, c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_void_p]
        L.topkv_bound_pages_layer.argtypes = [c_int, c_void_p, lp, bp, c_uint32, c_void_p, c_void_p, c_void_p]
        L.topkv_page_choice_workspace_bytes.argtypes = [lp, bp, ap, cp]
        L.topkv_page_choice_workspace_bytes.restype = c_int64
        L.topkv_choose_pages_layer.argtypes = [lp, bp, ap, cp, c_void_p, c_void_p, c_int64, c_void_p]
        L.topkv_attend_pages_layer.argtypes = [c_int, c_void_p, lp, bp, ap, cp, c_void_p, c_void_p, c_void_p, c_int64, c_void_p]
        ep = ctypes.POINTER(topkv_endpoint)
        L.topkv_select_transport.argtypes = [ep, ep, c_int, c_int]
        L.topkv_planning_rate.argtypes = [c_int]
        L.topkv_planning_rate.restype = c_double
        L.topkv_transport_name.argtypes = [c_int]
        L.topkv_transport_name.restype = ctypes.c_char_p
        L.topkv_copy_vector_bytes.argtypes = [c_int, c_int, c_void_p, lp, bp, c_void_p, c_int64]
        L.topkv_copy_grid_ctas.restype = c_int64
        L.topkv_copy_grid_ctas.argtypes = [c_int, c_void_p, lp, bp, c_void_p, c_int64, ctypes.POINTER(c_int32)]
        for fn in (L.topkv_pack_layers_to_host_pipelined, L.topkv_unpack_layers_from_host_pipelined):
            fn.argtypes = [c_int, c_int, c_void_p, lp, bp, c_void_p, c_int64, c_void_p, c_int64,
                           c_void_p, c_void_p, c_void_p]
        _lib = L
    return _lib


def _ptr(x) -> int | None:
    """torch tensor / numpy array / int / None -> address."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if hasattr(x, "data_ptr"):
        return x.data_ptr()
    if hasattr(x, "ctypes"):
        return x.ctypes.data
    raise TypeError(type(x))


def _stream(s) -> int | None:
    if s is None:
        return None
    if isinstance(s, int):
        return s or None
    return s.cuda_stream or None  # torch.cuda.Stream


def check(status: int) -> int:
    if status < 0:
        raise TopkvError(status)
    return status


# ---- constructors for the two descriptors -------------------------------------------------

def make_layout(L: int, F: int, H: int, D: int, E: int, P: int, num_pool_pages: int,
                wire_order: int = TOPKV_WIRE_TOKEN_KV, wire_layer_stride: int = 0,
                kind: int | None = None) -> topkv_layout:
    """Layout of the default page-major pool pool[l][page][c][t][h][d]."""
    lo = topkv_layout()
    lo.struct_size = ctypes.sizeof(topkv_layout)
    lo.kind = (TOPKV_KIND_MLA if F == 1 and H == 1 else TOPKV_KIND_GQA) if kind is None else kind
    lo.num_layers, lo.kv_factor, lo.num_kv_heads, lo.head_dim = L, F, H, D
    lo.elem_bytes, lo.page_tokens, lo.wire_order = E, P, wire_order
    lo.num_pool_pages = num_pool_pages
    lo.wire_layer_stride = wire_layer_stride
    check(topkv_layout_default_strides(lo))
    return lo


def make_batch(block_table, seq_lens, total_tokens: int = -1, cu_seq_lens=None,
               flags: int = 0, window_tokens: int = 0) -> topkv_batch:
    """block_table: device int32 [R][maxp]; seq_lens: device int32 [R]. The descriptor keeps a
    reference to the tensors it was built from."""
    b = topkv_batch()
    b.struct_size = ctypes.sizeof(topkv_batch)
    b.num_requests = int(block_table.shape[0])
    b.max_pages_per_req = int(block_table.shape[1]) if block_table.ndim == 2 else 0
    b.block_table = _ptr(block_table)
    b.seq_lens = _ptr(seq_lens)
    b.cu_seq_lens = _ptr(cu_seq_lens)
    b.total_tokens = total_tokens
    b.flags = flags
    b.window_tokens = window_tokens
    # The struct only holds addresses: keep the tensors alive with it, so that a temporary
    # passed here cannot be freed (and its memory reused) while the descriptor is in use.
    b._keepalive = (block_table, seq_lens, cu_seq_lens)
    return b


# ---- the C entry points, same names, same order ---------------------------------------------

def topkv_pack_layer(layer, src_pool, layout, batch, d_wire, wire_capacity_bytes, stream=None):
    return lib().topkv_pack_layer(layer, _ptr(src_pool), ctypes.byref(layout), ctypes.byref(batch),
                                  _ptr(d_wire), wire_capacity_bytes, _stream(stream))


def topkv_unpack_layer(layer, dst_pool, layout, batch, d_wire, wire_bytes, stream=None):
    return lib().topkv_unpack_layer(layer, _ptr(dst_pool), ctypes.byref(layout),
                                    ctypes.byref(batch), _ptr(d_wire), wire_bytes, _stream(stream))


def topkv_pack_layers(first_layer, num_layers, src_pool, layout, batch, d_wire, wire_capacity_bytes,
                      stream=None):
    return lib().topkv_pack_layers(first_layer, num_layers, _ptr(src_pool), ctypes.byref(layout),
                                   ctypes.byref(batch), _ptr(d_wire), wire_capacity_bytes,
                                   _stream(stream))


def topkv_unpack_layers(first_layer, num_layers, dst_pool, layout, batch, d_wire, wire_bytes,
                        stream=None):
    return lib().topkv_unpack_layers(first_layer, num_layers, _ptr(dst_pool), ctypes.byref(layout),
                                     ctypes.byref(batch), _ptr(d_wire), wire_bytes, _stream(stream))


def topkv_copy_grid_ctas(layer, pool, layout, batch, d_wire, wire_bytes):
    """(CTAs per layer or a negative status, compact grid or not)."""
    compact = c_int32(0)
    n = lib().topkv_copy_grid_ctas(layer, _ptr(pool), ctypes.byref(layout), ctypes.byref(batch), _ptr(d_wire),
                                   wire_bytes, ctypes.byref(compact))
    return int(n), bool(compact.value)


def topkv_copy_vector_bytes(first_layer, num_layers, pool, layout, batch, d_wire, wire_bytes):
    return lib().topkv_copy_vector_bytes(first_layer, num_layers, _ptr(pool), ctypes.byref(layout),
                                         ctypes.byref(batch), _ptr(d_wire), wire_bytes)


def topkv_pack_layer_to_host(layer, src_pool, layout, batch, h_pinned, host_capacity_bytes,
                             d_staging, staging_capacity_bytes, stream=None):
    return lib().topkv_pack_layer_to_host(layer, _ptr(src_pool), ctypes.byref(layout),
                                          ctypes.byref(batch), _ptr(h_pinned), host_capacity_bytes,
                                          _ptr(d_staging), staging_capacity_bytes, _stream(stream))


def topkv_unpack_layer_from_host(layer, dst_pool, layout, batch, h_pinned, host_bytes, d_staging,
                                 staging_capacity_bytes, stream=None):
    return lib().topkv_unpack_layer_from_host(layer, _ptr(dst_pool), ctypes.byref(layout),
                                              ctypes.byref(batch), _ptr(h_pinned), host_bytes,
                                              _ptr(d_staging), staging_capacity_bytes,
                                              _stream(stream))


def _events(events, n):
    """torch.cuda.Event list (entries may be None) -> C array of cudaEvent_t, or None."""
    if events is None:
        return None
    assert len(events) == n
    arr = (c_void_p * n)()
    for i, e in enumerate(events):
        if e is None:
            continue
        if not e.cuda_event:
            # torch creates the CUDA event only at its first record(): give it a handle now
            # (recording on the current stream; the library's own record replaces it)
            e.record()
        arr[i] = e.cuda_event
    return arr


def topkv_pack_layers_to_host_pipelined(first_layer, num_layers, src_pool, layout, batch, h_pinned,
                                        host_capacity_bytes, d_staging, staging_capacity_bytes,
                                        layer_ready=None, layer_done=None, side_stream=None):
    return lib().topkv_pack_layers_to_host_pipelined(
        first_layer, num_layers, _ptr(src_pool), ctypes.byref(layout), ctypes.byref(batch),
        _ptr(h_pinned), host_capacity_bytes, _ptr(d_staging), staging_capacity_bytes,
        _events(layer_ready, num_layers), _events(layer_done, num_layers), _stream(side_stream))


def topkv_unpack_layers_from_host_pipelined(first_layer, num_layers, dst_pool, layout, batch, h_pinned,
                                            host_bytes, d_staging, staging_capacity_bytes,
                                            layer_ready=None, layer_done=None, side_stream=None):
    return lib().topkv_unpack_layers_from_host_pipelined(
        first_layer, num_layers, _ptr(dst_pool), ctypes.byref(layout), ctypes.byref(batch),
        _ptr(h_pinned), host_bytes, _ptr(d_staging), staging_capacity_bytes,
        _events(layer_ready, num_layers), _events(layer_done, num_layers), _stream(side_stream))


def topkv_span_link_words(layout, batch):
    return lib().topkv_span_link_words(ctypes.byref(layout), ctypes.byref(batch))


def topkv_pack_layer_linked(layer, src_pool, layout, batch, d_wire, wire_capacity_bytes, link,
                            stream=None):
    return lib().topkv_pack_layer_linked(layer, _ptr(src_pool), ctypes.byref(layout),
                                         ctypes.byref(batch), _ptr(d_wire), wire_capacity_bytes,
                                         ctypes.byref(link), _stream(stream))


def topkv_unpack_layer_linked(layer, dst_pool, layout, batch, d_wire, wire_bytes, link, stream=None):
    return lib().topkv_unpack_layer_linked(layer, _ptr(dst_pool), ctypes.byref(layout),
                                           ctypes.byref(batch), _ptr(d_wire), wire_bytes,
                                           ctypes.byref(link), _stream(stream))


def topkv_relay_layers_linked(first_layer, num_layers, src_pool, src_layout, src_batch, dst_pool,
                              dst_layout, dst_batch, d_slab, slab_bytes, d_flags, flags_words,
                              first_epoch, stream=None):
    return lib().topkv_relay_layers_linked(
        first_layer, num_layers, _ptr(src_pool), ctypes.byref(src_layout), ctypes.byref(src_batch),
        _ptr(dst_pool), ctypes.byref(dst_layout), ctypes.byref(dst_batch), _ptr(d_slab), slab_bytes,
        _ptr(d_flags), flags_words, first_epoch, _stream(stream))


def topkv_layer_table_offsets(layout, table, num_requests):
    """Returns (status, offsets) with offsets a numpy int64 [num_layers + 1]."""
    import numpy as np
    off = np.zeros(table.num_layers + 1, dtype=np.int64)
    st = lib().topkv_layer_table_offsets(ctypes.byref(layout), ctypes.byref(table), num_requests,
                                         off.ctypes.data)
    return st, off


def topkv_pack_model_layers(first_layer, num_layers, src_pool, layout, batch, table, d_wire,
                            wire_capacity_bytes, stream=None):
    return lib().topkv_pack_model_layers(first_layer, num_layers, _ptr(src_pool), ctypes.byref(layout),
                                         ctypes.byref(batch), ctypes.byref(table), _ptr(d_wire),
                                         wire_capacity_bytes, _stream(stream))


def topkv_unpack_model_layers(first_layer, num_layers, dst_pool, layout, batch, table, d_wire,
                              wire_bytes, stream=None):
    return lib().topkv_unpack_model_layers(first_layer, num_layers, _ptr(dst_pool), ctypes.byref(layout),
                                           ctypes.byref(batch), ctypes.byref(table), _ptr(d_wire),
                                           wire_bytes, _stream(stream))


def topkv_pack_model_layers_to_host_pipelined(first_layer, num_layers, src_pool, layout, batch, table,
                                              h_pinned, host_capacity_bytes, d_staging,
                                              staging_capacity_bytes, layer_ready=None, layer_done=None,
                                              side_stream=None):
    return lib().topkv_pack_model_layers_to_host_pipelined(
        first_layer, num_layers, _ptr(src_pool), ctypes.byref(layout), ctypes.byref(batch),
        ctypes.byref(table), _ptr(h_pinned), host_capacity_bytes, _ptr(d_staging), staging_capacity_bytes,
        _events(layer_ready, num_layers), _events(layer_done, num_layers), _stream(side_stream))


def topkv_unpack_model_layers_from_host_pipelined(first_layer, num_layers, dst_pool, layout, batch, table,
                                                  h_pinned, host_bytes, d_staging,
                                                  staging_capacity_bytes, layer_ready=None,
                                                  layer_done=None, side_stream=None):
    return lib().topkv_unpack_model_layers_from_host_pipelined(
        first_layer, num_layers, _ptr(dst_pool), ctypes.byref(layout), ctypes.byref(batch),
        ctypes.byref(table), _ptr(h_pinned), host_bytes, _ptr(d_staging), staging_capacity_bytes,
        _events(layer_ready, num_layers), _events(layer_done, num_layers), _stream(side_stream))


def _two(ptrs, conv):
    arr = (c_void_p * 2)()
    arr[0], arr[1] = conv(ptrs[0]), conv(ptrs[1])
    return arr


def topkv_pack_layers_to_host_two_lanes(first_layer, num_layers, src_pool, layout, batch, h_pinned,
                                        host_capacity_bytes, d_stagings, staging_capacity_bytes,
                                        layer_ready=None, layer_done=None, side_streams=None):
    """d_stagings and side_streams: sequences of two device slabs / two streams."""
    return lib().topkv_pack_layers_to_host_two_lanes(
        first_layer, num_layers, _ptr(src_pool), ctypes.byref(layout), ctypes.byref(batch),
        _ptr(h_pinned), host_capacity_bytes, _two(d_stagings, _ptr), staging_capacity_bytes,
        _events(layer_ready, num_layers), _events(layer_done, num_layers), _two(side_streams, _stream))


def topkv_unpack_layers_from_host_two_lanes(first_layer, num_layers, dst_pool, layout, batch, h_pinned,
                                            host_bytes, d_stagings, staging_capacity_bytes,
                                            layer_ready=None, layer_done=None, side_streams=None):
    return lib().topkv_unpack_layers_from_host_two_lanes(
        first_layer, num_layers, _ptr(dst_pool), ctypes.byref(layout), ctypes.byref(batch),
        _ptr(h_pinned), host_bytes, _two(d_stagings, _ptr), staging_capacity_bytes,
        _events(layer_ready, num_layers), _events(layer_done, num_layers), _two(side_streams, _stream))


def topkv_pack_layer_to_host_noalloc(layer, src_pool, layout, batch, h_pinned,
                                     host_capacity_bytes, stream=None):
    """Staged pack-to-host for callers that may not allocate device memory: the staging slab
    is the library's built-in TOPKV_NOALLOC_STAGING_BYTES array. One slab per device, shared by
    all calls; make the first call on a device outside stream capture."""
    return lib().topkv_pack_layer_to_host_noalloc(
        layer, _ptr(src_pool), ctypes.byref(layout), ctypes.byref(batch), _ptr(h_pinned),
        host_capacity_bytes, _stream(stream))


def topkv_repage_layer(layer, src_pool, src_layout, src_batch, dst_pool, dst_layout, dst_batch,
                       stream=None):
    return lib().topkv_repage_layer(layer, _ptr(src_pool), ctypes.byref(src_layout),
                                    ctypes.byref(src_batch), _ptr(dst_pool),
                                    ctypes.byref(dst_layout), ctypes.byref(dst_batch),
                                    _stream(stream))


def topkv_attend_workspace_bytes(layout, batch, attention):
    return lib().topkv_attend_workspace_bytes(ctypes.byref(layout), ctypes.byref(batch),
                                              ctypes.byref(attention))


def topkv_attend_layer(layer, pool, layout, batch, attention, d_q, d_out, d_workspace, workspace_bytes,
                       stream=None):
    return lib().topkv_attend_layer(layer, _ptr(pool), ctypes.byref(layout), ctypes.byref(batch),
                                    ctypes.byref(attention), _ptr(d_q), _ptr(d_out), _ptr(d_workspace),
                                    workspace_bytes, _stream(stream))


def topkv_page_workspace_bytes(layout, batch, num_forks=0):
    return lib().topkv_page_workspace_bytes(ctypes.byref(layout), ctypes.byref(batch), num_forks)


def topkv_extend_requests(layout, batch, tables, d_new_tokens, d_workspace, workspace_bytes, stream=None):
    return lib().topkv_extend_requests(ctypes.byref(layout), ctypes.byref(batch), ctypes.byref(tables),
                                       _ptr(d_new_tokens), _ptr(d_workspace), workspace_bytes,
                                       _stream(stream))


def topkv_fork_requests(pool, layout, batch, tables, d_parents, d_children, num_forks, d_workspace,
                        workspace_bytes, stream=None):
    return lib().topkv_fork_requests(_ptr(pool), ctypes.byref(layout), ctypes.byref(batch),
                                     ctypes.byref(tables), _ptr(d_parents), _ptr(d_children), num_forks,
                                     _ptr(d_workspace), workspace_bytes, _stream(stream))


def topkv_free_requests(layout, batch, tables, d_rows, num_rows, stream=None):
    return lib().topkv_free_requests(ctypes.byref(layout), ctypes.byref(batch), ctypes.byref(tables),
                                     _ptr(d_rows), num_rows, _stream(stream))


def topkv_compact_pages(pool, layout, batch, tables, d_num_used, d_page_map, d_workspace,
                        workspace_bytes, stream=None):
    return lib().topkv_compact_pages(_ptr(pool), ctypes.byref(layout), ctypes.byref(batch),
                                     ctypes.byref(tables), _ptr(d_num_used), _ptr(d_page_map),
                                     _ptr(d_workspace), workspace_bytes, _stream(stream))


def topkv_copy_pages(first_layer, num_layers, pool, layout, d_src_pages, d_dst_pages, num_pages,
                     stream=None):
    return lib().topkv_copy_pages(first_layer, num_layers, _ptr(pool), ctypes.byref(layout),
                                  _ptr(d_src_pages), _ptr(d_dst_pages), num_pages, _stream(stream))


def topkv_append_layer(layer, pool, layout, batch, tokens, d_k, d_v, d_q, d_q_out, stream=None):
    return lib().topkv_append_layer(layer, _ptr(pool), ctypes.byref(layout), ctypes.byref(batch), ctypes.byref(tokens),
                                    _ptr(d_k), _ptr(d_v), _ptr(d_q), _ptr(d_q_out), _stream(stream))


def topkv_rotary_frequencies(count, base, kind=TOPKV_STRETCH_NONE, factor=1.0, original_tokens=0.0, slow=0.0, fast=0.0):
    """numpy float64 [count / 2], radians a position."""
    import numpy as np
    s = topkv_rotary_stretch()
    s.struct_size = ctypes.sizeof(topkv_rotary_stretch)
    s.kind, s.base, s.factor, s.original_tokens, s.slow, s.fast = kind, base, factor, original_tokens, slow, fast
    f = np.zeros(count // 2, dtype=np.float64)
    check(lib().topkv_rotary_frequencies(ctypes.byref(s), count, f.ctypes.data))
    return f


def topkv_rotary_turns(frequencies):
    """numpy uint64, one per frequency (radians a position)."""
    import numpy as np
    f = np.ascontiguousarray(frequencies, dtype=np.float64)
    turns = np.zeros(f.size, dtype=np.uint64)
    check(lib().topkv_rotary_turns(f.ctypes.data, f.size, turns.ctypes.data))
    return turns


def topkv_plan_prefixes(layout, batch, min_tokens, d_plan, stream=None):
    return lib().topkv_plan_prefixes(ctypes.byref(layout), ctypes.byref(batch), min_tokens, _ptr(d_plan), _stream(stream))


def topkv_set_sharing_bytes(nbytes):
    return lib().topkv_set_sharing_bytes(nbytes)


def topkv_attend_shared_workspace_bytes(layout, batch, attention):
    return lib().topkv_attend_shared_workspace_bytes(ctypes.byref(layout), ctypes.byref(batch), ctypes.byref(attention))


def topkv_attend_shared_layer(layer, pool, layout, batch, attention, d_plan, d_q, d_out, d_workspace, workspace_bytes,
                              stream=None):
    return lib().topkv_attend_shared_layer(layer, _ptr(pool), ctypes.byref(layout), ctypes.byref(batch),
                                           ctypes.byref(attention), _ptr(d_plan), _ptr(d_q), _ptr(d_out),
                                           _ptr(d_workspace), workspace_bytes, _stream(stream))


def topkv_bound_pages_layer(layer, pool, layout, batch, cache_type, d_bounds, d_steps, stream=None):
    return lib().topkv_bound_pages_layer(layer, _ptr(pool), ctypes.byref(layout), ctypes.byref(batch), cache_type,
                                         _ptr(d_bounds), _ptr(d_steps), _stream(stream))


def topkv_page_choice_workspace_bytes(layout, batch, attention, choice):
    return lib().topkv_page_choice_workspace_bytes(ctypes.byref(layout), ctypes.byref(batch), ctypes.byref(attention),
                                                   ctypes.byref(choice))


def topkv_choose_pages_layer(layout, batch, attention, choice, d_q, d_workspace, workspace_bytes, stream=None):
    return lib().topkv_choose_pages_layer(ctypes.byref(layout), ctypes.byref(batch), ctypes.byref(attention),
                                          ctypes.byref(choice), _ptr(d_q), _ptr(d_workspace), workspace_bytes, _stream(stream))


def topkv_attend_pages_layer(layer, pool, layout, batch, attention, choice, d_q, d_out, d_workspace, workspace_bytes,
                             stream=None):
    return lib().topkv_attend_pages_layer(layer, _ptr(pool), ctypes.byref(layout), ctypes.byref(batch),
                                          ctypes.byref(attention), ctypes.byref(choice), _ptr(d_q), _ptr(d_out),
                                          _ptr(d_workspace), workspace_bytes, _stream(stream))


def topkv_header_fill(header, request_id, model_id, layout, seq_len, crc_k, crc_v):
    return lib().topkv_header_fill(ctypes.byref(header), request_id, model_id, ctypes.byref(layout),
                                   seq_len, crc_k, crc_v)


def topkv_header_check(header, layout, seq_len, crc_k, crc_v):
    return lib().topkv_header_check(ctypes.byref(header), ctypes.byref(layout), seq_len, crc_k,
                                    crc_v)


def topkv_crc64(h_data, nbytes=None):
    """Host CRC-64 of a bytes object or a numpy array."""
    if isinstance(h_data, (bytes, bytearray)):
        buf = (ctypes.c_char * len(h_data)).from_buffer_copy(h_data)
        return lib().topkv_crc64(ctypes.addressof(buf), len(h_data))
    return lib().topkv_crc64(_ptr(h_data), h_data.nbytes if nbytes is None else nbytes)


def topkv_crc_workspace_bytes(layout, num_requests, max_pages_per_req):
    return lib().topkv_crc_workspace_bytes(ctypes.byref(layout), num_requests, max_pages_per_req)


def topkv_crc_begin(layout, batch, d_workspace, workspace_bytes, stream=None):
    return lib().topkv_crc_begin(ctypes.byref(layout), ctypes.byref(batch), _ptr(d_workspace),
                                 workspace_bytes, _stream(stream))


def topkv_pack_layer_crc(layer, src_pool, layout, batch, d_wire, wire_capacity_bytes, d_workspace,
                         workspace_bytes, stream=None):
    return lib().topkv_pack_layer_crc(layer, _ptr(src_pool), ctypes.byref(layout),
                                      ctypes.byref(batch), _ptr(d_wire), wire_capacity_bytes,
                                      _ptr(d_workspace), workspace_bytes, _stream(stream))


def topkv_unpack_layer_crc(layer, dst_pool, layout, batch, d_wire, wire_bytes, d_workspace,
                           workspace_bytes, stream=None):
    return lib().topkv_unpack_layer_crc(layer, _ptr(dst_pool), ctypes.byref(layout),
                                        ctypes.byref(batch), _ptr(d_wire), wire_bytes,
                                        _ptr(d_workspace), workspace_bytes, _stream(stream))


def topkv_crc_finish(layout, batch, d_workspace, workspace_bytes, d_crc_out, stream=None):
    return lib().topkv_crc_finish(ctypes.byref(layout), ctypes.byref(batch), _ptr(d_workspace),
                                  workspace_bytes, _ptr(d_crc_out), _stream(stream))


def topkv_pack_layer_to_host_crc(layer, src_pool, layout, batch, h_pinned, host_capacity_bytes,
                                 d_staging, staging_capacity_bytes, d_workspace, workspace_bytes,
                                 stream=None):
    return lib().topkv_pack_layer_to_host_crc(
        layer, _ptr(src_pool), ctypes.byref(layout), ctypes.byref(batch), _ptr(h_pinned),
        host_capacity_bytes, _ptr(d_staging), staging_capacity_bytes, _ptr(d_workspace),
        workspace_bytes, _stream(stream))


def topkv_unpack_layer_from_host_crc(layer, dst_pool, layout, batch, h_pinned, host_bytes,
                                     d_staging, staging_capacity_bytes, d_workspace,
                                     workspace_bytes, stream=None):
    return lib().topkv_unpack_layer_from_host_crc(
        layer, _ptr(dst_pool), ctypes.byref(layout), ctypes.byref(batch), _ptr(h_pinned), host_bytes,
        _ptr(d_staging), staging_capacity_bytes, _ptr(d_workspace), workspace_bytes, _stream(stream))


def topkv_retry(attempt, retries=2, backoff_ms=100):
    """attempt: a Python callable returning a topkv status; §3.1's policy by default."""
    cb = RETRY_ATTEMPT(lambda _ctx: int(attempt()))
    return lib().topkv_retry(cb, None, retries, backoff_ms)


def topkv_build_plan(batch, d_cu_seq_lens, stream=None):
    return lib().topkv_build_plan(ctypes.byref(batch), _ptr(d_cu_seq_lens), _stream(stream))


def topkv_validate_batch_host(layout, num_requests, max_pages_per_req, h_block_table, h_seq_lens,
                              require_disjoint):
    return lib().topkv_validate_batch_host(ctypes.byref(layout), num_requests, max_pages_per_req,
                                           _ptr(h_block_table), _ptr(h_seq_lens),
                                           int(require_disjoint))


def topkv_layout_default_strides(layout):
    return lib().topkv_layout_default_strides(ctypes.byref(layout))


def topkv_wire_layer_bytes(layout, total_tokens):
    return lib().topkv_wire_layer_bytes(ctypes.byref(layout), total_tokens)


def topkv_kv_bytes(layout, seq_len):
    return lib().topkv_kv_bytes(ctypes.byref(layout), seq_len)


def topkv_kv_bytes_layered(layout, specs, seq_len):
    """specs: sequence of (kind, param) pairs, one per layer, or a ctypes array of
    topkv_layer_spec."""
    if not isinstance(specs, ctypes.Array):
        arr = (topkv_layer_spec * len(specs))()
        for i, (kind, param) in enumerate(specs):
            arr[i].kind, arr[i].param = kind, param
        specs = arr
    return lib().topkv_kv_bytes_layered(ctypes.byref(layout), ctypes.addressof(specs), seq_len)


def topkv_model_transfer_s(nbytes, bandwidth_bytes_per_s, setup_s=0.0):
    return lib().topkv_model_transfer_s(nbytes, bandwidth_bytes_per_s, setup_s)


def topkv_model_t_eff_s(t_last_s, t_xfer_s, t_rem_s):
    return lib().topkv_model_t_eff_s(t_last_s, t_xfer_s, t_rem_s)


def topkv_model_hidden_fraction(layers, t_layer_compute_s, t_xfer_total_s):
    return lib().topkv_model_hidden_fraction(layers, t_layer_compute_s, t_xfer_total_s)


def topkv_select_transport(source, target, cluster_has_rdma, override_mode=0):
    return lib().topkv_select_transport(ctypes.byref(source), ctypes.byref(target),
                                        int(bool(cluster_has_rdma)), override_mode)


def topkv_planning_rate(mode):
    return lib().topkv_planning_rate(mode)


def topkv_transport_name(mode):
    return lib().topkv_transport_name(mode).decode()


def topkv_strerror(status):
    return lib().topkv_strerror(status).decode()


def topkv_version():
    return lib().topkv_version()


def topkv_last_cuda_error():
    return lib().topkv_last_cuda_error()


def topkv_device_error_flags():
    return lib().topkv_device_error_flags()


def topkv_reset_device_error_flags():
    return lib().topkv_reset_device_error_flags()


def topkv_kernel_launch_count():
    return lib().topkv_kernel_launch_count()


def topkv_set_host_leg_ctas(ctas):
    return lib().topkv_set_host_leg_ctas(ctas)


def topkv_set_kernel_variant(variant):
    return lib().topkv_set_kernel_variant(variant)
