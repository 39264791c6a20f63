"""Thin ctypes binding of libkvtier.so (include/kvtier.h).

Argument marshalling only: every step of the path runs in the CUDA library.
PyTorch is used for device memory, pinned host memory and streams.  There is no
fallback: if the library cannot be loaded, loading raises.
"""
import ctypes as C
import os
import struct

import numpy as np

from . import build as _build

KV_OK = 0
KV_ERR_INVALID_ARG = -1
KV_ERR_UNSUPPORTED_VARIANT = -2
KV_ERR_K_TOO_LARGE = -3
KV_ERR_NO_FREE_SLOT = -4
KV_ERR_BAD_HOST_SLOT = -5
KV_ERR_HOST_TIER_TOO_SMALL = -6
KV_ERR_CUDA = -7
KV_ERR_INTERNAL = -8
KV_ERR_UNIMPLEMENTED = -9
KV_ERR_TAGS_EXHAUSTED = -10
KV_AUTO, KV_MHA, KV_GQA, KV_MQA, KV_MLA = -1, 0, 1, 2, 3
KV_STATE_FREE, KV_STATE_RESIDENT = 0, 1
KV_POLICY_BAYESIAN, KV_POLICY_EMA, KV_POLICY_LRU = 0, 1, 2
KV_NONE = 0xFFFFFFFF
KV_DEV_BAD_INDEX = 16
KV_DEV_BAD_HEAD_VALUE = 64
KV_DEV_BAD_SPAN_VALUE = 128
KV_DEV_BLOCK_NOT_RESIDENT = 256
KV_DTYPE_BF16, KV_DTYPE_F16 = 0, 1
KV_LOC_HOST = 0x80000000


class kv_model_desc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in
                ("variant", "n_layers", "n_q_heads", "n_kv_heads", "head_dim", "d_latent",
                 "d_rope", "dtype_bits")]


class kv_partition_desc(C.Structure):
    _fields_ = [("model", kv_model_desc), ("block_tokens", C.c_int32), ("reserved", C.c_int32),
                ("blocks_per_layer", C.c_int64), ("d_slab", C.c_void_p), ("h_ring", C.c_void_p),
                ("ring_slots", C.c_uint64), ("h_meta", C.c_void_p)]


class kv_pool_desc(C.Structure):
    _fields_ = [("n_partitions", C.c_int32), ("reserved", C.c_int32),
                ("part", kv_partition_desc * 4),
                ("d_ema", C.c_void_p), ("d_decay", C.c_void_p), ("d_touch", C.c_void_p),
                ("d_last_epoch", C.c_void_p), ("d_pair", C.c_void_p), ("d_state", C.c_void_p),
                ("d_tag", C.c_void_p), ("d_score", C.c_void_p),
                ("d_hits", C.c_void_p), ("d_misses", C.c_void_p), ("d_P", C.c_void_p),
                ("alpha0", C.c_float), ("beta0", C.c_float),
                ("d_loc", C.c_void_p), ("n_tags", C.c_uint64),
                ("d_staging", C.c_void_p * 4), ("staging_bytes", C.c_uint64),
                ("max_promote", C.c_uint64),
                ("d_workspace", C.c_void_p), ("workspace_bytes", C.c_uint64),
                ("h_workspace", C.c_void_p), ("h_workspace_bytes", C.c_uint64)]


class kv_stats(C.Structure):
    _fields_ = [(n, C.c_uint64) for n in
                ("epochs", "events", "victims", "promoted", "admitted", "bytes_demoted",
                 "bytes_promoted", "bytes_dropped", "n_entries", "n_free", "kernel_launches", "host_waits", "gathered")]


class kv_select_stats(C.Structure):
    _fields_ = [(n, C.c_uint64) for n in ("selections", "hint_hits", "hint_misses", "reread_ctas")]


class kv_timing(C.Structure):
    _fields_ = [("pack_ms", C.c_double), ("unpack_ms", C.c_double),
                ("pack_launches", C.c_uint64), ("unpack_launches", C.c_uint64),
                ("pack_bytes", C.c_uint64), ("unpack_bytes", C.c_uint64),
                ("gather_ms", C.c_double), ("gather_launches", C.c_uint64), ("gather_bytes", C.c_uint64)]


class kv_slot_meta(C.Structure):
    _fields_ = [("tag", C.c_uint32), ("last_epoch", C.c_uint32), ("ema", C.c_float),
                ("decay", C.c_float), ("pair", C.c_uint32), ("demote_epoch", C.c_uint32)]


class kv_rope_desc(C.Structure):
    _fields_ = [("rot_dim", C.c_int32), ("rot_first", C.c_int32), ("interleaved", C.c_int32), ("n_axes", C.c_int32),
                ("axis", C.c_uint8 * 128), ("d_inv_freq", C.c_void_p)]


_stride = C.c_int64 * 2


class kv_append_desc(C.Structure):
    _fields_ = [("partition", C.c_int32), ("layer", C.c_int32), ("dtype", C.c_int32), ("reserved", C.c_int32),
                ("n_tokens", C.c_uint64),
                ("d_k", C.c_void_p), ("k_stride", _stride), ("d_v", C.c_void_p), ("v_stride", _stride),
                ("d_q", C.c_void_p), ("q_stride", _stride), ("d_q_out", C.c_void_p), ("q_out_stride", _stride),
                ("d_table", C.c_void_p), ("n_rows", C.c_uint64), ("d_slot", C.c_void_p), ("d_pos", C.c_void_p),
                ("rope", kv_rope_desc)]


class kv_attend_desc(C.Structure):
    _fields_ = [("partition", C.c_int32), ("layer", C.c_int32), ("dtype", C.c_int32), ("scale", C.c_float),
                ("n_seqs", C.c_uint32), ("n_groups", C.c_uint32),
                ("max_suffix", C.c_uint32), ("max_prefix", C.c_uint32), ("max_members", C.c_uint32),
                ("reserved", C.c_uint32),
                ("d_q", C.c_void_p), ("q_stride", _stride), ("d_out", C.c_void_p), ("out_stride", _stride),
                ("d_lse", C.c_void_p), ("d_table", C.c_void_p), ("n_rows", C.c_uint64),
                ("d_suffix", C.c_void_p), ("d_prefix", C.c_void_p), ("d_group", C.c_void_p),
                ("d_weight", C.c_void_p), ("d_scratch", C.c_void_p), ("scratch_bytes", C.c_uint64)]


SLOT_META_DTYPE = np.dtype([("tag", "<u4"), ("last_epoch", "<u4"), ("ema", "<f4"),
                            ("decay", "<f4"), ("pair", "<u4"), ("demote_epoch", "<u4")])

EXPORTS = ("kv_size_bytes", "kv_infer_variant", "kv_entry_bytes", "kv_workspace_bytes",
           "kv_pool_create", "kv_pool_destroy", "kv_epoch_score", "kv_epoch_score_select", "kv_epoch_events", "kv_epoch_counts",
           "kv_epoch_update", "kv_set_policy", "kv_set_lazy_decay", "kv_hash_entries", "kv_dedup_table_slots", "kv_dedup_digests", "kv_set_confidence_blend", "kv_reuse_estimate", "kv_head_importance_update", "kv_set_head_multipliers", "kv_head_importance", "kv_head_weights", "kv_prefetch_window_update", "kv_set_prefetch_window", "kv_prefetch_span", "kv_prefetch_window", "kv_prefetch_list", "kv_select_victims", "kv_select_victim_blocks", "kv_select_victims_static", "kv_demote",
           "kv_promote", "kv_set_deferred_packing", "kv_flush", "kv_join_promotions", "kv_max_batch_bytes", "kv_admit", "kv_get_stats", "kv_ring_query",
           "kv_last_demote_counts", "kv_device_status", "kv_timing_enable", "kv_timing_read",
           "kv_set_select_variant", "kv_selection_stats", "kv_demote_counted", "kv_victim_counts", "kv_set_gather_threshold", "kv_set_l2_residency", "kv_last_cuda_error", "kv_status_string",
           "kv_append", "kv_attend", "kv_attend_scratch_bytes", "kv_attention_score",
           "kv_version")

_lib = None


def load():
    """Loads (building first if the source is newer) libkvtier.so."""
    global _lib
    if _lib is not None:
        return _lib
    path = _build.build()
    if not os.path.exists(path):
        raise RuntimeError("libkvtier.so is missing and could not be built")
    L = C.CDLL(path)
    vp, u64, i32, i64, u32 = C.c_void_p, C.c_uint64, C.c_int32, C.c_int64, C.c_uint32
    L.kv_size_bytes.restype = i64
    L.kv_size_bytes.argtypes = [C.POINTER(kv_model_desc), i64, i32]
    L.kv_infer_variant.restype = i32
    L.kv_infer_variant.argtypes = [C.POINTER(kv_model_desc)]
    L.kv_entry_bytes.restype = i64
    L.kv_entry_bytes.argtypes = [C.POINTER(kv_model_desc), i32]
    L.kv_workspace_bytes.restype = i32
    L.kv_workspace_bytes.argtypes = [C.POINTER(kv_pool_desc), C.POINTER(u64), C.POINTER(u64)]
    L.kv_pool_create.restype = i32
    L.kv_pool_create.argtypes = [C.POINTER(kv_pool_desc), vp, C.POINTER(vp)]
    L.kv_pool_destroy.restype = i32
    L.kv_pool_destroy.argtypes = [vp]
    L.kv_epoch_score.restype = i32
    L.kv_epoch_score.argtypes = [vp, u32, vp, vp, u64, vp]
    L.kv_epoch_score_select.restype = i32
    L.kv_epoch_score_select.argtypes = [vp, u32, vp, vp, u64, u64, vp, vp]
    L.kv_epoch_events.restype = i32
    L.kv_epoch_events.argtypes = [vp, vp, vp, u64, vp]
    L.kv_epoch_counts.restype = vp
    L.kv_epoch_counts.argtypes = [vp]
    L.kv_epoch_update.restype = i32
    L.kv_epoch_update.argtypes = [vp, u32, vp]
    L.kv_set_policy.restype = i32
    L.kv_set_policy.argtypes = [vp, i32]
    L.kv_set_lazy_decay.restype = i32
    L.kv_set_lazy_decay.argtypes = [vp, i32]
    L.kv_hash_entries.restype = i32
    L.kv_hash_entries.argtypes = [vp, vp, u64, vp, vp]
    L.kv_dedup_table_slots.restype = u64
    L.kv_dedup_table_slots.argtypes = [u64]
    L.kv_dedup_digests.restype = i32
    L.kv_dedup_digests.argtypes = [vp, u64, vp, vp, vp, u64, vp, vp, vp]
    L.kv_set_confidence_blend.restype = i32
    L.kv_set_confidence_blend.argtypes = [vp, C.c_float, i32, vp]
    L.kv_reuse_estimate.restype = vp
    L.kv_reuse_estimate.argtypes = [vp]
    L.kv_head_importance_update.restype = i32
    L.kv_head_importance_update.argtypes = [vp, i32, vp, C.c_float, vp]
    L.kv_set_head_multipliers.restype = i32
    L.kv_set_head_multipliers.argtypes = [vp, i32, vp, vp]
    L.kv_head_importance.restype = vp
    L.kv_head_importance.argtypes = [vp, i32]
    L.kv_head_weights.restype = vp
    L.kv_head_weights.argtypes = [vp, i32]
    L.kv_set_l2_residency.restype = i32
    L.kv_set_l2_residency.argtypes = [vp, C.c_uint64]
    L.kv_prefetch_window_update.restype = i32
    L.kv_prefetch_window_update.argtypes = [vp, i32, vp, C.c_float, vp]
    L.kv_set_prefetch_window.restype = i32
    L.kv_set_prefetch_window.argtypes = [vp, i32, C.c_float, C.c_uint32, vp]
    L.kv_prefetch_span.restype = vp
    L.kv_prefetch_span.argtypes = [vp, i32]
    L.kv_prefetch_window.restype = vp
    L.kv_prefetch_window.argtypes = [vp, i32]
    L.kv_prefetch_list.restype = i32
    L.kv_prefetch_list.argtypes = [vp, i32, vp, C.c_uint64, C.c_uint64, i32, vp, C.c_uint64, vp, vp]
    L.kv_select_victims.restype = i32
    L.kv_select_victims.argtypes = [vp, u64, vp, vp]
    L.kv_select_victim_blocks.restype = i32
    L.kv_select_victim_blocks.argtypes = [vp, u64, vp, C.POINTER(u64), vp]
    L.kv_select_victims_static.restype = i32
    L.kv_select_victims_static.argtypes = [vp, vp, u64, u64, vp, vp, vp]
    L.kv_demote.restype = i32
    L.kv_demote.argtypes = [vp, vp, u64, u64, vp, vp]
    L.kv_promote.restype = i32
    L.kv_promote.argtypes = [vp, i32, vp, u64, u64, vp, vp]
    L.kv_set_deferred_packing.restype = i32
    L.kv_set_deferred_packing.argtypes = [vp, i32]
    L.kv_flush.restype = i32
    L.kv_flush.argtypes = [vp]
    L.kv_join_promotions.restype = i32
    L.kv_join_promotions.argtypes = [vp, vp]
    L.kv_max_batch_bytes.restype = u64
    L.kv_max_batch_bytes.argtypes = [vp, i32]
    L.kv_admit.restype = i32
    L.kv_admit.argtypes = [vp, u32, C.c_float, vp, u64, i32, C.POINTER(u64), vp]
    L.kv_get_stats.restype = i32
    L.kv_get_stats.argtypes = [vp, C.POINTER(kv_stats)]
    L.kv_ring_query.restype = i32
    L.kv_ring_query.argtypes = [vp, i32, C.POINTER(u64), C.POINTER(u64), vp]
    L.kv_last_demote_counts.restype = i32
    L.kv_last_demote_counts.argtypes = [vp, C.POINTER(u64 * 4)]
    L.kv_device_status.restype = i32
    L.kv_device_status.argtypes = [vp, vp, C.POINTER(u32)]
    L.kv_timing_enable.restype = i32
    L.kv_timing_enable.argtypes = [vp, i32]
    L.kv_timing_read.restype = i32
    L.kv_timing_read.argtypes = [vp, C.POINTER(kv_timing)]
    L.kv_set_select_variant.restype = i32
    L.kv_set_select_variant.argtypes = [vp, i32]
    L.kv_demote_counted.restype = i32
    L.kv_demote_counted.argtypes = [vp, vp, u64, vp, u64, vp, vp]
    L.kv_victim_counts.restype = vp
    L.kv_victim_counts.argtypes = [vp]
    L.kv_set_gather_threshold.restype = i32
    L.kv_set_gather_threshold.argtypes = [vp, u64]
    L.kv_selection_stats.restype = i32
    L.kv_selection_stats.argtypes = [vp, vp, vp]
    L.kv_append.restype = i32
    L.kv_append.argtypes = [vp, C.c_char_p, vp]   # (a packed kv_append_desc)
    L.kv_attend.restype = i32
    L.kv_attend.argtypes = [vp, C.c_char_p, vp]   # (a packed kv_attend_desc)
    L.kv_attend_scratch_bytes.restype = u64
    L.kv_attend_scratch_bytes.argtypes = [vp, i32, u32, u32, u32, u32, u32, i32]
    L.kv_attention_score.restype = i32
    L.kv_attention_score.argtypes = [vp, u32, C.c_float, u32, vp, vp, vp]
    L.kv_last_cuda_error.restype = i32
    L.kv_last_cuda_error.argtypes = [vp]
    L.kv_status_string.restype = C.c_char_p
    L.kv_status_string.argtypes = [i32]
    L.kv_version.restype = C.c_char_p
    L.kv_version.argtypes = []
    _lib = L
    return L


class KVError(RuntimeError):
    def __init__(self, status, what):
        self.status = status
        super().__init__("%s: %s (%d)" % (what, load().kv_status_string(status).decode(), status))


def model_desc(p) -> kv_model_desc:
    """kv_model_desc from a workloads.Partition (or anything with those fields)."""
    return kv_model_desc(p.variant, p.n_layers, p.n_q_heads, p.n_kv_heads, p.head_dim, p.d_latent,
                         p.d_rope, p.dtype_bits)


def kv_size_bytes(model: kv_model_desc, n_tokens: int, per_layer: bool = True) -> int:
    return load().kv_size_bytes(C.byref(model), n_tokens, 1 if per_layer else 0)


def kv_infer_variant(model: kv_model_desc) -> int:
    return load().kv_infer_variant(C.byref(model))


def kv_entry_bytes(model: kv_model_desc, block_tokens: int) -> int:
    return load().kv_entry_bytes(C.byref(model), block_tokens)


def _stream_ptr(s):
    return s.cuda_stream if s is not None else 0   # (the argument types make it a pointer)


def kv_dedup_table_slots(m: int) -> int:
    return int(load().kv_dedup_table_slots(int(m)))


def kv_dedup_digests(d_digests, m, d_canon, d_refcount, d_table, d_n_unique, d_status, stream=None) -> int:
    """First position per digest and reference counts; arguments are torch device tensors."""
    return load().kv_dedup_digests(d_digests.data_ptr(), int(m), d_canon.data_ptr(), d_refcount.data_ptr(),
                                   d_table.data_ptr(), int(d_table.numel()),
                                   d_n_unique.data_ptr() if d_n_unique is not None else None,
                                   d_status.data_ptr(), _stream_ptr(stream) if stream is not None else None)


def kv_select_victims_static(d_score, d_state, n, k, d_victims, d_status=None, stream=None) -> int:
    """Selection with the library's built-in scratch: for callers that cannot
    allocate a workspace.  Arguments are torch device tensors; returns the status."""
    return load().kv_select_victims_static(
        d_score.data_ptr(), d_state.data_ptr(), int(n), int(k),
        d_victims.data_ptr() if d_victims is not None else None,
        d_status.data_ptr() if d_status is not None else None, _stream_ptr(stream))


# The descriptions of kv_append and kv_attend are packed in one go (a call is a few microseconds of them).
_APPEND = struct.Struct("@iiiiQ" + "Pqq" * 4 + "PQPP%ds" % C.sizeof(kv_rope_desc))
_ATTEND = struct.Struct("@iiifIIIIIIPqqPqqPPQPPPPPQ")
_NO_ROPE = bytes(C.sizeof(kv_rope_desc))
assert _APPEND.size == C.sizeof(kv_append_desc) and _ATTEND.size == C.sizeof(kv_attend_desc)
_I64, _I32, _F32 = ("torch.int64", "torch.uint64"), ("torch.int32", "torch.uint32"), ("torch.float32",)
_dtypes = {}


def _is(dtype, names):
    """Whether a torch dtype is one of those names (torch is only imported where a pool is made)."""
    k = _dtypes.get(dtype)
    if k is None:
        k = _dtypes[dtype] = str(dtype)
    return k in names


def _element(what, dtype):
    if _is(dtype, ("torch.bfloat16",)):
        return KV_DTYPE_BF16
    if _is(dtype, ("torch.float16",)):
        return KV_DTYPE_F16
    raise TypeError("%s: elements of %s" % (what, dtype))


def _array(what, t, names, size):
    if not _is(t.dtype, names):
        raise TypeError("%s: a tensor of %s where %s is wanted" % (what, t.dtype, " or ".join(names)))
    if not t.is_contiguous() or (size is not None and t.numel() != size):
        raise ValueError("%s: an array %s where %s contiguous elements are wanted" % (what, tuple(t.shape), size))


def _table_rows(what, t, layers, heads):
    shape = t.shape
    if not _is(t.dtype, _I32):
        raise TypeError("%s: a table of %s" % (what, t.dtype))
    if len(shape) != 3 or shape[1] != layers or shape[2] != heads or not t.is_contiguous():
        raise ValueError("%s: a table %s where a contiguous (rows, %d, %d) is wanted" % (what, tuple(shape), layers, heads))
    return shape[0]


def _heads(what, t, n, heads, dim, dtype):
    """(address, token stride, head stride) of a [n][heads][dim] tensor; zeros without one."""
    if t is None:
        return 0, 0, 0
    s = t.stride()
    if t.dtype != dtype or t.shape != (n, heads, dim) or (dim > 1 and s[2] != 1):
        raise ValueError("%s: %s %s where %s (%d, %d, %d) with contiguous rows is wanted" %
                         (what, t.dtype, tuple(t.shape), dtype, n, heads, dim))
    return t.data_ptr(), s[0], s[1]


class kv_rope:
    """Rotary positions for kv_append: kv_rope_desc and the tensor it points to.  axis: the axis of
    position each pair follows (an int for all of them)."""

    def __init__(self, rot_dim, axis, inv_freq, first=0, interleaved=False, n_axes=None):
        half = int(rot_dim) // 2
        axis = [int(axis)] * half if isinstance(axis, int) else [int(x) for x in axis]
        if len(axis) != half or half > 128 or (inv_freq.numel() if inv_freq is not None else 0) < half:
            raise ValueError("kv_rope: %d axes and %s frequencies for %d pairs" %
                             (len(axis), inv_freq.numel() if inv_freq is not None else "no", half))
        if inv_freq is not None:
            _array("kv_rope", inv_freq, _F32, None)
        self.inv_freq = inv_freq
        self.n_axes = int(n_axes if n_axes is not None else (max(axis) + 1 if axis else 0))
        self.desc = kv_rope_desc(int(rot_dim), int(first), int(bool(interleaved)), self.n_axes,
                                 (C.c_uint8 * 128)(*axis), inv_freq.data_ptr() if inv_freq is not None else None)
        self.packed = bytes(self.desc)


class Pool:
    """A pool whose memory is owned by torch tensors and whose every operation is
    one call into the C library.  `parts` is a list of workloads.Partition."""

    def __init__(self, parts, n_tags, alpha0=1.0, beta0=1.0, staging_bytes=64 << 20,
                 max_promote=None, host_meta=True, device="cuda:0", stream=None):
        import torch
        self.torch = torch
        self.lib = load()
        self.device = torch.device(device)
        self.parts = list(parts)
        self.N = sum(p.n_entries for p in self.parts)
        self.n_tags = int(n_tags)
        self.max_promote = int(max_promote if max_promote is not None else self.N)
        self.staging_bytes = int(staging_bytes)
        dev = self.device

        def dz(n, dt):
            return torch.empty(max(int(n), 4), dtype=dt, device=dev)

        N = self.N
        self.ema = dz(N, torch.float32)
        self.decay = dz(N, torch.float32)
        self.touch = dz(N, torch.int32)
        self.last_epoch = dz(N, torch.int32)
        self.pair = dz(N, torch.uint8)
        self.state = dz(N, torch.uint8)
        self.tag = dz(N, torch.int32)
        self.score = dz(N, torch.float32)
        self.hits = dz(16, torch.int64)
        self.misses = dz(16, torch.int64)
        self.P = dz(16, torch.float32)
        self.loc = dz(self.n_tags, torch.int32)
        self.staging = [torch.empty(self.staging_bytes, dtype=torch.uint8, device=dev) for _ in range(4)]
        self.slabs, self.rings, self.metas = [], [], []
        d = kv_pool_desc()
        d.n_partitions = len(self.parts)
        self.entry_bytes = []
        for q, p in enumerate(self.parts):
            # sizes come from the library's own sizing calls (Eq. "unified"), not from the workload
            m = model_desc(p)
            eb = kv_entry_bytes(m, p.block_tokens)
            per_block = kv_size_bytes(m, p.block_tokens, per_layer=True)
            if eb <= 0 or per_block <= 0:
                raise KVError(min(eb, per_block), "kv_entry_bytes / kv_size_bytes")
            self.entry_bytes.append(eb)
            slab = torch.empty(p.n_layers * p.blocks_per_layer * per_block, dtype=torch.uint8, device=dev)
            ring = torch.empty(max(p.ring_slots * eb, 16), dtype=torch.uint8, pin_memory=True)
            meta = (torch.zeros(max(p.ring_slots * 24, 16), dtype=torch.uint8, pin_memory=True)
                    if host_meta else None)
            self.slabs.append(slab)
            self.rings.append(ring)
            self.metas.append(meta)
            d.part[q] = kv_partition_desc(model_desc(p), p.block_tokens, 0, p.blocks_per_layer,
                                          slab.data_ptr(), ring.data_ptr(), p.ring_slots,
                                          meta.data_ptr() if meta is not None else None)
        d.d_ema, d.d_decay = self.ema.data_ptr(), self.decay.data_ptr()
        d.d_touch, d.d_last_epoch = self.touch.data_ptr(), self.last_epoch.data_ptr()
        d.d_pair, d.d_state = self.pair.data_ptr(), self.state.data_ptr()
        d.d_tag, d.d_score = self.tag.data_ptr(), self.score.data_ptr()
        d.d_hits, d.d_misses, d.d_P = self.hits.data_ptr(), self.misses.data_ptr(), self.P.data_ptr()
        d.alpha0, d.beta0 = alpha0, beta0
        d.d_loc, d.n_tags = self.loc.data_ptr(), self.n_tags
        for b in range(4):
            d.d_staging[b] = self.staging[b].data_ptr()
        d.staging_bytes = self.staging_bytes
        d.max_promote = self.max_promote
        dev_b, host_b = C.c_uint64(0), C.c_uint64(0)
        rc = self.lib.kv_workspace_bytes(C.byref(d), C.byref(dev_b), C.byref(host_b))
        if rc != KV_OK:
            raise KVError(rc, "kv_workspace_bytes")
        self.workspace = torch.empty(max(dev_b.value, 16), dtype=torch.uint8, device=dev)
        self.h_workspace = torch.empty(max(host_b.value, 16), dtype=torch.uint8, pin_memory=True)
        d.d_workspace, d.workspace_bytes = self.workspace.data_ptr(), dev_b.value
        d.h_workspace, d.h_workspace_bytes = self.h_workspace.data_ptr(), host_b.value
        self.desc = d
        self.compute = stream if stream is not None else torch.cuda.Stream(device=dev)
        self.copy = torch.cuda.Stream(device=dev)        # D2H copies of demotions
        self.copy_h2d = torch.cuda.Stream(device=dev)    # H2D copies of promotions (overlap the D2H ones)
        self._h = C.c_void_p()
        with torch.cuda.device(dev):
            rc = self.lib.kv_pool_create(C.byref(d), _stream_ptr(self.compute), C.byref(self._h))
        if rc != KV_OK:
            raise KVError(rc, "kv_pool_create")

    def close(self):
        if getattr(self, "_h", None):
            self.sync()
            self.lib.kv_pool_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def sync(self):
        self.compute.synchronize()
        self.copy.synchronize()
        self.copy_h2d.synchronize()

    # -- the five calls, plus the harness extras; each returns the status --------
    def kv_epoch_score(self, epoch, d_ev_entry, d_ev_hit, n_events=None):
        n = int(n_events if n_events is not None else (d_ev_entry.numel() if d_ev_entry is not None else 0))
        return self.lib.kv_epoch_score(self._h, epoch,
                                       d_ev_entry.data_ptr() if n else None,
                                       d_ev_hit.data_ptr() if n else None, n, _stream_ptr(self.compute))

    def kv_epoch_score_select(self, epoch, d_ev_entry, d_ev_hit, n_events, k, d_victims):
        n = int(n_events)
        return self.lib.kv_epoch_score_select(self._h, epoch,
                                              d_ev_entry.data_ptr() if n else None,
                                              d_ev_hit.data_ptr() if n else None, n, int(k),
                                              d_victims.data_ptr() if k else None,
                                              _stream_ptr(self.compute))

    def kv_epoch_events(self, d_ev_entry, d_ev_hit, n_events=None):
        n = int(n_events if n_events is not None else (d_ev_entry.numel() if d_ev_entry is not None else 0))
        return self.lib.kv_epoch_events(self._h, d_ev_entry.data_ptr() if n else None,
                                        d_ev_hit.data_ptr() if n else None, n, _stream_ptr(self.compute))

    def kv_epoch_counts(self):
        """The 32 epoch counters as an int64 tensor aliasing the library's device memory."""
        addr = self.lib.kv_epoch_counts(self._h)
        off = addr - self.workspace.data_ptr()
        return self.workspace[off:off + 256].view(self.torch.int64)

    def kv_epoch_update(self, epoch):
        return self.lib.kv_epoch_update(self._h, epoch, _stream_ptr(self.compute))

    def kv_set_policy(self, policy):
        return self.lib.kv_set_policy(self._h, int(policy))

    def kv_hash_entries(self, d_ids, m, d_digests):
        """SHA-256 of the images of entries d_ids[:m] (None: entries 0..m-1) into d_digests (uint8 [m, 32])."""
        return self.lib.kv_hash_entries(self._h, d_ids.data_ptr() if d_ids is not None else None, int(m),
                                        d_digests.data_ptr(), _stream_ptr(self.compute))

    def kv_set_lazy_decay(self, on=True):
        return self.lib.kv_set_lazy_decay(self._h, int(bool(on)))

    def kv_set_confidence_blend(self, kappa, window):
        return self.lib.kv_set_confidence_blend(self._h, float(kappa), int(window), _stream_ptr(self.compute))

    def kv_reuse_estimate(self):
        """The 16 reuse estimates as a float32 tensor aliasing the library's device memory."""
        off = self.lib.kv_reuse_estimate(self._h) - self.workspace.data_ptr()
        return self.workspace[off:off + 64].view(self.torch.float32)

    def kv_head_importance_update(self, q, d_x, decay):
        return self.lib.kv_head_importance_update(self._h, int(q), d_x.data_ptr(), float(decay),
                                                  _stream_ptr(self.compute))

    def kv_set_head_multipliers(self, q, d_mult):
        return self.lib.kv_set_head_multipliers(self._h, int(q), d_mult.data_ptr() if d_mult is not None else None,
                                                _stream_ptr(self.compute))

    def _head_view(self, ptr, n):
        off = ptr - self.workspace.data_ptr()
        return self.workspace[off:off + 4 * n].view(self.torch.float32)

    def kv_head_importance(self, q):
        """Partition q's [layers][query heads] importance matrix (float32 tensor aliasing device memory)."""
        p = self.parts[q]
        qh = 1 if p.variant == KV_MLA else p.n_q_heads
        return self._head_view(self.lib.kv_head_importance(self._h, int(q)), p.n_layers * qh)

    def kv_head_weights(self, q):
        """Partition q's [layers][KV heads] score weights."""
        p = self.parts[q]
        return self._head_view(self.lib.kv_head_weights(self._h, int(q)), p.n_layers * p.heads)

    def kv_prefetch_window_update(self, q, d_span, decay):
        return self.lib.kv_prefetch_window_update(self._h, int(q), d_span.data_ptr() if d_span is not None else None,
                                                  float(decay), _stream_ptr(self.compute))

    def kv_set_prefetch_window(self, q, tokens, max_blocks):
        return self.lib.kv_set_prefetch_window(self._h, int(q), float(tokens), int(max_blocks),
                                               _stream_ptr(self.compute))

    def kv_prefetch_span(self, q):
        """Partition q's per-layer attention-span EMA in tokens (float32 tensor aliasing device memory)."""
        return self._head_view(self.lib.kv_prefetch_span(self._h, int(q)), self.parts[q].n_layers)

    def kv_prefetch_window(self, q):
        """Partition q's per-layer prefetch window in blocks (int32 view of the device's uint32 values)."""
        off = self.lib.kv_prefetch_window(self._h, int(q)) - self.workspace.data_ptr()
        return self.workspace[off:off + 4 * self.parts[q].n_layers].view(self.torch.int32)

    def kv_prefetch_list(self, q, d_table, n_pos, pos0, direction, d_out_slots, max_out, d_out_count):
        return self.lib.kv_prefetch_list(self._h, int(q), d_table.data_ptr() if d_table is not None else None,
                                         int(n_pos), int(pos0), int(direction),
                                         d_out_slots.data_ptr() if d_out_slots is not None else None, int(max_out),
                                         d_out_count.data_ptr() if d_out_count is not None else None,
                                         _stream_ptr(self.compute))

    def _attention(self, q):
        """(layers, key heads, query heads, elements of a query or key head, of a value head) of a partition."""
        d = self.__dict__.setdefault("_attention_dims", {})
        if q not in d:
            p = self.parts[q]
            d[q] = ((p.n_layers, 1, p.n_q_heads, p.d_latent + p.d_rope, p.d_latent) if p.variant == KV_MLA
                    else (p.n_layers, p.heads, p.n_q_heads, p.head_dim, p.head_dim))
        return d[q]

    def kv_append(self, q, layer, d_k, d_v, d_table, d_slot, d_q=None, d_q_out=None, rope=None, d_pos=None, stream=None):
        """d_k, d_v, d_q, d_q_out: [tokens, heads, dim] (any strides but the last); d_slot int64 [tokens];
        d_pos int32 [axes, tokens]; rope: kv_rope."""
        what = "kv_append"
        layers, H, QH, dk, dv = self._attention(q)
        n, dt = d_slot.shape[0], d_k.dtype
        rows = _table_rows(what, d_table, layers, H)
        _array(what, d_slot, _I64, n)
        if d_pos is not None and rope is not None:
            _array(what, d_pos, _I32, rope.n_axes * n)
        elif d_pos is not None:
            _array(what, d_pos, _I32, None)
        desc = _APPEND.pack(q, layer, _element(what, dt), 0, n, *_heads(what, d_k, n, H, dk, dt), *_heads(what, d_v, n, H, dv, dt),
                            *_heads(what, d_q, n, QH, dk, dt), *_heads(what, d_q_out, n, QH, dk, dt), d_table.data_ptr(), rows,
                            d_slot.data_ptr(), d_pos.data_ptr() if d_pos is not None else 0,
                            rope.packed if rope is not None else _NO_ROPE)
        return self.lib.kv_append(self._h, desc, _stream_ptr(stream if stream is not None else self.compute))

    def kv_attend_scratch_bytes(self, q, n_seqs, n_groups=0, max_suffix=0, max_prefix=0, max_members=0, weights=False):
        return int(self.lib.kv_attend_scratch_bytes(self._h, int(q), int(n_seqs), int(n_groups), int(max_suffix),
                                                    int(max_prefix), int(max_members), int(bool(weights))))

    def kv_attend(self, q, layer, d_q, d_out, d_table, d_suffix, max_suffix, scale, d_scratch, d_prefix=None,
                  d_group=None, max_prefix=0, max_members=0, d_lse=None, d_weight=None, stream=None):
        """d_q, d_out: [sequences, query heads, dim]; d_suffix [sequences, 2], d_prefix [groups, 2] and d_group
        [groups + 1] int32; d_lse float32 [sequences, query heads]; d_weight int64 [n_tags]."""
        what = "kv_attend"
        layers, _, QH, dk, dv = self._attention(q)
        n, dt = d_q.shape[0], d_q.dtype
        rows = _table_rows(what, d_table, layers, _)
        _array(what, d_suffix, _I32, 2 * n)
        groups = 0
        if d_prefix is not None:
            groups = d_prefix.shape[0]
            _array(what, d_prefix, _I32, 2 * groups)
            if d_group is None:
                raise ValueError("kv_attend: %d prefixes without groups" % groups)
            _array(what, d_group, _I32, groups + 1)
        if d_lse is not None:
            _array(what, d_lse, _F32, n * QH)
        if d_weight is not None:
            _array(what, d_weight, _I64, None)
            if d_weight.numel() < self.n_tags:
                raise ValueError("kv_attend: weights of %d handles, where %d may be named" % (d_weight.numel(), self.n_tags))
        if not d_scratch.is_contiguous():
            raise ValueError("kv_attend: the scratch has to be contiguous")
        desc = _ATTEND.pack(q, layer, _element(what, dt), scale, n, groups, max_suffix, max_prefix, max_members, 0,
                            *_heads(what, d_q, n, QH, dk, dt), *_heads(what, d_out, n, QH, dv, dt),
                            d_lse.data_ptr() if d_lse is not None else 0, d_table.data_ptr(), rows, d_suffix.data_ptr(),
                            d_prefix.data_ptr() if d_prefix is not None else 0, d_group.data_ptr() if d_prefix is not None else 0,
                            d_weight.data_ptr() if d_weight is not None else 0, d_scratch.data_ptr(), d_scratch.nbytes)
        return self.lib.kv_attend(self._h, desc, _stream_ptr(stream if stream is not None else self.compute))

    def kv_attention_score(self, epoch, decay, protect, d_weight, d_acc):
        """d_weight int64 [n_tags] (cleared), d_acc float32 [n_tags]."""
        _array("kv_attention_score", d_weight, _I64, None)
        _array("kv_attention_score", d_acc, _F32, None)
        if d_weight.numel() < self.n_tags or d_acc.numel() < self.n_tags:
            raise ValueError("kv_attention_score: arrays of fewer than %d handles" % self.n_tags)
        return self.lib.kv_attention_score(self._h, epoch, decay, protect, d_weight.data_ptr(), d_acc.data_ptr(), _stream_ptr(self.compute))

    def kv_set_l2_residency(self, budget_bytes):
        return self.lib.kv_set_l2_residency(self._h, int(budget_bytes))

    def kv_select_victims(self, k, d_victims):
        return self.lib.kv_select_victims(self._h, int(k), d_victims.data_ptr() if k else None,
                                          _stream_ptr(self.compute))

    def kv_select_victim_blocks(self, k_blocks, d_victims, wait=True):
        """Returns (status, number of entries written).  wait=False passes no place for the
        number: the call then never blocks, and the entries per partition are in
        kv_victim_counts() once the compute stream has run (the number returned is 0)."""
        n = C.c_uint64(0)
        rc = self.lib.kv_select_victim_blocks(self._h, int(k_blocks), d_victims.data_ptr() if k_blocks else None,
                                              C.byref(n) if wait else None, _stream_ptr(self.compute))
        return rc, n.value

    def kv_demote(self, d_victims, m, batch_bytes):
        return self.lib.kv_demote(self._h, d_victims.data_ptr() if m else None, int(m), int(batch_bytes),
                                  _stream_ptr(self.compute), _stream_ptr(self.copy))

    def kv_demote_counted(self, d_victims, m, counts, batch_bytes):
        c = (C.c_uint64 * 4)(*([int(x) for x in counts] + [0] * (4 - len(counts))))
        return self.lib.kv_demote_counted(self._h, d_victims.data_ptr() if m else None, int(m), C.byref(c),
                                          int(batch_bytes), _stream_ptr(self.compute), _stream_ptr(self.copy))

    def kv_victim_counts(self):
        """Victims per partition of the last selection (read after synchronising the compute stream)."""
        addr = self.lib.kv_victim_counts(self._h)
        return [int(x) for x in (C.c_uint64 * 4).from_address(addr)][:len(self.parts)]

    def kv_promote(self, partition, h_slots, batch_bytes):
        h_slots = np.ascontiguousarray(h_slots, dtype=np.uint64)
        return self.lib.kv_promote(self._h, partition, h_slots.ctypes.data if h_slots.size else None, h_slots.size, int(batch_bytes), _stream_ptr(self.compute),
                                   _stream_ptr(self.copy_h2d))

    def kv_admit(self, epoch, decay, d_new_pairs, fill_pattern=True):
        n = C.c_uint64(0)
        rc = self.lib.kv_admit(self._h, epoch, decay, d_new_pairs.data_ptr(), d_new_pairs.numel(),
                               1 if fill_pattern else 0, C.byref(n), _stream_ptr(self.compute))
        return rc, n.value

    def kv_set_gather_threshold(self, run_bytes):
        return self.lib.kv_set_gather_threshold(self._h, int(run_bytes))

    def kv_set_deferred_packing(self, on=True):
        return self.lib.kv_set_deferred_packing(self._h, 1 if on else 0)

    def kv_flush(self):
        return self.lib.kv_flush(self._h)

    def kv_join_promotions(self, stream=None):
        return self.lib.kv_join_promotions(self._h, _stream_ptr(stream if stream is not None else self.compute))

    def kv_max_batch_bytes(self, partition=0):
        return int(self.lib.kv_max_batch_bytes(self._h, partition))

    def kv_get_stats(self):
        s = kv_stats()
        rc = self.lib.kv_get_stats(self._h, C.byref(s))
        if rc != KV_OK:
            raise KVError(rc, "kv_get_stats")
        return {n: int(getattr(s, n)) for n, _ in kv_stats._fields_}

    def kv_ring_query(self, partition, want_live=True):
        cur, nl = C.c_uint64(0), C.c_uint64(0)
        live = np.zeros(self.parts[partition].ring_slots, dtype=np.uint8) if want_live else None
        rc = self.lib.kv_ring_query(self._h, partition, C.byref(cur), C.byref(nl),
                                    live.ctypes.data_as(C.c_void_p) if live is not None and live.size else None)
        if rc != KV_OK:
            raise KVError(rc, "kv_ring_query")
        return cur.value, nl.value, live

    def kv_last_demote_counts(self):
        c = (C.c_uint64 * 4)()
        self.lib.kv_last_demote_counts(self._h, C.byref(c))
        return [int(x) for x in c]

    def kv_device_status(self):
        bits = C.c_uint32(0)
        rc = self.lib.kv_device_status(self._h, _stream_ptr(self.compute), C.byref(bits))
        if rc != KV_OK:
            raise KVError(rc, "kv_device_status")
        return bits.value

    def kv_set_select_variant(self, variant):
        return self.lib.kv_set_select_variant(self._h, int(variant))

    def kv_selection_stats(self):
        s = kv_select_stats()
        rc = self.lib.kv_selection_stats(self._h, _stream_ptr(self.compute), C.byref(s))
        if rc != KV_OK:
            raise KVError(rc, "kv_selection_stats")
        return {n: int(getattr(s, n)) for n, _ in kv_select_stats._fields_}

    def kv_timing_enable(self, on=True):
        return self.lib.kv_timing_enable(self._h, 1 if on else 0)

    def kv_timing_read(self):
        t = kv_timing()
        rc = self.lib.kv_timing_read(self._h, C.byref(t))
        if rc != KV_OK:
            raise KVError(rc, "kv_timing_read")
        return {n: getattr(t, n) for n, _ in kv_timing._fields_}

    def ring_meta(self, partition):
        """numpy view of the pinned per-slot metadata mirror (after sync)."""
        return self.metas[partition].numpy().view(SLOT_META_DTYPE)[: self.parts[partition].ring_slots]
