"""ctypes binding of libptstore.so: same names as the C ABI, argument marshalling only.

torch is used for device memory and streams; every step of the path runs in the library's kernels.
Importing this module loads the library and raises if it has not been built (there is no fallback).
"""
import ctypes as C
import os
import struct

import torch

from . import build as _build

OK, E_INVAL, E_CUDA, E_NOMEM, E_LIMIT = 0, -1, -2, -3, -4
S_NOSPACE, S_TABLE_FULL, S_BOUNDS, S_STATE, S_TIMEOUT, S_INFLIGHT = 1, 2, 4, 8, 16, 32
PIN, NO_TOUCH = 1, 2
PINNED_LIST = 1
ASYNC_COPY = 1
COPY_BULK, COPY_VECTOR = 0, 1
EVICT_GDSF = 2
TIER_HBM, TIER_HOST = 0, 1


def lookup_lanes(n):
    return (n & 0xFF) << 8


def copy_variant(v):
    return (v & 0xF) << 16


def copy_ctas_per_sm(c):
    return (c & 0xFF) << 20


class Config(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("flags", C.c_uint32),
                ("num_layers", C.c_uint32), ("num_kv_heads", C.c_uint32), ("head_dim", C.c_uint32),
                ("elem_bytes", C.c_uint32), ("block_tokens", C.c_uint32), ("max_requests", C.c_uint32),
                ("max_batch_blocks", C.c_uint64), ("salt", C.c_uint64),
                ("hbm_pool", C.c_void_p), ("host_pool", C.c_void_p),
                ("hbm_blocks", C.c_uint32), ("host_blocks", C.c_uint32),
                ("table_slots", C.c_uint64), ("workspace", C.c_void_p), ("workspace_bytes", C.c_uint64),
                ("device", C.c_int32), ("reserved", C.c_int32)]


class PagedCache(C.Structure):
    _fields_ = [("layer_base", C.c_void_p), ("kv_stride_bytes", C.c_uint64), ("block_stride_bytes", C.c_uint64),
                ("num_blocks", C.c_uint32), ("reserved", C.c_uint32)]


class Stats(C.Structure):
    _fields_ = [("epoch", C.c_uint64), ("live_nodes", C.c_uint64 * 2), ("free_blocks", C.c_uint64 * 2),
                ("max_displacement", C.c_uint64), ("query_blocks", C.c_uint64), ("probes_issued", C.c_uint64),
                ("slots_visited", C.c_uint64), ("blocks_matched", C.c_uint64), ("blocks_fetched", C.c_uint64 * 2),
                ("blocks_inserted", C.c_uint64), ("blocks_denied", C.c_uint64), ("blocks_dropped", C.c_uint64 * 2),
                ("blocks_demoted", C.c_uint64), ("far_keys", C.c_uint64), ("blocks_promoted", C.c_uint64), ("gdsf_clock", C.c_uint64), ("blocks_fetched_distinct", C.c_uint64)]


KV_BF16, KV_FP16, KV_PACKED, KV_LATENT_BF16, KV_LATENT_FP16 = 0, 1, 2, 4, 5
LATENT_ROPE = 64


class KvCache(C.Structure):
    _fields_ = [("base", C.c_void_p), ("kv_stride_bytes", C.c_uint64), ("block_stride_bytes", C.c_uint64),
                ("num_blocks", C.c_uint32), ("block_tokens", C.c_uint32), ("num_kv_heads", C.c_uint32), ("head_dim", C.c_uint32),
                ("format", C.c_uint32), ("reserved", C.c_uint32), ("k_scale", C.c_float), ("v_scale", C.c_float)]


class Attend(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("dtype", C.c_uint32), ("q", C.c_void_p), ("q_token_stride", C.c_int64), ("q_head_stride", C.c_int64),
                ("out", C.c_void_p), ("out_token_stride", C.c_int64), ("out_head_stride", C.c_int64), ("token_offsets", C.c_void_p),
                ("lengths", C.c_void_p), ("block_tables", C.c_void_p), ("requests", C.c_int32), ("max_blocks", C.c_int32), ("num_heads", C.c_int32),
                ("tokens", C.c_int32), ("max_new", C.c_int32), ("scale", C.c_float), ("wait_polls", C.c_uint32), ("reserved", C.c_uint32)]


class LatentAttend(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("wait_polls", C.c_uint32), ("q_latent", C.c_void_p), ("q_latent_token_stride", C.c_int64),
                ("q_latent_head_stride", C.c_int64), ("q_rope", C.c_void_p), ("q_rope_token_stride", C.c_int64), ("q_rope_head_stride", C.c_int64),
                ("out", C.c_void_p), ("out_token_stride", C.c_int64), ("out_head_stride", C.c_int64), ("lse", C.c_void_p), ("token_offsets", C.c_void_p),
                ("lengths", C.c_void_p), ("block_tables", C.c_void_p), ("requests", C.c_int32), ("max_blocks", C.c_int32), ("num_heads", C.c_int32),
                ("tokens", C.c_int32), ("max_new", C.c_int32), ("scale", C.c_float)]


class ExpandedAttend(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("dtype", C.c_uint32), ("q", C.c_void_p), ("q_token_stride", C.c_int64), ("q_head_stride", C.c_int64),
                ("k", C.c_void_p), ("k_token_stride", C.c_int64), ("k_head_stride", C.c_int64), ("k_rope", C.c_void_p), ("k_rope_token_stride", C.c_int64),
                ("v", C.c_void_p), ("v_token_stride", C.c_int64), ("v_head_stride", C.c_int64), ("out", C.c_void_p), ("out_token_stride", C.c_int64),
                ("out_head_stride", C.c_int64), ("token_offsets", C.c_void_p), ("key_offsets", C.c_void_p), ("requests", C.c_int32), ("heads", C.c_int32),
                ("tokens", C.c_int32), ("keys", C.c_int32), ("max_new", C.c_int32), ("scale", C.c_float), ("wait_polls", C.c_uint32), ("reserved", C.c_uint32)]


class AttendWeights(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("dtype", C.c_uint32), ("q", C.c_void_p), ("q_token_stride", C.c_int64), ("q_head_stride", C.c_int64),
                ("lse", C.c_void_p), ("token_offsets", C.c_void_p), ("lengths", C.c_void_p), ("block_tables", C.c_void_p), ("requests", C.c_int32),
                ("max_blocks", C.c_int32), ("num_heads", C.c_int32), ("tokens", C.c_int32), ("weights", C.c_void_p), ("weights_request_stride", C.c_int64),
                ("weights_head_stride", C.c_int64), ("width", C.c_int32), ("max_new", C.c_int32), ("accumulate", C.c_uint32), ("scale", C.c_float),
                ("wait_polls", C.c_uint32), ("reserved", C.c_uint32)]


EXPORTS = ["ptstore_workspace_bytes", "ptstore_create", "ptstore_destroy", "ptstore_hash", "ptstore_lookup",
           "ptstore_fetch", "ptstore_insert", "ptstore_release", "ptstore_evict", "ptstore_status", "ptstore_stats",
           "ptstore_launch_count", "ptstore_last_cuda_error", "ptstore_strerror", "ptstore_fetch_static", "ptstore_promote", "ptstore_evict_async", "ptstore_join", "ptstore_stats_enqueue", "ptstore_lookup_fetch",
           "ptstore_reserve", "ptstore_set_wait_limit", "ptstore_time_next_copy", "ptstore_copy_probe",
           "ptstore_insert_after_lookup", "ptstore_resumed_inserts", "ptstore_kv_chunk_bytes", "ptstore_assign_blocks", "ptstore_map_slots",
           "ptstore_kv_write", "ptstore_kv_read", "ptstore_attend_workspace_bytes", "ptstore_attend",
           "ptstore_latent_write", "ptstore_latent_read", "ptstore_latent_workspace_bytes", "ptstore_latent_attend",
           "ptstore_expanded_attend", "ptstore_attend_lse", "ptstore_attend_weights", "ptstore_select_tokens", "ptstore_kv_compact"]


def _load():
    path = _build.LIB
    if not os.path.exists(path):
        raise ImportError("libptstore.so is not built: run paper_2607_22648_b200/build.py (needs nvcc)")
    lib = C.CDLL(path)
    vp, i32, u32, u64 = C.c_void_p, C.c_int32, C.c_uint32, C.c_uint64
    lib.ptstore_workspace_bytes.restype = u64
    lib.ptstore_workspace_bytes.argtypes = [C.POINTER(Config)]
    lib.ptstore_create.argtypes = [C.POINTER(Config), C.POINTER(vp), vp]
    lib.ptstore_destroy.argtypes = [vp]
    lib.ptstore_hash.argtypes = [vp, vp, vp, i32, i32, vp, vp]
    lib.ptstore_lookup.argtypes = [vp, vp, vp, i32, i32, u32, vp, vp, vp]
    lib.ptstore_fetch.argtypes = [vp, vp, vp, i32, i32, C.POINTER(PagedCache), vp, vp]
    lib.ptstore_lookup_fetch.argtypes = [vp, vp, vp, i32, i32, u32, C.POINTER(PagedCache), vp, vp, vp, vp]
    lib.ptstore_reserve.argtypes = [vp, C.c_int64, i32, vp, i32, u32, vp, vp, i32, vp]
    lib.ptstore_set_wait_limit.argtypes = [vp, u32]
    lib.ptstore_time_next_copy.argtypes = [vp, vp, vp]
    lib.ptstore_copy_probe.argtypes = [vp, vp, u64, i32, u32, i32, u32, i32, i32, vp, vp]
    lib.ptstore_insert.argtypes = [vp, vp, vp, i32, i32, C.POINTER(PagedCache), vp, vp, vp, vp]
    lib.ptstore_insert_after_lookup.argtypes = [vp, vp, vp, i32, i32, C.POINTER(PagedCache), vp, vp, vp, vp]
    lib.ptstore_resumed_inserts.restype = u64
    lib.ptstore_resumed_inserts.argtypes = [vp]
    lib.ptstore_release.argtypes = [vp, vp, vp, i32, i32, vp]
    lib.ptstore_evict.argtypes = [vp, i32, i32, vp, vp, vp]
    lib.ptstore_evict_async.argtypes = [vp, i32, i32, vp, vp, vp]
    lib.ptstore_join.argtypes = [vp, vp]
    lib.ptstore_promote.argtypes = [vp, vp, vp, i32, i32, u32, i32, vp, vp]
    lib.ptstore_status.argtypes = [vp, vp, C.POINTER(u32)]
    lib.ptstore_stats.argtypes = [vp, vp, C.POINTER(Stats)]
    lib.ptstore_stats_enqueue.argtypes = [vp, vp, vp]
    lib.ptstore_launch_count.restype = u64
    lib.ptstore_launch_count.argtypes = [vp]
    lib.ptstore_last_cuda_error.argtypes = [vp]
    lib.ptstore_fetch_static.argtypes = [vp, u32, u32, u64, vp, vp, i32, i32, C.POINTER(PagedCache), vp, vp, vp]
    i64 = C.c_int64
    lib.ptstore_kv_chunk_bytes.restype = u64
    lib.ptstore_kv_chunk_bytes.argtypes = [u32, u32, u32, u32]
    lib.ptstore_assign_blocks.argtypes = [vp, vp, i32, i32, vp, i32, vp, i32, vp, vp, vp, vp, vp]
    lib.ptstore_map_slots.argtypes = [vp, vp, i32, i32, i32, vp, i32, i32, i64, vp, vp, vp, vp, vp]
    lib.ptstore_kv_write.argtypes = [vp, i64, i64, vp, i64, i64, i64, u32, vp, vp, vp, vp]
    lib.ptstore_kv_read.argtypes = [vp, vp, i64, u32, vp, i64, i64, vp, i64, i64, vp, vp]
    lib.ptstore_attend_workspace_bytes.restype = u64
    lib.ptstore_attend_workspace_bytes.argtypes = [u32]
    lib.ptstore_attend.argtypes = [vp, vp, vp, u64, vp, vp]
    lib.ptstore_latent_write.argtypes = [vp, i64, vp, i64, i64, vp, vp, vp, vp]
    lib.ptstore_latent_read.argtypes = [vp, vp, i64, vp, i64, vp, i64, vp, vp]
    lib.ptstore_latent_workspace_bytes.restype = u64
    lib.ptstore_latent_workspace_bytes.argtypes = [u32]
    lib.ptstore_latent_attend.argtypes = [vp, vp, vp, u64, vp, vp]
    lib.ptstore_expanded_attend.argtypes = [vp, vp, vp]
    lib.ptstore_attend_lse.argtypes = [vp, vp, vp, u64, vp, vp, vp]
    lib.ptstore_attend_weights.argtypes = [vp, vp, vp, vp]
    lib.ptstore_select_tokens.argtypes = [vp, i64, i64, vp, i32, i32, i32, i32, i32, i32, vp, vp, vp, i64, i64, vp, vp]
    lib.ptstore_kv_compact.argtypes = [vp, vp, vp, i32, i32, vp, i32, vp, i32, vp, vp]
    lib.ptstore_strerror.restype = C.c_char_p
    lib.ptstore_strerror.argtypes = [C.c_int]
    return lib


lib = _load()


class PTStoreError(RuntimeError):
    def __init__(self, code, what):
        super().__init__("%s: %s (%d)" % (what, lib.ptstore_strerror(code).decode(), code))
        self.code = code


def _ptr(t):
    return t.data_ptr() if t is not None else None


def _stream():
    return torch.cuda.current_stream().cuda_stream


class PagedKV:
    """A vLLM-style paged cache: one uint8 tensor [2, num_blocks, chunk_bytes] per layer, plus the
    device array of layer pointers the library wants."""

    def __init__(self, layers, num_blocks, chunk_bytes, device="cuda", tensors=None):
        self.tensors = tensors if tensors is not None else [
            torch.empty((2, num_blocks, chunk_bytes), dtype=torch.uint8, device=device) for _ in range(layers)]
        self.num_blocks = num_blocks
        self.ptrs = torch.tensor([t.data_ptr() for t in self.tensors], dtype=torch.int64, device=device)
        t0 = self.tensors[0]
        self.desc = PagedCache(self.ptrs.data_ptr(), t0.stride(0) * t0.element_size(), t0.stride(1) * t0.element_size(),
                               num_blocks, 0)


PROBE_READ, PROBE_WRITE, PROBE_COPY, PROBE_MIX = 0, 1, 2, 3


def copy_probe(src, dst, nbytes, mode, writes_x100=100, stages=3, stage_bytes=32768, ctas_per_sm=1, scatter=True, status=None):
    """ptstore_copy_probe: one launch of the bulk copy ring over plain buffers (uint8 device tensors) in one traffic pattern."""
    if status is None:
        status = torch.zeros(1, dtype=torch.int32, device=src.device)
    rc = lib.ptstore_copy_probe(_ptr(src), _ptr(dst), nbytes, mode, writes_x100, stages, stage_bytes, ctas_per_sm, 1 if scatter else 0,
                                _ptr(status), _stream())
    if rc:
        raise PTStoreError(rc, "ptstore_copy_probe")
    return status


STATIC_MAX_REQUESTS, STATIC_MAX_PAIRS = 1024, 65536


def fetch_static(hbm_pool, hbm_blocks, layers, chunk_bytes, ids, matched, cache, block_tables, status_out=None):
    """ptstore_fetch_static: the gather for callers that may not allocate device memory.  Needs no store
    handle; scratch is a fixed array inside the library (limits STATIC_MAX_REQUESTS / STATIC_MAX_PAIRS).
    Calls that overlap on the GPU race on that array; the first call per device should precede any stream
    capture.  Raises PTStoreError on a refused call."""
    R, mb = ids.shape
    rc = lib.ptstore_fetch_static(_ptr(hbm_pool), hbm_blocks, layers, chunk_bytes, _ptr(ids), _ptr(matched), R, mb,
                                  C.byref(cache.desc), _ptr(block_tables), _ptr(status_out), _stream())
    if rc:
        raise PTStoreError(rc, "ptstore_fetch_static")


# ---- operators around the paged cache: no store handle, work on the stream and device that are current -------------------------------
# A decode step calls these once per layer with kernels of ten microseconds, so the checks are written out flat and the C structs
# are packed as bytes.
_KV_DTYPES = {torch.bfloat16: KV_BF16, torch.float16: KV_FP16}
_KV_CACHE = struct.Struct("PQQIIIIIIff")
_ATTEND = struct.Struct("IIPqqPqqPPPiiiiifII")
_LATENT_ATTEND = struct.Struct("IIPqqPqqPqqPPPPiiiiif")
_EXPANDED_ATTEND = struct.Struct("IIPqqPqqPqPqqPqqPPiiiiifII")
assert _EXPANDED_ATTEND.size == C.sizeof(ExpandedAttend)
_ATTEND_WEIGHTS = struct.Struct("IIPqqPPPPiiiiPqqiiIfII")
assert _ATTEND_WEIGHTS.size == C.sizeof(AttendWeights)
assert _LATENT_ATTEND.size == C.sizeof(LatentAttend)
assert _KV_CACHE.size == C.sizeof(KvCache) and _ATTEND.size == C.sizeof(Attend)
_ATTEND_SIZE = C.sizeof(Attend)
_raw_stream = torch._C._cuda_getCurrentRawStream
_device = torch.cuda.current_device


def _check(rc, what):
    if rc:
        raise PTStoreError(rc, what)


def _vec(t, dtype, n, dev, what):
    """n contiguous elements on the current device, or pinned; returns their address."""
    if t.dtype is not dtype or t.numel() != n or not t.is_contiguous():
        raise ValueError("%s: needs a contiguous %s vector of %d elements" % (what, dtype, n))
    if t.get_device() != dev:
        _elsewhere(t, what)
    return t.data_ptr()


def _table(t, R, dev, what):
    if t.dtype is not torch.int32 or t.dim() != 2 or t.shape[0] != R or not t.is_contiguous():
        raise ValueError("%s: needs a contiguous int32 tensor of %d rows" % (what, R))
    if t.get_device() != dev:
        _elsewhere(t, what)
    return t.data_ptr()


def _elsewhere(t, what):
    if t.is_cuda:
        raise ValueError("%s: is on another device than the current one" % what)
    if not t.is_pinned():
        raise ValueError("%s: needs device or pinned memory" % what)


def _on_device(t, dev, what):
    """What kernels fetch by bulk copies and tensor maps lies in device memory."""
    if t.get_device() != dev:
        raise ValueError("%s: needs memory of the current device" % what)


def _rows(t, heads, dim, n, dtype, dev, what):
    """[n][heads][dim] rows of 16-bit elements, any token and head strides; returns the address."""
    if t.dtype is not dtype or t.shape != (n, heads, dim) or t.stride(2) != 1:
        raise ValueError("%s: needs a %s tensor [%d, %d, %d], contiguous along the last axis" % (what, dtype, n, heads, dim))
    if t.get_device() != dev:
        _elsewhere(t, what)
    return t.data_ptr()


def _kv_dtype(t, what):
    code = _KV_DTYPES.get(t.dtype)
    if code is None or t.dim() != 3:
        raise ValueError("%s: needs a bfloat16 or float16 tensor [tokens, heads, dim]" % what)
    return code


class KVLayout:
    """How a layer's K and V lie in the chunks of a PagedKV: kv heads, head size, tokens per block and format.  k_scale / v_scale are the
    tensor scales of KV_PACKED (powers of two).  KV_LATENT_BF16 / _FP16: heads 1, dim the latent vector's and LATENT_ROPE; a layer has one
    chunk per block, so layer i lies in half i % 2 of the PagedKV's (and the store's) layer i // 2."""

    def __init__(self, heads, dim, block_tokens, format=KV_BF16, k_scale=1.0, v_scale=1.0):
        self.heads, self.dim, self.block_tokens, self.format = heads, dim, block_tokens, format
        self.k_scale, self.v_scale = k_scale, v_scale
        self.latent = format in (KV_LATENT_BF16, KV_LATENT_FP16)
        self.chunk_bytes = int(lib.ptstore_kv_chunk_bytes(format, block_tokens, heads, dim))
        if self.chunk_bytes == 0:
            raise PTStoreError(E_INVAL, "ptstore_kv_chunk_bytes")

    def store_args(self):
        """dim and elem_bytes for a PTStore that holds chunks of this layout (the store moves opaque bytes)."""
        return {"dim": self.dim * 9 // 16, "elem_bytes": 1} if self.format == KV_PACKED else {"dim": self.dim, "elem_bytes": 2}

    def of(self, cache, layer, dev=None):
        """The C descriptor of one layer of a PagedKV, as bytes."""
        half = 0
        if self.latent:
            layer, half = layer >> 1, layer & 1
        if not 0 <= layer < len(cache.tensors):
            raise ValueError("layer %d of a cache of %d layers" % (layer, len(cache.tensors)))
        t = cache.tensors[layer]
        if t.get_device() != (_device() if dev is None else dev):
            _elsewhere(t, "cache")
        size, shape, stride = t.element_size(), t.shape, t.stride()
        if len(shape) == 3:
            inner = shape[2] if stride[2] == 1 or shape[2] == 1 else 0
        else:
            inner = 1
            for n, s in zip(shape[:1:-1], stride[:1:-1]):        # the axes of a chunk, last first
                if s != inner and n != 1:
                    inner = 0
                inner *= n
        if len(shape) < 2 or shape[0] != 2 or inner * size != self.chunk_bytes:
            raise ValueError("cache: needs [2, blocks, chunk] with contiguous chunks of %d bytes" % self.chunk_bytes)
        return _KV_CACHE.pack(t.data_ptr() + half * stride[0] * size, stride[0] * size, stride[1] * size, shape[1], self.block_tokens, self.heads, self.dim, self.format, 0,
                              self.k_scale, self.v_scale)


def assign_blocks(lengths, held, block_tables, free_ids, free_count, block_tokens, held_out=None, free_count_out=None, status=None):
    """ptstore_assign_blocks: grows and shrinks block-table rows to the lengths, from and to the stack free_ids[:free_count].  held (None:
    nothing held yet) and free_count are updated in place unless held_out / free_count_out are given.  Returns (held, free_count)."""
    dev, i32, R = _device(), torch.int32, lengths.numel()
    if held_out is None:
        held_out = held if held is not None else torch.empty_like(lengths)
    if free_count_out is None:
        free_count_out = free_count
    _check(lib.ptstore_assign_blocks(_vec(lengths, i32, R, dev, "lengths"), None if held is None else _vec(held, i32, R, dev, "held"), R, block_tokens,
                                     _table(block_tables, R, dev, "block_tables"), block_tables.shape[1], _vec(free_ids, i32, free_ids.numel(), dev, "free_ids"),
                                     free_ids.numel(), _vec(free_count, i32, 1, dev, "free_count"), _vec(held_out, i32, R, dev, "held_out"),
                                     _vec(free_count_out, i32, 1, dev, "free_count_out"), None if status is None else _vec(status, i32, 1, dev, "status"),
                                     _raw_stream(dev)), "ptstore_assign_blocks")
    return held_out, free_count_out


def map_slots(lengths, done, block_tables, block_tokens, max_tokens, done_unit=1, min_new=0, token_offsets=None, slots=None, positions=None,
              status=None):
    """ptstore_map_slots: the new tokens of a batch.  done (tokens, times done_unit; None: none) are in the cache already; after a lookup
    pass its matched lengths with done_unit=block_tokens, min_new=1.  Returns (token_offsets [R+1], slots int64 [max_tokens], positions)."""
    dev, i32, R = _device(), torch.int32, lengths.numel()
    if token_offsets is None:
        token_offsets = torch.empty(R + 1, dtype=i32, device="cuda")
        offsets_at = token_offsets.data_ptr()
    else:
        offsets_at = _vec(token_offsets, i32, R + 1, dev, "token_offsets")
    if slots is None:
        slots = torch.empty(max_tokens, dtype=torch.int64, device="cuda")
        slots_at = slots.data_ptr()
    else:
        slots_at = _vec(slots, torch.int64, max_tokens, dev, "slots")
    if positions is None:
        positions = torch.empty(max_tokens, dtype=i32, device="cuda")
        positions_at = positions.data_ptr()
    else:
        positions_at = _vec(positions, i32, max_tokens, dev, "positions")
    _check(lib.ptstore_map_slots(_vec(lengths, i32, R, dev, "lengths"), None if done is None else _vec(done, i32, R, dev, "done"), done_unit, min_new, R,
                                 _table(block_tables, R, dev, "block_tables"), block_tables.shape[1], block_tokens, max_tokens,
                                 offsets_at, slots_at, positions_at, None if status is None else _vec(status, i32, 1, dev, "status"),
                                 _raw_stream(dev)), "ptstore_map_slots")
    return token_offsets, slots, positions


def kv_write(layout, cache, layer, k, v, slots, status=None):
    """ptstore_kv_write: rows k, v [tokens, heads, dim] into one layer of the paged cache at `slots` (int64; -1 skips a row)."""
    dev, n, code, k_stride, v_stride = _device(), slots.numel(), _kv_dtype(k, "k"), k.stride(), v.stride()
    _check(lib.ptstore_kv_write(_rows(k, layout.heads, layout.dim, n, k.dtype, dev, "k"), k_stride[0], k_stride[1],
                                _rows(v, layout.heads, layout.dim, n, k.dtype, dev, "v"), v_stride[0], v_stride[1], n, code,
                                _vec(slots, torch.int64, n, dev, "slots"), layout.of(cache, layer, dev),
                                None if status is None else _vec(status, torch.int32, 1, dev, "status"), _raw_stream(dev)), "ptstore_kv_write")


def kv_read(layout, cache, layer, slots, dtype, k=None, v=None, status=None):
    """ptstore_kv_read: the values at `slots` as rows [tokens, heads, dim]; rows whose slot is -1 are left as they were.  Returns (k, v)."""
    dev, n, heads, dim = _device(), slots.numel(), layout.heads, layout.dim
    if k is None:
        k = torch.empty((n, heads, dim), dtype=dtype, device="cuda")
        k_at, k_stride = k.data_ptr(), (heads * dim, dim)
    else:
        k_at, k_stride = _rows(k, heads, dim, n, dtype, dev, "k"), k.stride()
    if v is None:
        v = torch.empty((n, heads, dim), dtype=dtype, device="cuda")
        v_at, v_stride = v.data_ptr(), (heads * dim, dim)
    else:
        v_at, v_stride = _rows(v, heads, dim, n, dtype, dev, "v"), v.stride()
    code = _kv_dtype(k, "k")
    _check(lib.ptstore_kv_read(layout.of(cache, layer, dev), _vec(slots, torch.int64, n, dev, "slots"), n, code, k_at, k_stride[0], k_stride[1],
                               v_at, v_stride[0], v_stride[1], None if status is None else _vec(status, torch.int32, 1, dev, "status"), _raw_stream(dev)), "ptstore_kv_read")
    return k, v


def attend_workspace(layout):
    """A workspace for attend on the current device.  Calls that share one must not overlap; they may differ in every size."""
    n = int(lib.ptstore_attend_workspace_bytes(layout.dim))
    raw = torch.zeros(n + 256, dtype=torch.uint8, device="cuda")
    at = -raw.data_ptr() % 256
    return raw[at:at + n]


def attend(layout, cache, layer, q, token_offsets, lengths, block_tables, max_new, scale=None, out=None, workspace=None, status=None, wait_polls=0, lse=None):
    """ptstore_attend: causal attention of the new tokens q [tokens, num_heads, dim] over the paged cache (which holds their own K/V
    already).  Request r owns rows token_offsets[r] .. token_offsets[r+1]-1 and lengths[r] tokens of cache; max_new (host) is at least the
    rows of any request.  workspace: from attend_workspace (a program that calls often keeps one per stream).  wait_polls: polls of the kernels' bounded
    waits, 0 for the built-in limit.  lse: float32 [tokens, num_heads] that receives the logarithms of the rows' sums (ptstore_attend_lse), for attend_weights.
    Returns out."""
    dev, i32, code = _device(), torch.int32, _kv_dtype(q, "q")
    R, (T, heads, dim) = lengths.numel(), q.shape
    if out is None:
        out = torch.empty((T, heads, dim), dtype=q.dtype, device=q.device)
    if workspace is None:
        workspace = attend_workspace(layout)
    elif workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError("workspace: needs contiguous memory on the current device")
    _on_device(q, dev, "q")
    desc = layout.of(cache, layer, dev)
    _on_device(cache.tensors[layer], dev, "cache")
    q_stride, o_stride = q.stride(), out.stride()
    args = _ATTEND.pack(_ATTEND_SIZE, code, _rows(q, heads, layout.dim, T, q.dtype, dev, "q"), q_stride[0], q_stride[1],
                        _rows(out, heads, layout.dim, T, q.dtype, dev, "out"), o_stride[0], o_stride[1],
                        _vec(token_offsets, i32, R + 1, dev, "token_offsets"), _vec(lengths, i32, R, dev, "lengths"),
                        _table(block_tables, R, dev, "block_tables"), R, block_tables.shape[1], heads, T, max_new,
                        layout.dim ** -0.5 if scale is None else scale, wait_polls, 0)
    work, room, bits = workspace.data_ptr(), workspace.numel() * workspace.element_size(), None if status is None else _vec(status, i32, 1, dev, "status")
    if lse is None:
        _check(lib.ptstore_attend(args, desc, work, room, bits, _raw_stream(dev)), "ptstore_attend")
    else:
        _check(lib.ptstore_attend_lse(args, desc, work, room, _vec(lse, torch.float32, T * heads, dev, "lse"), bits, _raw_stream(dev)), "ptstore_attend_lse")
    return out


_LATENT_DTYPES = {KV_LATENT_BF16: torch.bfloat16, KV_LATENT_FP16: torch.float16}


def _latent_dtype(layout):
    if not layout.latent:
        raise ValueError("layout: needs KV_LATENT_BF16 or KV_LATENT_FP16")
    return _LATENT_DTYPES[layout.format]


def _rows2(t, dim, n, dtype, dev, what):
    """[n][dim] rows of 16-bit elements, any token stride; returns the address."""
    if t.dtype is not dtype or t.shape != (n, dim) or t.stride(1) != 1:
        raise ValueError("%s: needs a %s tensor [%d, %d], contiguous along the last axis" % (what, dtype, n, dim))
    if t.get_device() != dev:
        _elsewhere(t, what)
    return t.data_ptr()


def latent_write(layout, cache, layer, latent, rope, slots, status=None):
    """ptstore_latent_write: rows latent [tokens, dim - 64], rope [tokens, 64] into one layer of the paged cache at `slots` (int64; -1 skips a row)."""
    dev, n, dtype = _device(), slots.numel(), _latent_dtype(layout)
    _check(lib.ptstore_latent_write(_rows2(latent, layout.dim - LATENT_ROPE, n, dtype, dev, "latent"), latent.stride(0), _rows2(rope, LATENT_ROPE, n, dtype, dev, "rope"),
                                    rope.stride(0), n, _vec(slots, torch.int64, n, dev, "slots"), layout.of(cache, layer, dev),
                                    None if status is None else _vec(status, torch.int32, 1, dev, "status"), _raw_stream(dev)), "ptstore_latent_write")


def latent_read(layout, cache, layer, slots, latent=None, rope=None, status=None):
    """ptstore_latent_read: the rows at `slots`; rows whose slot is -1 are left as they were.  Returns (latent [tokens, dim - 64], rope [tokens, 64])."""
    dev, n, dtype = _device(), slots.numel(), _latent_dtype(layout)
    if latent is None:
        latent = torch.empty((n, layout.dim - LATENT_ROPE), dtype=dtype, device="cuda")
    if rope is None:
        rope = torch.empty((n, LATENT_ROPE), dtype=dtype, device="cuda")
    _check(lib.ptstore_latent_read(layout.of(cache, layer, dev), _vec(slots, torch.int64, n, dev, "slots"), n,
                                   _rows2(latent, layout.dim - LATENT_ROPE, n, dtype, dev, "latent"), latent.stride(0),
                                   _rows2(rope, LATENT_ROPE, n, dtype, dev, "rope"), rope.stride(0),
                                   None if status is None else _vec(status, torch.int32, 1, dev, "status"), _raw_stream(dev)), "ptstore_latent_read")
    return latent, rope


def latent_workspace(layout):
    """A workspace for latent_attend on the current device.  Calls that share one must not overlap; they may differ in every size."""
    _latent_dtype(layout)
    raw = torch.empty(int(lib.ptstore_latent_workspace_bytes(layout.dim)) + 256, dtype=torch.uint8, device="cuda")
    return raw[-raw.data_ptr() % 256:]


def latent_attend(layout, cache, layer, q_latent, q_rope, token_offsets, lengths, block_tables, max_new, scale, out=None, lse=None, workspace=None, status=None,
                  wait_polls=0):
    """ptstore_latent_attend: causal attention of the new tokens over the latent cache (which holds their own rows already), absorbed form.
    q_latent [tokens, num_heads, dim - 64] (q times the key projection), q_rope [tokens, num_heads, 64]; scale: that of the scores, 1 / sqrt of the
    size of a head that is not absorbed.  out [tokens, num_heads, dim - 64], to be multiplied by the value projection.  lse: float32 [tokens, num_heads]
    that receives the logarithms of the rows' sums.  The rest as for attend; workspace: from latent_workspace.  Returns out."""
    dev, i32, dtype, L = _device(), torch.int32, _latent_dtype(layout), layout.dim - LATENT_ROPE
    if q_latent.dim() != 3:
        raise ValueError("q_latent: needs a tensor [tokens, heads, dim]")
    R, (T, heads, _) = lengths.numel(), q_latent.shape
    if out is None:
        out = torch.empty((T, heads, L), dtype=dtype, device=q_latent.device)
    if workspace is None:
        workspace = latent_workspace(layout)
    elif workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError("workspace: needs contiguous memory on the current device")
    desc = layout.of(cache, layer, dev)
    _on_device(cache.tensors[layer >> 1], dev, "cache")
    ql, qr, o = q_latent.stride(), q_rope.stride(), out.stride()
    at = _rows(q_latent, heads, L, T, dtype, dev, "q_latent"), _rows(q_rope, heads, LATENT_ROPE, T, dtype, dev, "q_rope"), _rows(out, heads, L, T, dtype, dev, "out")
    if at[2] == at[0] and ((T > 1 and o[0] != ql[0]) or (T > 0 and heads > 1 and o[1] != ql[1])):
        raise ValueError("out: is q_latent with other strides")
    args = _LATENT_ATTEND.pack(_LATENT_ATTEND.size, wait_polls, at[0], ql[0], ql[1], at[1], qr[0], qr[1], at[2], o[0], o[1],
                               0 if lse is None else _vec(lse, torch.float32, T * heads, dev, "lse"), _vec(token_offsets, i32, R + 1, dev, "token_offsets"),
                               _vec(lengths, i32, R, dev, "lengths"), _table(block_tables, R, dev, "block_tables"), R, block_tables.shape[1], heads, T, max_new, scale)
    _check(lib.ptstore_latent_attend(args, desc, workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                     None if status is None else _vec(status, i32, 1, dev, "status"), _raw_stream(dev)), "ptstore_latent_attend")
    return out


def expanded_attend(q, k, k_rope, v, token_offsets, key_offsets, max_new, scale=None, out=None, status=None, wait_polls=0):
    """ptstore_expanded_attend: causal attention of the new tokens q [tokens, heads, 192] over the requests' keys k [keys, heads, 128] and k_rope [keys, 64] (shared by the heads; q's
    last 64 elements meet them) and values v [keys, heads, 128], the last keys of a request being its rows' own.  k and v may be views of one tensor, and their head
    strides 0.  Request r owns rows token_offsets[r] .. and keys key_offsets[r] ..; scale: 192 ** -0.5 by default.  Returns out [tokens, heads, 128]."""
    dev, i32, code = _device(), torch.int32, _kv_dtype(q, "q")
    R, (T, heads, _), dtype = token_offsets.numel() - 1, q.shape, q.dtype
    if k.dim() != 3 or R < 0:
        raise ValueError("k: needs a tensor [keys, heads, 128], token_offsets at least one entry")
    N = k.shape[0]
    if out is None:
        out = torch.empty((T, heads, 128), dtype=dtype, device=q.device)
    for t, what in ((q, "q"), (k, "k"), (k_rope, "k_rope"), (v, "v")):
        _on_device(t, dev, what)
    qs, ks, rs, vs, os_ = q.stride(), k.stride(), k_rope.stride(), v.stride(), out.stride()
    args = _EXPANDED_ATTEND.pack(_EXPANDED_ATTEND.size, code, _rows(q, heads, 192, T, dtype, dev, "q"), qs[0], qs[1], _rows(k, heads, 128, N, dtype, dev, "k"), ks[0], ks[1],
                                 _rows2(k_rope, 64, N, dtype, dev, "k_rope"), rs[0], _rows(v, heads, 128, N, dtype, dev, "v"), vs[0], vs[1],
                                 _rows(out, heads, 128, T, dtype, dev, "out"), os_[0], os_[1], _vec(token_offsets, i32, R + 1, dev, "token_offsets"),
                                 _vec(key_offsets, i32, R + 1, dev, "key_offsets"), R, heads, T, N, max_new, 192 ** -0.5 if scale is None else scale, wait_polls, 0)
    _check(lib.ptstore_expanded_attend(args, None if status is None else _vec(status, i32, 1, dev, "status"), _raw_stream(dev)), "ptstore_expanded_attend")
    return out


def _weights(t, R, heads, dev, what):
    """[R][heads][width] 32-bit floats, any request and head strides; returns the address."""
    if t.dtype is not torch.float32 or t.dim() != 3 or t.shape[0] != R or t.shape[1] != heads or (t.stride(2) != 1 and t.shape[2] > 1):
        raise ValueError("%s: needs a float32 tensor [%d, %d, width], contiguous along the last axis" % (what, R, heads))
    if t.get_device() != dev:
        _elsewhere(t, what)
    return t.data_ptr()


def attend_weights(layout, cache, layer, q, lse, token_offsets, lengths, block_tables, max_new, weights, scale=None, accumulate=True, status=None, wait_polls=0):
    """ptstore_attend_weights: adds to weights [requests, kv heads, width] what the rows of q [tokens, num_heads, dim] gave to every cached token; lse from attend or
    latent_attend (of a latent cache q is the latent and the rotary part side by side, and scale has no default).  accumulate=False: writes
    instead, zeros behind a request's tokens.  Returns weights."""
    dev, i32, code = _device(), torch.int32, _kv_dtype(q, "q")
    R, (T, heads, _) = lengths.numel(), q.shape
    if scale is None:
        if layout.latent:
            raise ValueError("scale: has no default for a latent cache")
        scale = layout.dim ** -0.5
    desc, at = layout.of(cache, layer, dev), _weights(weights, R, layout.heads, dev, "weights")
    q_stride, w_stride = q.stride(), weights.stride()
    args = _ATTEND_WEIGHTS.pack(_ATTEND_WEIGHTS.size, code, _rows(q, heads, layout.dim, T, q.dtype, dev, "q"), q_stride[0], q_stride[1],
                                _vec(lse, torch.float32, T * heads, dev, "lse"), _vec(token_offsets, i32, R + 1, dev, "token_offsets"),
                                _vec(lengths, i32, R, dev, "lengths"), _table(block_tables, R, dev, "block_tables"), R, block_tables.shape[1], heads, T, at,
                                w_stride[0], w_stride[1], weights.shape[2], max_new, 1 if accumulate else 0, scale, wait_polls, 0)
    _check(lib.ptstore_attend_weights(args, desc, None if status is None else _vec(status, i32, 1, dev, "status"), _raw_stream(dev)), "ptstore_attend_weights")
    return weights


def select_tokens(weights, lengths, budget, first, recent, kept=None, lengths_out=None, weights_out=None, status=None):
    """ptstore_select_tokens: of every request longer than `budget` the tokens each kv head keeps, its first `first`, last `recent` and the ones with the largest weights in between.
    weights [requests, kv heads, width] float32; the kept tokens' weights go to weights_out (weights itself by default).  Returns (kept int32 [requests, kv heads, budget],
    ascending, -1 behind the last; lengths_out int32 [requests]; weights_out).  A budget beyond width keeps all."""
    dev, i32, R = _device(), torch.int32, lengths.numel()
    if weights.dim() != 3:
        raise ValueError("weights: needs a float32 tensor [requests, heads, width]")
    heads, width = weights.shape[1:]
    if kept is None:
        kept = torch.empty((R, heads, max(budget, 0)), dtype=i32, device="cuda")
    if lengths_out is None:
        lengths_out = torch.empty(R, dtype=i32, device="cuda")
    if weights_out is None:
        weights_out = weights
    elif weights_out.shape != weights.shape:
        raise ValueError("weights_out: needs the shape of weights")
    w, o, at = weights.stride(), weights_out.stride(), _vec(kept, i32, R * heads * max(budget, 0), dev, "kept")
    chosen, wide = None, budget
    if budget > width > 0 and first >= 0 and recent >= 0 and first + recent <= budget:
        # the library takes a budget of at most width: nothing has to go, and what is written of a row of `kept` is as wide as a row of weights
        chosen = torch.empty((R, heads, width), dtype=i32, device="cuda")
        at, budget, first, recent = chosen.data_ptr(), width, 0, 0
    _check(lib.ptstore_select_tokens(_weights(weights, R, heads, dev, "weights"), w[0], w[1], _vec(lengths, i32, R, dev, "lengths"), R, heads, width, budget, first, recent,
                                     at, _vec(lengths_out, i32, R, dev, "lengths_out"),
                                     _weights(weights_out, R, heads, dev, "weights_out"), o[0], o[1], None if status is None else _vec(status, i32, 1, dev, "status"),
                                     _raw_stream(dev)), "ptstore_select_tokens")
    if chosen is not None:
        rows = kept.view(R, heads, wide)
        rows[:, :, :width] = chosen
        rows[:, :, width:] = -1
    return kept, lengths_out, weights_out


def kv_compact(layout, cache, layer, kept, lengths, block_tables, to_tables=None, status=None):
    """ptstore_kv_compact: in one layer of the cache, token i < lengths[r] of request r and kv head h becomes its token kept[r, h, i] (int32 [requests, kv heads, n]).  to_tables None: in
    place (kept ascends, and no block belongs to two requests); else the tokens go to the blocks of to_tables, none of which block_tables names."""
    dev, i32, R = _device(), torch.int32, lengths.numel()
    if kept.dim() != 3 or kept.shape[0] != R or kept.shape[1] != layout.heads:
        raise ValueError("kept: needs an int32 tensor [%d, %d, n]" % (R, layout.heads))
    to = block_tables if to_tables is None else to_tables
    _check(lib.ptstore_kv_compact(layout.of(cache, layer, dev), _vec(kept, i32, kept.numel(), dev, "kept"), _vec(lengths, i32, R, dev, "lengths"), R, kept.shape[2],
                                  _table(block_tables, R, dev, "block_tables"), block_tables.shape[1], _table(to, R, dev, "to_tables"), to.shape[1],
                                  None if status is None else _vec(status, i32, 1, dev, "status"), _raw_stream(dev)), "ptstore_kv_compact")


class PTStore:
    """One store on one GPU.  Allocates pool and workspace with torch and hands them to the library."""

    def __init__(self, layers, heads, dim, block_tokens, hbm_blocks, max_requests, max_batch_blocks, elem_bytes=2,
                 host_blocks=0, table_slots=None, salt=0, flags=0, device=None, hbm_pool=None, host_pool=None):
        if device is None:
            device = torch.cuda.current_device()       # one process per GPU: the rank's own device
        self.device = torch.device("cuda", device)
        self.layers, self.block_tokens = layers, block_tokens
        self.chunk_bytes = block_tokens * heads * dim * elem_bytes
        self.block_bytes = 2 * layers * self.chunk_bytes
        self.hbm_blocks, self.host_blocks = hbm_blocks, host_blocks
        n = hbm_blocks + host_blocks
        self.table_slots = table_slots or max(int(n / 0.7) + 1, n + 2)
        self.hbm_pool = hbm_pool if hbm_pool is not None else torch.empty(hbm_blocks * self.block_bytes, dtype=torch.uint8,
                                                                         device=self.device)
        self.host_pool = host_pool
        host_ptr = None
        if host_blocks:
            if self.host_pool is None:
                self.host_pool = torch.empty(host_blocks * self.block_bytes, dtype=torch.uint8, pin_memory=True)
            host_ptr = self.host_pool.data_ptr()   # pinned memory shares the unified address space
        cfg = Config(C.sizeof(Config), flags, layers, heads, dim, elem_bytes, block_tokens, max_requests,
                     max_batch_blocks, salt, self.hbm_pool.data_ptr(), host_ptr, hbm_blocks, host_blocks,
                     self.table_slots, None, 0, device, 0)
        need = lib.ptstore_workspace_bytes(C.byref(cfg))
        if need == 0:
            raise PTStoreError(E_INVAL, "ptstore_workspace_bytes")
        self.workspace = torch.empty(need + 256, dtype=torch.uint8, device=self.device)
        base = (self.workspace.data_ptr() + 255) // 256 * 256
        cfg.workspace, cfg.workspace_bytes = base, need
        self.cfg = cfg
        h = C.c_void_p()
        with torch.cuda.device(self.device):
            rc = lib.ptstore_create(C.byref(cfg), C.byref(h), _stream())
        if rc:
            raise PTStoreError(rc, "ptstore_create")
        self.h = h

    def close(self):
        if getattr(self, "h", None):
            torch.cuda.synchronize(self.device)
            lib.ptstore_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc, what):
        if rc:
            raise PTStoreError(rc, what)

    # every method takes device tensors (int32 tokens/ids/tables, int64 offsets) and returns device tensors
    def hash(self, tokens, offsets, max_blocks):
        R = offsets.numel() - 1
        keys = torch.empty((R, max_blocks), dtype=torch.int64, device=self.device)
        self._check(lib.ptstore_hash(self.h, _ptr(tokens), _ptr(offsets), R, max_blocks, _ptr(keys), _stream()), "ptstore_hash")
        return keys

    def lookup(self, tokens, offsets, max_blocks, flags=0, matched=None, ids=None):
        R = offsets.numel() - 1
        if matched is None:
            matched = torch.empty(R, dtype=torch.int32, device=self.device)
        if ids is None:
            ids = torch.empty((R, max_blocks), dtype=torch.int32, device=self.device)
        self._check(lib.ptstore_lookup(self.h, _ptr(tokens), _ptr(offsets), R, max_blocks, flags, _ptr(matched), _ptr(ids),
                                       _stream()), "ptstore_lookup")
        return matched, ids

    def fetch(self, ids, matched, cache, block_tables):
        R, mb = ids.shape
        self._check(lib.ptstore_fetch(self.h, _ptr(ids), _ptr(matched), R, mb, C.byref(cache.desc), _ptr(block_tables),
                                      _stream()), "ptstore_fetch")

    def lookup_fetch(self, tokens, offsets, max_blocks, cache, block_tables, flags=0, matched=None, ids=None):
        R = offsets.numel() - 1
        if matched is None:
            matched = torch.empty(R, dtype=torch.int32, device=self.device)
        if ids is None:
            ids = torch.empty((R, max_blocks), dtype=torch.int32, device=self.device)
        self._check(lib.ptstore_lookup_fetch(self.h, _ptr(tokens), _ptr(offsets), R, max_blocks, flags, C.byref(cache.desc),
                                             _ptr(block_tables), _ptr(matched), _ptr(ids), _stream()), "ptstore_lookup_fetch")
        return matched, ids

    def reserve(self, want_free, minus=None, flags=0, max_victims=0, n_evicted=None, victims=None, headroom=0):
        """Evicts need + headroom blocks from HBM if need = want_free - sum(minus) - free HBM blocks is positive, decided on
        the device."""
        if n_evicted is None:
            n_evicted = torch.zeros(2, dtype=torch.int32, device=self.device)
        if victims is None and max_victims:
            victims = torch.full((2 * max_victims,), -1, dtype=torch.int32, device=self.device)
        self._check(lib.ptstore_reserve(self.h, int(want_free), int(headroom), _ptr(minus), minus.numel() if minus is not None else 0, flags,
                                        _ptr(n_evicted), _ptr(victims), max_victims, _stream()), "ptstore_reserve")
        return n_evicted, victims

    def time_next_copy(self, before, after):
        """before / after: torch.cuda.Event(enable_timing=True) that have been recorded once (so that they exist)."""
        self._check(lib.ptstore_time_next_copy(self.h, before.cuda_event, after.cuda_event), "ptstore_time_next_copy")

    def set_wait_limit(self, polls):
        self._check(lib.ptstore_set_wait_limit(self.h, polls), "ptstore_set_wait_limit")

    def insert(self, tokens, offsets, max_blocks, cache=None, block_tables=None, ids=None, new_blocks=None, after_lookup=False):
        """after_lookup: ptstore_insert_after_lookup (reuses the keys of the last lookup if it saw these very tensors)."""
        R = offsets.numel() - 1
        if ids is None:
            ids = torch.empty((R, max_blocks), dtype=torch.int32, device=self.device)
        if new_blocks is None:
            new_blocks = torch.empty(R, dtype=torch.int32, device=self.device)
        desc = C.byref(cache.desc) if cache is not None else None
        fn = lib.ptstore_insert_after_lookup if after_lookup else lib.ptstore_insert
        self._check(fn(self.h, _ptr(tokens), _ptr(offsets), R, max_blocks, desc, _ptr(block_tables),
                       _ptr(ids), _ptr(new_blocks), _stream()), "ptstore_insert")
        return ids, new_blocks

    def resumed_inserts(self):
        return int(lib.ptstore_resumed_inserts(self.h))

    def release(self, ids, matched):
        R, mb = ids.shape
        self._check(lib.ptstore_release(self.h, _ptr(ids), _ptr(matched), R, mb, _stream()), "ptstore_release")

    def evict(self, tier, n, want_victims=True, n_evicted=None, victims=None, asynchronous=False):
        if n_evicted is None:
            n_evicted = torch.zeros(2, dtype=torch.int32, device=self.device)
        if victims is None and want_victims:
            victims = torch.full((max(2 * n, 1),), -1, dtype=torch.int32, device=self.device)
        fn = lib.ptstore_evict_async if asynchronous else lib.ptstore_evict
        self._check(fn(self.h, tier, n, _ptr(n_evicted), _ptr(victims), _stream()), "ptstore_evict")
        return n_evicted, victims

    def join(self):
        self._check(lib.ptstore_join(self.h, _stream()), "ptstore_join")

    def promote(self, ids, matched, flags, max_promote, n_promoted=None):
        """Rewrites `ids` in place; returns the device counter of blocks moved."""
        R, mb = ids.shape
        if n_promoted is None:
            n_promoted = torch.zeros(1, dtype=torch.int32, device=self.device)
        self._check(lib.ptstore_promote(self.h, _ptr(ids), _ptr(matched), R, mb, flags, max_promote, _ptr(n_promoted), _stream()),
                    "ptstore_promote")
        return n_promoted

    def status(self):
        out = C.c_uint32(0)
        self._check(lib.ptstore_status(self.h, _stream(), C.byref(out)), "ptstore_status")
        return out.value

    def stats(self):
        out = Stats()
        self._check(lib.ptstore_stats(self.h, _stream(), C.byref(out)), "ptstore_stats")
        return out

    def stats_enqueue(self, pinned_bytes):
        """Writes the counters into `pinned_bytes` (a pinned uint8 host tensor of sizeof(Stats)) without blocking;
        read it with Stats.from_buffer_copy(...) once the stream (or a later event) has completed."""
        self._check(lib.ptstore_stats_enqueue(self.h, pinned_bytes.data_ptr(), _stream()), "ptstore_stats_enqueue")

    def launch_count(self):
        return int(lib.ptstore_launch_count(self.h))
