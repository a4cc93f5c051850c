"""ctypes binding of libtriattn.so (include/triattn.h).

Argument marshalling only: every step of the attention passes runs in the HIP
kernels of the library.  Torch tensors provide device memory and the stream.
The library must have been built (``python -m paper_2507_21526_amd.build``);
loading raises ``RuntimeError`` otherwise -- there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libtriattn.so")
HEADER_PATH = os.path.join(os.path.dirname(_PKG), "include", "triattn.h")

TA_OK = 0
TA_ERR_INVALID_ARG = 1
TA_ERR_UNSUPPORTED = 2
TA_ERR_BUFFER_TOO_SMALL = 3
TA_ERR_WORKSPACE = 4
TA_ERR_SCHEDULE_MISMATCH = 5
TA_ERR_HIP = 6

TRIANGLE = 0
CAUSAL = 1
BLOCKSPARSE = 2
OUT_BF16 = 0
OUT_F32 = 1

HDR_WORDS, ITEM_WORDS, MERGE_WORDS = 16, 12, 8


class ScheduleInfo(ctypes.Structure):
    _fields_ = [
        ("version", ctypes.c_int32),
        ("kind", ctypes.c_int32),
        ("tile", ctypes.c_int32),
        ("batch", ctypes.c_int32),
        ("sink", ctypes.c_int32),
        ("window", ctypes.c_int32),
        ("last", ctypes.c_int32),
        ("splits_requested", ctypes.c_int32),
        ("total_tokens", ctypes.c_int64),
        ("words", ctypes.c_int64),
        ("n_items", ctypes.c_int32),
        ("n_last_items", ctypes.c_int32),
        ("n_merge_items", ctypes.c_int32),
        ("n_last_rows", ctypes.c_int32),
        ("n_partial_rows", ctypes.c_int32),
        ("max_splits", ctypes.c_int32),
        ("kept_tiles_per_qhead", ctypes.c_int64),
        ("max_item_tiles", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
    ]

    def as_dict(self):
        return {name: getattr(self, name) for name, _ in self._fields_}


class TriAttnError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"status {status}: {message}")
        self.status = status


_lib = None


def lib():
    """Load libtriattn.so; raise if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            f"{LIB_PATH} is missing: build it with "
            "`python -m paper_2507_21526_amd.build` (no fallback path exists)")
    L = ctypes.CDLL(LIB_PATH)
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    pinfo = ctypes.POINTER(ScheduleInfo)
    L.ta_abi_version.restype = i32
    L.ta_abi_version.argtypes = []
    L.ta_last_error.restype = ctypes.c_char_p
    L.ta_last_error.argtypes = []
    L.ta_build_schedule.restype = ctypes.c_int
    L.ta_build_schedule.argtypes = [i32, vp, i32, i32, i32, i32, i32, i32, vp,
                                    i64, pinfo]
    L.ta_workspace_bytes.restype = ctypes.c_size_t
    L.ta_workspace_bytes.argtypes = [pinfo, i32, i32]
    L.triangle_attn_fwd.restype = ctypes.c_int
    L.triangle_attn_fwd.argtypes = [vp, vp, vp, vp, i32, vp, vp, pinfo, i64,
                                    i32, i32, i32, ctypes.c_float, vp,
                                    ctypes.c_size_t, vp]
    L.triangle_attn_fwd_noalloc.restype = ctypes.c_int
    L.triangle_attn_fwd_noalloc.argtypes = [vp, vp, vp, vp, i32, vp, vp, pinfo, i64,
                                            i32, i32, i32, ctypes.c_float, vp]
    L.triangle_attn_tiles.restype = ctypes.c_int
    L.triangle_attn_tiles.argtypes = list(L.triangle_attn_fwd.argtypes)
    L.triangle_attn_merge.restype = ctypes.c_int
    L.triangle_attn_merge.argtypes = [vp, i32, vp, vp, pinfo, i64, i32, i32,
                                      vp, ctypes.c_size_t, vp]
    L.causal_attn_fwd.restype = ctypes.c_int
    L.causal_attn_fwd.argtypes = [vp, vp, vp, vp, i32, vp, vp, pinfo, i64,
                                  i32, i32, i32, ctypes.c_float, vp]
    L.ta_build_blocksparse_schedule.restype = ctypes.c_int
    L.ta_build_blocksparse_schedule.argtypes = [vp, i32, i32, vp, vp, i32, vp, i64,
                                                pinfo]
    L.blocksparse_attn_fwd.restype = ctypes.c_int
    L.blocksparse_attn_fwd.argtypes = list(L.triangle_attn_fwd.argtypes)
    L.ta_probe_workspace_bytes.restype = ctypes.c_size_t
    L.ta_probe_workspace_bytes.argtypes = [pinfo, i32]
    L.region_grad_probe.restype = ctypes.c_int
    L.region_grad_probe.argtypes = [vp, vp, vp, vp, vp, vp, pinfo, i64, i32, i32,
                                    i32, ctypes.c_float, i32, i32, i32, vp, vp,
                                    ctypes.c_size_t, vp]
    L.ta_region_grad_workspace_bytes.restype = ctypes.c_size_t
    L.ta_region_grad_workspace_bytes.argtypes = [pinfo, i32, i32]
    L.region_grad_sums.restype = ctypes.c_int
    L.region_grad_sums.argtypes = [vp, vp, vp, vp, vp, pinfo, i64, i32, i32, i32,
                                   ctypes.c_float, i32, i32, i32, vp, vp,
                                   ctypes.c_size_t, vp]
    L.scored_attn_fwd.restype = ctypes.c_int
    L.scored_attn_fwd.argtypes = [vp, vp, vp, vp, i32, vp, vp, pinfo, i64, i32, i32, i32,
                                  ctypes.c_float, ctypes.c_float, vp, vp, ctypes.c_size_t, vp]
    L.ta_page_map.restype = ctypes.c_int
    L.ta_page_map.argtypes = [vp, vp, i32, i32, vp, i32, vp, i32, vp, vp, vp, vp, i64, vp, vp]
    L.kv_cache_write.restype = ctypes.c_int
    L.kv_cache_write.argtypes = [vp, vp, i64, i64, i64, i64, vp, i64, vp, vp, i64, i32, i32, i32,
                                 vp]
    L.kv_cache_write_q8.restype = ctypes.c_int
    L.kv_cache_write_q8.argtypes = [vp, vp, i64, i64, i64, i64, vp, i64, vp, vp, vp, vp, i64, i32,
                                    i32, i32, vp]
    L.kv_cache_read.restype = ctypes.c_int
    L.kv_cache_read.argtypes = [vp, vp, vp, i32, i32, vp, vp, vp, vp, i64, i64, i64, i64, i64, i64,
                                i32, i32, i32, vp]
    L.kv_cache_read_q8.restype = ctypes.c_int
    L.kv_cache_read_q8.argtypes = [vp, vp] + list(L.kv_cache_read.argtypes)
    L.ta_paged_workspace_bytes.restype = ctypes.c_size_t
    L.ta_paged_workspace_bytes.argtypes = [i32, i64, i32, i32, i32, i32, i32]
    L.paged_attn_fwd.restype = ctypes.c_int
    L.paged_attn_fwd.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp, vp, i32, i32, vp, i32, i64, i32,
                                 i32, i32, i64, i32, ctypes.c_float, ctypes.c_float, vp, vp,
                                 ctypes.c_size_t, vp]
    L.ta_paged_q8_workspace_bytes.restype = ctypes.c_size_t
    L.ta_paged_q8_workspace_bytes.argtypes = list(L.ta_paged_workspace_bytes.argtypes)
    L.paged_attn_fwd_q8.restype = ctypes.c_int
    L.paged_attn_fwd_q8.argtypes = [vp, vp] + list(L.paged_attn_fwd.argtypes)
    L.ta_region_counts.restype = ctypes.c_int
    L.ta_region_counts.argtypes = [vp, i32, i32, i32, i32, vp]
    L.ta_region_grad_mean.restype = ctypes.c_int
    L.ta_region_grad_mean.argtypes = [vp, i32, vp, vp]
    L.ta_select_triangle_layers.restype = ctypes.c_int
    L.ta_select_triangle_layers.argtypes = [vp, i32, i32, vp]
    _lib = L
    return L


def ta_last_error() -> str:
    return lib().ta_last_error().decode()


def ta_abi_version() -> int:
    return int(lib().ta_abi_version())


def _check(status):
    if status != TA_OK:
        raise TriAttnError(status, ta_last_error())


def _kind(kind) -> int:
    if kind in (TRIANGLE, "triangle"):
        return TRIANGLE
    if kind in (CAUSAL, "causal"):
        return CAUSAL
    if kind in (BLOCKSPARSE, "blocksparse"):
        return BLOCKSPARSE
    raise ValueError(f"unknown kind {kind!r}")


def ta_build_schedule(kind, cu_seqlens, sink, window, last, tile, splits=0):
    """Build a schedule on the host: returns (int32 words, ScheduleInfo)."""
    L = lib()
    cu = np.ascontiguousarray(np.asarray(cu_seqlens, dtype=np.int32))
    info = ScheduleInfo()
    _check(L.ta_build_schedule(_kind(kind), cu.ctypes.data, cu.size - 1, sink,
                               window, last, tile, splits, None, 0,
                               ctypes.byref(info)))
    words = np.zeros(info.words, dtype=np.int32)
    _check(L.ta_build_schedule(_kind(kind), cu.ctypes.data, cu.size - 1, sink,
                               window, last, tile, splits, words.ctypes.data,
                               words.size, ctypes.byref(info)))
    return words, info


def ta_build_blocksparse_schedule(cu_seqlens, tile, qtile_ptr, ktile_idx,
                                  max_tiles_per_item=0):
    """Build a block-sparse schedule on the host from per-q-tile k-tile
    lists in CSR form: returns (int32 words, ScheduleInfo)."""
    L = lib()
    cu = np.ascontiguousarray(np.asarray(cu_seqlens, dtype=np.int32))
    ptr = np.ascontiguousarray(np.asarray(qtile_ptr, dtype=np.int32))
    idx = np.ascontiguousarray(np.asarray(ktile_idx, dtype=np.int32))
    idx_p = idx.ctypes.data if idx.size else None
    info = ScheduleInfo()
    _check(L.ta_build_blocksparse_schedule(cu.ctypes.data, cu.size - 1, tile,
                                           ptr.ctypes.data, idx_p, max_tiles_per_item,
                                           None, 0, ctypes.byref(info)))
    words = np.zeros(info.words, dtype=np.int32)
    _check(L.ta_build_blocksparse_schedule(cu.ctypes.data, cu.size - 1, tile,
                                           ptr.ctypes.data, idx_p, max_tiles_per_item,
                                           words.ctypes.data, words.size,
                                           ctypes.byref(info)))
    return words, info


def ta_workspace_bytes(info: ScheduleInfo, hq: int, head_dim: int) -> int:
    return int(lib().ta_workspace_bytes(ctypes.byref(info), hq, head_dim))


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    import torch
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _out_dtype(o):
    import torch
    if o.dtype == torch.bfloat16:
        return OUT_BF16
    if o.dtype == torch.float32:
        return OUT_F32
    raise ValueError(f"o must be bf16 or fp32, got {o.dtype}")


def _check_tensors(q, k, v, o, lse, sched_dev, info, workspace=None, extra=()):
    """Validate what the C interface cannot see: dtypes, contiguity, shapes
    and devices of the torch tensors whose raw pointers are passed.  Raises
    ValueError before anything is enqueued (a wrong shape or a strided view
    would otherwise be misread, or read out of bounds, by the kernels).
    extra: (name, tensor, dtype, shape) of further operands."""
    import torch
    named = [("q", q), ("k", k), ("v", v), ("o", o)]
    for name, t in named:
        if not isinstance(t, torch.Tensor):
            raise ValueError(f"{name} must be a torch tensor")
    for name, t in (("q", q), ("k", k), ("v", v)):
        if t.dtype != torch.bfloat16:
            raise ValueError(f"{name} must be bfloat16, got {t.dtype}")
        if t.dim() != 3:
            raise ValueError(f"{name} must be [tokens, heads, head_dim], got {tuple(t.shape)}")
    _out_dtype(o)
    total, hq, d = q.shape
    if k.shape[0] != total or v.shape[0] != total:
        raise ValueError(f"k and v must have {total} tokens like q, got "
                         f"{k.shape[0]} and {v.shape[0]}")
    if k.shape != v.shape:
        raise ValueError(f"k {tuple(k.shape)} and v {tuple(v.shape)} differ")
    if k.shape[2] != d:
        raise ValueError(f"k/v head_dim {k.shape[2]} != q head_dim {d}")
    if tuple(o.shape) != tuple(q.shape):
        raise ValueError(f"o must have q's shape {tuple(q.shape)}, got {tuple(o.shape)}")
    if lse is not None:
        named.append(("lse", lse))
        if lse.dtype != torch.float32 or tuple(lse.shape) != (hq, total):
            raise ValueError(f"lse must be float32 [{hq}, {total}], got "
                             f"{lse.dtype} {tuple(lse.shape)}")
    named.append(("sched_dev", sched_dev))
    if not isinstance(sched_dev, torch.Tensor) or sched_dev.dtype != torch.int32:
        raise ValueError("sched_dev must be an int32 tensor of schedule words")
    if sched_dev.numel() != info.words:
        raise ValueError(f"sched_dev holds {sched_dev.numel()} words, the schedule "
                         f"info says {info.words}")
    if workspace is not None:
        named.append(("workspace", workspace))
    for name, t, dtype, shape in extra:
        named.append((name, t))
        if t.dtype != dtype or tuple(t.shape) != tuple(shape):
            raise ValueError(f"{name} must be {dtype} {tuple(shape)}, got "
                             f"{t.dtype} {tuple(t.shape)}")
    for name, t in named:
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
    dev = q.device
    for name, t in named:
        if t.device != dev:
            raise ValueError(f"{name} is on {t.device}, q on {dev}: all operands "
                             "must be on one device")
    if dev.type != "cuda":
        raise ValueError(f"operands must be on a GPU, got {dev}")


def triangle_attn_fwd(q, k, v, o, lse, sched_dev, info, softmax_scale,
                      workspace, stream=None):
    """Enqueue Triangle attention on ``stream`` (torch current stream if None).

    q [T, Hq, d], k/v [T, Hkv, d] bf16 cuda tensors; o [T, Hq, d] bf16/fp32;
    lse [Hq, T] fp32 or None; sched_dev int32 cuda tensor of the schedule
    words; workspace uint8 cuda tensor of >= ta_workspace_bytes bytes or None.
    """
    _check_tensors(q, k, v, o, lse, sched_dev, info, workspace)
    total, hq, d = q.shape
    hkv = k.shape[1]
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().triangle_attn_fwd(
        _ptr(q), _ptr(k), _ptr(v), _ptr(o), _out_dtype(o), _ptr(lse),
        _ptr(sched_dev), ctypes.byref(info), total, hq, hkv, d,
        float(softmax_scale), _ptr(workspace), ws_bytes, _stream(stream)))


def triangle_attn_fwd_noalloc(q, k, v, o, lse, sched_dev, info, softmax_scale,
                              stream=None):
    """Triangle attention without a workspace argument: the split partials
    go to the library's own per-GPU scratch array (no allocation in the
    call; at most TA_NOALLOC_SCRATCH_BYTES of partials).  Calls that overlap
    on one GPU race on that array."""
    _check_tensors(q, k, v, o, lse, sched_dev, info)
    total, hq, d = q.shape
    hkv = k.shape[1]
    _check(lib().triangle_attn_fwd_noalloc(
        _ptr(q), _ptr(k), _ptr(v), _ptr(o), _out_dtype(o), _ptr(lse),
        _ptr(sched_dev), ctypes.byref(info), total, hq, hkv, d,
        float(softmax_scale), _stream(stream)))


def triangle_attn_tiles(q, k, v, o, lse, sched_dev, info, softmax_scale,
                        workspace, stream=None):
    """Enqueue the attention pass of Triangle attention (no merge)."""
    _check_tensors(q, k, v, o, lse, sched_dev, info, workspace)
    total, hq, d = q.shape
    hkv = k.shape[1]
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().triangle_attn_tiles(
        _ptr(q), _ptr(k), _ptr(v), _ptr(o), _out_dtype(o), _ptr(lse),
        _ptr(sched_dev), ctypes.byref(info), total, hq, hkv, d,
        float(softmax_scale), _ptr(workspace), ws_bytes, _stream(stream)))


def triangle_attn_merge(o, lse, sched_dev, info, workspace, stream=None):
    """Enqueue the merge of the Last-row split partials into o / lse."""
    import torch
    _out_dtype(o)
    total, hq, d = o.shape
    named = [("o", o), ("sched_dev", sched_dev)]
    if lse is not None:
        named.append(("lse", lse))
        if lse.dtype != torch.float32 or tuple(lse.shape) != (hq, total):
            raise ValueError(f"lse must be float32 [{hq}, {total}]")
    if workspace is not None:
        named.append(("workspace", workspace))
    if sched_dev.dtype != torch.int32 or sched_dev.numel() != info.words:
        raise ValueError("sched_dev must hold the schedule's int32 words")
    for name, t in named:
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        if t.device != o.device:
            raise ValueError(f"{name} is on {t.device}, o on {o.device}")
    if o.device.type != "cuda":
        raise ValueError(f"operands must be on a GPU, got {o.device}")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().triangle_attn_merge(
        _ptr(o), _out_dtype(o), _ptr(lse), _ptr(sched_dev), ctypes.byref(info),
        total, hq, d, _ptr(workspace), ws_bytes, _stream(stream)))


def blocksparse_attn_fwd(q, k, v, o, lse, sched_dev, info, softmax_scale,
                         workspace, stream=None):
    """Enqueue block-sparse causal attention (tiles + merge)."""
    _check_tensors(q, k, v, o, lse, sched_dev, info, workspace)
    total, hq, d = q.shape
    hkv = k.shape[1]
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().blocksparse_attn_fwd(
        _ptr(q), _ptr(k), _ptr(v), _ptr(o), _out_dtype(o), _ptr(lse),
        _ptr(sched_dev), ctypes.byref(info), total, hq, hkv, d,
        float(softmax_scale), _ptr(workspace), ws_bytes, _stream(stream)))


def causal_attn_fwd(q, k, v, o, lse, sched_dev, info, softmax_scale,
                    stream=None):
    """Enqueue dense causal attention on ``stream``; arguments as above."""
    _check_tensors(q, k, v, o, lse, sched_dev, info)
    total, hq, d = q.shape
    hkv = k.shape[1]
    _check(lib().causal_attn_fwd(
        _ptr(q), _ptr(k), _ptr(v), _ptr(o), _out_dtype(o), _ptr(lse),
        _ptr(sched_dev), ctypes.byref(info), total, hq, hkv, d,
        float(softmax_scale), _stream(stream)))


def _launch(device, stream, fn, *args):
    """fn(*args, stream) with the GPU of the operands current, on its current
    stream if None; a stream of another GPU is refused.  (The stream's handle is
    asked for without building a Stream object: a microsecond of a call that
    enqueues one short kernel in eight.)"""
    import torch
    index = device.index
    if stream is None:
        handle = torch._C._cuda_getCurrentRawStream(index)
    elif stream.device != device:
        raise ValueError(f"stream is on {stream.device}, operands on {device}")
    else:
        handle = stream.cuda_stream
    if torch._C._cuda_getDevice() == index:
        status = fn(*args, handle)
    else:
        with torch.cuda.device(device):
            status = fn(*args, handle)
    if status != TA_OK:
        raise TriAttnError(status, ta_last_error())


def _check_operands(named, dev):
    """named: (name, tensor, dtype, shape or None: any)."""
    import torch
    tensor = torch.Tensor
    for name, t, dtype, shape in named:
        if (isinstance(t, tensor) and t.dtype is dtype and t.device == dev and t.is_contiguous()
                and (shape is None or t.shape == shape)):
            continue
        if not isinstance(t, tensor):
            raise ValueError(f"{name} must be a torch tensor")
        if t.dtype != dtype:
            raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
        if shape is not None and t.shape != shape:
            raise ValueError(f"{name} must be {shape}, got {tuple(t.shape)}")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        if t.device != dev:
            raise ValueError(f"{name} is on {t.device}, not on {dev}: all operands must be on "
                             "one device")


def _check_gpu(dev):
    if dev.type != "cuda":
        raise ValueError(f"operands must be on a GPU, got {dev}")


def _check_vector(name, t):
    if t.dim() != 1:
        raise ValueError(f"{name} must have one dimension, got {tuple(t.shape)}")


def _check_table(t, batch):
    if t.dim() != 2 or t.shape[0] != batch:
        raise ValueError(f"block_table must be ({batch}, pages), got {tuple(t.shape)}")


def _addr(t):
    return None if t is None else t.data_ptr()


def _nbytes(t):
    return 0 if t is None else t.numel() * t.element_size()


def scored_attn_fwd(q, k, v, o, lse, sched_dev, info, softmax_scale, softcap, slopes, workspace,
                    stream=None):
    """Enqueue prefill attention with modified scores over a schedule of any
    kind: softcap * tanh(x / softcap) where softcap is given, minus slopes[h]
    times the distance from key to row where slopes (float32 [Hq]) are.  Other
    arguments as triangle_attn_fwd."""
    _check_tensors(q, k, v, o, lse, sched_dev, info, workspace)
    total, hq, d = q.shape
    if slopes is not None:
        import torch
        _check_operands([("slopes", slopes, torch.float32, (hq,))], q.device)
    cap = 0.0 if softcap is None else float(softcap)
    _launch(q.device, stream, lib().scored_attn_fwd, q.data_ptr(), k.data_ptr(), v.data_ptr(),
            o.data_ptr(), _out_dtype(o), _addr(lse), sched_dev.data_ptr(), ctypes.byref(info),
            total, hq, k.shape[1], d, float(softmax_scale), cap, _addr(slopes), _addr(workspace),
            _nbytes(workspace))


# status bits of page_map (state[1])
MAP_NO_PAGES = 1
MAP_TABLE_WIDTH = 2
MAP_BAD_LENGTH = 4
MAP_SLOT_COUNT = 8
MAP_BAD_FREE = 16


def page_map(cached_lens, new_lens, block_table, free_pages, n_free, page_size, kv_lens, cu_new,
             slots, state, stream=None):
    """Enqueue the pages and slots of one step, all int32 cuda tensors.

    cached_lens, new_lens [B]: tokens that the requests hold and get;
    block_table [B, W]: gets the pages taken; free_pages [F] with its first
    n_free [1] entries free, taken from the end.  Outputs: kv_lens [B], cu_new
    [B + 1], slots [any length >= the new tokens; -1 behind the last] and
    state [2]: free pages left, and MAP_* status bits (0: done; otherwise
    nothing was taken and every slot is -1).  Nothing is read back to the host.
    """
    import torch
    i32 = torch.int32
    if not isinstance(cached_lens, torch.Tensor) or cached_lens.dim() != 1:
        raise ValueError("cached_lens must be a tensor [requests]")
    b, dev = cached_lens.shape[0], cached_lens.device
    _check_operands([("cached_lens", cached_lens, i32, (b,)), ("new_lens", new_lens, i32, (b,)),
                     ("block_table", block_table, i32, None), ("free_pages", free_pages, i32, None),
                     ("n_free", n_free, i32, (1,)), ("kv_lens", kv_lens, i32, (b,)),
                     ("cu_new", cu_new, i32, (b + 1,)), ("slots", slots, i32, None),
                     ("state", state, i32, (2,))], dev)
    _check_table(block_table, b)
    _check_vector("free_pages", free_pages)
    _check_vector("slots", slots)
    _check_gpu(dev)
    _launch(dev, stream, lib().ta_page_map, cached_lens.data_ptr(), new_lens.data_ptr(), b,
            int(page_size), block_table.data_ptr(), block_table.shape[1], free_pages.data_ptr(),
            free_pages.shape[0], n_free.data_ptr(), kv_lens.data_ptr(), cu_new.data_ptr(),
            slots.data_ptr(), slots.shape[0], state.data_ptr())


def _cache_shape(k_cache):
    import torch
    if not isinstance(k_cache, torch.Tensor) or k_cache.dim() != 4:
        raise ValueError("k_cache must be a tensor [pages, heads, page_size, head_dim]")
    return tuple(k_cache.shape)


def _cache_operands(torch, k_cache, v_cache, k_scale, v_scale):
    """Operands of a cache [pages, heads, page_size, head_dim]: bf16, or
    float8_e4m3fn with scales float8_e8m0fnu [pages, heads, page_size].  (The
    module is handed in: an import statement of its own costs a short call a
    quarter of a microsecond.)"""
    shape = _cache_shape(k_cache)
    if k_scale is None and v_scale is None:
        return shape, [("k_cache", k_cache, torch.bfloat16, shape),
                       ("v_cache", v_cache, torch.bfloat16, shape)]
    return shape, [("k_cache", k_cache, torch.float8_e4m3fn, shape),
                   ("v_cache", v_cache, torch.float8_e4m3fn, shape),
                   ("k_scale", k_scale, torch.float8_e8m0fnu, shape[:3]),
                   ("v_scale", v_scale, torch.float8_e8m0fnu, shape[:3])]


def _rows(torch, k, v):
    """Shape and (token, head) strides of k, v [tokens, heads, head_dim] bf16 of
    any token and head stride."""
    for name, t in (("k", k), ("v", v)):
        if not isinstance(t, torch.Tensor) or t.dtype != torch.bfloat16:
            raise ValueError(f"{name} must be a bfloat16 tensor")
        if t.dim() != 3:
            raise ValueError(f"{name} must be [tokens, heads, head_dim], got {tuple(t.shape)}")
    shape = k.shape
    if shape != v.shape:
        raise ValueError(f"k {tuple(shape)} and v {tuple(v.shape)} differ")
    total, heads, d = shape
    ks, kh, kd = k.stride()
    vs, vh, vd = v.stride()
    if d > 1 and (kd != 1 or vd != 1):
        raise ValueError(f"the last dimension of {'k' if kd != 1 else 'v'} must be contiguous")
    if v.device != k.device:
        raise ValueError(f"v is on {v.device}, k on {k.device}")
    # (the stride of a dimension of one says nothing)
    if total < 2:
        ks = vs = 0
    if heads < 2:
        kh = vh = 0
    return shape, (ks, kh, vs, vh)


def kv_cache_write(k, v, slots, k_cache, v_cache, stream=None, k_scale=None, v_scale=None):
    """Enqueue the write of k, v [T, Hkv, d] bf16 (views with any token and
    head stride that is a multiple of 8) into the slots [T] int32 of the caches
    [pages, Hkv, page_size, d] bf16.  Rows with a negative slot are skipped;
    the slots of one call are distinct.

    With k_scale and v_scale [pages, Hkv, page_size] float8_e8m0fnu the caches
    are float8_e4m3fn and the rows quantised, each with a scale of its own
    (kv_cache_write_q8).
    """
    import torch
    (total, hkv, d), strides = _rows(torch, k, v)
    dev = k.device
    shape, named = _cache_operands(torch, k_cache, v_cache, k_scale, v_scale)
    pages, ch, page_size, cd = shape
    if (ch, cd) != (hkv, d):
        raise ValueError(f"the caches have {ch} heads of {cd}, k has {hkv} of {d}")
    named.append(("slots", slots, torch.int32, (total,)))
    _check_operands(named, dev)
    _check_gpu(dev)
    if k_scale is None:
        _launch(dev, stream, lib().kv_cache_write, k.data_ptr(), v.data_ptr(),
                *strides, slots.data_ptr(), total, k_cache.data_ptr(),
                v_cache.data_ptr(), pages, hkv, page_size, d)
    else:
        _launch(dev, stream, lib().kv_cache_write_q8, k.data_ptr(), v.data_ptr(),
                *strides, slots.data_ptr(), total, k_cache.data_ptr(),
                k_scale.data_ptr(), v_cache.data_ptr(), v_scale.data_ptr(), pages, hkv, page_size,
                d)


def kv_cache_read(k_cache, v_cache, block_table, cu, k, v, starts=None, stream=None, k_scale=None,
                  v_scale=None):
    """Enqueue cached rows back into k, v [T, Hkv, d] bf16 (views with any
    token and head stride that is a multiple of 8): rows cu[b] .. cu[b + 1) get
    positions starts[b], starts[b] + 1, .. of request b.

    caches [pages, Hkv, page_size, d]: bf16, or float8_e4m3fn with k_scale,
    v_scale [pages, Hkv, page_size] float8_e8m0fnu; block_table [B, W], cu [B +
    1] and starts [B] (None: 0) int32.  Rows from cu[B] on are left as they are;
    rows that no page of the cache holds are NaN.
    """
    import torch
    (total, hkv, d), strides = _rows(torch, k, v)
    dev = k.device
    shape, named = _cache_operands(torch, k_cache, v_cache, k_scale, v_scale)
    pages, ch, page_size, cd = shape
    if (ch, cd) != (hkv, d):
        raise ValueError(f"the caches have {ch} heads of {cd}, k has {hkv} of {d}")
    if not isinstance(cu, torch.Tensor) or cu.dim() != 1 or cu.shape[0] < 1:
        raise ValueError("cu must be a tensor [requests + 1]")
    b = cu.shape[0] - 1
    i32 = torch.int32
    named += [("cu", cu, i32, (b + 1,)), ("block_table", block_table, i32, None)]
    if starts is not None:
        named.append(("starts", starts, i32, (b,)))
    _check_operands(named, dev)
    _check_table(block_table, b)
    _check_gpu(dev)
    rest = (block_table.data_ptr(), b, block_table.shape[1], cu.data_ptr(), _addr(starts),
            k.data_ptr(), v.data_ptr(), *strides, total, pages, hkv, page_size, d)
    if k_scale is None:
        _launch(dev, stream, lib().kv_cache_read, k_cache.data_ptr(), v_cache.data_ptr(), *rest)
    else:
        _launch(dev, stream, lib().kv_cache_read_q8, k_cache.data_ptr(), k_scale.data_ptr(),
                v_cache.data_ptr(), v_scale.data_ptr(), *rest)


def ta_paged_workspace_bytes(batch, total_tokens, ragged, prefix, hq, hkv, head_dim) -> int:
    return int(lib().ta_paged_workspace_bytes(batch, total_tokens, int(ragged), int(prefix), hq,
                                              hkv, head_dim))


def ta_paged_q8_workspace_bytes(batch, total_tokens, ragged, prefix, hq, hkv, head_dim) -> int:
    return int(lib().ta_paged_q8_workspace_bytes(batch, total_tokens, int(ragged), int(prefix), hq,
                                                 hkv, head_dim))


def paged_attn_fwd(q, k_cache, v_cache, o, lse, kv_lens, cu_q, block_table, prefix_pages,
                   prefix_len, softmax_scale, softcap, slopes, workspace, stream=None,
                   k_scale=None, v_scale=None):
    """Enqueue attention of q [T, Hq, d] over the caches [pages, Hkv,
    page_size, d], all bf16 (o bf16 or fp32).  With k_scale and v_scale [pages,
    Hkv, page_size] float8_e8m0fnu the caches are float8_e4m3fn (kv_cache_write)
    and the workspace is of >= ta_paged_q8_workspace_bytes bytes.

    kv_lens [B] int32: own keys of each request, this call's tokens among
    them; cu_q [B + 1] int32 or None (one row a request); block_table [B, W]
    int32; prefix_pages [>= ceil(prefix_len / page_size)] int32 and prefix_len:
    keys that come before every request's own (None and 0: none); lse [Hq, T]
    fp32 or None; softcap and slopes as scored_attn_fwd, or None; workspace
    uint8 of >= ta_paged_workspace_bytes bytes.
    """
    import torch
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError("q must be a tensor [tokens, heads, head_dim]")
    total, hq, d = q.shape
    dev = q.device
    if not isinstance(o, torch.Tensor):
        raise ValueError("o must be a torch tensor")
    out = _out_dtype(o)
    shape, caches = _cache_operands(torch, k_cache, v_cache, k_scale, v_scale)
    pages, hkv, page_size, cd = shape
    if cd != d:
        raise ValueError(f"the caches have head_dim {cd}, q {d}")
    if not isinstance(kv_lens, torch.Tensor) or kv_lens.dim() != 1:
        raise ValueError("kv_lens must be a tensor [requests]")
    b = kv_lens.shape[0]
    i32 = torch.int32
    named = [("q", q, torch.bfloat16, None), *caches, ("o", o, o.dtype, (total, hq, d)),
             ("kv_lens", kv_lens, i32, (b,)), ("block_table", block_table, i32, None)]
    if lse is not None:
        named.append(("lse", lse, torch.float32, (hq, total)))
    if cu_q is not None:
        named.append(("cu_q", cu_q, i32, (b + 1,)))
    elif total != b:
        raise ValueError(f"q has {total} rows for {b} requests of one each (pass cu_q)")
    prefix_len = int(prefix_len)
    if prefix_len < 0:
        raise ValueError(f"prefix_len {prefix_len} < 0")
    if prefix_len > 0:
        named.append(("prefix_pages", prefix_pages, i32, None))
    if workspace is not None:
        named.append(("workspace", workspace, workspace.dtype, None))
    if slopes is not None:
        named.append(("slopes", slopes, torch.float32, (hq,)))
    _check_operands(named, dev)
    _check_table(block_table, b)
    if prefix_len > 0:
        _check_vector("prefix_pages", prefix_pages)
    _check_gpu(dev)
    if prefix_len > 0 and prefix_pages.shape[0] * page_size < prefix_len:
        raise ValueError(f"{prefix_pages.shape[0]} prefix pages of {page_size} hold no "
                         f"{prefix_len} keys")
    if k_scale is None:
        fn, held = lib().paged_attn_fwd, (k_cache.data_ptr(), v_cache.data_ptr())
    else:
        fn = lib().paged_attn_fwd_q8
        held = (k_cache.data_ptr(), k_scale.data_ptr(), v_cache.data_ptr(), v_scale.data_ptr())
    _launch(dev, stream, fn, q.data_ptr(), *held, o.data_ptr(), out, _addr(lse),
            kv_lens.data_ptr(), _addr(cu_q), block_table.data_ptr(), b, block_table.shape[1],
            prefix_pages.data_ptr() if prefix_len > 0 else None, prefix_len, total, hq, hkv, d,
            pages, page_size, float(softmax_scale), 0.0 if softcap is None else float(softcap),
            _addr(slopes), _addr(workspace), _nbytes(workspace))


class PagedPlan:
    """The workspace of attention over a paged cache for calls of so many
    requests and query rows.  Lengths, tables and the prefix's length may
    change from call to call; calls that may overlap need plans of their own,
    and a captured call needs its plan as long as its graph."""

    def __init__(self, batch, total_tokens, hq, hkv, head_dim, prefix=False, ragged=False,
                 device="cuda", q8=False):
        """prefix: whether calls have a shared prefix; ragged: whether they
        give cu_q (otherwise every request has one row); q8: whether the caches
        hold 8 bits (k_scale and v_scale are then given)."""
        import torch
        size = ta_paged_q8_workspace_bytes if q8 else ta_paged_workspace_bytes
        nbytes = size(batch, total_tokens, ragged, prefix, hq, hkv, head_dim)
        self.workspace = (torch.empty(nbytes, dtype=torch.uint8, device=device)
                          if nbytes > 0 else None)

    def run(self, q, k_cache, v_cache, o, kv_lens, block_table, cu_q=None, prefix_pages=None,
            prefix_len=0, lse=None, softmax_scale=None, softcap=None, slopes=None, stream=None,
            k_scale=None, v_scale=None):
        if softmax_scale is None:
            softmax_scale = 1.0 / float(q.shape[-1]) ** 0.5
        paged_attn_fwd(q, k_cache, v_cache, o, lse, kv_lens, cu_q, block_table, prefix_pages,
                       prefix_len, softmax_scale, softcap, slopes, self.workspace, stream,
                       k_scale, v_scale)
        return o


def ta_probe_workspace_bytes(info: ScheduleInfo, hq: int) -> int:
    return int(lib().ta_probe_workspace_bytes(ctypes.byref(info), hq))


def region_grad_probe(q, k, v, dout, lse, sched_dev, info, softmax_scale, sink,
                      window, last, region_sums, workspace, stream=None):
    """Enqueue the region-contribution probe on ``stream``.

    q, dout [T, Hq, d], k/v [T, Hkv, d] bf16 cuda tensors; lse [Hq, T] fp32
    (the causal normaliser); sched_dev/info a causal schedule; region_sums
    float64 cuda tensor [Hq, 3] (streaming, middle, last) that receives the
    per-head sums of A_ij <dO_i, V_j>; workspace uint8 cuda tensor of >=
    ta_probe_workspace_bytes bytes or None.
    """
    import torch
    if lse is None:
        raise ValueError("the probe needs the causal LSE [Hq, T]")
    if not isinstance(dout, torch.Tensor) or dout.dtype != torch.bfloat16:
        raise ValueError(f"dout must be a bfloat16 tensor, got {getattr(dout, 'dtype', dout)}")
    _check_tensors(q, k, v, dout, lse, sched_dev, info, workspace,
                   extra=(("region_sums", region_sums, torch.float64, (q.shape[1], 3)),))
    total, hq, d = q.shape
    hkv = k.shape[1]
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().region_grad_probe(
        _ptr(q), _ptr(k), _ptr(v), _ptr(dout), _ptr(lse), _ptr(sched_dev),
        ctypes.byref(info), total, hq, hkv, d, float(softmax_scale), sink, window,
        last, _ptr(region_sums), _ptr(workspace), ws_bytes, _stream(stream)))


def ta_region_grad_workspace_bytes(info: ScheduleInfo, hq: int, hkv: int) -> int:
    return int(lib().ta_region_grad_workspace_bytes(ctypes.byref(info), hq, hkv))


def region_grad_sums(q, k, v, dout, sched_dev, info, softmax_scale, sink, window, last,
                     region_sums, workspace, stream=None):
    """Enqueue the region-contribution sums on ``stream`` without a given LSE.

    Arguments as region_grad_probe minus lse; workspace uint8 cuda tensor of
    >= ta_region_grad_workspace_bytes bytes or None.
    """
    import torch
    if not isinstance(dout, torch.Tensor) or dout.dtype != torch.bfloat16:
        raise ValueError(f"dout must be a bfloat16 tensor, got {getattr(dout, 'dtype', dout)}")
    _check_tensors(q, k, v, dout, None, sched_dev, info, workspace,
                   extra=(("region_sums", region_sums, torch.float64, (q.shape[1], 3)),))
    total, hq, d = q.shape
    hkv = k.shape[1]
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().region_grad_sums(
        _ptr(q), _ptr(k), _ptr(v), _ptr(dout), _ptr(sched_dev), ctypes.byref(info), total,
        hq, hkv, d, float(softmax_scale), sink, window, last, _ptr(region_sums),
        _ptr(workspace), ws_bytes, _stream(stream)))


def ta_region_counts(cu_seqlens, sink, window, last) -> np.ndarray:
    """Pairs per head in the (streaming, middle, last) sections."""
    cu = np.ascontiguousarray(np.asarray(cu_seqlens, dtype=np.int32))
    out = np.zeros(3, dtype=np.int64)
    _check(lib().ta_region_counts(cu.ctypes.data, cu.size - 1, sink, window, last,
                                  out.ctypes.data))
    return out


def ta_region_grad_mean(region_sums, counts) -> np.ndarray:
    """Grad per section from host per-head sums [Hq, 3] and the counts."""
    sums = np.ascontiguousarray(np.asarray(region_sums, dtype=np.float64))
    cnt = np.ascontiguousarray(np.asarray(counts, dtype=np.int64))
    assert sums.ndim == 2 and sums.shape[1] == 3 and cnt.shape == (3,)
    out = np.zeros(3, dtype=np.float64)
    _check(lib().ta_region_grad_mean(sums.ctypes.data, sums.shape[0], cnt.ctypes.data,
                                     out.ctypes.data))
    return out


def region_grad(q, k, v, dout, cu_seqlens, sink, window, last, tile=128,
                softmax_scale=None, stream=None):
    """Grad(M-hat, l) of one layer for the (streaming, middle, last)
    sections, and the per-head sums behind it: one pass sums A_ij <dO_i, V_j>
    per head and section, carrying each row's softmax normaliser along, and
    the library divides by Hq times the section's pair count.  Returns (grad
    [3], sums [Hq, 3]) as numpy float64; synchronises the stream to read
    them."""
    import torch
    total, hq, d = q.shape
    if softmax_scale is None:
        softmax_scale = 1.0 / float(d) ** 0.5
    plan = Plan("causal", cu_seqlens, 0, 1, 0, tile, hq, d, device=q.device)
    # (tensors and head counts that do not fit are refused by the call below)
    hkv = k.shape[1] if getattr(k, "ndim", 0) == 3 else 0
    nbytes = ta_region_grad_workspace_bytes(plan.info, hq, hkv)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=q.device) if nbytes else None
    sums = torch.empty((hq, 3), dtype=torch.float64, device=q.device)
    region_grad_sums(q, k, v, dout, plan.sched, plan.info, softmax_scale, sink, window,
                     last, sums, ws, stream)
    counts = ta_region_counts(cu_seqlens, sink, window, last)
    (stream or torch.cuda.current_stream()).synchronize()
    sums_host = sums.cpu().numpy()
    return ta_region_grad_mean(sums_host, counts), sums_host


def ta_select_triangle_layers(grad_middle, n_triangle) -> list:
    """The n_triangle layers with the smallest |Grad(middle)|, ascending."""
    g = np.ascontiguousarray(np.asarray(grad_middle, dtype=np.float64))
    out = np.zeros(max(int(n_triangle), 1), dtype=np.int32)
    _check(lib().ta_select_triangle_layers(g.ctypes.data if g.size else None, g.size,
                                           int(n_triangle), out.ctypes.data))
    return [int(x) for x in out[:int(n_triangle)]]


class Plan:
    """A schedule built once and uploaded to the device, plus its workspace.

    Buffers come from torch; the plan can be reused for every call with the
    same (cu_seqlens, sink, window, last, tile, splits, hq, head_dim).
    """

    def __init__(self, kind, cu_seqlens, sink, window, last, tile, hq,
                 head_dim, splits=0, device="cuda", blocks=None):
        """blocks: (qtile_ptr, ktile_idx) for kind "blocksparse" (splits is
        then the work bound per item)."""
        import torch
        self.kind = _kind(kind)
        if self.kind == BLOCKSPARSE:
            if blocks is None:
                raise ValueError("a block-sparse plan needs blocks=(qtile_ptr, ktile_idx)")
            self.words, self.info = ta_build_blocksparse_schedule(
                cu_seqlens, tile, blocks[0], blocks[1], splits)
        else:
            self.words, self.info = ta_build_schedule(self.kind, cu_seqlens, sink,
                                                      window, last, tile, splits)
        self.sched = torch.from_numpy(self.words).to(device)
        nbytes = ta_workspace_bytes(self.info, hq, head_dim)
        self.workspace = (torch.empty(nbytes, dtype=torch.uint8, device=device)
                          if nbytes > 0 else None)

    def run(self, q, k, v, o, lse=None, softmax_scale=None, stream=None, softcap=None,
            slopes=None):
        """softcap, slopes: modified scores (scored_attn_fwd); plain scores
        where neither is given (or softcap is 0)."""
        if softmax_scale is None:
            softmax_scale = 1.0 / float(q.shape[-1]) ** 0.5
        if softcap or slopes is not None:
            scored_attn_fwd(q, k, v, o, lse, self.sched, self.info, softmax_scale, softcap,
                            slopes, self.workspace, stream)
        elif self.kind == TRIANGLE:
            triangle_attn_fwd(q, k, v, o, lse, self.sched, self.info,
                              softmax_scale, self.workspace, stream)
        elif self.kind == BLOCKSPARSE:
            blocksparse_attn_fwd(q, k, v, o, lse, self.sched, self.info,
                                 softmax_scale, self.workspace, stream)
        else:
            causal_attn_fwd(q, k, v, o, lse, self.sched, self.info,
                            softmax_scale, stream)
        return o


def attention(kind, q, k, v, cu_seqlens, sink=0, window=1, last=0, tile=128,
              splits=0, softmax_scale=None, out_dtype=None, return_lse=False, softcap=None,
              slopes=None):
    """Allocate outputs with torch and run one pass (convenience wrapper)."""
    import torch
    out_dtype = out_dtype or torch.bfloat16
    plan = Plan(kind, cu_seqlens, sink, window, last, tile, q.shape[1],
                q.shape[2], splits, device=q.device)
    o = torch.empty(q.shape, dtype=out_dtype, device=q.device)
    lse = (torch.empty((q.shape[1], q.shape[0]), dtype=torch.float32,
                       device=q.device) if return_lse else None)
    plan.run(q, k, v, o, lse, softmax_scale, softcap=softcap, slopes=slopes)
    return (o, lse) if return_lse else o
