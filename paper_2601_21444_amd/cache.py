"""The key/value cache held in 4 bits (include/apbv_cache.h): argument marshalling only, as binding.py for include/apbv.h; the
plain call is marshalled in native code there and here.  What a call that names a ``stream`` allocates is memory of that stream.

A serving program keeps, for all layers, the block table ``[requests, max_blocks]``, the requests' lengths and the list of free
pages, and an :class:`ApbvCache` per layer.  A step is ``apbv_cache_map`` once, then in every layer ``apbv_cache_store`` of the
new rows and ``apbv_cache_attention``; ``apbv_cache_load`` reads a cached prefix back as bf16.
"""
from __future__ import annotations

import ctypes
import operator
from typing import NamedTuple, Optional

import torch

from . import binding
from .binding import ApbvCacheStruct, ApbvError, _check_buffer, _new, _stream_ptr, load_library, tensor_view

CACHE_MAX_REQUESTS = 4096      # APBV_CACHE_MAX_REQUESTS of include/apbv_cache.h


class ApbvCache(NamedTuple):
    """The cache of one layer: codes ``[pages, KV heads, page_size, d/2]`` and scales ``[pages, KV heads, page_size, d/32]``, uint8.
    Pages may be strided (a slice of an allocation that holds several layers), alike for K and V; what lies inside one is dense."""
    k_codes: torch.Tensor
    v_codes: torch.Tensor
    k_scales: torch.Tensor
    v_scales: torch.Tensor

    @property
    def n_pages(self) -> int:
        return self.k_codes.shape[0]

    @property
    def n_kv_heads(self) -> int:
        return self.k_codes.shape[1]

    @property
    def page_size(self) -> int:
        return self.k_codes.shape[2]

    @property
    def head_dim(self) -> int:
        return self.k_codes.shape[3] * 2


def apbv_cache_empty(n_pages: int, n_kv_heads: int, head_dim: int, page_size: int = 64, *, device="cuda") -> ApbvCache:
    """A cache of uninitialised pages."""
    if page_size not in (16, 32, 64, 128, 256) or head_dim not in (64, 128):
        raise ValueError("page_size is 16, 32, 64, 128 or 256 and head_dim 64 or 128")

    def new(width):
        return torch.empty((n_pages, n_kv_heads, page_size, width), dtype=torch.uint8, device=device)
    return ApbvCache(new(head_dim // 2), new(head_dim // 2), new(head_dim // 32), new(head_dim // 32))


def _cache_view(cache: ApbvCache, device: torch.device):
    """(apbv_cache, KV heads, head_dim) of a cache whose tensors fit one another and live on `device`."""
    pages, heads, page, half = cache.k_codes.shape
    for name, t, width in (("k_codes", cache.k_codes, half), ("v_codes", cache.v_codes, half),
                           ("k_scales", cache.k_scales, half // 16), ("v_scales", cache.v_scales, half // 16)):
        if t.dtype is not torch.uint8:
            raise TypeError(f"{name}: expected a {torch.uint8} tensor")
        if t.device != device:
            raise ValueError(f"{name}: must live on {device}")
        if tuple(t.shape) != (pages, heads, page, width):
            raise ValueError(f"{name}: expected shape {(pages, heads, page, width)}")
        if t.numel() > 0 and (t.stride(3) != 1 or t.stride(2) != width or (heads > 1 and t.stride(1) != page * width)):
            raise ValueError(f"{name}: a page must be dense")
    c, s = cache.k_codes.stride(0), cache.k_scales.stride(0)
    if cache.v_codes.stride(0) != c or cache.v_scales.stride(0) != s:
        raise ValueError("K and V must have the same distance between pages")
    return ApbvCacheStruct(cache.k_codes.data_ptr(), cache.v_codes.data_ptr(), cache.k_scales.data_ptr(), cache.v_scales.data_ptr(),
                           pages, c, s, page), heads, half * 2


def _check_ints(t: torch.Tensor, name: str, shape, device: torch.device) -> None:
    if not isinstance(t, torch.Tensor) or t.dtype is not torch.int32:
        raise TypeError(f"{name}: expected a {torch.int32} tensor")
    if not t.is_cuda or t.device != device:
        raise ValueError(f"{name}: must live on {device}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: expected shape {tuple(shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")


def _check_table(t: torch.Tensor, n: int, device: torch.device):
    """Table [n, max_blocks] -> (stride of a row, max_blocks)."""
    if not isinstance(t, torch.Tensor) or t.dtype is not torch.int32:
        raise TypeError(f"block_table: expected a {torch.int32} tensor")
    if not t.is_cuda or t.device != device:
        raise ValueError(f"block_table: must live on {device}")
    if t.dim() != 2 or t.shape[0] != n or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError("block_table: expected [requests, max_blocks], blocks contiguous")
    return t.stride(0), t.shape[1]


def _rows_device(t: torch.Tensor, name: str, stream: Optional[torch.cuda.Stream]) -> torch.device:
    """The device of a call: a GPU, and that of the stream the call is enqueued on."""
    if not t.is_cuda:
        raise ValueError(f"{name}: must live on a GPU")
    on = torch.cuda.current_device() if stream is None else stream.device.index
    if t.device.index != on:
        raise ValueError(f"{name}: lives on {t.device}, the stream of the call on cuda:{on}")
    return t.device


def apbv_cache_map(old_lengths: torch.Tensor, new_lengths: torch.Tensor, block_table: torch.Tensor, free_pages: torch.Tensor,
                   free_count: torch.Tensor, page_size: int, max_new_tokens: int, *, lengths_out: Optional[torch.Tensor] = None,
                   starts_out: Optional[torch.Tensor] = None, slots_out: Optional[torch.Tensor] = None,
                   free_count_out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """Grows and shrinks every request from ``old_lengths`` to ``new_lengths``; see apbv_cache_map in include/apbv_cache.h.
    ``block_table`` and ``free_pages`` are updated in place.  Returns ``(lengths, starts, slots, free_count)``; ``lengths_out``
    may be ``old_lengths`` and ``free_count_out`` ``free_count``, which updates a step's state in place."""
    lib = load_library()
    if stream is None and lengths_out is not None and starts_out is not None and slots_out is not None and free_count_out is not None:
        st = binding._native.cache_map(old_lengths, new_lengths, block_table, free_pages, free_count, page_size, max_new_tokens,
                                       lengths_out, starts_out, slots_out, free_count_out)
        if st is not None:
            if st != 0:
                raise ApbvError(st, "apbv_cache_map")
            return lengths_out, starts_out, slots_out, free_count_out
    dev = _rows_device(old_lengths, "old_lengths", stream)
    n, max_new = old_lengths.numel(), operator.index(max_new_tokens)
    _check_ints(old_lengths, "old_lengths", (n,), dev)
    _check_ints(new_lengths, "new_lengths", (n,), dev)
    _check_ints(free_count, "free_count", (1,), dev)
    _check_ints(free_pages, "free_pages", (free_pages.numel(),), dev)
    stride, max_blocks = _check_table(block_table, n, dev)
    for name, t, size in (("lengths_out", lengths_out, n), ("starts_out", starts_out, n + 1), ("slots_out", slots_out, max(max_new, 0)),
                          ("free_count_out", free_count_out, 1)):
        _check_buffer(t, name, torch.int32, size, dev)

    def new(size):
        return _new(size, torch.int32, dev, stream)
    lengths_out = new(n) if lengths_out is None else lengths_out
    starts_out = new(n + 1) if starts_out is None else starts_out
    slots_out = new(max(max_new, 0)) if slots_out is None else slots_out
    free_count_out = new(1) if free_count_out is None else free_count_out
    st = lib.apbv_cache_map(n, operator.index(page_size), max_blocks, old_lengths.data_ptr(), new_lengths.data_ptr(), block_table.data_ptr(), stride,
                            free_pages.data_ptr() if free_pages.numel() else None, free_pages.numel(), free_count.data_ptr(), max_new,
                            lengths_out.data_ptr(), starts_out.data_ptr(), slots_out.data_ptr() if max_new > 0 else None,
                            free_count_out.data_ptr(), _stream_ptr(stream))
    if st != 0:
        raise ApbvError(st, "apbv_cache_map")
    return lengths_out, starts_out, slots_out, free_count_out


def apbv_cache_store(cache: ApbvCache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, *,
                     stream: Optional[torch.cuda.Stream] = None) -> ApbvCache:
    """Writes the rows ``k``, ``v`` ``[tokens, KV heads, d]`` into the cache at ``slots [tokens]``; see apbv_cache_store in
    include/apbv_cache.h.  Returns the cache."""
    lib = load_library()
    if stream is None and type(cache) is ApbvCache:
        st = binding._native.cache_store(cache, k, v, slots)
        if st is not None:
            if st != 0:
                raise ApbvError(st, "apbv_cache_store")
            return cache
    dev = _rows_device(k, "k", stream)
    view, heads, d = _cache_view(cache, dev)
    views = []
    for name, t in (("k", k), ("v", v)):
        if t.dim() != 3 or t.shape[1:] != (heads, d) or t.device != dev:
            raise ValueError(f"{name}: expected [tokens, {heads}, {d}] on {dev}")
        views.append(tensor_view(t)[0])
    _check_ints(slots, "slots", (k.shape[0],), dev)
    st = lib.apbv_cache_store(ctypes.byref(view), heads, d, *views, slots.data_ptr() if slots.numel() else None, _stream_ptr(stream))
    if st != 0:
        raise ApbvError(st, "apbv_cache_store")
    return cache


def apbv_cache_load(cache: ApbvCache, slots: torch.Tensor, *, k_out: Optional[torch.Tensor] = None, v_out: Optional[torch.Tensor] = None,
                    stream: Optional[torch.cuda.Stream] = None):
    """The rows at ``slots [tokens]`` as the bf16 values they stand for, ``(k, v)`` of ``[tokens, KV heads, d]``; see apbv_cache_load in
    include/apbv_cache.h."""
    lib = load_library()
    if stream is None and type(cache) is ApbvCache and k_out is not None and v_out is not None:
        st = binding._native.cache_load(cache, slots, k_out, v_out)
        if st is not None:
            if st != 0:
                raise ApbvError(st, "apbv_cache_load")
            return k_out, v_out
    dev = _rows_device(slots, "slots", stream)
    view, heads, d = _cache_view(cache, dev)
    n = slots.numel()
    _check_ints(slots, "slots", (n,), dev)
    _check_buffer(k_out, "k_out", torch.bfloat16, (n, heads, d), dev)
    _check_buffer(v_out, "v_out", torch.bfloat16, (n, heads, d), dev)
    if k_out is None:
        k_out = _new((n, heads, d), torch.bfloat16, dev, stream)
    if v_out is None:
        v_out = _new((n, heads, d), torch.bfloat16, dev, stream)
    st = lib.apbv_cache_load(ctypes.byref(view), heads, d, n, *(t.data_ptr() if n else None for t in (slots, k_out, v_out)), _stream_ptr(stream))
    if st != 0:
        raise ApbvError(st, "apbv_cache_load")
    return k_out, v_out


def apbv_cache_attention_workspace_bytes(n_requests: int, n_rows: int, n_q_heads: int, n_kv_heads: int, head_dim: int, max_q: int) -> int:
    return int(load_library().apbv_cache_attention_workspace_bytes(n_requests, n_rows, n_q_heads, n_kv_heads, head_dim, max_q))


def apbv_cache_attention(q: torch.Tensor, cache: ApbvCache, block_table: torch.Tensor, lengths: torch.Tensor, softmax_scale: float, *,
                         q_starts: Optional[torch.Tensor] = None, max_q: Optional[int] = None, causal: bool = True,
                         return_lse: bool = False, out: Optional[torch.Tensor] = None, lse_out: Optional[torch.Tensor] = None,
                         workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """Attention of the rows ``q [rows, Hq, d]`` of many requests over their cached keys; see apbv_cache_attention in
    include/apbv_cache.h.  Without ``q_starts`` every request has ``rows / requests`` rows (one: a decoding step); with it and
    without ``max_q`` a request is taken to have up to all of them, which takes single tokens two to three times as long.  Returns
    ``out [rows, Hq, d]`` bf16 (and ``lse [Hq, rows]`` fp32), the layouts of apbv_merge_lse."""
    lib = load_library()
    if stream is None and type(cache) is ApbvCache and out is not None and workspace is not None and not (return_lse and lse_out is None):
        st = binding._native.cache_attention(q, cache, block_table, lengths, softmax_scale, q_starts, max_q, causal, out, lse_out, workspace)
        if st is not None:
            if st != 0:
                raise ApbvError(st, "apbv_cache_attention")
            return (out, lse_out) if return_lse else out
    dev = _rows_device(q, "q", stream)
    view, heads, d = _cache_view(cache, dev)
    if q.dim() != 3 or q.shape[2] != d:
        raise ValueError(f"q: expected [rows, heads, {d}]")
    rows, hq, _ = q.shape
    n = lengths.numel()
    _check_ints(lengths, "lengths", (n,), dev)
    stride, max_blocks = _check_table(block_table, n, dev)
    if q_starts is not None:
        _check_ints(q_starts, "q_starts", (n + 1,), dev)
    if max_q is None:
        max_q = rows // max(n, 1) if q_starts is None else rows
    qv = tensor_view(q)[0]
    _check_buffer(out, "out", torch.bfloat16, (rows, hq, d), dev)
    _check_buffer(lse_out, "lse_out", torch.float32, (hq, rows), dev)
    _check_buffer(workspace, "workspace", torch.uint8, 0, dev)
    if out is None:
        out = _new((rows, hq, d), torch.bfloat16, dev, stream)
    if return_lse and lse_out is None:
        lse_out = _new((hq, rows), torch.float32, dev, stream)
    if workspace is None:
        workspace = _new(max(apbv_cache_attention_workspace_bytes(n, rows, hq, heads, d, max_q), 256), torch.uint8, dev, stream,
                         returned=False)
    st = lib.apbv_cache_attention(ctypes.byref(view), n, hq, heads, d, qv, block_table.data_ptr(), stride, max_blocks, lengths.data_ptr(),
                                  q_starts.data_ptr() if q_starts is not None else None, operator.index(max_q), int(bool(causal)),
                                  float(softmax_scale), out.data_ptr() if rows else None, lse_out.data_ptr() if lse_out is not None else None,
                                  workspace.data_ptr(), workspace.numel(), _stream_ptr(stream))
    if st != 0:
        raise ApbvError(st, "apbv_cache_attention")
    return (out, lse_out) if return_lse else out
