"""Attention of requests that share cached prefixes (include/apbv_shared.h): argument marshalling only, as binding.py for
include/apbv.h; the plain call is marshalled in native code there and here.  What a call that names a ``stream`` allocates is memory of
that stream.

A server that answers many questions about one video keeps the video's keys once, in pages that a row of a prefix table names, and the
questions' and answers' own keys in pages of their own requests (``apbv_cache_map``, ``apbv_cache_append``).
"""
from __future__ import annotations

import ctypes
import operator
from typing import Optional

import torch

from . import binding
from .binding import ApbvError, _check_buffer, _new, _stream_ptr, load_library, tensor_view
from .cache import ApbvCache, _cache_view, _check_ints, _check_table, _rows_device


def apbv_cache_shared_attention_workspace_bytes(n_groups: int, n_requests: int, n_rows: int, n_q_heads: int, n_kv_heads: int, head_dim: int,
                                                max_q: int) -> int:
    return int(load_library().apbv_cache_shared_attention_workspace_bytes(n_groups, n_requests, n_rows, n_q_heads, n_kv_heads, head_dim, max_q))


def apbv_cache_shared_attention(q: torch.Tensor, cache: ApbvCache, prefix_table: torch.Tensor, prefix_lengths: torch.Tensor,
                                block_table: torch.Tensor, lengths: torch.Tensor, softmax_scale: float, *,
                                group_starts: Optional[torch.Tensor] = None, q_starts: Optional[torch.Tensor] = None,
                                max_q: Optional[int] = None, causal: bool = True, return_lse: bool = False,
                                out: Optional[torch.Tensor] = None, lse_out: Optional[torch.Tensor] = None,
                                workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """Attention of the rows ``q [rows, Hq, d]`` of many requests over the prefix of their group and their own keys; see
    apbv_cache_shared_attention in include/apbv_shared.h.  ``prefix_table [groups, blocks]`` and ``prefix_lengths [groups]`` name the
    prefixes, ``group_starts [groups + 1]`` the first request of each group (without it all groups have equally many); the others are
    those of ``apbv_cache_attention``.  Returns ``out [rows, Hq, d]`` bf16 (and ``lse [Hq, rows]`` fp32)."""
    lib = load_library()
    if stream is None and type(cache) is ApbvCache and out is not None and workspace is not None and not (return_lse and lse_out is None):
        st = binding._native.cache_shared_attention(q, cache, prefix_table, prefix_lengths, block_table, lengths, softmax_scale, group_starts, q_starts,
                                                    max_q, causal, out, lse_out, workspace)
        if st is not None:
            if st != 0:
                raise ApbvError(st, "apbv_cache_shared_attention")
            return (out, lse_out) if return_lse else out
    dev = _rows_device(q, "q", stream)
    view, heads, d = _cache_view(cache, dev)
    if q.dim() != 3 or q.shape[2] != d:
        raise ValueError(f"q: expected [rows, heads, {d}]")
    rows, hq, _ = q.shape
    n, groups = lengths.numel(), prefix_lengths.numel()
    _check_ints(lengths, "lengths", (n,), dev)
    _check_ints(prefix_lengths, "prefix_lengths", (groups,), dev)
    stride, max_blocks = _check_table(block_table, n, dev)
    prefix_stride, max_prefix_blocks = _check_table(prefix_table, groups, dev, "prefix_table")
    if group_starts is not None:
        _check_ints(group_starts, "group_starts", (groups + 1,), dev)
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
        workspace = _new(max(apbv_cache_shared_attention_workspace_bytes(groups, n, rows, hq, heads, d, max_q), 256), torch.uint8, dev, stream,
                         returned=False)
    st = lib.apbv_cache_shared_attention(ctypes.byref(view), groups, n, hq, heads, d, qv, prefix_table.data_ptr(), prefix_stride, max_prefix_blocks,
                                         prefix_lengths.data_ptr(), group_starts.data_ptr() if group_starts is not None else None,
                                         block_table.data_ptr(), stride, max_blocks, lengths.data_ptr(),
                                         q_starts.data_ptr() if q_starts is not None else None, operator.index(max_q), int(bool(causal)),
                                         float(softmax_scale), out.data_ptr() if rows else None, lse_out.data_ptr() if lse_out is not None else None,
                                         workspace.data_ptr(), workspace.numel(), _stream_ptr(stream))
    if st != 0:
        raise ApbvError(st, "apbv_cache_shared_attention")
    return (out, lse_out) if return_lse else out
