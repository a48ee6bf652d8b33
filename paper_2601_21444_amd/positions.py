"""Positions of queries and keys (include/apbv_positions.h): argument marshalling only, as binding.py for include/apbv.h; the plain
call is marshalled in native code there and here.  What a call that names a ``stream`` allocates is memory of that stream.

A program keeps an :class:`ApbvRotation` per layer (or one for all, where rows are not normed).  The prefill turns a block's queries and
keys with ``apbv_rotate``; a serving step turns its queries and puts its keys and values into the cache with ``apbv_cache_append``.
"""
from __future__ import annotations

import ctypes
import math
import operator
from typing import Optional, Sequence

import torch

from . import binding
from .binding import ApbvError, ApbvTensor, _check_buffer, _new, _stream_ptr, load_library, tensor_view
from .cache import ApbvCache, _cache_view, _check_ints, _rows_device

_NO_ROWS = ApbvTensor(None, 0, 0, 0, 0)


class ApbvRotationStruct(ctypes.Structure):
    """Mirror of ``apbv_rotation`` in include/apbv_positions.h."""
    _fields_ = [
        ("inv_freq", ctypes.c_void_p), ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p),
        ("eps", ctypes.c_float),
        ("rot_dim", ctypes.c_int32), ("n_axes", ctypes.c_int32), ("adjacent", ctypes.c_int32),
        ("axis", ctypes.c_uint8 * 64),
    ]


class ApbvRotation:
    """What is done with rows of ``head_dim`` elements; see apbv_rotation in include/apbv_positions.h.

    ``inv_freq [rot_dim / 2]`` float32: a frequency per pair.  ``axis``: the axis of the positions that each pair goes with (without it
    there is one).  ``adjacent``: pairs are neighbours, not ``rot_dim / 2`` elements apart.  ``q_weight``, ``k_weight`` ``[head_dim]``
    bf16: rows are normed with them first.  The memory of the tensors is kept, not copied: what is written into it later
    counts.  A tensor that is given other memory (a module's parameter, when the module is moved or cast) wants a new rotation."""

    def __init__(self, inv_freq: torch.Tensor, head_dim: int, *, axis: Optional[Sequence[int]] = None, adjacent: bool = False,
                 q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6):
        head_dim = operator.index(head_dim)
        if head_dim not in (64, 128):
            raise ValueError("head_dim is 64 or 128")
        if not isinstance(inv_freq, torch.Tensor) or inv_freq.dtype is not torch.float32:
            raise TypeError(f"inv_freq: expected a {torch.float32} tensor")
        if inv_freq.dim() != 1 or not inv_freq.is_contiguous():
            raise ValueError("inv_freq: expected a dense vector")
        pairs = inv_freq.numel()
        if pairs < 8 or 2 * pairs > head_dim or pairs % 8:
            raise ValueError(f"inv_freq: expected a multiple of 8 entries, {head_dim // 2} at most")
        axes = [0] * pairs if axis is None else [operator.index(a) for a in axis]
        if len(axes) != pairs or min(axes) < 0 or max(axes) > 3:
            raise ValueError(f"axis: expected {pairs} numbers from 0 to 3")
        for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
            if w is None:
                continue
            if not isinstance(w, torch.Tensor) or w.dtype is not torch.bfloat16:
                raise TypeError(f"{name}: expected a {torch.bfloat16} tensor")
            if tuple(w.shape) != (head_dim,) or not w.is_contiguous() or w.device != inv_freq.device or w.data_ptr() % 16:
                raise ValueError(f"{name}: expected a dense vector of {head_dim}, 16-byte aligned, on {inv_freq.device}")
        eps = float(eps)
        if not (eps >= 0.0 and math.isfinite(eps)):
            raise ValueError("eps: expected a finite number, not negative")
        # (tensors of its own on that memory: theirs may be replaced, which would free what the addresses below name)
        inv_freq, q_weight, k_weight = (None if t is None else t.detach() for t in (inv_freq, q_weight, k_weight))
        self.inv_freq, self.q_weight, self.k_weight, self.head_dim = inv_freq, q_weight, k_weight, head_dim
        self._made_of = (inv_freq, head_dim, axes, bool(adjacent), q_weight, k_weight, eps)
        self.n_axes, self.rot_dim, self.device = max(axes) + 1, 2 * pairs, inv_freq.device
        self._struct = ApbvRotationStruct(inv_freq.data_ptr(), *(w.data_ptr() if w is not None else None for w in (q_weight, k_weight)), eps,
                                          2 * pairs, self.n_axes, int(bool(adjacent)), (ctypes.c_uint8 * 64)(*axes))
        self._plan = (ctypes.addressof(self._struct), self.n_axes, head_dim, inv_freq.get_device())      # for the native marshalling

    def __reduce__(self):                                             # (a copy has an apbv_rotation of its own)
        return _rotation_of, self._made_of


def _rotation_of(inv_freq, head_dim, axis, adjacent, q_weight, k_weight, eps) -> ApbvRotation:
    return ApbvRotation(inv_freq, head_dim, axis=axis, adjacent=adjacent, q_weight=q_weight, k_weight=k_weight, eps=eps)


def _check_rotation(r: ApbvRotation, d: int, device: torch.device) -> None:
    if not isinstance(r, ApbvRotation):
        raise TypeError("rotation: expected an ApbvRotation")
    if r.head_dim != d:
        raise ValueError(f"rotation: of rows of {r.head_dim} elements, these have {d}")
    if r.device != device:
        raise ValueError(f"rotation: must live on {device}")


def _check_positions(t: torch.Tensor, n_axes: int, tokens: int, device: torch.device) -> int:
    """[tokens] (all axes the same) or [n_axes or more, tokens] -> distance of the axes."""
    if not isinstance(t, torch.Tensor) or t.dtype is not torch.int32:
        raise TypeError(f"positions: expected a {torch.int32} tensor")
    if not t.is_cuda or t.device != device:
        raise ValueError(f"positions: must live on {device}")
    if tuple(t.shape) != (tokens,) and (t.dim() != 2 or t.shape[1] != tokens or t.shape[0] < n_axes):
        raise ValueError(f"positions: expected [{tokens}] or [{n_axes}, {tokens}]")
    if tokens > 1 and t.stride(-1) != 1:
        raise ValueError("positions: tokens must be contiguous")
    return t.stride(0) if t.dim() == 2 else 0


def apbv_rotate(q: Optional[torch.Tensor], k: Optional[torch.Tensor], positions: torch.Tensor, rotation: ApbvRotation, *,
                q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """Norms and turns the rows of ``q [tokens, Hq, d]`` and ``k [tokens, Hkv, d]`` (either may be None) by ``positions``
    ``[tokens]`` or ``[axes, tokens]`` int32; see apbv_rotate in include/apbv_positions.h.  Returns ``(q_out, k_out)``, dense; an output
    may be its own input, where that is dense."""
    lib = load_library()
    if stream is None and type(rotation) is ApbvRotation:
        st = binding._native.rotate(q, k, positions, rotation._plan, q_out, k_out)
        if st is not None:
            if st != 0:
                raise ApbvError(st, "apbv_rotate")
            return q_out if q is not None else None, k_out if k is not None else None
    if q is None and k is None:
        raise ValueError("q and k: one of them is needed")
    one = k if q is None else q
    dev = _rows_device(one, "k" if q is None else "q", stream)
    if one.dim() != 3:
        raise ValueError("q, k: expected [tokens, heads, head_dim]")
    n, _, d = one.shape
    for name, t, out in (("q", q, q_out), ("k", k, k_out)):
        if t is None:
            continue
        if t.dim() != 3 or t.shape[0] != n or t.shape[2] != d or t.device != dev:
            raise ValueError(f"{name}: expected [{n}, heads, {d}] on {dev}")
        _check_buffer(out, name + "_out", torch.bfloat16, t.shape, dev)
    _check_rotation(rotation, d, dev)
    stride = _check_positions(positions, rotation.n_axes, n, dev)
    views = [_NO_ROWS if t is None else tensor_view(t)[0] for t in (q, k)]
    if q is not None and q_out is None:
        q_out = _new(q.shape, torch.bfloat16, dev, stream)
    if k is not None and k_out is None:
        k_out = _new(k.shape, torch.bfloat16, dev, stream)
    if q is None:
        q_out = None
    if k is None:
        k_out = None
    st = lib.apbv_rotate(q.shape[1] if q is not None else 0, k.shape[1] if k is not None else 0, d, ctypes.byref(rotation._struct), *views,
                         positions.data_ptr() if n else None, stride, q_out.data_ptr() if q_out is not None else None,
                         k_out.data_ptr() if k_out is not None else None, _stream_ptr(stream))
    if st != 0:
        raise ApbvError(st, "apbv_rotate")
    return q_out, k_out


def apbv_cache_append(cache: ApbvCache, q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor,
                      positions: torch.Tensor, rotation: ApbvRotation, *, q_out: Optional[torch.Tensor] = None,
                      stream: Optional[torch.cuda.Stream] = None):
    """A step's queries turned into ``q_out``, its keys (turned) and values written into the cache at ``slots [tokens]``; see
    apbv_cache_append in include/apbv_positions.h.  Returns ``q_out`` (None without ``q``)."""
    lib = load_library()
    if stream is None and type(cache) is ApbvCache and type(rotation) is ApbvRotation:
        st = binding._native.cache_append(cache, q, k, v, slots, positions, rotation._plan, q_out)
        if st is not None:
            if st != 0:
                raise ApbvError(st, "apbv_cache_append")
            return q_out if q is not None else None
    dev = _rows_device(k, "k", stream)
    view, heads, d = _cache_view(cache, dev)
    n = k.shape[0]
    views = []
    for name, t in (("k", k), ("v", v)):
        if t.dim() != 3 or tuple(t.shape) != (n, heads, d) or t.device != dev:
            raise ValueError(f"{name}: expected [tokens, {heads}, {d}] on {dev}")
        views.append(tensor_view(t)[0])
    if q is not None:
        if q.dim() != 3 or q.shape[0] != n or q.shape[2] != d or q.device != dev:
            raise ValueError(f"q: expected [{n}, heads, {d}] on {dev}")
        _check_buffer(q_out, "q_out", torch.bfloat16, q.shape, dev)
    _check_ints(slots, "slots", (n,), dev)
    _check_rotation(rotation, d, dev)
    stride = _check_positions(positions, rotation.n_axes, n, dev)
    qv = _NO_ROWS if q is None else tensor_view(q)[0]
    if q is None:
        q_out = None
    elif q_out is None:
        q_out = _new(q.shape, torch.bfloat16, dev, stream)
    st = lib.apbv_cache_append(ctypes.byref(view), q.shape[1] if q is not None else 0, heads, d, ctypes.byref(rotation._struct), qv, *views,
                               positions.data_ptr() if n else None, stride, slots.data_ptr() if n else None,
                               q_out.data_ptr() if q_out is not None else None, _stream_ptr(stream))
    if st != 0:
        raise ApbvError(st, "apbv_cache_append")
    return q_out
