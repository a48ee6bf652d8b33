"""Plain fp64 oracle of the 4-bit key/value cache (include/apbv_cache.h), written from its definitions: loops and tables, no
tiles, no sharing of work, no online softmax.  Test infrastructure only."""
from __future__ import annotations

import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
LARGEST_BF16 = float(np.uint32(0x7F7F0000).view(np.float32))


def encode(x):
    """float64 rows [..., d] of bf16 values -> (codes [..., d] of 0..15, scale bytes [..., d/32])."""
    x = np.where(np.isnan(x), 0.0, np.clip(x, -LARGEST_BF16, LARGEST_BF16))
    blocks = x.reshape(x.shape[:-1] + (x.shape[-1] // 32, 32))
    codes = np.zeros(blocks.shape, np.uint8)
    scales = np.zeros(blocks.shape[:-1], np.uint8)
    for i in np.ndindex(scales.shape):
        m = np.abs(blocks[i]).max()
        s = -125
        if m > 0:
            s = int(np.floor(np.log2(m))) - 2
            if m > 7.0 * 2.0 ** s:
                s += 1
            s = min(max(s, -125), 125)
        scales[i] = s + 127
        y = np.abs(blocks[i]) / 2.0 ** s
        dist = np.abs(y[:, None] - MAGNITUDES[None, :])
        near = dist == dist.min(1, keepdims=True)
        even = near & (np.arange(8) % 2 == 0)                    # of two magnitudes equally near the one with the even code
        code = np.where(even.any(1), even.argmax(1), near.argmax(1)).astype(np.uint8)
        codes[i] = code | (np.signbit(blocks[i]).astype(np.uint8) << 3)
    return codes.reshape(x.shape), scales


def decode(codes, scales):
    """The values that codes [..., d] and scale bytes [..., d/32] stand for."""
    v = np.where(codes & 8, -1.0, 1.0) * MAGNITUDES[codes & 7]
    return v * np.repeat(2.0 ** (scales.astype(np.float64) - 127.0), 32, axis=-1)


def pack(codes):
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def unpack(packed):
    return np.stack((packed & 15, packed >> 4), -1).reshape(packed.shape[:-1] + (2 * packed.shape[-1],))


def cache_map(old, new, table, free_pages, free_count, page, max_new):
    """One request after the other.  -> lengths, starts, slots, free_count; table and free_pages (lists) change in place."""
    n, cap, capacity = len(old), len(table[0]) * page, len(free_pages)
    blocks = lambda x: -(-x // page)
    old = [min(max(o, 0), cap) for o in old]
    count = min(max(free_count, 0), capacity)
    for b in range(n):
        if 0 <= new[b] < old[b]:
            for i in range(blocks(new[b]), blocks(old[b])):
                if count < capacity:
                    free_pages[count] = table[b][i]
                    count += 1
    lengths, starts, slots = list(old), [0], [-1] * max_new
    tokens = pages = taken = 0
    for b in range(n):
        grown = max(new[b] - old[b], 0)
        need = blocks(new[b]) - blocks(old[b]) if old[b] < new[b] <= cap else 0
        tokens, pages = tokens + grown, pages + need
        if 0 <= new[b] <= cap and (grown == 0 or (tokens <= max_new and (need == 0 or pages <= count))):
            lengths[b] = new[b]
            for i in range(need):
                table[b][blocks(old[b]) + i] = free_pages[count - 1 - taken]
                taken += 1
            for i in range(grown):
                pos = old[b] + i
                slots[tokens - grown + i] = table[b][pos // page] * page + pos % page
        starts.append(min(tokens, max_new))
    return lengths, starts, slots, count - taken


def attention(q, k, v, scale, causal):
    """One request: q [n, Hq, d], k and v [len, Hkv, d] float64 -> out, lse [Hq, n], and sum_j w_j |v_j| (for error bounds)."""
    n, hq, d = q.shape
    length, hkv, _ = k.shape
    group = hq // hkv
    out, spread, lse = np.zeros((n, hq, d)), np.zeros((n, hq, d)), np.full((hq, n), -np.inf)
    for h in range(hq):
        kh, vh = k[:, h // group], v[:, h // group]
        for i in range(n):
            seen = length - n + i + 1 if causal else length
            if seen <= 0:
                continue
            s = scale * (kh[:seen] @ q[i, h])
            w = np.exp(s - s.max())
            lse[h, i] = s.max() + np.log(w.sum())
            w /= w.sum()
            out[i, h] = w @ vh[:seen]
            spread[i, h] = w @ np.abs(vh[:seen])
    return out, lse, spread
