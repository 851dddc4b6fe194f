"""Oracle for the operators around a paged cache of keys and values: their definitions in 64 bits, request by request.

Test infrastructure only: imported by tests/, never by the product path.  Caches are given as [blocks, heads, place, D]
arrays whatever their strides on the device.
"""
from __future__ import annotations

import math

import numpy as np


def block_tables(cached, fresh, free, tables, tokens, blocks, block_size):
    """-> tables, lengths, starts, positions, slots, taken (the given tables are left alone)."""
    tables = np.array(tables, dtype=np.int64).reshape(len(cached), -1) if len(cached) else np.zeros((0, 0), np.int64)
    lengths, starts, used = [], [0], 0
    positions, slots = np.zeros(tokens, np.int64), np.full(tokens, -1, np.int64)
    for b in range(len(cached)):
        room = tables.shape[1] * block_size
        c = min(max(int(cached[b]), 0), room)
        n = min(max(int(fresh[b]), 0), room - c, tokens - starts[-1])
        have, need = -(-c // block_size), -(-(c + n) // block_size)
        for j in range(have, need):
            tables[b, j] = free[used] if used < len(free) else -1
            used += 1
        for i in range(n):
            p = c + i
            block = tables[b, p // block_size]
            positions[starts[-1] + i] = p
            if 0 <= block < blocks:
                slots[starts[-1] + i] = block * block_size + p % block_size
        lengths.append(c + n)
        starts.append(starts[-1] + n)
    return tables, np.array(lengths, np.int64), np.array(starts), positions, slots, np.array([min(used, len(free)), used])


def frequencies(rotary_dim, base=10000.0, factor=1.0, low=0.0, high=0.0, original=0.0):
    out = []
    for i in range(rotary_dim // 2):
        f = base ** (-2.0 * i / rotary_dim)
        waves = original * f / (2 * math.pi)          # how many fit into the original context
        keep = 0.0 if low == high == 0 else min(1.0, max(0.0, (waves - low) / (high - low)))
        out.append((1 - keep) * f / factor + keep * f)
    return out


def rotary(x, positions, freqs, interleaved=False, inverse=False, magnitude=1.0):
    """x[T, H, D] -> the same, its first 2 * len(freqs) elements of each head turned."""
    y = np.array(x, dtype=np.float64)
    n = len(freqs)
    a = np.asarray(positions, np.float64)[:, None, None] * np.asarray(freqs, np.float64)
    c, s = magnitude * np.cos(a), magnitude * np.sin(a) * (-1 if inverse else 1)
    i0, i1 = (np.arange(0, 2 * n, 2), np.arange(1, 2 * n, 2)) if interleaved else (np.arange(n), np.arange(n, 2 * n))
    x0, x1 = y[..., i0].copy(), y[..., i1].copy()
    y[..., i0], y[..., i1] = x0 * c - x1 * s, x1 * c + x0 * s
    return y


def stored(cache, rows, slots):
    """The cache with rows[t] in slot slots[t]; slots outside it are skipped."""
    cache = np.array(cache, dtype=np.float64)
    blocks, _, size, _ = cache.shape
    for t, s in enumerate(slots):
        if 0 <= s < blocks * size:
            cache[s // size, :, s % size] = rows[t]
    return cache


def seen_keys(n, position, row, block_size, blocks, causal, window):
    """The keys that the query at `position` sees of a request with n of them whose row of the table is `row`."""
    j = np.arange(n)
    ok = np.ones(n, bool)
    if causal:
        ok &= j <= position
    if window:
        ok &= j > position - window
    page = np.asarray(row, np.int64)[j // block_size] if n else j
    return j[ok & (page >= 0) & (page < blocks)]


def attention(q, k_cache, v_cache, tables, lengths, starts, scale, causal=True, window=0):
    """-> out [T, H, D], lse [T, H], weight [T, H, D] = sum_j softmax_j |v_j|, small [T, H, D] = sum_j |v_j| / sum_j exp(s_j - max s) and
    top [T, H], the largest of scale * sum_d |q_d k_jd|: what bounds of rounding errors are made of.  Rows of no request: NaN."""
    T, H, D = q.shape
    blocks, kv_heads, size, _ = k_cache.shape
    share = H // kv_heads
    out, weight, small = (np.full((T, H, D), np.nan) for _ in range(3))
    lse, top = np.full((T, H), np.nan), np.zeros((T, H))
    tables = np.asarray(tables, np.int64).reshape(len(lengths), -1) if len(lengths) else None
    for b in range(len(lengths)):
        n = min(max(int(lengths[b]), 0), tables.shape[1] * size)
        first, end = (min(max(int(s), 0), T) for s in (starts[b], starts[b + 1]))
        for t in range(first, end):
            j = seen_keys(n, n - (end - first) + t - first, tables[b], size, blocks, causal, window)
            for h in range(H):
                if len(j) == 0:
                    out[t, h], weight[t, h], small[t, h], lse[t, h] = 0, 0, 0, -np.inf
                    continue
                k = k_cache[tables[b, j // size], h // share, j % size].astype(np.float64)
                v = v_cache[tables[b, j // size], h // share, j % size].astype(np.float64)
                x = np.asarray(q[t, h], np.float64)
                s = scale * (k @ x)
                m = s.max()
                e = np.exp(s - m)
                out[t, h], weight[t, h], small[t, h] = e @ v / e.sum(), e @ np.abs(v) / e.sum(), np.abs(v).sum(0) / e.sum()
                lse[t, h] = m + np.log(e.sum())
                top[t, h] = (abs(scale) * (np.abs(k) @ np.abs(x))).max()
    return out, lse, weight, small, top
