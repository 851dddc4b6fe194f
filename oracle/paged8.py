"""Oracle for the paged cache in 8 bits: its definitions in 64 bits, block by block.

Test infrastructure only: imported by tests/, never by the product path.  Codes are bytes in [blocks, heads, place, D] arrays whatever their
strides on the device, scales [blocks, heads].
"""
from __future__ import annotations

import math

import numpy as np

LARGEST = {"e4m3": 448.0, "int8": 127.0}


def _e4m3():
    out = np.zeros(256)
    for c in range(128):
        e, m = c >> 3, c & 7
        out[c] = math.ldexp(m, -9) if e == 0 else math.ldexp(8 + m, e - 10)
    out[127] = np.nan
    out[128:] = -out[:128]
    return out


E4M3 = _e4m3()
_ORDER = E4M3[:127]      # of the codes without a sign, ascending


def values(codes, code):
    codes = np.asarray(codes)
    return E4M3[codes.view(np.uint8)] if code == "e4m3" else codes.view(np.int8).astype(np.float64)


def coded(y, code):
    """The codes nearest to y, as bytes; of two the one that is even (e4m3: whose last bit is 0).  NaN: 0x7f of e4m3."""
    y = np.asarray(y, np.float64)
    if code == "int8":
        return np.rint(y).astype(np.int8).view(np.uint8)
    a = np.minimum(np.abs(np.nan_to_num(y, nan=0.0)), 448.0)
    hi = np.clip(np.searchsorted(_ORDER, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = _ORDER[hi] - a, a - _ORDER[lo]
    c = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo).astype(np.uint8)
    c = np.where(np.isnan(y), np.uint8(127), c)
    return c | (np.signbit(y).astype(np.uint8) << 7)


def least_power(most, code):
    """The least e, -126 or more, with most <= largest code * 2^e."""
    if most == 0:
        return -126
    m, e = math.frexp(most / LARGEST[code])      # (exact: the largest code has few bits)
    e = e - 1 if math.ldexp(LARGEST[code], e - 1) >= most else e
    while math.ldexp(LARGEST[code], e) < most:
        e += 1
    return max(-126, e)


def cut(x, code, dtype, scale):
    """Numbers whose code over `scale` would stand for an infinity of dtype, cut to the largest that does not."""
    top = {"f16": 65504.0, "bf16": float(2.0**127 * (2 - 2.0**-7)), "f32": float(np.finfo(np.float32).max)}[dtype]
    grid = _ORDER if code == "e4m3" else np.arange(128.0)
    limit = max(v * scale for v in grid if v * scale <= top)
    return np.copysign(np.minimum(np.abs(x), limit), x)


def store(x, codes, scales, tables, lengths, starts, code, dtype):
    """-> codes, scales after x[T, H, D] were stored (the given ones are left alone)."""
    codes, scales = np.array(codes).view(np.uint8).copy(), np.array(scales, np.float64)
    blocks, heads, size, _ = codes.shape
    T = len(x)
    tables = np.asarray(tables, np.int64).reshape(len(lengths), -1) if len(lengths) else None
    for b in range(len(lengths)):
        n = min(max(int(lengths[b]), 0), tables.shape[1] * size)
        first, end = (min(max(int(s), 0), T) for s in (starts[b], starts[b + 1]))
        p0 = n - (end - first)
        begin = max(p0, 0)
        for j in range(begin // size, -(-n // size)):
            lo, hi = max(begin - j * size, 0), min(size, n - j * size)
            page = tables[b, j]
            if hi <= lo or not 0 <= page < blocks:
                continue
            rows = np.asarray(x[first + j * size + lo - p0:first + j * size + hi - p0], np.float64)
            for h in range(heads):
                here, before = rows[:, h], scales[page, h]
                bad = not np.isfinite(here).all()
                power = -126 if bad else least_power(np.abs(here).max(), code)
                if lo:
                    if not np.isfinite(before) or (before and math.ceil(math.log2(abs(before))) > 127):
                        bad = True
                    elif before:
                        m, e = math.frexp(abs(before))
                        power = max(power, e - 1 if m == 0.5 else e)
                if bad:
                    scales[page, h] = np.nan
                    codes[page, h, lo:hi] = 0
                    continue
                scale = math.ldexp(1.0, power)
                if lo and scale != before:
                    codes[page, h, :lo] = coded(values(codes[page, h, :lo], code) * (before / scale), code)
                codes[page, h, lo:hi] = coded(cut(here, code, dtype, scale) / scale, code)
                scales[page, h] = scale
    return codes, scales


def numbers(codes, scales, code):
    """What the codes of a cache stand for."""
    with np.errstate(invalid="ignore"):
        return values(codes, code) * np.asarray(scales, np.float64)[:, :, None, None]


def read(cache, tables, lengths, starts, T):
    """Rows [T, H, D] of a cache of numbers; None: nobody's (as a mask beside them)."""
    blocks, heads, size, dim = cache.shape
    out, mine = np.zeros((T, heads, dim)), np.zeros(T, bool)
    tables = np.asarray(tables, np.int64).reshape(len(lengths), -1) if len(lengths) else None
    for b in range(len(lengths)):
        n = min(max(int(lengths[b]), 0), tables.shape[1] * size)
        first, end = (min(max(int(s), 0), T) for s in (starts[b], starts[b + 1]))
        for t in range(first, end):
            mine[t] = True
            p = n - (end - t)
            page = tables[b, p // size] if p >= 0 else -1
            out[t] = cache[page, :, p % size] if 0 <= page < blocks else 0
    return out, mine
