"""Plain NumPy forms, in 64 bits, of rows held in 4 bits (e2m1, one power of two per
32 elements).  Written from the definition; nothing here is shared with the GPU path."""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
EXP_LOW, EXP_HIGH = -100, 125


def block_exponent(x):
    """Least e of EXP_LOW .. EXP_HIGH with max |x| <= 6 * 2^e, of blocks in the last axis; None stands for NaN (255)."""
    top = np.abs(x.astype(np.float64)).max(axis=-1)
    e = np.full(top.shape, EXP_LOW)
    for i in range(EXP_LOW, EXP_HIGH):
        e = np.where(top > 6.0 * 2.0 ** i, i + 1, e)
    return e


def codes_of(x):
    """Codes of the values next to x (|x| > 6: 6), ties to the even code, the sign in bit 3."""
    a = np.minimum(np.abs(x.astype(np.float64)), 6.0)
    d = np.abs(a[..., None] - GRID)
    near = d == d.min(axis=-1, keepdims=True)
    low = near.argmax(axis=-1)
    tie = near.sum(axis=-1) > 1
    return (np.where(tie & (low % 2 == 1), low + 1, low) + 8 * np.signbit(x)).astype(np.uint8)


def quantise(x):
    """(bytes [..][64], exponent bytes [..][4]) of rows of 128; a block that is not finite: 255 and code 0."""
    x = np.asarray(x).astype(np.float64)
    blocks = x.reshape(*x.shape[:-1], -1, 32)
    odd = ~np.isfinite(blocks).all(axis=-1)
    blocks = np.where(odd[..., None], 0.0, blocks)
    e = block_exponent(blocks)
    codes = codes_of(blocks * 2.0 ** -e[..., None].astype(np.float64)).reshape(x.shape)
    return codes[..., 0::2] | (codes[..., 1::2] << 4), np.where(odd, 255, e + 127).astype(np.uint8)


def values_of(packed, exps):
    """What rows stand for, in 64 bits."""
    codes = np.stack([packed & 15, packed >> 4], axis=-1).reshape(*packed.shape[:-1], -1)
    v = np.where(codes >= 8, -1.0, 1.0) * GRID[codes & 7]
    scale = np.where(exps == 255, np.nan, 2.0 ** (exps.astype(np.float64) - 127.0))
    return (v.reshape(*v.shape[:-1], -1, 32) * scale[..., None]).reshape(v.shape)


def held(x):
    """What rows of 128 stand for once they are held."""
    return values_of(*quantise(x))


# ---------------------------------------------------------------------------
# Pages: plain loops over the table
# ---------------------------------------------------------------------------
def fork(table, page, source=None, keep=None):
    out = np.full_like(table, -1)
    b, columns = table.shape
    for q in range(b):
        s = q if source is None else int(source[q])
        if not 0 <= s < b:
            continue
        for c in range(columns):
            if keep is None or c * page < int(keep[q]):
                out[q, c] = table[s, c]
    return out


def holders(table, num_pages):
    count = np.zeros(num_pages, int)
    for e in table.ravel():
        if 0 <= e < num_pages:
            count[e] += 1
    return count


def reserve(table, page, num_pages, rows, start=None, counts=None):
    """(out, pairs, totals, granted)."""
    b, columns = table.shape
    count = holders(table, num_pages)
    free = [p for p in range(num_pages) if count[p] == 0]
    out, pairs, granted, taken, wanted = table.copy(), [], np.zeros(b, int), 0, 0
    for q in range(b):
        s = 0 if start is None else int(start[q])
        n = rows if counts is None else min(max(int(counts[q]), 0), rows)
        lo, hi = max(s, 0), min(s + n, columns * page)
        need = []
        for c in range(lo // page, -(-hi // page)) if hi > lo else ():
            e = int(table[q, c])
            if not 0 <= e < num_pages:
                need.append((c, None))
            elif count[e] > 1:
                need.append((c, None if lo <= c * page and hi >= (c + 1) * page else e))
        wanted += len(need)
        if need and wanted > len(free):
            continue
        granted[q] = 1
        for c, e in need:
            out[q, c] = free[taken]
            if e is not None:
                pairs.append((e, free[taken]))
            taken += 1
    return out, pairs, (len(pairs), len(free) - taken), granted


def compact(table, num_pages):
    """(out, pairs, totals)."""
    used = holders(table, num_pages) > 0
    live = int(used.sum())
    away = [p for p in range(live, num_pages) if used[p]]
    to = [p for p in range(live) if not used[p]]
    place = dict(zip(away, to))
    out = np.array([[place.get(int(e), int(e)) if 0 <= e < num_pages else -1 for e in row] for row in table], np.int32)
    return out.reshape(table.shape), list(zip(away, to)), (len(away), live)


# ---------------------------------------------------------------------------
# Rotary positions
# ---------------------------------------------------------------------------
def frequencies(rot, base=10000.0, rule=0, factor=1.0, low=0.0, high=1.0, length=1):
    """Radians a position, in extended precision."""
    x = np.longdouble
    pi = x("3.14159265358979323846264338327950288")
    b = x(base)
    if rule == 2 and rot > 2:
        b = b * x(factor) ** (x(rot) / x(rot - 2))
    f = b ** (-x(2) * np.arange(rot // 2).astype(x) / x(rot))
    if rule == 1:
        f = f / x(factor)
    if rule == 3:
        s = np.clip((x(length) * f / (2 * pi) - x(low)) / (x(high) - x(low)), 0, 1)
        f = f * (s + (1 - s) / x(factor))
    return f


def rotate(x, positions, f, half, amplitude=1.0, inverse=False):
    """x [..][heads][d] of rows at `positions` [..], in 64 bits."""
    rot = 2 * len(f)
    angle = np.asarray(positions).astype(np.longdouble)[..., None] * f
    c, s = np.cos(angle).astype(float)[..., None, :], np.sin(angle).astype(float)[..., None, :]
    s = -s if inverse else s
    out = np.asarray(x, np.float64).copy()
    a, b = (out[..., :rot // 2].copy(), out[..., rot // 2:rot].copy()) if half else (out[..., 0:rot:2].copy(), out[..., 1:rot:2].copy())
    u, v = amplitude * (a * c - b * s), amplitude * (b * c + a * s)
    if half:
        out[..., :rot // 2], out[..., rot // 2:rot] = u, v
    else:
        out[..., 0:rot:2], out[..., 1:rot:2] = u, v
    return out
