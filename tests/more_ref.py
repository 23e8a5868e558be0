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
