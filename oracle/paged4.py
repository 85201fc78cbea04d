"""Rows of a 4-bit pool in 64 bits, from the definition: blocks of 32 values, each a code of a sign and one of eight
magnitudes under the block's power of two.  NumPy."""
from __future__ import annotations

import numpy as np

D, ROW = 128, 68
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
RANGE = {"bf16": (-120, 125), "fp16": (-14, 13)}  # of a scale's exponent
NONE = 255  # scale byte of a block that is not finite


def exponent(top, dtype):
    """The least e with top <= 7 2^e, cut to the type's range."""
    lo, hi = RANGE[dtype]
    e = np.full(np.shape(top), lo, np.int64)
    for _ in range(hi - lo):
        more = (top > np.ldexp(7.0, e)) & (e < hi)
        if not more.any():
            break
        e += more
    return e


def encode(x, dtype):
    """x [..., 128] -> codes uint8 [..., 64], scale bytes uint8 [..., 4]."""
    b = np.asarray(x, np.float64).reshape(*np.shape(x)[:-1], 4, 32)
    finite = np.isfinite(b).all(-1)
    b = np.where(finite[..., None], b, 0.0)
    e = exponent(np.abs(b).max(-1), dtype)
    y = np.ldexp(np.abs(b), -e[..., None])
    mid = (GRID[1:] + GRID[:-1]) / 2
    code = np.zeros(y.shape, np.uint8)
    for i, m in enumerate(mid):  # a tie between codes i and i + 1 goes to the even one
        code += (y > m) | ((y == m) & (i % 2 == 1))
    code |= (np.signbit(b).astype(np.uint8) << 3)
    code = np.where(finite[..., None], code, 0).astype(np.uint8).reshape(*np.shape(x)[:-1], D)
    return code[..., 0::2] | code[..., 1::2] << 4, np.where(finite, e + 127, NONE).astype(np.uint8)


def decode(codes, scales):
    """The values, in 64 bits."""
    c = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], D)
    x = np.where(c & 8, -GRID[c & 7], GRID[c & 7]).reshape(*codes.shape[:-1], 4, 32)
    scale = np.where(scales == NONE, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return (x * scale[..., None]).reshape(*codes.shape[:-1], D)


def pool(x, dtype):
    """Rows [..., page, 128] -> bytes [..., page * 68]."""
    codes, scales = encode(x, dtype)
    return np.concatenate([codes.reshape(*codes.shape[:-2], -1), scales.reshape(*scales.shape[:-2], -1)], -1)


def rows(data, page):
    """Bytes [..., page * 68] -> (codes [..., page, 64], scales [..., page, 4])."""
    return (data[..., :64 * page].reshape(*data.shape[:-1], page, 64),
            data[..., 64 * page:].reshape(*data.shape[:-1], page, 4))
