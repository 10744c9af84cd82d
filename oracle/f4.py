"""Oracle of the 4-bit float (e2m1) products with microscales and of the expert layer: numpy, 64 bits (test infrastructure).

Codes are two per byte, low half = even column.  A scale belongs to 32 columns (a power of two, byte - 127, 255 = NaN)
or, by16, to 16 columns (e4m3); four scales of a row make a word, stored [word][row].  The quantizer's arithmetic is
binary32 by definition; everything behind it is computed in 64 bits.
"""
from __future__ import annotations

import numpy as np

from . import f8

FLOOR = np.float32(2.0 ** -60)
LARGEST = np.finfo(np.float32).max
MAGNITUDES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
_VALUES = np.concatenate([MAGNITUDES, -MAGNITUDES])


def group_of(by16: bool) -> int:
    return 16 if by16 else 32


def words_of(cols: int, by16: bool) -> int:
    return -(-cols // (4 * group_of(by16)))


def encode(y: np.ndarray) -> np.ndarray:
    """Nearest code (ties to the even code, magnitudes beyond 6 saturate)."""
    y = np.asarray(y, dtype=np.float64)
    m = np.minimum(np.abs(y), 6.0)
    step = np.where(m < 2, 0.5, np.where(m < 4, 1.0, 2.0))
    near = np.round(m / step) * step
    return np.searchsorted(MAGNITUDES, near).astype(np.uint8) | (np.signbit(y).astype(np.uint8) << 3)


def pack(codes: np.ndarray) -> np.ndarray:
    rows, cols = codes.shape
    c = np.zeros((rows, (cols + 1) // 2 * 2), dtype=np.uint8)
    c[:, :cols] = codes
    return c[:, 0::2] | (c[:, 1::2] << 4)


def unpack(packed: np.ndarray, cols: int) -> np.ndarray:
    return np.stack([packed & 15, packed >> 4], axis=2).reshape(packed.shape[0], -1)[:, :cols]


def scale_value(byte: np.ndarray, by16: bool) -> np.ndarray:
    if by16:
        return f8.decode(byte & 0x7F)
    return np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127))


def to_words(byte: np.ndarray) -> np.ndarray:
    """[rows][groups] bytes to [word][row]."""
    rows, n = byte.shape
    b = np.zeros((rows, -(-n // 4) * 4), dtype=np.uint8)
    b[:, :n] = byte
    return np.ascontiguousarray(b.view("<u4").T)


def from_words(words: np.ndarray, rows: int) -> np.ndarray:
    return np.ascontiguousarray(words[:, :rows].T).astype("<u4").view(np.uint8)


def quantize(x: np.ndarray, by16: bool = False, factor=None):
    """(packed codes [rows, ceil(cols / 2)], words of scales) of float32 values."""
    x = np.asarray(x, dtype=np.float32)
    rows, cols = x.shape
    g = group_of(by16)
    n = -(-cols // g)
    v = np.zeros((rows, n * g), dtype=np.float32)
    v[:, :cols] = x
    v = v.reshape(rows, n, g)
    with np.errstate(all="ignore"):
        a = np.abs(v).max(axis=2)
        if by16:
            r = np.minimum(np.float32(1) / np.float32(1 if factor is None else factor), LARGEST)      # (NaN stays)
            byte = np.maximum(f8.encode(a * (r / np.float32(6))), 1)
            byte = np.where(np.isfinite(a), byte, 0x7F).astype(np.uint8)
            inv = np.minimum(r / f8.decode(byte).astype(np.float32), LARGEST)
        else:
            m, e = np.frexp(np.maximum(a, FLOOR).astype(np.float64) / 6)
            e = np.where(m == 0.5, e - 1, e)                   # 2^e is the next power of two
            byte = np.where(np.isfinite(a), e + 127, 255).astype(np.uint8)
            inv = np.where(np.isfinite(a), 2.0 ** -e.astype(np.float64), 0).astype(np.float32)
        y = v * inv[:, :, None]                                # binary32
    return pack(encode(y).reshape(rows, -1)[:, :cols]), to_words(byte)


def values(packed, words, cols: int, by16: bool = False, factor=None):
    """What codes and scales stand for, in 64 bits."""
    rows = packed.shape[0]
    n = -(-cols // group_of(by16))
    s = scale_value(from_words(words, rows)[:, :n], by16)
    v = _VALUES[unpack(packed, cols)] * np.repeat(s, group_of(by16), axis=1)[:, :cols]
    return v if factor is None else v * np.float64(factor)


def product(a, b):
    """(C, the sum of the terms' magnitudes) of two matrices of values."""
    return a @ b.T, np.abs(a) @ np.abs(b).T


def experts(a, b, starts, n: int):
    """(C, magnitudes) of the rows of every segment; rows outside are NaN (not written).  b: values [E * n, K]."""
    c = np.full((a.shape[0], n), np.nan)
    mag = np.zeros_like(c)
    for e in range(len(starts) - 1):
        lo, hi = starts[e], starts[e + 1]
        c[lo:hi], mag[lo:hi] = product(a[lo:hi], b[e * n:(e + 1) * n])
    return c, mag


def entered(v, by16=None):
    """How far from itself a value of a row of activations may enter the layer's products: 2^-20 of the largest of its group
    or, by 16, 2^-37 of the row's largest where that is more; 2^-144 where these are less.  None: the more of both kinds."""
    if by16 is None:
        return np.maximum(entered(v, False), entered(v, True))
    group = group_of(by16)
    m = np.zeros(-(-v.size // group) * group)
    m[:v.size] = np.abs(v)
    largest = np.repeat(m.reshape(-1, group).max(axis=1), group)[:v.size]
    return np.maximum(largest * 2.0 ** -20, m.max() * 2.0 ** -37 if by16 else 0) + 2.0 ** -144


def layer(x, ids, w, w1, w2, gated: bool, by16=None):
    """(Out, how far a binary32 evaluation may be off, before the last rounding).  w1 [E, up * H, D], w2 [E, D, H] values.

    Counted: one last place (2^-23 of the magnitudes: an addition may cut) per term of a sum; silu's slope is at most
    1.1 and its own evaluation 8 last places; what values of x and hidden values may be off when they enter a product (`entered`).
    """
    E, D, H = w2.shape
    out, off = np.zeros(x.shape), np.zeros(x.shape)
    last = 2.0 ** -23
    for t in range(ids.shape[0]):
        for j in range(ids.shape[1]):
            e = ids[t, j]
            if e < 0 or e >= E:
                continue
            p = 1.0 if w is None else float(w[t, j])
            up, mag = w1[e] @ x[t], np.abs(w1[e]) @ np.abs(x[t])
            err = (D + 4) * last * mag + np.abs(w1[e]) @ entered(x[t], by16)
            g, ge = up[:H], err[:H]
            with np.errstate(over="ignore"):
                s = g / (1 + np.exp(-g))
            u, ue = (up[H:], err[H:]) if gated else (np.ones(H), np.zeros(H))
            h = s * u
            he = 1.1 * ge * (np.abs(u) + ue) + np.abs(s) * ue + np.abs(h) * 8 * last
            he += entered(np.abs(h) + he, by16)
            out[t] += p * (w2[e] @ h)
            off[t] += abs(p) * (np.abs(w2[e]) @ (he + (H + ids.shape[1] + 4) * last * np.abs(h)))
    return out, off
