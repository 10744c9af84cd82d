"""Oracle of the e4m3 product with block scales and of the expert layer: numpy, 64 bits (test infrastructure).

Codes are e4m3 (bias 7, largest 448, no infinity, 0x7F / 0xFF = NaN).  Scales are stored [block of
columns][row] ("groups") or [block of rows][block of columns] ("blocks"), blocks of 128.  The quantizer's
arithmetic is binary32 by definition; everything behind it is computed in 64 bits.
"""
from __future__ import annotations

import numpy as np

BLOCK = 128
FLOOR = np.float32(2.0 ** -60)


def blocks_of(n: int) -> int:
    return -(-n // BLOCK)


def decode_table() -> np.ndarray:
    """The 256 values."""
    out = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = np.nan if (c & 0x7F) == 0x7F else (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
        out[c] = -v if c & 0x80 else v
    return out


_TABLE = decode_table()


def decode(codes: np.ndarray) -> np.ndarray:
    return _TABLE[codes]


def encode(y: np.ndarray) -> np.ndarray:
    """Nearest code (ties to the even mantissa, values beyond 448 saturate, NaN -> 0x7F) of float values."""
    y = np.asarray(y, dtype=np.float64)
    mag = np.abs(y)
    _, e = np.frexp(mag)
    step = np.ldexp(1.0, np.maximum(e - 4, -9))
    mag = np.minimum(np.where(np.isfinite(mag), np.round(np.where(np.isfinite(mag), mag, 0) / step) * step, 448.0), 448.0)
    codes = np.searchsorted(_TABLE[:127], mag).astype(np.uint8) | (np.signbit(y).astype(np.uint8) << 7)
    return np.where(np.isnan(y), np.uint8(0x7F), codes)


def scale_of(a: np.ndarray, pow2: bool):
    """(scale, inverse) in binary32 of block maxima."""
    with np.errstate(all="ignore"):
        a = np.maximum(a.astype(np.float32), FLOOR)            # NaN stays
        s = a / np.float32(448)
        if not pow2:
            return s, np.float32(448) / a
        bits = s.view(np.uint32)
        up = ((bits.astype(np.uint64) + 0x7FFFFF) & 0xFF800000).astype(np.uint32).view(np.float32)
        s = np.where(np.isnan(s), s, up)
        return s, np.float32(1) / s


def quantize(x: np.ndarray, blocks: bool = False, pow2: bool = False):
    """(codes [rows, cols], scales) of float32 values."""
    x = np.asarray(x, dtype=np.float32)
    rows, cols = x.shape
    rb, cb = blocks_of(rows), blocks_of(cols)
    h = BLOCK if blocks else 1
    pad = np.zeros(((rb * BLOCK if blocks else rows), cb * BLOCK), dtype=np.float32)
    pad[:rows, :cols] = x
    v = pad.reshape(-1, h, cb, BLOCK)
    s, inv = scale_of(np.abs(v).max(axis=(1, 3), keepdims=True), pow2)
    with np.errstate(all="ignore"):
        y = v * inv                                            # binary32
    q = encode(y).reshape(pad.shape)[:rows, :cols]
    s = s.reshape(-1, cb)
    return q, (s if blocks else np.ascontiguousarray(s.T))


def values(codes: np.ndarray, scales: np.ndarray, blocks: bool = False) -> np.ndarray:
    """What codes and scales stand for, in 64 bits."""
    rows, cols = codes.shape
    s = scales.astype(np.float64)
    s = np.repeat(s, BLOCK, axis=0)[:rows] if blocks else s.T[:rows]
    return decode(codes) * np.repeat(s, BLOCK, axis=1)[:, :cols]


def product(a, sa, b, sb, b_rows: bool = False):
    """(C, the sum of the terms' magnitudes) of codes and scales."""
    va, vb = values(a, sa), values(b, sb, blocks=not b_rows)
    return va @ vb.T, np.abs(va) @ np.abs(vb).T


def experts(a, sa, b, sb, starts, n: int):
    """(C, magnitudes) of the rows of every segment; rows outside are NaN (not written)."""
    va = values(a, sa)
    c = np.full((a.shape[0], n), np.nan)
    mag = np.zeros_like(c)
    for e in range(len(starts) - 1):
        lo, hi = starts[e], starts[e + 1]
        vb = values(b[e * n:(e + 1) * n], sb[e * blocks_of(n):(e + 1) * blocks_of(n)], blocks=True)
        c[lo:hi] = va[lo:hi] @ vb.T
        mag[lo:hi] = np.abs(va[lo:hi]) @ np.abs(vb).T
    return c, mag


def experts_wgrad(a, sa, b, sb, starts):
    va, vb = values(a, sa), values(b, sb)
    seg = [slice(starts[e], starts[e + 1]) for e in range(len(starts) - 1)]
    return (np.concatenate([va[:, s] @ vb[:, s].T for s in seg]),
            np.concatenate([np.abs(va[:, s]) @ np.abs(vb[:, s]).T for s in seg]))


def sort_rows(n: int, E: int, align: int) -> int:
    return (n + min(n, E) * (align - 1)) // align * align


def sort(ids: np.ndarray, E: int, align: int, rows: int):
    """(starts, source, slot) of the stable sort by expert number."""
    flat = ids.reshape(-1)
    starts = np.zeros(E + 1, dtype=np.int32)
    source = np.full(rows, -1, dtype=np.int32)
    slot = np.full(flat.size, -1, dtype=np.int32)
    at = 0
    for e in range(E):
        starts[e] = at
        mine = np.flatnonzero(flat == e)
        source[at:at + mine.size] = mine
        slot[mine] = np.arange(at, at + mine.size)
        at += -(-mine.size // align) * align
    starts[E] = at
    return starts, source, slot.reshape(ids.shape)


def gather(x, source, topk: int, w=None):
    out = np.zeros((source.size, x.shape[1]))
    has = source >= 0
    out[has] = x[source[has] // topk].astype(np.float64)
    if w is not None:
        out[has] *= w.reshape(-1)[source[has], None].astype(np.float64)
    return out


def combine(y, slot, w=None):
    out = np.zeros((slot.shape[0], y.shape[1]))
    for j in range(slot.shape[1]):
        has = slot[:, j] >= 0
        t = y[slot[has, j]].astype(np.float64)
        out[has] += t if w is None else t * w[has, j, None].astype(np.float64)
    return out


def combine_grad(dout, y, slot, w):
    """(dY, dw); rows of y that no pair takes get zeros."""
    dy, dw = np.zeros(y.shape), np.zeros(slot.shape)
    for j in range(slot.shape[1]):
        has = slot[:, j] >= 0
        d = dout[has].astype(np.float64)
        dy[slot[has, j]] = d if w is None else d * w[has, j, None].astype(np.float64)
        dw[has, j] = (d * y[slot[has, j]].astype(np.float64)).sum(1)
    return dy, dw
