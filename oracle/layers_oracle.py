"""The layer operators in plain numpy, 64 bits throughout: microscaled formats by
search among all values of their elements, a layer's products as matrix
products."""
from __future__ import annotations

import numpy as np

BLOCK = 32
NAN_SCALE = 255


def _grid(fmt: str) -> np.ndarray:
    """The non-negative values of the elements in order: a value's place is its code."""
    if fmt == "mxfp4":
        return np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    small = [m * 2.0 ** -9 for m in range(8)]
    return np.array(small + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:-1])


GRID = {f: _grid(f) for f in ("mxfp4", "mxfp8")}
LARGEST = {f: g[-1] for f, g in GRID.items()}


def scale_exponent(top: float, fmt: str) -> int:
    """The smallest s >= -127 with top <= LARGEST 2^s."""
    if top == 0:
        return -127
    _, e = np.frexp(top)
    s = int(e) - 12
    while top > np.ldexp(LARGEST[fmt], s):
        s += 1
    return max(s, -127)


def quantize(x, fmt: str):
    """(rows, cols) -> (codes (rows, blocks, 32) one per element, scales (rows,
    blocks)), both uint8; elements behind the last column are zeros."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    blocks = -(-cols // BLOCK)
    v = np.zeros((rows, blocks * BLOCK))
    v[:, :cols] = x
    v = v.reshape(rows, blocks, BLOCK)
    codes = np.zeros(v.shape, np.uint8)
    scales = np.zeros((rows, blocks), np.uint8)
    sign_bit = 8 if fmt == "mxfp4" else 128
    grid = GRID[fmt]
    mid = (grid[1:] + grid[:-1]) / 2
    for r in range(rows):
        for b in range(blocks):
            u = v[r, b]
            finite = np.isfinite(u)
            if fmt == "mxfp4" and not finite.all():
                scales[r, b] = NAN_SCALE
                continue
            a = np.where(finite, np.abs(u), 0.0)
            s = scale_exponent(a.max(), fmt)
            q = np.ldexp(a, -s)
            lo, hi = np.searchsorted(mid, q, side="left"), np.searchsorted(mid, q, side="right")
            c = np.where((lo != hi) & (hi % 2 == 1), lo, hi)       # a tie goes to the even code
            if fmt == "mxfp8":
                c = np.where((a > 0) & (c == 0), 1, c)
                c = np.where(finite, c, 127)
            codes[r, b] = (c + np.where(np.signbit(u) & finite, sign_bit, 0)).astype(np.uint8)
            scales[r, b] = s + 127
    return codes, scales


def pack(codes, fmt: str):
    """One code per element -> the bytes of a row."""
    rows = codes.shape[0]
    if fmt == "mxfp8":
        return codes.reshape(rows, -1)
    c = codes.reshape(rows, -1, 2)
    return (c[:, :, 0] | (c[:, :, 1] << 4)).astype(np.uint8)


def unpack(packed, fmt: str):
    rows = packed.shape[0]
    if fmt == "mxfp4":
        packed = np.stack([packed & 15, packed >> 4], 2)
    return packed.reshape(rows, -1, BLOCK)


def values(codes, scales, cols: int, fmt: str) -> np.ndarray:
    """What codes (one per element) and scales stand for."""
    n = len(GRID[fmt])
    table = np.concatenate([GRID[fmt], [np.nan] * (128 - n)]) if fmt == "mxfp8" else GRID[fmt]
    half = len(table)
    v = table[codes % half] * np.where(codes >= half, -1.0, 1.0)
    s = scales[:, :codes.shape[1]].astype(np.int64)
    v = np.ldexp(v, (s - 127)[:, :, None].astype(np.int32))
    v[s == NAN_SCALE] = np.nan
    return v.reshape(v.shape[0], -1)[:, :cols]


def half_step(v, scales, fmt: str) -> np.ndarray:
    """The most that rounding to an element may move each of the values v (rows,
    cols) in blocks with these scales."""
    v = np.abs(np.asarray(v, np.float64))
    rows, cols = v.shape
    s = np.repeat(scales.astype(np.int64) - 127, BLOCK, axis=1)[:, :cols].astype(np.int32)
    q = np.ldexp(v, -s)
    _, e = np.frexp(q)
    least, bits = (0, 1) if fmt == "mxfp4" else (-6, 3)       # exponent of the smallest normal, mantissa bits
    step = np.ldexp(1.0, np.maximum(e - 1, least) - bits)
    # an MXFP8 value below half the smallest element is moved up to it
    half = step / 2 if fmt == "mxfp4" else np.where(q < 2.0 ** -10, 2.0 ** -9, step / 2)
    return np.ldexp(half, s)


def linear(x, w, bias=None, relu=False):
    z = np.asarray(x, np.float64) @ np.asarray(w, np.float64).T
    if bias is not None:
        z = z + np.asarray(bias, np.float64)
    return np.where(z <= 0, 0.0, z) if relu else z


def linear_magnitude(x, w, bias=None):
    """The sum of the terms' magnitudes, which bounds every partial sum."""
    return linear(np.abs(x), np.abs(w), None if bias is None else np.abs(bias))


def backward(dz, x, w, relu=False):
    """(dx, dw, db) of z = x w^T + bias; relu: x is a ReLU's output and dx the
    gradient of its input."""
    dz, x, w = (np.asarray(v, np.float64) for v in (dz, x, w))
    dx = dz @ w
    return np.where(x != 0, dx, 0.0) if relu else dx, dz.T @ x, dz.sum(0)
