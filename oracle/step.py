"""The operators of a training step from their definitions, in 64 bits with numpy: what tests compare the kernels with.

Nothing here is shared with the product.  Matrices are float64 arrays; 8-bit values come as the numbers they stand for.
"""
from __future__ import annotations

import numpy as np

LARGEST = {"e4m3": 448.0, "e5m2": 57344.0}
# mantissa bits, exponent of the smallest normal number
_FORMAT = {"e4m3": (3, -6), "e5m2": (2, -14)}


def philox4x32(counter, key, rounds: int = 10):
    """Philox4x32 (Salmon, Moraes, Dror, Shaw, SC 2011): four arrays of 32-bit words as uint64, two key words."""
    c = [np.asarray(w, dtype=np.uint64) for w in counter]
    k = [int(w) for w in key]
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(rounds):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> half) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> half) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return c


def keep_mask(rows: int, cols: int, p: float, seed: int, offset: int):
    """(which elements are kept, the factor of those)"""
    t = round(p * 65536)
    groups = -(-cols // 8)
    r, g = np.meshgrid(np.arange(rows, dtype=np.uint64), np.arange(groups, dtype=np.uint64), indexing="ij")
    words = philox4x32([g, r, np.full_like(g, offset % 2 ** 32), np.full_like(g, offset // 2 ** 32)],
                       [seed % 2 ** 32, seed // 2 ** 32])
    bits = np.stack([w >> np.uint64(s) & np.uint64(0xFFFF) for w in words for s in (0, 16)], axis=-1)
    keep = bits.reshape(rows, groups * 8)[:, :cols] >= t
    return keep, (65536 / (65536 - t) if t < 65536 else 0.0)


def dropout(x, p, seed, offset):
    keep, scale = keep_mask(*x.shape, p, seed, offset)
    return np.where(keep, np.where(keep, x, 0.0) * scale, 0.0)


def norm_forward(x, residual, weight, eps, p, seed, offset):
    """(h, rstd, y)"""
    h = dropout(x, p, seed, offset)
    if residual is not None:
        h = h + residual
    rstd = 1 / np.sqrt((h * h).mean(axis=1) + eps)
    return h, rstd, h * rstd[:, None] * weight


def norm_backward(dy, dh, h, rstd, weight, p, seed, offset):
    """(dres, dx, dweight)"""
    xhat, g = h * rstd[:, None], dy * weight
    dres = rstd[:, None] * (g - xhat * (g * xhat).mean(axis=1, keepdims=True))
    if dh is not None:
        dres = dres + dh
    return dres, dropout(dres, p, seed, offset), (dy * xhat).sum(axis=0)


def round_to(x, fmt):
    """To the nearest value of an 8-bit format, ties to even; |x| at most the largest."""
    bits, low = _FORMAT[fmt]
    with np.errstate(invalid="ignore"):
        _, power = np.frexp(x)
        step = np.exp2(np.maximum(power - 1, low) - bits)
        return np.where(np.isfinite(x), np.rint(x / step) * step, np.nan)


def quantize(x, fmt, blocks: bool):
    """(8-bit values, biased exponents [rows or rows of blocks][blocks of columns])"""
    rows, cols = x.shape
    tall, wide = (128 if blocks else 1), 128
    up, left = -(-rows // tall), -(-cols // wide)
    q, e = np.empty_like(x), np.empty((up, left), dtype=np.int64)
    for i in range(up):
        for j in range(left):
            at = (slice(i * tall, (i + 1) * tall), slice(j * wide, (j + 1) * wide))
            most = np.abs(x[at]).max()
            if not np.isfinite(most):
                e[i, j], q[at] = 255, np.nan
                continue
            power = -126
            if most > 0:
                power = max(power, int(np.frexp(most / LARGEST[fmt])[1]) - 1)
                if most > LARGEST[fmt] * 2.0 ** power:
                    power += 1
            e[i, j], q[at] = power + 127, round_to(x[at] * 2.0 ** -power, fmt)
    return q, e


def words_of(e):
    """Exponents [rows][blocks] as the bytes [ceil(blocks / 4)][rows][4]; 127 behind the last block."""
    rows, blocks = e.shape
    out = np.full((-(-blocks // 4), rows, 4), 127, dtype=np.uint8)
    for b in range(blocks):
        out[b // 4, :, b % 4] = e[:, b]
    return out


def scaled(q, scales, blocks: bool):
    """The numbers that 8-bit values with scales stand for."""
    rows, cols = q.shape
    out = np.empty_like(q)
    for b in range(-(-cols // 128)):
        byte = scales[b // 4, :, b % 4].astype(np.float64)
        f = np.where(byte == 255, np.nan, np.exp2(byte - 127))
        out[:, b * 128:(b + 1) * 128] = q[:, b * 128:(b + 1) * 128] * np.repeat(f, 128 if blocks else 1)[:rows, None]
    return out


def product(a, a_scales, b, b_scales, b_blocks: bool):
    return scaled(a, a_scales, False) @ scaled(b, b_scales, b_blocks).T
