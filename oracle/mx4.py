"""4-bit rows with a power of two for each block of 32 columns, in float64.

Each block: e = the least whole number >= -127 with max |x| <= 6 2^e; a code is
the nearest of {0, 0.5, 1, 1.5, 2, 3, 4, 6} to |x| 2^-e, ties to the one whose
place in that list is even; the value is the code times 2^e. A block that is
not finite has NaN for a scale. Layout of codes and scales: include/dstd.h.
"""

import numpy as np

BLOCK = 32
LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def blocks_of(cols):
    return -(-cols // BLOCK)


def scale_bytes(rows, cols):
    return -(-rows // 128) * -(-blocks_of(cols) // 4) * 512


def scale_place(r, b, cols):
    """Byte of the scale of block b of row r."""
    tiles = -(-blocks_of(cols) // 4)
    return ((r // 128) * tiles + b // 4) * 512 + (r % 32) * 16 + (r % 128 // 32) * 4 + b % 4


def round_block(x):
    """(codes 0..15, exponent or None) of up to 32 numbers."""
    x = np.asarray(x, np.float64)
    top = np.abs(x).max() if x.size else 0.0
    if not np.isfinite(x).all():
        return np.zeros(x.size, int), None
    e = -127
    while top > 6.0 * 2.0 ** e:
        e += 1
    d = np.abs(np.abs(x)[:, None] * 2.0 ** -e - LEVELS[None, :])
    near = d.argmin(1)
    tie = (near < 7) & (d[np.arange(x.size), np.minimum(near + 1, 7)] == d[np.arange(x.size), near]) & (near % 2 == 1)
    code = near + tie
    return code + 8 * np.signbit(x), e


def quantize(x):
    """(codes [R, K], exponents [R, blocks] with NaN for blocks that are not finite, values [R, K])."""
    x = np.asarray(x, np.float64)
    R, K = x.shape
    codes, e = np.zeros((R, K), int), np.zeros((R, blocks_of(K)))
    for r in range(R):
        for b in range(blocks_of(K)):
            c, k = round_block(x[r, b * BLOCK:(b + 1) * BLOCK])
            codes[r, b * BLOCK:(b + 1) * BLOCK] = c
            e[r, b] = np.nan if k is None else k
    return codes, e, value_of(codes, e)


def value_of(codes, e):
    sign = 1.0 - 2.0 * (codes >= 8)
    return sign * LEVELS[codes % 8] * np.repeat(2.0 ** e, BLOCK, axis=1)[:, :codes.shape[1]]


def pack(codes, e):
    """Bytes of rows of codes, and of their scales."""
    R, K = codes.shape
    n = blocks_of(K)
    q = np.zeros((R, n * BLOCK), np.uint8)
    q[:, :K] = codes
    scale = np.zeros(scale_bytes(R, K), np.uint8)
    for r in range(R):
        for b in range(n):
            scale[scale_place(r, b, K)] = 255 if np.isnan(e[r, b]) else int(e[r, b]) + 127
    return q[:, 0::2] | q[:, 1::2] << 4, scale


def unpack(q, scale, K):
    """Codes and exponents of bytes."""
    q = np.asarray(q)
    R, n = q.shape[0], blocks_of(K)
    codes = np.zeros((R, q.shape[1] * 2), int)
    codes[:, 0::2], codes[:, 1::2] = q & 15, q >> 4
    r, b = np.arange(R)[:, None], np.arange(n)[None, :]
    byte = np.asarray(scale)[scale_place(r, b, K)].astype(np.float64)
    return codes[:, :K], np.where(byte == 255, np.nan, byte - 127)
