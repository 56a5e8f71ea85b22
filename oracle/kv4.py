"""The 4-bit key-value cache, in float64.  TEST INFRASTRUCTURE ONLY (nothing on the product path
imports this).

32 neighbouring dimensions of a cached row are kept as an exponent and multiples of its power of
two: with a the largest magnitude among them, e is the least integer from -60 to 125 with
a <= 7 2^e, and the multiples are the nearest to x 2^-e among 0, 0.5, 1, 1.5, 2, 3, 4 and 6 with
either sign, ties to the one at an even place of that list.  A row that is not finite is all NaN.
"""

from __future__ import annotations

import numpy as np

KV4_CODES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def kv4_quantise(x):
    """(codes 0 .. 15 [..., hd], scale bytes [..., hd / 32]) of float32 rows x."""
    x = np.asarray(x, np.float64)
    g = x.reshape(*x.shape[:-1], -1, 32)
    ok = np.isfinite(x).all(-1)[..., None]
    a = np.where(ok, np.abs(g).max(-1, initial=0.0), 0.0)
    e = np.full(a.shape, -60)
    for i in range(-60, 126):
        e = np.where(a > 7.0 * 2.0 ** e, i, e)
    mult = np.abs(np.where(ok[..., None], g, 0.0)) / 2.0 ** e[..., None].astype(np.float64)
    far = np.abs(mult[..., None] - KV4_CODES)
    # the nearest, of two as near the even place
    near = far.min(-1, keepdims=True)
    place = np.where(far == near, np.arange(8) + 8 * (np.arange(8) % 2), 99).argmin(-1)
    code = np.where(ok[..., None], place + 8 * np.signbit(g), 0)
    return (code.reshape(x.shape).astype(np.uint8), np.where(ok, e + 127, 255).astype(np.uint8))


def kv4_values(x):
    """The float64 values that the cache holds for rows x."""
    code, byte = kv4_quantise(x)
    mult = np.where(code >= 8, -1.0, 1.0) * KV4_CODES[code & 7]
    scale = np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127))
    return mult * np.repeat(scale, 32, -1)


def kv4_block(rows):
    """The bytes of one block from its page's rows [page, hd], keys and values."""
    code, byte = kv4_quantise(rows)
    page, hd = code.shape
    pairs = code[:, 0::2] + 16 * code[:, 1::2]
    keys, values = bytearray(pairs.tobytes()), bytearray()
    for part in (pairs, byte):
        for s in range(0, page, 4):
            for d in range(part.shape[1]):
                values += bytes(part[s:s + 4, d])
    return np.frombuffer(bytes(keys) + byte.tobytes(), np.uint8), np.frombuffer(bytes(values), np.uint8)
