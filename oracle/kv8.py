"""Rotary positions, the 8-bit key-value cache and attention over it, in float64.
TEST INFRASTRUCTURE ONLY (nothing on the product path imports this).

A cached row of head_dim values x is kept as one step and integer multiples of it: with
a = max(max_d |x_d|, 2^-60) the step is a / 127 in float32 and the integers are the nearest
to 127 x_d / a, ties to even.  A row that is not finite is all NaN.
"""

from __future__ import annotations

import math

import numpy as np

LEAST = 2.0 ** -60


def kv8_quantise(x):
    """(integers int64 [..., hd], steps float32 [...]) of float32 rows x."""
    x = np.asarray(x, np.float64)
    a = np.maximum(np.max(np.abs(x), axis=-1, keepdims=True), LEAST)
    ok = np.isfinite(a)
    with np.errstate(invalid="ignore"):
        n = np.where(ok, np.rint(127.0 * x / np.where(ok, a, 1.0)), 0.0)
        step = np.where(ok, a / 127.0, np.nan)[..., 0].astype(np.float32)
    return n.astype(np.int64), step


def kv8_values(x):
    """The float64 values that the cache holds for rows x."""
    n, step = kv8_quantise(x)
    return n * step.astype(np.float64)[..., None]


def kv8_block(rows):
    """The bytes of one block from its page's rows [page, hd], keys and values: codes position
    by position (keys), and four positions side by side (values); then the steps."""
    n, step = kv8_quantise(rows)
    page, hd = n.shape
    code = (n + 128).astype(np.uint8)
    keys, values = bytearray(), bytearray()
    for s in range(page):
        keys += bytes(code[s])
    for s in range(0, page, 4):
        for d in range(hd):
            values += bytes(code[s:s + 4, d])
    tail = step.astype("<f4").tobytes()
    return np.frombuffer(bytes(keys) + tail, np.uint8), np.frombuffer(bytes(values) + tail, np.uint8)


def rope_steps(dim, base, scaling="plain", factor=1.0, original=0.0, low=0.0, high=0.0):
    """Angle steps of the pairs and the factor on cosines and sines."""
    f, mult = [], 1.0
    if scaling == "ramp":
        mult = 1.0 + 0.1 * math.log(factor)
    for j in range(dim // 2):
        b = base ** (-2.0 * j / dim)
        if scaling == "linear":
            b /= factor
        elif scaling == "base":
            b = (base * factor ** (dim / (dim - 2))) ** (-2.0 * j / dim)
        elif scaling == "bands":
            lo, hi = (low, high) if high else (1.0, 4.0)
            turns = original * b / (2 * math.pi)
            keep = min(max((turns - lo) / (hi - lo), 0.0), 1.0)
            b = (1 - keep) * b / factor + keep * b
        elif scaling == "ramp":
            lo, hi = (low, high) if high else (1.0, 32.0)

            def at(t):
                return dim * math.log(original / (t * 2 * math.pi)) / (2 * math.log(base))
            j_lo, j_hi = max(math.floor(at(hi)), 0), min(math.ceil(at(lo)), dim - 1)
            m = min(max((j - j_lo) / max(j_hi - j_lo, 0.001), 0.0), 1.0)
            b = m * b / factor + (1 - m) * b
        f.append(b)
    return np.array(f), mult


def rope_pairs(x, cos, sin, layout):
    """x [T, H, hd] with its first 2 n dimensions turned by cos, sin [T, n], in x's dtype: every
    product and sum is rounded to it."""
    n = cos.shape[1]
    out = x.copy()
    first, second = (slice(0, n), slice(n, 2 * n)) if layout == "half" else \
        (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    a, b = x[..., first], x[..., second]
    c, s = cos[:, None], sin[:, None]
    out[..., first] = a * c - b * s
    out[..., second] = a * s + b * c
    return out


def attend_rows(q, K, V, seen, scale):
    """One sequence: q [T, Hq, hd] over K, V [n, Hkv, hd]; row t sees the positions where
    seen[t] is true; zeros where that is none.  Returns the output, the same with |v| in place
    of v, and the largest sum_d |q_d k_d| * scale of each row and head."""
    T, Hq, hd = q.shape
    G = Hq // K.shape[1]
    out, mag, dots = np.zeros((T, Hq, hd)), np.zeros((T, Hq, hd)), np.zeros((T, Hq))
    for t in range(T):
        at = np.flatnonzero(seen[t])
        if not at.size:
            continue
        for h in range(Hq):
            k, v = K[at, h // G], V[at, h // G]
            s = k @ q[t, h] * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            out[t, h], mag[t, h] = p @ v, p @ np.abs(v)
            dots[t, h] = np.max(np.abs(k) @ np.abs(q[t, h])) * abs(scale)
    return out, mag, dots
