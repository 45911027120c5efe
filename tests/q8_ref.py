"""The 8-bit cache in plain numpy, fp64 throughout: one (sequence, kv head) at a
time, one block at a time, from the definitions.  Shares nothing with the
library but the format."""
from __future__ import annotations

import math

import numpy as np

MOST = {"e4m3": 448.0, "i8": 127.0}


def round_code(y, code):
    """y / 1 to the nearest code (ties to even), as the value it stands for."""
    y = np.asarray(y, np.float64)
    if code == "i8":
        return np.where(np.isnan(y), 0.0, np.rint(np.clip(y, -127, 127)))
    y = np.clip(y, -448.0, 448.0)
    with np.errstate(divide="ignore", invalid="ignore"):
        _, e = np.frexp(np.abs(y))  # |y| in [2^(e-1), 2^e)
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.rint(y / step) * step


def scale_of(values, code):
    """The scale of a block with these live values (the least power of two from
    2^-126 up that holds the largest finite magnitude)."""
    v = np.abs(np.asarray(values, np.float64))
    v = v[np.isfinite(v)]
    a = float(v.max()) if v.size else 0.0
    e = -126
    while a > MOST[code] * math.ldexp(1.0, e):
        e += 1
    return math.ldexp(1.0, e)


def quantise(rows, code):
    """rows [n][Dh] of one block -> (codes as values, scale)."""
    s = scale_of(rows, code)
    return round_code(np.asarray(rows, np.float64) / s, code), s


def gather(pool, idx, n, k, code, block, codes, scales):
    """One head's Tier-1 block, in place: codes [k][Dh], scales [ceil(k / block)]."""
    N = pool.shape[0]
    at = np.clip(np.arange(k) if idx is None else idx[:k], 0, N - 1)
    n = min(max(n, 0), k)
    for j in range(-(-n // block)):
        lo, hi = j * block, min((j + 1) * block, n)
        codes[lo:hi], scales[j] = quantise(pool[at[lo:hi]], code)


def append(codes, scales, count, new, code, block):
    """One head's ring after new [T][Dh], in place; returns the new count."""
    W, T = codes.shape[0], new.shape[0]
    count = max(count, 0)
    taken = {(count + t) % W: t for t in range(T)}
    filled = min(count + T, W)
    for j in sorted({s // block for s in taken}):
        lo, hi = j * block, min((j + 1) * block, filled)
        rows = np.empty((hi - lo, codes.shape[1]))
        for s in range(lo, hi):
            rows[s - lo] = new[taken[s]] if s in taken else codes[s] * scales[j]
        codes[lo:hi], scales[j] = quantise(rows, code)
    return count + T


def values(codes, scales, block, n):
    """The first n rows' values."""
    return codes[:n] * scales[np.arange(n) // block, None]


def read(codes, scales, block, count):
    """Rows in the order written, oldest first."""
    R = codes.shape[0]
    n, first = min(max(count, 0), R), count % R if count > R else 0
    at = (first + np.arange(n)) % R
    return codes[at] * scales[at // block, None]


def attend(q, K, V, scale):
    """softmax(scale q K^T) V of one head, and an entrywise bound of what a
    kernel may be off: the products take q and the weights with 22 bits (q
    against the head's largest element, weights to 2^-38 of the largest), sums
    of n terms in fp32 are off by at most n 2^-24 of the terms' magnitudes, and
    exp2's argument is rounded to 2^-24 of itself, its result to 2^-23."""
    if K.shape[0] == 0:
        return np.zeros(V.shape[1]), np.zeros(V.shape[1])
    z = scale * (K @ q)
    p = np.exp(z - z.max())
    l = p.sum()
    out = (p[:, None] * V).sum(axis=0) / l
    n, d = K.shape
    mags = abs(scale) * (np.abs(K) @ np.abs(q))
    dz = mags * ((d + 8) * 2.0 ** -24 + 2.0 ** -21) + abs(scale) * np.abs(K).sum(axis=1) * np.abs(q).max() * 2.0 ** -36
    dz = dz.max() + 2.0 ** -22 * (np.abs(z).max() + 2)
    w = np.expm1(2 * dz) + 2.0 ** -20 + (n + 64) * 2.0 ** -24
    bound = ((p[:, None] * np.abs(V)).sum(axis=0) / l + np.abs(out)) * w + 2.0 ** -36 * np.abs(V).sum(axis=0)
    return out, bound + 1e-30
