"""The 4-bit cache in plain numpy, fp64 throughout, from the definitions: one row,
one group of 32 dims at a time.  Shares nothing with the library but the format."""
from __future__ import annotations

import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
GROUP = 32


def round_code(y):
    """Code 0 .. 15 of y: the nearest magnitude, of two the one with the even code."""
    y = np.asarray(y, np.float64)
    mag = np.abs(y)
    code = np.zeros(y.shape, np.int64)
    for c in range(1, 8):
        mid = (MAGNITUDES[c - 1] + MAGNITUDES[c]) / 2
        code = np.where((mag > mid) | ((mag == mid) & (c % 2 == 0)), c, code)
    return code + 8 * np.signbit(y)


def scale_byte(values):
    """Of a group with these values: the least s >= 1 whose 6 * 2^(s - 127) holds the
    largest finite magnitude; 255 with a NaN among them."""
    v = np.asarray(values, np.float64)
    if np.isnan(v).any():
        return 255
    v = np.abs(v[np.isfinite(v)])
    a, s = float(v.max()) if v.size else 0.0, 1
    while a > 6 * np.ldexp(1.0, s - 127):
        s += 1
    return s


def quantise(rows):
    """rows [n][Dh] -> (codes [n][Dh], scale bytes [n][Dh / 32])."""
    rows = np.asarray(rows, np.float64)
    n, d = rows.shape
    codes, scales = np.zeros((n, d), np.int64), np.zeros((n, d // GROUP), np.int64)
    for r in range(n):
        for g in range(d // GROUP):
            x = rows[r, g * GROUP:(g + 1) * GROUP]
            s = scales[r, g] = scale_byte(x)
            if s != 255:
                codes[r, g * GROUP:(g + 1) * GROUP] = round_code(np.clip(x / np.ldexp(1.0, s - 127), -6, 6))
    return codes, scales


def pack(codes):
    """Codes two to a byte, the even dim in the low half."""
    return (codes[..., 0::2] + 16 * codes[..., 1::2]).astype(np.uint8)


def unpack(b):
    b = np.asarray(b).astype(np.int64)
    return np.stack([b & 15, b >> 4], axis=-1).reshape(*b.shape[:-1], -1)


def values(codes, scales):
    """Of codes [..][Dh] under scale bytes [..][Dh / 32]."""
    v = MAGNITUDES[codes & 7] * np.where(codes >= 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, np.asarray(scales, np.int64) - 127))
    return v * np.repeat(s, GROUP, axis=-1)


def append(ring, scales, count, new):
    """One head's ring (packed codes [W][Dh / 2], bytes [W][Dh / 32]) after new
    [T][Dh], in place; returns the new count."""
    W, count = ring.shape[0], max(count, 0)
    c, s = quantise(new)
    for t in range(len(new)):
        ring[(count + t) % W], scales[(count + t) % W] = pack(c[t]), s[t]
    return count + len(new)


def newest(R, count, rows):
    """Where the newest `rows` rows lie, in the order written."""
    m = min(max(count, 0), R, rows)
    return [(count - m + r) % R for r in range(m)]


def attend(q, K, V, scale):
    """softmax(scale q K^T) V of one head, and an entrywise bound of what a kernel may
    be off.  Products of the parts are exact; one MFMA sums 32 of them and what was
    there with at most 2^-22 of the magnitudes (fp32 rounding is 2^-24, and its inner
    sums keep two bits less): a score takes up to Dh / 16 of them in a row, an output
    3 for 16 rows.  q and p keep 24 bits, exp2's argument is rounded to 2^-24 of
    itself, its result to 2^-23."""
    if K.shape[0] == 0:
        return np.zeros(V.shape[1]), np.zeros(V.shape[1])
    z = scale * (K @ q)
    p = np.exp(z - z.max())
    l = p.sum()
    out = (p[:, None] * V).sum(axis=0) / l
    n, d = K.shape
    mags = abs(scale) * (np.abs(K) @ np.abs(q))
    dz = mags.max() * (d / 16 + 2) * 2.0 ** -22 + 2.0 ** -22 * (np.abs(z).max() + 2)
    w = np.expm1(2 * dz) + 2.0 ** -20 + (3 * n / 16 + 64) * 2.0 ** -22
    return out, ((p[:, None] * np.abs(V)).sum(axis=0) / l + np.abs(out)) * w + 1e-30
