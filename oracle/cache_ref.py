"""Oracle of the calls around the paged cache, in NumPy float64 from their
definitions: rotary positions, 4-bit blocks, attention.  Test infrastructure
only; it shares no code with the HIP library.
"""
from __future__ import annotations

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def rope_frequencies(r, theta, scaling="plain", factor=1.0, original=8192,
                     low=1.0, high=4.0):
    """Radians a position, for the r / 2 pairs."""
    i = np.arange(r // 2, dtype=np.float64)
    if scaling == "ntk":
        theta = theta * factor ** (r / (r - 2))
    f = theta ** (-2.0 * i / r)
    if scaling == "linear":
        return f / factor
    if scaling == "bands":
        turns = original * f / (2 * np.pi)
        g = np.clip((turns - low) / (high - low), 0.0, 1.0)
        return g * f + (1 - g) * f / factor
    if scaling == "yarn":
        def pair(t):
            return r / 2 * np.log(original / (2 * np.pi * t)) / np.log(theta)
        lo, hi = max(np.floor(pair(high)), 0.0), min(np.ceil(pair(low)), r - 1.0)
        if hi == lo:
            hi += 0.001
        g = 1 - np.clip((i - lo) / (hi - lo), 0.0, 1.0)
        return g * f + (1 - g) * f / factor
    return f


def rope_angles(n_pos, *args, **kw):
    return np.arange(n_pos, dtype=np.float64)[:, None] * rope_frequencies(*args, **kw)


def rotate(x, cos, sin, interleaved, transpose=False):
    """x [..., heads, d]; cos, sin [..., r / 2] of each token."""
    x = np.asarray(x, dtype=np.float64)
    h = cos.shape[-1]
    c, s = cos[..., None, :], sin[..., None, :]
    if transpose:
        s = -s
    y = x.copy()
    if interleaved:
        a, b = x[..., 0:2 * h:2], x[..., 1:2 * h:2]
        y[..., 0:2 * h:2], y[..., 1:2 * h:2] = a * c - b * s, b * c + a * s
    else:
        a, b = x[..., :h], x[..., h:2 * h]
        y[..., :h], y[..., h:2 * h] = a * c - b * s, b * c + a * s
    return y


def mxfp4_encode(x):
    """Codes (0..15) and scale bytes of blocks of 32 along the last axis."""
    x = np.asarray(x, dtype=np.float64)
    blk = x.reshape(x.shape[:-1] + (x.shape[-1] // 32, 32))
    codes = np.zeros(blk.shape, dtype=np.uint8)
    byte = np.full(blk.shape[:-1], 1, dtype=np.uint8)
    for at in np.ndindex(blk.shape[:-1]):
        v = blk[at]
        if not np.all(np.isfinite(v)):
            byte[at] = 255
            continue
        m = np.abs(v).max()
        e = -126
        if m > 0:
            e = int(np.floor(np.log2(m))) - 2
            if m > 7 * 2.0 ** e:
                e += 1
            e = max(e, -126)
        byte[at] = e + 127
        for j in range(32):
            a = abs(v[j]) / 2.0 ** e
            off = np.abs(E2M1 - a)
            near = np.flatnonzero(off == off.min())
            code = near[0] if near.size == 1 or near[0] % 2 == 0 else near[1]
            codes[at + (j,)] = code | (8 if np.signbit(v[j]) else 0)
    return codes.reshape(x.shape), byte


def mxfp4_pack(codes, byte, row_bytes):
    """Rows [..., row_bytes] of codes [..., n] and bytes [..., n / 32]; bytes
    past the scales are 0."""
    n = codes.shape[-1]
    row = np.zeros(codes.shape[:-1] + (row_bytes,), dtype=np.uint8)
    row[..., :n // 2] = codes[..., 0::2] | (codes[..., 1::2] << 4)
    row[..., n // 2:n // 2 + n // 32] = byte
    return row


def mxfp4_decode(row, n):
    """float64 values of packed rows; NaN throughout a block of byte 255."""
    codes = np.empty(row.shape[:-1] + (n,), dtype=np.uint8)
    codes[..., 0::2], codes[..., 1::2] = row[..., :n // 2] & 15, row[..., :n // 2] >> 4
    byte = row[..., n // 2:n // 2 + n // 32]
    scale = np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127))
    v = E2M1[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    return v * np.repeat(scale, 32, -1)


def attend(q, k, v, n_new, scale, ok=None):
    """q [n_new][Hq][d], k and v [n][H][d] (the new tokens last), ok [n]
    marks the slots that exist.  Returns out, lse and, for the tolerances,
    the weighted mean of |v| and the largest sum of |scale q k| a row has."""
    n, H, d = k.shape
    Hq = q.shape[1]
    out = np.zeros(q.shape)
    mag = np.zeros(q.shape)
    lse = np.full((Hq, n_new), -np.inf)
    size = np.zeros((Hq, n_new))
    for c in range(n_new):
        see = np.arange(n) <= n - n_new + c
        if ok is not None:
            see &= ok
        if not see.any():
            continue
        for h in range(Hq):
            kk, vv = k[see, h * H // Hq], v[see, h * H // Hq]
            s = scale * (kk @ q[c, h])
            size[h, c] = scale * np.max(np.abs(kk) @ np.abs(q[c, h]))
            top = s.max()
            if top == -np.inf:
                continue
            w = np.exp(s - top)
            lse[h, c] = top + np.log(w.sum())
            w /= w.sum()
            out[c, h], mag[c, h] = w @ vv, w @ np.abs(vv)
    return out, lse, mag, size
