"""CPU oracle of the 4-bit window cache, rotary embedding by several axes, accumulated attention weights and eviction -- TEST
INFRASTRUCTURE ONLY.

The definitions written out in NumPy, in 64 bits; only what the interface defines in single precision (cosine, sine and the
turned rows that a 4-bit cache is made from) is rounded to it.  Shares nothing with the HIP path.  Pinned in
tests/test_kv4_pins.py by enumeration of the grid, closed forms and brute force.
"""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = 32
NO_NUMBER = 255


def quantise(x):
    """[..., d] -> codes uint8 [..., d/2], scales uint8 [..., d/32]."""
    x = np.asarray(x, np.float64)
    b = x.reshape(x.shape[:-1] + (-1, BLOCK))
    top = np.abs(b).max(-1)
    e = np.ones(top.shape, np.int64)
    good = np.isfinite(top)                   # (NaN: the maximum is NaN)
    for _ in range(254):                      # the least scale that holds the block
        e = np.where(good & (top > 7.0 * 2.0 ** (e - 127.0)) & (e < 254), e + 1, e)
    y = np.abs(np.where(good[..., None], b, 0.0)) / 2.0 ** (e - 127.0)[..., None]
    dist = np.abs(y[..., None] - GRID)
    near = dist.min(-1, keepdims=True)
    # of two equally near numbers, the one with the even code
    tie = np.where(dist == near, np.arange(8) % 2, 2)
    code = np.argmin(tie, -1) + np.where(np.signbit(b) & good[..., None], 8, 0)
    code = code.reshape(x.shape).astype(np.uint8)
    return code[..., 0::2] | code[..., 1::2] << 4, np.where(good, e, NO_NUMBER).astype(np.uint8)


def values(codes, scales):
    """What codes [..., d/2] and scales [..., d/32] stand for, float64 [..., d]."""
    n = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[:-1] + (-1,)).astype(np.int64)
    v = np.where(n & 8, -1.0, 1.0) * GRID[n & 7]
    s = np.where(scales == NO_NUMBER, np.nan, 2.0 ** (np.maximum(scales, 1) - 127.0))
    return (v.reshape(v.shape[:-1] + (-1, BLOCK)) * s[..., None]).reshape(v.shape)


def angles(pos, axis_of_pair, head_dim, base):
    """[n][head_dim/2] angles: pos [n], or [n][3] with axis_of_pair [head_dim/2]."""
    theta = np.array([float(np.float32(base)) ** (-2.0 * i / head_dim) for i in range(head_dim // 2)])
    p = np.asarray(pos, np.float64)
    p = p[:, None] if axis_of_pair is None else p[:, np.minimum(axis_of_pair, 2)]
    return p * theta


def _turn(x, c, s, style, t):
    half = x.shape[-1] // 2
    a, b = (x[..., :half], x[..., half:]) if style == 0 else (x[..., 0::2], x[..., 1::2])
    a, b, c, s = (np.asarray(v, t) for v in (a, b, c, s))
    ra, rb = a * c - b * s, b * c + a * s
    return np.concatenate([ra, rb], -1) if style == 0 else np.stack([ra, rb], -1).reshape(x.shape)


def rope(x, pos, axis_of_pair, base, style):
    """x [n][heads][d] turned, in 64 bits."""
    ang = angles(pos, axis_of_pair, x.shape[-1], base)[:, None]
    return _turn(x, np.cos(ang), np.sin(ang), style, np.float64)


def rope_single(x, pos, axis_of_pair, base, style):
    """The same in single precision, every operation rounded: the rows that a 4-bit cache is made from."""
    ang = angles(pos, axis_of_pair, x.shape[-1], base)[:, None]
    return _turn(x, np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32), style, np.float32)


def attention(q, k, v, pos, scale):
    """One stream: q [n][hq][d], k, v [kv][hkv][d], pos [n] (clamped to the last entry; negative: sees nothing).
    Returns out [n][hq][d], lse [n][hq] and p [n][hq][kv]."""
    n, hq, _ = q.shape
    group = hq // k.shape[1]
    kv = k.shape[0]
    out, lse, p = np.zeros(q.shape), np.full((n, hq), -np.inf), np.zeros((n, hq, kv))
    for t in range(n):
        m = min(int(pos[t]), kv - 1) + 1
        for h in range(hq):
            if m <= 0:
                continue
            s = scale * (k[:m, h // group] @ q[t, h])
            with np.errstate(invalid="ignore"):
                top = s.max()
                w = np.exp(s - top)
                lse[t, h] = top + np.log(w.sum())
                p[t, h, :m] = w / w.sum()
                out[t, h] = p[t, h, :m] @ v[:m, h // group]
    return out, lse, p


def evict(weight, n, budget, n_first, n_last):
    """Indices of the entries 0..n-1 that stay, ascending."""
    keep = min(n, budget)

    def key(j):
        if j < n_first or j >= n - n_last:
            return (0, 0.0, j)
        return (2, 0.0, j) if np.isnan(weight[j]) else (1, -weight[j], j)

    return sorted(sorted(range(n), key=key)[:keep])
