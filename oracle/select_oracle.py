"""CPU oracle of the operators of long windows (norms per head with rotary embedding, corrections by a table of frequencies, block bounds,
selection of blocks, attention over them) -- TEST INFRASTRUCTURE ONLY.

The definitions written out in NumPy, floating numbers in 64 bits, whole numbers as Python's.  Shares nothing with the HIP path.
Pinned in tests/test_select_pins.py by closed forms, bounds and brute force.
"""
from __future__ import annotations

import math

import numpy as np

NO_NUMBER = 255


def norm(x, weight, eps):
    """[..., d] normed over its last axis; weight None: as it is."""
    x = np.asarray(x, np.float64)
    if weight is None:
        return x
    top = np.abs(x).max(-1, keepdims=True)
    s = np.where(np.isfinite(top) & (top > 0), top, 1.0)       # (squares of any number stay numbers)
    return x / s / np.sqrt(((x / s) ** 2).mean(-1, keepdims=True) + eps / s / s) * np.asarray(weight, np.float64)


def turn(x, pos, axis_of_pair, inv_freq, rotary, style, amplitude=1.0):
    """x [n][heads][d]: pair by pair."""
    x = np.array(x, np.float64)
    out = x.copy()
    for i in range(rotary // 2):
        a, b = (i, i + rotary // 2) if style == 0 else (2 * i, 2 * i + 1)
        p = np.asarray(pos, np.float64) if axis_of_pair is None else np.asarray(pos, np.float64)[:, min(int(axis_of_pair[i]), 2)]
        angle = (p * float(inv_freq[i]))[:, None]
        c, s = amplitude * np.cos(angle), amplitude * np.sin(angle)
        out[..., a] = x[..., a] * c - x[..., b] * s
        out[..., b] = x[..., b] * c + x[..., a] * s
    return out


def power(top):
    """The least k >= -95 with top <= 127 * 2^k."""
    k = -95
    while top > math.ldexp(127.0, k):
        k += 1
    return k


def block_bounds(keys):
    """keys [n][d], n >= 1 -> hi, lo (lists of whole numbers), scale byte."""
    keys = np.asarray(keys, np.float64)
    if not np.isfinite(keys).all():
        return [0] * keys.shape[1], [0] * keys.shape[1], NO_NUMBER
    k = power(float(np.abs(keys).max()))
    hi = [math.ceil(math.ldexp(float(v), -k)) for v in keys.max(0)]
    lo = [math.floor(math.ldexp(float(v), -k)) for v in keys.min(0)]
    return hi, lo, k + 127


def query_codes(q):
    """q [group][d] -> whole numbers [group][d]."""
    q = np.asarray(q, np.float64)
    if not np.isfinite(q).all():
        return np.zeros(q.shape, np.int64)
    k = power(float(np.abs(q).max()))
    return np.rint(np.ldexp(q, -k)).astype(np.int64)


def block_score(codes, hi, lo, byte):
    """A Python number that orders the blocks of a query (infinite: a block without numbers)."""
    if byte == NO_NUMBER:
        return math.inf
    hi, lo = np.asarray(hi, np.int64), np.asarray(lo, np.int64)
    best = max(int(np.maximum(row * hi, row * lo).sum()) for row in codes)
    return math.ldexp(float(best), int(byte) - 127)


def select(scores, n, n_select, n_first, n_last):
    """The list of a query with n candidates."""
    fixed = [b for b in range(n) if b < n_first or b >= n - n_last]
    others = sorted((b for b in range(n) if b not in set(fixed)), key=lambda b: (-scores[b], b))
    kept = sorted(fixed + others[:max(0, n_select - len(fixed))])
    return kept + [-1] * (n_select - len(kept))


def candidates(pos, kv_len, size):
    last = min(pos, kv_len - 1)
    return last // size + 1 if last >= 0 else 0


def seen(listed, pos, kv_len, size):
    """The entries that a query reads, ascending."""
    last = min(pos, kv_len - 1)
    return [j for b in sorted({int(b) for b in listed if b >= 0 and int(b) * size <= last}) for j in range(b * size, min((b + 1) * size - 1, last) + 1)]


def attend(q, keys, values, scale):
    """q [group][d] over keys, values [n][d] -> out [group][d], lse [group]."""
    q = np.asarray(q, np.float64)
    if len(keys) == 0:
        return np.zeros(q.shape), np.full(q.shape[0], -np.inf)
    with np.errstate(invalid="ignore", over="ignore"):
        x = scale * (q[:, None] * np.asarray(keys, np.float64)[None]).sum(-1)
        m = x.max(-1, keepdims=True)
        p = np.exp(x - m)
        total = p.sum(-1, keepdims=True)
        out = (p[..., None] * np.asarray(values, np.float64)[None]).sum(1) / total
    return out, (m + np.log(total))[:, 0]
