"""Pins of oracle/select_oracle.py: closed forms, bounds that have to hold, brute force, and the other oracles where they meet."""
import itertools
import math

import numpy as np
import pytest

from oracle import codecsight_oracle as oc
from oracle import kv4_oracle as ko
from oracle import select_oracle as so

RNG = np.random.default_rng(11)


def test_norm_closed_forms():
    x = RNG.normal(size=(5, 3, 32))
    w = RNG.normal(size=32)
    y = so.norm(x, np.ones(32), 1e-12)
    assert np.allclose((y ** 2).mean(-1), 1.0, rtol=1e-9)
    assert np.allclose(so.norm(1e30 * x, w, 1e-6), so.norm(x, w, 0.0), rtol=1e-12)          # scale-free
    assert np.allclose(so.norm(x, w, 1e-6)[2, 1], [x[2, 1, c] / math.sqrt(sum(v * v for v in x[2, 1]) / 32 + 1e-6) * w[c] for c in range(32)])
    assert np.array_equal(so.norm(np.zeros((1, 8)), np.ones(8), 1e-6), np.zeros((1, 8)))
    assert np.isnan(so.norm(np.array([[1.0, np.nan]]), np.ones(2), 1e-6)).all()
    assert so.norm(x, None, 1e-6) is not None and np.array_equal(so.norm(x, None, 1e-6), x)


@pytest.mark.parametrize("style", [0, 1])
def test_turn_against_the_other_oracles_and_its_group(style):
    n, h, d = 6, 2, 32
    x, pos = RNG.normal(size=(n, h, d)), RNG.integers(-900, 900, n)
    full = np.array([1e4 ** (-2.0 * i / d) for i in range(d // 2)])
    assert np.allclose(so.turn(x, pos, None, full, d, style), ko.rope(x, pos, None, 1e4, style), atol=1e-9)
    pos3, axis = RNG.integers(-90, 90, (n, 3)), np.arange(16) % 3
    assert np.allclose(so.turn(x, pos3, axis, full, d, style), ko.rope(x, pos3, axis, 1e4, style), atol=1e-9)
    f = RNG.random(8)
    both = so.turn(so.turn(x, pos, None, f, 16, style), 5 - pos, None, f, 16, style)
    assert np.allclose(both, so.turn(x, np.full(n, 5), None, f, 16, style))                  # R(5 - p) R(p) = R(5)
    assert np.array_equal(both[..., 16:], x[..., 16:])
    twice = so.turn(x, pos, None, f, 16, style, 2.0)
    assert np.allclose(twice[..., :16], 2 * so.turn(x, pos, None, f, 16, style)[..., :16]) and np.array_equal(twice[..., 16:], x[..., 16:])


def test_powers():
    for k in range(-95, 122):
        assert so.power(math.ldexp(127.0, k)) == k
        assert so.power(math.nextafter(math.ldexp(127.0, k), math.inf)) == k + 1
    assert so.power(0.0) == -95 and so.power(2.0 ** 128) == 122


def test_bounds_hold_and_are_tight():
    for n, d, gain in ((1, 4, 1.0), (7, 9, 1e-20), (64, 16, 1e18), (3, 5, 1e-33)):
        keys = RNG.normal(size=(n, d)) * gain
        hi, lo, byte = so.block_bounds(keys)
        s = 2.0 ** (byte - 127)
        assert 32 <= byte <= 249 and max(map(abs, hi + lo)) <= 127
        for c in range(d):
            assert lo[c] * s <= keys[:, c].min() and keys[:, c].max() <= hi[c] * s
            assert (hi[c] - 1) * s < keys[:, c].max() and keys[:, c].min() < (lo[c] + 1) * s
        assert byte == 32 or np.abs(keys).max() > 127 * s / 2
    assert so.block_bounds([[1e-44, -1e-44]]) == ([1, 0], [0, -1], 32)
    assert so.block_bounds([[1.0, np.inf]])[2] == so.block_bounds([[np.nan, 0.0]])[2] == 255


def test_score_bounds_every_product():
    for _ in range(30):
        q, keys = RNG.normal(size=(3, 8)), RNG.normal(size=(5, 8))
        codes = so.query_codes(q)
        f = 2.0 ** so.power(float(np.abs(q).max()))
        score = so.block_score(codes, *so.block_bounds(keys))
        assert score * f >= max(float(f * c @ k) for c in codes for k in keys) - 1e-12
        assert np.abs(codes * f - q).max() <= f / 2
    # one key a block whose numbers are whole: the bound is the product
    codes = so.query_codes(np.array([[127.0, -3.0], [1.0, 2.0]]))
    assert so.block_score(codes, *so.block_bounds(np.array([[64.0, -100.0]]))) == 127 * 64 + 300
    assert so.block_score(codes, [0, 0], [0, 0], 255) == math.inf


def test_selection_by_brute_force():
    for trial in range(300):
        n, k = int(RNG.integers(0, 8)), int(RNG.integers(1, 6))
        first = int(RNG.integers(0, k + 1))
        last = int(RNG.integers(0, k - first + 1))
        scores = RNG.integers(-2, 3, max(n, 1)).astype(float)
        got = so.select(scores, n, k, first, last)
        m = min(n, k)
        must = {b for b in range(n) if b < first or b >= n - last}
        # of all lists that hold the fixed blocks, the one with the largest scores, then the lowest indexes
        best = max((s for s in itertools.combinations(range(n), m) if must <= set(s)), key=lambda s: (sorted((scores[b] for b in s if b not in must), reverse=True), [-b for b in s]))
        assert got == list(best) + [-1] * (k - m)


def test_all_blocks_are_full_attention():
    n, hq, hkv, d, size = 45, 4, 2, 8, 16
    q, k, v = RNG.normal(size=(n, hq, d)), RNG.normal(size=(n, hkv, d)), RNG.normal(size=(n, hkv, d))
    want = oc.full_causal(q, k, v, 0.3)
    for t in range(n):
        listed = so.select([0.0] * 3, so.candidates(t, n, size), 5, 0, 0)
        rows = so.seen(listed, t, n, size)
        assert rows == list(range(t + 1))
        for g in range(hkv):
            out, lse = so.attend(q[t, 2 * g:2 * g + 2], k[rows, g], v[rows, g], 0.3)
            assert np.allclose(out, want[t, 2 * g:2 * g + 2], atol=1e-12)


def test_what_a_list_leaves():
    assert so.seen([2, -1, 0, 2, 9], 40, 100, 16) == list(range(16)) + list(range(32, 41))
    assert so.seen([2, 1], 15, 100, 16) == [] and so.seen([0], -1, 100, 16) == [] and so.seen([0], 5, 0, 16) == []
    assert so.seen([1], 31, 20, 16) == [16, 17, 18, 19]
    out, lse = so.attend(np.ones((2, 3)), np.zeros((0, 3)), np.zeros((0, 3)), 1.0)
    assert np.array_equal(out, np.zeros((2, 3))) and np.all(lse == -np.inf)
    out, lse = so.attend(np.zeros((1, 3)), np.ones((4, 3)), np.arange(12.0).reshape(4, 3), 1.0)
    assert np.allclose(out, [[4.5, 5.5, 6.5]]) and np.allclose(lse, [math.log(4)])
