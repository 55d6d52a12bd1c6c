"""Pins of oracle/kv4_oracle.py, and what the plain forms of perf/operators.py compute against it (both on the CPU)."""
import itertools
import math

import numpy as np
import pytest
import torch

from oracle import codecsight_oracle as oc
from oracle import kv4_oracle as ko


def test_every_code_round_trips_at_every_scale():
    row = np.concatenate([ko.GRID, -ko.GRID, ko.GRID, -ko.GRID])
    for e in (1, 2, 90, 127, 200, 253):
        x = row * 2.0 ** (e - 127.0)
        codes, scales = ko.quantise(x)
        assert scales.tolist() == [e]
        assert np.array_equal(ko.values(codes, scales), x)


def test_nearest_and_ties_to_even_codes():
    # 6 fixes the scale at 1; ties between neighbours go to 0, 1, 1, 2, 2, 4, 4 (even codes)
    mids = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    for eps, want in ((0.0, [0, 1, 1, 2, 2, 4, 4]), (1e-6, [0.5, 1, 1.5, 2, 3, 4, 6]), (-1e-6, [0, 0.5, 1, 1.5, 2, 3, 4])):
        x = np.zeros(32)
        x[0], x[1:8] = 6.0, mids + eps
        codes, scales = ko.quantise(x)
        assert ko.values(codes, scales)[1:8].tolist() == want
        assert (-ko.values(*ko.quantise(-x)))[1:8].tolist() == want


@pytest.mark.parametrize("top,e,stored", [(6.0, 127, 6.0), (7.0, 127, 6.0), (7.0000005, 128, 8.0), (3.5, 126, 3.0), (3.6, 127, 4.0), (0.0, 1, 0.0),
                                          (1e-45, 1, 0.0), (3.0e38, 253, 2.0 ** 128)])      # (3.53 scales: 4, past the largest fp32 number)
def test_scale_of_a_block(top, e, stored):
    x = np.zeros(64)
    x[5] = np.float64(np.float32(top))
    codes, scales = ko.quantise(x)
    assert scales.tolist() == [e, 1] and ko.values(codes, scales)[5] == stored


def test_error_of_a_block_is_a_sixth_of_its_largest():
    rng = np.random.default_rng(0)
    x = rng.normal(size=(200, 64)) * np.exp(rng.normal(size=(200, 1)) * 5)
    err = np.abs(ko.values(*ko.quantise(x)) - x).reshape(-1, 32)
    # half a step is at most 1 scale (between 4 and 6, or 7 stored as 6) and the largest is above 3.5 scales
    assert np.all(err.max(-1) <= np.abs(x).reshape(-1, 32).max(-1) / 3.5)


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_blocks_without_numbers(bad):
    x = np.ones(96)
    x[40] = bad
    codes, scales = ko.quantise(x)
    assert scales[1] == 255 and scales[0] != 255 and scales[2] != 255
    v = ko.values(codes, scales)
    assert np.isnan(v[32:64]).all() and np.array_equal(v[:32], np.ones(32)) and np.array_equal(v[64:], np.ones(32))


@pytest.mark.parametrize("style", [0, 1])
def test_rotation_is_the_one_of_the_reused_keys(style):
    rng = np.random.default_rng(3)
    x = rng.normal(size=(5, 3, 64))
    pos = rng.integers(0, 50000, 5)
    assert np.allclose(ko.rope(x, pos, None, 1e6, style), oc.rotate(x, pos[:, None], 1e6, style), atol=1e-9)
    axis = rng.integers(0, 3, 32)
    same = np.repeat(pos[:, None], 3, 1)
    assert np.array_equal(ko.rope(x, same, axis, 1e6, style), ko.rope(x, pos, None, 1e6, style))
    assert np.allclose(ko.rope(ko.rope(x, same, axis, 1e6, style), -same, axis, 1e6, style), x, atol=1e-12)
    assert np.abs(ko.rope_single(x.astype(np.float32), pos, None, 1e6, style) - ko.rope(x.astype(np.float32), pos, None, 1e6, style)).max() < 1e-5


def test_attention_against_loops_and_torch():
    rng = np.random.default_rng(4)
    n, hq, hkv, d, kv = 6, 4, 2, 8, 9
    q, k, v = rng.normal(size=(n, hq, d)), rng.normal(size=(kv, hkv, d)), rng.normal(size=(kv, hkv, d))
    pos = np.array([3, 8, 0, 5, 20, -1])
    out, lse, p = ko.attention(q, k, v, pos, 0.3)
    for t, h in itertools.product(range(n), range(hq)):
        seen = [j for j in range(kv) if j <= pos[t]]
        e = [math.exp(0.3 * float(np.dot(q[t, h], k[j, h // 2]))) for j in seen]
        for c in range(d):
            assert out[t, h, c] == pytest.approx(sum(x * v[j, h // 2, c] for x, j in zip(e, seen)) / sum(e) if seen else 0.0)
        assert lse[t, h] == (pytest.approx(math.log(sum(e))) if seen else -math.inf)
    assert np.allclose(p.sum(-1), [[1.0] * hq] * 5 + [[0.0] * hq])
    full = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q[:, :1].transpose(1, 0, 2)), torch.from_numpy(k[:n, :1].transpose(1, 0, 2)),
                                                            torch.from_numpy(v[:n, :1].transpose(1, 0, 2)), is_causal=True, scale=0.3)
    assert np.allclose(ko.attention(q[:, :1], k[:n, :1], v[:n, :1], np.arange(n), 0.3)[0][:, 0], full[0].numpy())


def test_evict_against_brute_force():
    rng = np.random.default_rng(5)
    for _ in range(200):
        n = int(rng.integers(0, 9))
        w = rng.choice([0.0, -0.0, 1.0, 1.0, 2.5, -np.inf, np.inf, np.nan], n)
        budget, first, last = int(rng.integers(1, 9)), int(rng.integers(0, 4)), int(rng.integers(0, 4))
        kept = ko.evict(w, n, budget, first, last)
        assert kept == sorted(set(kept)) and len(kept) == min(n, budget)
        order = lambda j: (2, 0) if j < first or j >= n - last else (0, 0) if np.isnan(w[j]) else (1, w[j])
        for a in kept:                        # nothing that went is better than what stayed
            for b in set(range(n)) - set(kept):
                assert order(a) > order(b) or (order(a) == order(b) and a < b)


# ---- the plain forms that the timing cases hold the kernels to

@pytest.fixture
def plain(monkeypatch):
    from perf import operators
    monkeypatch.setattr(operators, "DEV", "cpu")
    monkeypatch.setattr(operators, "own", False)
    return operators


def test_plain_quantisation_is_the_oracles(plain):
    rng = np.random.default_rng(6)
    x = (rng.normal(size=(300, 64)) * np.exp(rng.normal(size=(300, 1)) * 8)).astype(np.float32)
    x[:8] = np.float32(3.5) * 2.0 ** np.arange(8)[:, None]
    x[8:16, ::3] = 0
    codes, scales, v = plain._quantise(torch.from_numpy(x))
    want_c, want_s = ko.quantise(x)
    assert np.array_equal(scales.numpy(), want_s)
    assert np.array_equal(ko.values(codes.numpy(), want_s), ko.values(want_c, want_s)) and np.array_equal(v.numpy(), ko.values(want_c, want_s))


@pytest.mark.parametrize("axes", ["none", "sections", "interleaved"])
@pytest.mark.parametrize("style", ["half", "pairs"])
def test_plain_append_and_move_are_the_oracles(plain, axes, style):
    c = plain._append("x", 5, q_heads=4, kv_heads=2, head_dim=64, dtype="f32", axes=axes, style=style, layout="slot")
    s = plain.prepare(c, 1)
    q, k, v = plain.run(s)
    axis, st = plain._axis_of_pair(axes, 32), 0 if style == "half" else 1
    pos = s["pos"].numpy()
    assert np.abs(q.numpy() - ko.rope(s["q"].numpy().reshape(5, 4, 64).astype(float), pos, axis, 1e6, st)).max() < 1e-5
    assert np.array_equal(k[0].numpy(), ko.values(*ko.quantise(ko.rope_single(s["k"].numpy().reshape(5, 2, 64), pos, axis, 1e6, st))))
    assert np.array_equal(v[0].numpy(), ko.values(*ko.quantise(s["v"].numpy().reshape(5, 2, 64))))
    c = plain._move("x", 6, 2, kv_heads=2, head_dim=64, axes=axes, style=style)
    s = plain.prepare(c, 2)
    src = s["src"].long()
    before = [ko.values(s["codes"][i][:, src].numpy(), s["scales"][i][:, src].numpy()) for i in range(2)]
    k, v = plain.run(s)
    turned = np.stack([ko.rope_single(before[0][l].astype(np.float32), s["delta"].numpy(), axis, 1e6, st) for l in range(2)])
    assert np.array_equal(k.float().numpy(), ko.values(*ko.quantise(turned))) and np.array_equal(v.float().numpy(), before[1])


def test_plain_attention_weights_and_eviction_are_the_oracles(plain):
    c = plain._attn("x", 3, 7, 40, q_heads=4, kv_heads=2, head_dim=64, dtype="f32", where="spread")
    s = plain.prepare(c, 3)
    out, lse = plain.run(s)
    w = dict(plain._weights("x", 3, 7, 40, q_heads=4, kv_heads=2, head_dim=64, dtype="f32", where="spread", lse=False, decay=0.5))
    sw = plain.prepare(w, 3)
    got = plain.run(sw)
    for st, i in ((s, 0), (sw, 1)):
        q0 = 0
        for b in range(3):
            rows = plain._slots(st, b)
            k = ko.values(st["codes"][0][0, rows].numpy(), st["scales"][0][0, rows].numpy())
            n = st["nq"][b]
            v = ko.values(st["codes"][1][0, rows].numpy(), st["scales"][1][0, rows].numpy()) if i == 0 else k
            o, l, p = ko.attention(st["q"][q0:q0 + n].numpy().astype(float), k, v, st["q_pos"][q0:q0 + n].numpy(), 0.125)
            if i == 0:
                assert np.abs(out[q0:q0 + n].numpy() - o).max() < 1e-5 and np.abs(lse[q0:q0 + n].numpy() - l).max() < 1e-5
            else:
                want = 0.5 * st["weight"][b, :st["kv"][b]].numpy() + p.sum((0, 1))
                assert np.abs(got[b, :st["kv"][b]].numpy() - want).max() < 1e-4
            q0 += n
    c = plain._evict("x", 4, 50, 23, n_last=5, ragged=0.9)
    s = plain.prepare(c, 4)
    kept, src, dst, delta, kv_new, weight_new = plain.run(s)
    for b in range(4):
        n = int(s["kv_len"][b])
        want = ko.evict(s["weight"][b].numpy(), n, 23, 4, 5)
        assert kept[b].tolist() == want + [-1] * (23 - len(want)) and kv_new[b] == len(want)
        assert src[b, :len(want)].tolist() == [int(s["old"][b, j // 16]) * 16 + j % 16 for j in want]
        assert dst[b, :len(want)].tolist() == [int(s["new"][b, i // 16]) * 16 + i % 16 for i in range(len(want))]
        assert delta[b, :len(want)].tolist() == [i - j for i, j in enumerate(want)]
        assert weight_new[b, :len(want)].tolist() == s["weight"][b][want].tolist()
