"""Queries, keys and values that are no numbers, or infinite, and calls at the edges of what is accepted, over the 4-bit window cache,
against oracle/kv4_oracle.py (needs an MI355X).  Tolerances as in tests/test_gpu_kv4.py."""
import math
import os
import re

import numpy as np
import pytest
import torch

from oracle import kv4_oracle as ko
from tests.test_gpu_kv4 import AXES, B, CACHES, DEV, U, Batch, cs, dev, pool, say, single, strides  # noqa: F401 (cs: fixture)

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------ attention weights

@pytest.mark.parametrize("dtype,cache", CACHES)
@pytest.mark.parametrize("given", [True, False])
def test_attn_weights_without_numbers_reach_only_what_their_rows_see(cs, dtype, cache, given):
    """Stream 0: one head of one query is NaN, and sees entries 0..100.  Stream 1: key 30 is NaN, and the queries see up to 40 at most.
    Stream 2: an ordinary one.  The entries that a row without statistics sees are NaN, all others what the finite rows give."""
    say("attention weights, NaN in a query and in a key", dtype, cache, given)
    b = Batch(cs, 170, 8, 2, 128, [300, 90, 150], [40, 12, 21], dtype, cache=cache, where="any", bad=[(1, 30, 0, 5)])
    rng = np.random.default_rng(171)
    b.pos = [rng.integers(0, 300, 40), rng.integers(0, 41, 12), rng.integers(0, 150, 21)]
    b.pos[0][7], b.pos[0][8], b.pos[1][3] = 100, 299, 40
    b.q_pos = dev(np.concatenate(b.pos).astype(np.int32))
    b.q64[7, 3, 11] = np.nan
    b.q[7, 3, 11] = math.nan
    before = torch.rand((3, 16 * b.max_blocks), device=DEV)
    lse = None
    if given:
        lse = np.concatenate([b.oracle(s)[2] for s in range(3)]).astype(np.float32)
        assert np.isnan(lse[7, 3]) and np.isfinite(lse[8]).all()
        lse = dev(lse)
    got = b.weights(before, 0.5, lse=lse).double().cpu().numpy()
    for s, n in enumerate(b.kv):
        _, _, _, p, e = b.oracle(s)
        add, old = p.sum((0, 1)), 0.5 * before[s, :n].double().cpu().numpy()
        assert int(np.isnan(add).sum()) == (101, 41, 0)[s]
        assert np.array_equal(np.isnan(got[s, :n]), np.isnan(add)), s
        ok = ~np.isnan(add)
        slack = (np.nan_to_num(p) * (2 * np.nan_to_num(e) + 16 * U)[..., None]).sum((0, 1))
        tol = slack + (len(b.pos[s]) * b.hq / 16 + 80) * U * (np.nan_to_num(add) + old)
        assert np.all(np.abs(got[s, :n] - old - np.nan_to_num(add))[ok] <= tol[ok] + 1e-30), s


def test_attn_weights_take_statistics_without_numbers_from_the_attention_call(cs):
    say("attention, then weights, one query head NaN")
    b = Batch(cs, 172, 28, 4, 128, [400], [64], "bf16", where="tail")
    b.pos[0][:] = np.arange(64) * 6
    b.q_pos = dev(b.pos[0].astype(np.int32))
    b.q64[20, 9] = np.nan
    b.q[20, 9] = math.nan
    _, lse = b.attend()
    assert np.argwhere(np.isnan(lse.cpu().numpy())).tolist() == [[20, 9]]
    got = b.weights(None, 1.0, lse=lse)[0].cpu().numpy()
    assert np.isnan(got[:121]).all() and np.isfinite(got[121:400]).all()

# ------------------------------------------------------------------------------------------ attention over infinite values

def put_value(b, s, j, x):
    """Entry j of stream s gets the value row x [n_kv_heads][head_dim]."""
    c, e = ko.quantise(x)
    slot = int(b.table[s, j // 16]) * 16 + j % 16
    b.pool[1][slot], b.scales[1][slot] = dev(c), dev(e)
    with np.errstate(over="ignore"):
        b.v[s][j] = ko.values(c, e).astype(np.float32)     # (2^128 reads as infinity)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,kv,nq", [
    (8, 2, 128, [200, 40], [60, 20]), (8, 2, 64, [200, 40], [60, 20]),                  # many rows
    (8, 2, 128, [200, 40], [3, 1]), (8, 2, 64, [200, 40], [3, 1]),                      # few rows
    (16, 1, 64, [4700, 30], [30, 17]), (7, 1, 128, [9000, 30], [2, 1]),                 # sweeps in pieces
])
def test_kv4_attention_over_infinite_values(cs, hq, hkv, d, kv, nq, dtype):
    """Values past the largest finite number, the last one that a query sees among them: infinite in the columns that hold them, for the queries
    that see them, NaN where infinities of both signs meet, and nothing of it in other columns or queries."""
    say("kv4 attention, infinite values", hq, hkv, d, kv, nq, dtype)
    b = Batch(cs, 173, hq, hkv, d, kv, nq, dtype, where="sorted", layout="slot")
    last = [n - 1 for n in kv]
    b.pos[0][-1], b.pos[1][-1] = last
    b.pos[0][0] = kv[0] // 4
    b.q_pos = dev(np.concatenate(b.pos).astype(np.int32))
    rng = np.random.default_rng(174)
    for s, j, cols in ((0, kv[0] // 2, {3: 1, 40: -1}), (0, kv[0] // 2 + 5, {40: 1, d - 1: -1}), (0, last[0], {17: 1}), (1, last[1], {0: -1, 33: 1})):
        x = rng.normal(size=(hkv, d))
        for c, sign in cols.items():
            x[-1, c] = sign * 3.2e38
        put_value(b, s, j, x)
    out, lse = b.attend()
    seen = 0
    for s in range(2):
        rows, want, stat, p, e = b.oracle(s)
        got = out[rows].double().cpu().numpy()
        for kind in (np.isnan, np.isposinf, np.isneginf):
            assert np.array_equal(kind(got), kind(want)), (s, kind)
        seen += int(np.isinf(want).sum())
        ok = np.isfinite(want)
        v = np.abs(np.repeat(b.v[s], hq // hkv, 1))
        mass = np.einsum("thj,jhc->thc", p, np.where(np.isfinite(v), v, 0.0))
        rel = 2 * e + (8 + 2 * (kv[s] / 16 + 64)) * U + (2 * B if dtype == "bf16" else 0.0)
        tol = rel[..., None] * mass + (B if dtype == "bf16" else 2 * U) * np.abs(np.where(ok, want, 0.0))
        assert np.all(np.abs(np.where(ok, got, 0.0) - np.where(ok, want, 0.0)) <= tol + 1e-30)
        assert np.all(np.isfinite(lse[rows].cpu().numpy()))
    assert seen > 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq", [60, 3])
def test_kv4_infinite_keys_reach_only_the_queries_that_see_them(cs, nq, dtype):
    say("kv4 attention, an infinite key", nq, dtype)
    b = Batch(cs, 176, 4, 1, 128, [200], [nq], dtype, where="tail")
    b.pos[0][:] = np.linspace(0, 199, nq).astype(int)
    b.q_pos = dev(b.pos[0].astype(np.int32))
    x = b.k[0][150].copy()
    x[0, 7], x[0, 90] = 3.2e38, -3.2e38
    c, e = ko.quantise(x)
    slot = int(b.table[0, 150 // 16]) * 16 + 150 % 16
    b.pool[0][slot], b.scales[0][slot] = dev(c), dev(e)
    out, lse = b.attend()
    n = int((b.pos[0] < 150).sum())                        # (in order: the queries that do not see the entry)
    want, stat, p = ko.attention(b.q64[:n], b.k[0], b.v[0], b.pos[0][:n], b.scale)
    mass = np.einsum("thj,jhc->thc", p, np.abs(np.repeat(b.v[0], 4, 1)))
    size = b.scale * max(float((np.abs(b.q64[:n, h]) @ np.abs(b.k[0][:150, 0]).T).max()) for h in range(4))
    err = 2 * ((128 / 8 + 8) * U * size + 8 * U * size) + (8 + 2 * (200 / 16 + 64)) * U
    assert np.all(np.abs(out[:n].double().cpu().numpy() - want) <= (err + (2 * B if dtype == "bf16" else 0.0)) * mass + (B if dtype == "bf16" else 2 * U) * np.abs(want))
    assert np.all(np.abs(lse[:n].double().cpu().numpy() - stat) <= err + 8 * U * np.abs(stat))

# ------------------------------------------------------------------------------------------ a shift of 0

@pytest.mark.parametrize("style", [0, 1])
@pytest.mark.parametrize("d,axes,in_place", [(64, "one", False), (128, "one", True), (128, "sections", False), (192, "one", False), (256, "interleaved", True)])
def test_kv4_rerotate_by_nothing_keeps_every_row(cs, d, axes, in_place, style):
    """Codes and scales of any kind, blocks without numbers and infinite elements among them, behind a shift of 0."""
    say("kv4 rerotate by 0", d, axes, in_place, style)
    n, layers, hkv = 128, 2, 2
    rng = np.random.default_rng(d)
    axis = AXES[axes](d // 2)
    codes = rng.integers(0, 256, (2, layers, 2 * n, hkv, d // 2)).astype(np.uint8)
    scales = rng.integers(0, 256, (2, layers, 2 * n, hkv, d // 32)).astype(np.uint8)
    scales[:, :, ::3] = rng.choice([0, 1, 252, 253, 254, 255], scales[:, :, ::3].shape)
    kc, vc, ks, vs = (dev(t) for t in (*codes, *scales))
    perm = rng.permutation(2 * n).astype(np.int32)
    src, dst = perm[:n], perm[n:]
    cs.cs_kv4_rerotate(kc, ks, None if in_place else vc, None if in_place else vs, dev(src), None if in_place else dev(dst),
                       dev(np.zeros((n, 3) if axis is not None else (n,), np.int32)), None if axis is None else dev(axis), n, layers, hkv, d, 2 * n * hkv * d, hkv * d, d,
                       1e6, style)
    to = src if in_place else dst
    with np.errstate(over="ignore"):
        want = ko.values(codes[0], scales[0]).astype(np.float32)
        got = ko.values(kc.cpu().numpy(), ks.cpu().numpy()).astype(np.float32)
    want[:, to] = want[:, src]
    assert np.isinf(want).any() and np.isnan(want).any()
    assert np.array_equal(got, want, equal_nan=True)


def test_kv4_rerotate_turns_only_the_pairs_of_an_axis_that_moved(cs):
    say("kv4 rerotate, one axis of two moved")
    d, n = 128, 40
    rng = np.random.default_rng(175)
    axis = np.repeat([0, 1], 32).astype(np.uint8)          # pairs 32..63: elements 32..63 and 96..127
    codes = rng.integers(0, 256, (1, 2 * n, 1, d // 2)).astype(np.uint8)
    scales = rng.integers(100, 140, (1, 2 * n, 1, d // 32)).astype(np.uint8)
    scales[:, ::2, :, 1] = 255
    delta = np.zeros((n, 3), np.int32)
    delta[:, 0] = -5
    kc, ks = dev(codes), dev(scales)
    at = np.arange(n, dtype=np.int32)
    cs.cs_kv4_rerotate(kc, ks, None, None, dev(at), None, dev(delta), dev(axis), n, 1, 1, d, 2 * n * d, d, d, 1e6, 0)
    before, after = (ko.values(c, s)[0, :n, 0] for c, s in ((codes, scales), (kc.cpu().numpy(), ks.cpu().numpy())))
    still = np.r_[32:64, 96:128]
    assert np.array_equal(after[:, still], before[:, still], equal_nan=True) and np.isnan(before[0, 32:64]).all()
    turned = ko.values(*ko.quantise(ko.rope_single(ko.values(codes, scales)[0, :n].astype(np.float32), delta, axis, 1e6, 0)))[:, 0]
    moved = np.r_[0:32, 64:96]
    assert np.array_equal(after[:, moved], turned[:, moved])

# ------------------------------------------------------------------------------------------ many heads

@pytest.mark.parametrize("n", [1, 3])
def test_rope_refresh_scatter_of_the_most_heads(cs, n):
    """65,535 query heads beside key and value heads, the same for few and for many tokens."""
    say("rope, 65,535 query heads, tokens:", n)
    hq, hkv, d = 65535, 3, 64
    rng = np.random.default_rng(n)
    x64, x = single(rng.normal(size=(n, (hq + 2 * hkv) * d)), torch.bfloat16)
    pos = rng.integers(0, 50000, n).astype(np.int32)
    out = torch.full((n, hq, d), 5.0, dtype=torch.bfloat16, device=DEV)
    kc, vc = (pool("slot", 1, n, hkv, d // 2) for _ in range(2))
    ks, vs = (pool("slot", 1, n, hkv, d // 32) for _ in range(2))
    _, sl, sh = strides(kc)
    q, k, v = x[:, :hq * d], x[:, hq * d:(hq + hkv) * d], x[:, (hq + hkv) * d:]
    row = (hq + 2 * hkv) * d
    cs.cs_rope_refresh_scatter(q, out, k, v, dev(np.arange(n, dtype=np.int32)), dev(pos), None, kc, vc, ks, vs, n, hq, hkv, d, row, row, row, sl, sh, 1e6, 0, cs.CS_BF16,
                               cs.CS_KV4)
    q64 = x64[:, :hq * d].reshape(n, hq, d)
    pair = np.abs(q64[..., :d // 2]) + np.abs(q64[..., d // 2:])
    pair = np.concatenate([pair, pair], -1)
    want = ko.rope(q64, pos, None, 1e6, 0)
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= 4 * U * pair + B * (np.abs(want) + 4 * U * pair))
    k64, v64 = (x64[:, a * d:(a + hkv) * d].reshape(n, hkv, d) for a in (hq, hq + hkv))
    for c, s, w in ((kc, ks, ko.rope_single(k64.astype(np.float32), pos, None, 1e6, 0)), (vc, vs, v64)):
        wc, ws = ko.quantise(w)
        assert np.array_equal(s[0].cpu().numpy(), ws) and np.array_equal(ko.values(c[0].cpu().numpy(), ws), ko.values(wc, ws))

# ------------------------------------------------------------------------------------------ attention weights: steps that are sorted out

def weights_route(b):
    """(steps of each stream, shares, whether each stream's steps are sorted out, most steps that can be), as attn_weights.hip has them."""
    with open(os.path.join(os.path.dirname(b.cs.__file__), "csrc", "attn_weights.hip")) as f:
        text = f.read()
    k = {n: int(re.search(rf"\b{n} = (\d+)", text).group(1)) for n in ("kStep", "kListed", "kFewSteps", "kGroups", "kLeast")}
    tile, group = 128 if b.cache == "f32" else 256, b.hq // b.hkv
    jobs = -(-b.max_blocks * 16 // tile) * len(b.kv) * b.hkv
    chunks = max(1, min(k["kGroups"] // jobs, -(-(b.n_q * group // len(b.kv)) // k["kStep"]) // k["kLeast"]))
    steps = [-(-n * group // k["kStep"]) for n in b.nq]
    return steps, chunks, [k["kFewSteps"] * chunks < s <= k["kListed"] for s in steps], k["kListed"]


def weights_oracle(b, s):
    """Weights, log-sum-exp and the slack of the weights of stream s, as Batch.oracle and check_weights have them, in whole matrices."""
    at, group = sum(b.nq[:s]), b.hq // b.hkv
    n, kv = b.nq[s], max(0, b.kv[s])
    add, slack, lse = np.zeros(kv), np.zeros(kv), np.full((n, b.hq), -np.inf)
    seen = np.arange(kv)[None] <= np.minimum(b.pos[s], kv - 1)[:, None]
    for h in range(b.hq if n and kv else 0):
        q, k = b.q64[at:at + n, h], b.k[s][:, h // group]
        x = np.where(seen, b.scale * (q @ k.T), -np.inf)
        some = seen.any(1)
        top = np.where(some, x.max(1), 0.0)
        w = np.exp(x - top[:, None])
        lse[some, h] = (top + np.log(np.where(some, w.sum(1), 1.0)))[some]
        p = w / np.where(some, w.sum(1), 1.0)[:, None]
        size = b.scale * (np.abs(q) @ np.abs(k).T).max(1)
        e = (b.d / 8 + 8) * U * size + 4 * U * (np.where(some, np.abs(lse[:, h]), 0.0) + size)
        add += p.sum(0)
        slack += (p * (2 * e + 16 * U)[:, None]).sum(0)
    return add, lse, slack + (n * b.hq / 16 + 80) * U * add


SORTED = [
    # hq, hkv, d, kv, nq, which streams' steps are sorted out
    (28, 4, 128, [300] + [20 + i for i in range(39)], [120] + [1] * 39, [True] + [False] * 39),            # a long stream beside many short ones
    (24, 8, 64, [540 + 10 * i for i in range(24)], [200 + i for i in range(24)], [True] * 24),            # a token's three rows in two steps
    (56, 8, 64, [4000], [450], [True]),                                                                    # ... its seven rows; many tiles
    (16, 1, 64, [40] + [7] * 39, [4000] + [1] * 39, [True] + [False] * 39),                                # 2,000 steps
    (16, 1, 64, [40] + [7] * 39, [4200] + [1] * 39, [False] * 40),                                         # 2,100: more than the list holds
]


@pytest.mark.parametrize("dtype,cache", CACHES)
@pytest.mark.parametrize("i", range(len(SORTED)))
def test_attn_weights_of_steps_that_are_sorted_out(cs, i, dtype, cache):
    hq, hkv, d, kv, nq, which = SORTED[i]
    b = Batch(cs, 180 + i, hq, hkv, d, kv, nq, dtype, cache=cache, layout=("head", "slot")[i % 2], where="any", extra=i % 3)
    steps, chunks, is_sorted, most = weights_route(b)
    say("attention weights, sorted steps", SORTED[i][:3], dtype, cache, "steps up to", max(steps), "shares", chunks)
    assert is_sorted == which and (any(which) or max(steps) > most)
    want = [weights_oracle(b, s) for s in range(len(kv))]
    lse = dev(np.concatenate([w[1] for w in want] + [np.full((i % 3, hq), np.nan)]).astype(np.float32))
    before = torch.rand((len(kv), 16 * b.max_blocks), device=DEV)
    for stat in (None, lse):
        got = b.weights(before, 0.75, lse=stat)
        for s, n in enumerate(kv):
            add, _, tol = want[s]
            old = 0.75 * before[s, :n].double().cpu().numpy()
            err = np.abs(got[s, :n].double().cpu().numpy() - old - add)
            assert np.all(err <= tol + (len(b.pos[s]) * b.hq / 16 + 80) * U * old + 1e-30), (s, float(err.max()))
            assert bool((got[s, n:] == 9.0).all())
        assert torch.equal(got, b.weights(before, 0.75, lse=stat))
