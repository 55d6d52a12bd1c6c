"""The 4-bit window cache and what goes with it (rotary embedding by axes, attention, attention weights, eviction) against
oracle/kv4_oracle.py, through the C ABI (needs an MI355X).

Tolerances.  u = 2^-24 (half a step of fp32), b = 2^-8 (of bf16).  A score is a sum of d products in fp32 accumulators and, for fp32
queries, of 3 d parts: it is off by at most e = (d/8 + 8) u scale sum_c |q_c k_c|, and the exponent's argument by 4 u |argument|
more.  A weight is off by that (relative), by 4 u from the exponential, and by b where it is rounded to bf16."""
import math
import sys

import numpy as np
import pytest
import torch

from oracle import codecsight_oracle as oc
from oracle import kv4_oracle as ko

pytestmark = pytest.mark.gpu
DEV = "cuda"
U, B = 2.0 ** -24, 2.0 ** -8


@pytest.fixture(scope="module")
def cs():
    from paper_2604_06036_amd import binding
    binding.lib()
    return binding


def say(*what):
    print("[case]", *what, flush=True)
    sys.stdout.flush()


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def pool(layout, layers, n_slots, heads, width, dtype=torch.uint8, fill=0):
    shape = (layers, n_slots, heads, width) if layout == "slot" else (layers, heads, n_slots, width)
    t = torch.full(shape, fill, dtype=dtype, device=DEV)
    return t if layout == "slot" else t.transpose(1, 2)


def strides(codes):
    return tuple(2 * codes.stride(i) for i in range(3))


def single(x, t):
    """float64 of numbers rounded to the torch type, and the tensor."""
    r = torch.from_numpy(np.asarray(x, np.float32)).to(t)
    return r.to(torch.float32).numpy().astype(np.float64), r.to(DEV)


AXES = {"one": lambda half: None, "sections": lambda half: np.repeat([0, 1, 2], [half // 4, 3 * half // 8, half - half // 4 - 3 * half // 8]).astype(np.uint8),
        "interleaved": lambda half: (np.arange(half) % 3).astype(np.uint8), "past": lambda half: (np.arange(half) % 5).astype(np.uint8)}


# ------------------------------------------------------------------------------------------ rotary embedding with the write

@pytest.mark.parametrize("n,hq,hkv,d,dtype,cache,axes,style,layout,fused", [
    (1, 28, 4, 128, "bf16", "kv4", "sections", 0, "head", True),
    (37, 4, 2, 64, "bf16", "kv4", "interleaved", 0, "slot", True),
    (37, 4, 2, 64, "bf16", "kv4", "past", 1, "head", False),
    (130, 2, 1, 64, "f32", "kv4", "one", 0, "slot", True),
    (65, 3, 3, 128, "f32", "kv4", "sections", 1, "slot", False),
    (9, 2, 2, 192, "f32", "kv4", "interleaved", 0, "head", True),
    (9, 1, 2, 256, "bf16", "kv4", "one", 1, "slot", True),
    (2500, 8, 2, 128, "bf16", "kv4", "sections", 0, "head", True),
    (50, 4, 2, 128, "bf16", "same", "sections", 0, "slot", True),
    (50, 5, 1, 80, "f32", "same", "interleaved", 1, "head", False),
    (3, 2, 2, 16, "bf16", "same", "one", 0, "slot", False),
    (40000, 2, 1, 64, "bf16", "same", "one", 0, "slot", True),
    (33, 0, 2, 64, "bf16", "kv4", "sections", 0, "slot", True),       # keys and values only
    (33, 4, 0, 64, "f32", "kv4", "sections", 0, "slot", True),        # queries only
])
def test_rope_refresh_scatter(cs, n, hq, hkv, d, dtype, cache, axes, style, layout, fused):
    say("rope", n, hq, hkv, d, dtype, cache, axes, style, layout)
    rng = np.random.default_rng(n + d)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    code = cs.CS_BF16 if dtype == "bf16" else cs.CS_F32
    axis = AXES[axes](d // 2)
    pos = rng.integers(-70000, 70000, (n, 3) if axis is not None else (n,)).astype(np.int32)
    pos[0] = 0
    x64, x = single(rng.normal(size=(n, (hq + 2 * hkv) * d)) * np.exp(rng.normal(size=(n, 1)) * 3), t)
    if fused:        # slices of one projection
        q, k, v = x[:, :hq * d], x[:, hq * d:(hq + hkv) * d], x[:, (hq + hkv) * d:]
    else:
        q, k, v = (p.contiguous() for p in (x[:, :hq * d], x[:, hq * d:(hq + hkv) * d], x[:, (hq + hkv) * d:]))
    n_slots = n + 19
    slot = rng.permutation(n_slots)[:n].astype(np.int32)
    slot[rng.random(n) < 0.1] = -1
    four = cache == "kv4"
    w = d // 2 if four else d
    kc, vc = (pool(layout, 1, n_slots, max(1, hkv), w, torch.uint8 if four else t, 7) for _ in range(2))
    ks, vs = (pool(layout, 1, n_slots, max(1, hkv), d // 32, torch.uint8, 9) if four else None for _ in range(2))
    sl, sh = (2 * kc.stride(1), 2 * kc.stride(2)) if four else (kc.stride(1), kc.stride(2))
    out = torch.full((n, max(1, hq), d), 5.0, dtype=t, device=DEV)
    none = lambda c, v_: v_ if c else None
    cs.cs_rope_refresh_scatter(none(hq, q), none(hq, out), none(hkv, k), none(hkv, v), none(hkv, dev(slot)), dev(pos), None if axis is None else dev(axis), none(hkv, kc),
                               none(hkv, vc), none(hkv, ks), none(hkv, vs), n, hq, hkv, d, q.stride(0), k.stride(0), v.stride(0), sl, sh, 1e6, style, code,
                               cs.CS_KV4 if four else code)
    torch.cuda.synchronize()
    q64, k64, v64 = (p.reshape(n, -1, d) for p in (x64[:, :hq * d], x64[:, hq * d:(hq + hkv) * d], x64[:, (hq + hkv) * d:]))
    half = d // 2

    def near(got, x_, what):       # products and their sum are rounded (3 u of |a| + |b|, with the cosine's own u), then the storage
        want = ko.rope(x_, pos, axis, 1e6, style)
        pair = np.abs(x_).reshape(n, -1, 2, half).sum(2) if style == 0 else np.abs(x_).reshape(n, -1, half, 2).sum(3)
        pair = np.concatenate([pair, pair], -1) if style == 0 else np.repeat(pair, 2, -1)
        tol = 4 * U * pair + (B if dtype == "bf16" else 0) * (np.abs(want) + 4 * U * pair)
        err = np.abs(got.double().cpu().numpy() - want)
        assert np.all(err <= tol), (what, float((err - tol).max()))

    if hq:
        near(out, q64, "q")
    if not hkv:
        return
    live = np.flatnonzero(slot >= 0)
    at = slot[live]
    other = np.setdiff1d(np.arange(n_slots), at)
    if four:
        turned = ko.rope_single(k64.astype(np.float32), pos, axis, 1e6, style)
        for got_c, got_s, want in ((kc, ks, turned), (vc, vs, v64)):
            c, s = got_c[0].cpu().numpy(), got_s[0].cpu().numpy()
            wc, ws = ko.quantise(want[live])
            assert np.array_equal(s[at], ws)
            assert np.array_equal(ko.values(c[at], s[at]), ko.values(wc, ws))
            assert np.all(c[other] == 7) and np.all(s[other] == 9)
    else:
        full = torch.zeros((n, hkv, d), dtype=t, device=DEV)
        full[live] = kc[0][at]
        whole = k64.copy()
        whole[slot < 0] = 0
        near(full, whole, "k")
        assert torch.equal(vc[0][at], v.reshape(n, hkv, d)[live])
        assert bool((kc[0][other] == 7).all()) and bool((vc[0][other] == 7).all())


@pytest.mark.parametrize("n,hq,hkv,d,cache", [(6000, 7, 2, 128, "kv4"), (9000, 5, 1, 64, "kv4"), (6000, 5, 3, 128, "same")])
def test_rope_refresh_scatter_several_heads_a_thread(cs, n, hq, hkv, d, cache):
    test_rope_refresh_scatter(cs, n, hq, hkv, d, "bf16", cache, "sections", 0, "head", True)


def test_rope_in_place_and_its_transpose(cs):
    say("rope in place")
    rng = np.random.default_rng(1)
    n, h, d = 77, 6, 128
    axis = AXES["sections"](64)
    pos = rng.integers(0, 5000, (n, 3)).astype(np.int32)
    x = torch.from_numpy(rng.normal(size=(n, h + 2, d)).astype(np.float32)).to(DEV)
    keep = x.clone()
    args = lambda p: (x, x, None, None, None, dev(p), dev(axis), None, None, None, None, n, h, 0, d, x.stride(0), 0, 0, 0, 0, 1e4, 0, cs.CS_F32, cs.CS_F32)
    cs.cs_rope_refresh_scatter(*args(pos))
    turned = x.clone()
    assert torch.equal(x[:, h:], keep[:, h:]) and not torch.equal(x[:, :h], keep[:, :h])
    cs.cs_rope_refresh_scatter(*args(-pos))
    assert float((x - keep).abs().max()) <= 16 * U * float(keep.abs().max()) * 2
    # <g, R x> = <R^T g, x>: the gradient of the results is mapped by the same call with negated positions
    g = torch.from_numpy(rng.normal(size=(n, h + 2, d)).astype(np.float32)).to(DEV)
    left = (g[:, :h].double() * turned[:, :h].double()).sum()
    x.copy_(g)
    cs.cs_rope_refresh_scatter(*args(-pos))
    right = (x[:, :h].double() * keep[:, :h].double()).sum()
    assert abs(float(left - right)) <= 8 * U * float((g[:, :h].abs().double() * keep[:, :h].abs().double()).sum()) * 2


def test_keys_without_positions_and_without_numbers(cs):
    say("plain 4-bit write, NaN and infinities")
    rng = np.random.default_rng(2)
    n, hkv, d = 40, 2, 128
    k = rng.normal(size=(n, hkv, d)).astype(np.float32)
    v = rng.normal(size=(n, hkv, d)).astype(np.float32) * 1e-30
    k[3, 1, 40], k[5, 0, 127], v[7, 1, 0] = np.nan, np.inf, -np.inf
    v[8] = 0
    v[9, 0, :32] = 7 * 2.0 ** -20
    v[10, 0, :4] = [1e-45, 2e-38, 3.5e-38, -1e-44]
    for style in (0, 1):
        kc, vc = (pool("head", 1, n, hkv, d // 2) for _ in range(2))
        ks, vs = (pool("head", 1, n, hkv, d // 32) for _ in range(2))
        cs.cs_rope_refresh_scatter(None, None, dev(k), dev(v), dev(np.arange(n, dtype=np.int32)), None, None, kc, vc, ks, vs, n, 0, hkv, d, 0, hkv * d, hkv * d,
                                   2 * kc.stride(1), 2 * kc.stride(2), 1e6, style, cs.CS_F32, cs.CS_KV4)
        ko_, vo_ = (torch.zeros((1, n, hkv, d), device=DEV) for _ in range(2))
        cs.cs_kv4_gather(kc, ks, vc, vs, dev(np.arange(n, dtype=np.int32)), n, 1, hkv, d, 0, 2 * kc.stride(1), 2 * kc.stride(2), ko_, vo_, cs.CS_F32)
        for got, s, x in ((ko_, ks, k), (vo_, vs, v)):
            want = ko.values(*ko.quantise(x))
            assert np.array_equal(got[0].cpu().numpy(), want.astype(np.float32), equal_nan=True)
            assert np.array_equal(s[0].cpu().numpy(), ko.quantise(x)[1])


# ------------------------------------------------------------------------------------------ rows as numbers, position correction

def test_gather_every_code_and_scale(cs):
    say("gather: all 16 codes x 256 scales")
    codes = (np.arange(256 * 16) % 256).reshape(256, 1, 16).astype(np.uint8)          # every pair of codes
    row = np.concatenate([codes, np.roll(codes, 1, 0)], -1)                            # head_dim 64
    scales = np.stack([np.arange(256), 255 - np.arange(256)], -1).reshape(256, 1, 2).astype(np.uint8)
    slot = np.arange(256, dtype=np.int32)
    slot[17] = -1
    for t, dt in ((torch.float32, cs.CS_F32), (torch.bfloat16, cs.CS_BF16)):
        out = torch.full((1, 256, 1, 64), 3.0, dtype=t, device=DEV)
        cs.cs_kv4_gather(dev(row), dev(scales), None, None, dev(slot), 256, 1, 1, 64, 0, 64, 64, out, None, dt)
        with np.errstate(over="ignore"):
            want = ko.values(row, scales).astype(np.float32)
        want[17] = 3.0
        assert np.array_equal(out[0].float().cpu().numpy(), torch.from_numpy(want).to(t).float().numpy(), equal_nan=True)


@pytest.mark.parametrize("n,layers,hkv,d,axes,style,layout,in_place", [
    (1, 1, 1, 64, "one", 0, "slot", False), (300, 3, 4, 128, "one", 0, "head", False), (77, 2, 2, 128, "sections", 1, "slot", False),
    (77, 5, 3, 64, "interleaved", 0, "slot", True), (33, 2, 1, 192, "sections", 0, "head", False), (33, 2, 2, 256, "one", 1, "slot", True),
    (5000, 2, 8, 128, "one", 0, "slot", False)])
def test_kv4_rerotate(cs, n, layers, hkv, d, axes, style, layout, in_place):
    say("kv4 rerotate", n, layers, hkv, d, axes, style, layout, in_place)
    rng = np.random.default_rng(n + d)
    n_slots = 2 * n + 3
    axis = AXES[axes](d // 2)
    codes = [pool(layout, layers, n_slots, hkv, d // 2) for _ in range(2)]
    scales = [pool(layout, layers, n_slots, hkv, d // 32) for _ in range(2)]
    for c, s in zip(codes, scales):
        c.copy_(dev(rng.integers(0, 256, tuple(c.shape)).astype(np.uint8)))
        s.copy_(dev(rng.integers(100, 140, tuple(s.shape)).astype(np.uint8)))
    scales[0][0, 0, 0, 0] = 255
    scales[0][-1, 1, -1, -1] = 0
    before = [[t.cpu().numpy() for t in ts] for ts in (codes, scales)]
    perm = rng.permutation(n_slots).astype(np.int32)
    src, dst = perm[:n].copy(), perm[n:2 * n].copy()
    if n > 5:
        src[3] = -1
        dst[4] = -1
    delta = rng.integers(-4000, 4000, (n, 3) if axis is not None else (n,)).astype(np.int32)
    delta[n // 2] = 0
    layer, slot, head = strides(codes[0])
    cs.cs_kv4_rerotate(codes[0], scales[0], None if in_place else codes[1], None if in_place else scales[1], dev(src), None if in_place else dev(dst), dev(delta),
                       None if axis is None else dev(axis), n, layers, hkv, d, layer, slot, head, 1e6, style)
    to = src if in_place else dst
    live = (src >= 0) & (to >= 0)
    after = [[t.cpu().numpy() for t in ts] for ts in (codes, scales)]
    for l in range(layers):
        k = ko.values(before[0][0][l, src[live]], before[1][0][l, src[live]])
        with np.errstate(invalid="ignore"):
            wc, ws = ko.quantise(ko.rope_single(k.astype(np.float32), delta[live], axis, 1e6, style))
        assert np.array_equal(after[1][0][l, to[live]], ws)
        assert np.array_equal(ko.values(after[0][0][l, to[live]], ws), ko.values(wc, ws), equal_nan=True)
        zero = np.flatnonzero(live)[np.all(delta[live].reshape(int(live.sum()), -1) == 0, 1)]
        for z in zero:
            assert np.array_equal(ko.values(after[0][0][l, to[z]], after[1][0][l, to[z]]), ko.values(before[0][0][l, src[z]], before[1][0][l, src[z]]), equal_nan=True)
        rest = np.setdiff1d(np.arange(n_slots), to[live])
        assert np.array_equal(after[0][0][l, rest], before[0][0][l, rest]) and np.array_equal(after[1][0][l, rest], before[1][0][l, rest])
        for i in range(2):
            want = before[i][1][l].copy()
            if not in_place:
                want[to[live]] = before[i][1][l, src[live]]
            assert np.array_equal(after[i][1][l], want)


@pytest.mark.parametrize("d,pad,shift,in_place", [(64, 32, 0, False), (64, 0, 1, False), (64, 0, 1, True), (128, 64, 0, False), (128, 32, 0, True),
                                                   (128, 0, 2, False), (128, 0, 1, True)])
def test_kv4_rerotate_scales_at_any_byte(cs, d, pad, shift, in_place):
    """Rows that lie `pad` elements apart and scales that start `shift` bytes into their memory: what dense, aligned pools give."""
    say("kv4 rerotate, scales anywhere", d, pad, shift, in_place)
    n, layers, hkv = 37, 2, 3
    rng = np.random.default_rng(d + pad + shift)
    n_slots, row = 2 * n, hkv * d + pad
    perm = rng.permutation(n_slots).astype(np.int32)
    src, dst, delta = dev(perm[:n].copy()), dev(perm[n:].copy()), dev(rng.integers(-400, 400, (n,)).astype(np.int32))
    got = []
    fill = [rng.integers(lo, hi, (layers, n_slots, hkv, d // per)).astype(np.uint8) for lo, hi, per in ((0, 256, 2), (0, 256, 2), (1, 255, 32), (1, 255, 32))]
    for r, off in ((hkv * d, 0), (row, shift)):
        ts, flats = [], []
        for x, per in zip(fill, (2, 2, 32, 32)):
            start = off if per == 32 else 0
            flat = torch.full((start + layers * n_slots * r // per,), 7, dtype=torch.uint8, device=DEV)
            t = torch.as_strided(flat, x.shape, (n_slots * r // per, r // per, d // per, 1), start)
            t.copy_(dev(x))
            ts.append(t)
            flats.append(flat)
        cs.cs_kv4_rerotate(ts[0], ts[2], None if in_place else ts[1], None if in_place else ts[3], src, None if in_place else dst, delta, None, n, layers,
                           hkv, d, n_slots * r, r, d, 1e6, 0)
        got.append([t.cpu().numpy() for t in ts])
        for flat, t in zip(flats, ts):                     # nothing beside the rows is written
            t.fill_(7)
            assert bool((flat == 7).all())
    assert not np.array_equal(got[0][0], fill[0])
    for a, b in zip(*got):
        assert np.array_equal(a, b)


# ------------------------------------------------------------------------------------------ attention, attention weights

class Batch:
    """A batch over a paged cache.  Rows of the pool that no window holds, and rows past a window's end in its last block, are NaN."""

    def __init__(self, cs, seed, hq, hkv, d, kv, nq, dtype, cache="kv4", layout="head", where="any", gain=1.0, extra=0, bad=()):
        rng = np.random.default_rng(seed)
        self.cs, self.hq, self.hkv, self.d, self.kv, self.nq, self.dtype, self.cache = cs, hq, hkv, d, kv, nq, dtype, cache
        t = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.code = cs.CS_BF16 if dtype == "bf16" else cs.CS_F32
        need = [max(0, -(-n // 16)) for n in kv]
        self.max_blocks = max(1, max(need)) + 1
        n_slots = 16 * (sum(need) + 2)
        ids = rng.permutation(sum(need) + 2)
        table = np.full((len(kv), self.max_blocks), ids[-1], np.int32)       # a block of NaN
        at = 0
        for s, m in enumerate(need):
            table[s, :m] = ids[at:at + m]
            at += m
        self.n_q = sum(nq) + extra
        self.q64, self.q = single(rng.normal(size=(self.n_q, hq, d)) * gain, t)
        kv64 = [rng.normal(size=(n_slots, hkv, d)) for _ in range(2)]
        slots = [np.array([table[s, j // 16] * 16 + j % 16 for j in range(max(0, n))], np.int64) for s, n in enumerate(kv)]
        used = np.concatenate(slots).astype(int)
        for i, x in enumerate(kv64):
            x[np.setdiff1d(np.arange(n_slots), used)] = np.nan
        for s, j, i, c in bad:                 # (stream, entry, 0 key / 1 value, element)
            kv64[i][slots[s][j], :, c] = np.nan
        if cache == "kv4":
            self.pool, self.scales, self.k, self.v = [], [], None, None
            for x in kv64:
                c, e = ko.quantise(x)
                pc, ps = pool(layout, 1, n_slots, hkv, d // 2), pool(layout, 1, n_slots, hkv, d // 32)
                pc.copy_(dev(c[None]))
                ps.copy_(dev(e[None]))
                self.pool.append(pc[0])
                self.scales.append(ps[0])
            x64 = [ko.values(*ko.quantise(x)) for x in kv64]
            self.stride = (2 * self.pool[0].stride(0), 2 * self.pool[0].stride(1))
        else:
            x64, self.pool, self.scales = [], [], [None, None]
            for x in kv64:
                r64, r = single(x, t)
                pc = pool(layout, 1, n_slots, hkv, d, t)
                pc.copy_(r[None])
                self.pool.append(pc[0])
                x64.append(r64)
            self.stride = (self.pool[0].stride(0), self.pool[0].stride(1))
        self.k = [x64[0][sl] for sl in slots]
        self.v = [x64[1][sl] for sl in slots]
        pos = []
        for n, m in zip(kv, nq):
            if where == "tail":
                pos.append(np.arange(n - m, n))
            elif where == "sorted":
                pos.append(np.sort(rng.integers(0, max(1, n), m)))
            else:                              # no order, some that see nothing, some past the end (clamped)
                p = rng.integers(0, max(1, n), m)
                p[rng.random(m) < 0.1] = -1
                p[rng.random(m) < 0.1] = n + 5
                pos.append(p)
        self.pos = pos
        self.q_pos = dev(np.concatenate(pos + [np.full(extra, 3)]).astype(np.int32))
        self.cu_q = dev(np.cumsum([0] + nq).astype(np.int32))
        self.kv_len, self.table = dev(np.array(kv, np.int32)), dev(table)
        self.scale = 1.0 / math.sqrt(d)

    def attend(self, lse=True, ws_fill=0xA5):
        cs = self.cs
        out = torch.full((self.n_q, self.hq, self.d), 9.0, dtype=self.q.dtype, device=DEV)
        stat = torch.full((self.n_q, self.hq), 9.0, device=DEV) if lse else None
        nbytes = cs.cs_kv4_window_attn_workspace(self.n_q, len(self.kv), self.hq, self.hkv, self.d, self.max_blocks)
        ws = torch.full((nbytes,), ws_fill, dtype=torch.uint8, device=DEV) if nbytes else None
        cs.cs_kv4_window_attn(self.q, self.pool[0], self.scales[0], self.pool[1], self.scales[1], self.cu_q, self.q_pos, self.kv_len, self.table, self.max_blocks, 16, out,
                              stat, self.n_q, len(self.kv), self.hq, self.hkv, self.d, *self.stride, self.scale, self.code, ws)
        torch.cuda.synchronize()
        return out, stat

    def weights(self, before, decay, lse=None, in_place=False):
        cs = self.cs
        out = before if in_place else torch.full((len(self.kv), 16 * self.max_blocks), 9.0, device=DEV)
        ws = torch.full((cs.cs_attn_weights_workspace(self.n_q, len(self.kv), self.hq, self.hkv, self.d, self.max_blocks),), 0xFF, dtype=torch.uint8, device=DEV)
        cs.cs_attn_weights(self.q, lse, self.pool[0], self.scales[0], self.cu_q, self.q_pos, self.kv_len, self.table, self.max_blocks, 16, before, out, decay, self.n_q,
                           len(self.kv), self.hq, self.hkv, self.d, *self.stride, self.scale, self.code, cs.CS_KV4 if self.cache == "kv4" else self.code, ws)
        torch.cuda.synchronize()
        return out

    def oracle(self, s):
        at = sum(self.nq[:s])
        q = self.q64[at:at + self.nq[s]]
        with np.errstate(invalid="ignore", over="ignore"):
            out, lse, p = ko.attention(q, self.k[s], self.v[s], self.pos[s], self.scale)
        group = self.hq // self.hkv
        k = np.nan_to_num(np.repeat(self.k[s], group, 1))
        e = np.zeros((len(q), self.hq))          # the largest error of a score of each row
        for h in range(self.hq):
            if len(k):
                e[:, h] = (self.d / 8 + 8) * U * self.scale * (np.abs(q[:, h]) @ np.abs(k[:, h]).T).max(-1, initial=0.0)
        top = np.where(np.isfinite(lse), np.abs(lse), 0.0) + e / (self.d / 8 + 8) / U      # no argument is larger
        return slice(at, at + self.nq[s]), out, lse, p, e + 4 * U * top

    def check(self, out, stat):
        done = 0
        for s in range(len(self.kv)):
            rows, want, lse, p, e = self.oracle(s)
            if self.kv[s] <= 0:
                assert bool((out[rows] == 9).all())
                continue
            got = out[rows].double().cpu().numpy()
            assert np.array_equal(np.isnan(got), np.isnan(want)), s
            v = np.abs(np.nan_to_num(np.repeat(self.v[s], self.hq // self.hkv, 1)))
            mass = np.einsum("thj,jhc->thc", np.nan_to_num(p), v)
            n = self.kv[s] / 16 + 64             # additions on the way into a sum
            rel = 2 * e + (8 + 2 * n) * U + (2 * B if self.dtype == "bf16" else 0.0)
            tol = rel[..., None] * mass + (B if self.dtype == "bf16" else 2 * U) * np.abs(np.nan_to_num(want))
            err = np.where(np.isnan(want), 0, np.abs(got - np.nan_to_num(want)))
            assert np.all(err <= tol + 1e-30), (s, float(err.max()), float((err / (tol + 1e-30)).max()))
            if stat is not None:
                g = stat[rows].double().cpu().numpy()
                assert np.array_equal(np.isneginf(g), np.isneginf(lse))
                ok = np.isfinite(lse)
                assert np.array_equal(np.isnan(g), np.isnan(lse))
                assert np.all(np.abs(g - np.where(ok, lse, 0))[ok] <= (e + (8 + n) * U + 4 * U * np.abs(np.where(ok, lse, 0)))[ok])
            done += 1
        tail = sum(self.nq)
        assert bool((out[tail:] == 9).all()) and (stat is None or bool((stat[tail:] == 9).all()))
        return done

    def check_weights(self, got, before, decay):
        for s in range(len(self.kv)):
            _, _, _, p, e = self.oracle(s)
            n = max(0, self.kv[s])
            g = got[s].double().cpu().numpy()
            assert np.all(g[n:] == 9.0) if before is not got else True
            add = np.nan_to_num(p).sum((0, 1))
            old = before[s].double().cpu().numpy()[:n] * decay if before is not None and decay else np.zeros(n)
            slack = (np.nan_to_num(p) * (2 * e + 16 * U)[..., None]).sum((0, 1))
            tol = slack + (len(self.pos[s]) * self.hq / 16 + 80) * U * (add + np.abs(old))
            assert np.all(np.abs(g[:n] - old - add) <= tol + 1e-30), (s, float((np.abs(g[:n] - old - add) / (tol + 1e-30)).max()))


SHAPES = [
    # hq, hkv, d, kv, nq, where, layout
    (28, 4, 128, [919], [1], "tail", "head"),
    (28, 4, 128, [1], [1], "tail", "slot"),
    (2, 1, 64, [65], [65], "tail", "slot"),
    (8, 2, 128, [200, 0, 63, 64, 17], [33, 4, 1, 64, 17], "any", "head"),
    (8, 2, 64, [129, 1, 16, 300], [40, 1, 0, 21], "any", "slot"),
    (7, 1, 128, [500], [100], "sorted", "head"),
    (16, 1, 64, [333, 70], [9, 70], "any", "head"),
    (3, 3, 128, [31, 32, 33], [31, 32, 33], "tail", "slot"),
    (32, 8, 128, [100 + 7 * i for i in range(70)], [1] * 70, "tail", "head"),
    (4, 4, 64, [40 + i for i in range(130)], [i % 3 for i in range(130)], "any", "slot"),
    (28, 4, 128, [2500, 300], [1, 2], "tail", "head"),
    (4, 1, 128, [5000], [3], "any", "slot"),
    (12, 3, 64, [3000, 1], [5, 1], "any", "head"),
    (16, 4, 64, [2439, 800], [60, 45], "any", "slot"),                      # many rows, sweeps in pieces
    (8, 2, 64, [30 + 3 * i for i in range(66)], [20] * 66, "sorted", "head"),    # more streams than lanes, many rows
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_kv4_window_attn(cs, i, dtype):
    hq, hkv, d, kv, nq, where, layout = SHAPES[i]
    say("kv4 attention", dtype, SHAPES[i])
    b = Batch(cs, i, hq, hkv, d, kv, nq, dtype, layout=layout, where=where, extra=i % 3)
    b.check(*b.attend())
    out, _ = b.attend()
    again, none = b.attend(lse=False, ws_fill=0)
    assert none is None and torch.equal(out, again)


# sweeps cut into pieces, and their joins
LONG = [
    (7, 1, 64, [9000], [2], "any", "head"),                                 # few rows, many pieces
    (16, 2, 128, [9300, 0, 5], [1, 1, 2], "any", "slot"),
    (8, 2, 128, [4600, 30], [30, 17], "any", "head"),                       # many rows, many pieces
    (16, 1, 64, [4700], [9], "any", "slot"),
    (8, 1, 64, [3000, 1500, 20, 0], [150, 1, 1, 3], "any", "head"),         # streams of very different numbers of rows
    (4, 4, 128, [1700, 900, 1800], [70, 200, 90], "sorted", "slot"),        # few pieces
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("i", range(len(LONG)))
def test_kv4_window_attn_in_pieces(cs, i, dtype):
    hq, hkv, d, kv, nq, where, layout = LONG[i]
    say("kv4 attention in pieces", dtype, LONG[i])
    b = Batch(cs, 50 + i, hq, hkv, d, kv, nq, dtype, layout=layout, where=where, extra=i % 3)
    out, lse = b.attend()
    b.check(out, lse)
    again, stat = b.attend(ws_fill=0xFF)
    assert torch.equal(out, again) and torch.equal(lse, stat)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gain", [4.0, 30.0])
def test_kv4_window_attn_peaked(cs, dtype, gain):
    say("kv4 attention, scores times", gain)
    b = Batch(cs, 77, 8, 2, 128, [700, 90], [60, 90], dtype, where="any", gain=gain)
    b.check(*b.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_kv4_window_attn_maximum_at_the_end(cs, dtype):
    """A last key far above the others: the reference maximum moves in the last tile."""
    say("kv4 attention, late outlier")
    b = Batch(cs, 78, 4, 1, 64, [400], [3], dtype, where="tail")
    k = b.k[0]
    k[399] = 0
    k[399, :, :] = 6.0
    c, e = ko.quantise(k[399:400])
    slot = int(b.table[0, 399 // 16]) * 16 + 399 % 16
    b.pool[0][slot] = dev(c)[0]
    b.scales[0][slot] = dev(e)[0]
    b.check(*b.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_kv4_entries_without_numbers_reach_only_those_that_see_them(cs, dtype):
    say("kv4 attention, NaN inside the windows")
    bad = [(0, 70, 0, 5), (0, 90, 1, 40), (0, 130, 1, 100), (1, 20, 1, 1), (2, 0, 0, 0)]
    b = Batch(cs, 79, 8, 2, 128, [200, 21, 40], [60, 21, 5], dtype, where="any", bad=bad)
    out, stat = b.attend()
    b.check(out, stat)
    assert bool(torch.isnan(out.float()).any()) and not bool(torch.isnan(out.float()).all())


def test_kv4_attention_equals_attention_over_the_gathered_rows(cs):
    """The same batch through cs_window_prefill_attn, on a bf16 cache of the numbers that the codes stand for."""
    say("kv4 attention beside the 16-bit call")
    b = Batch(cs, 80, 28, 4, 128, [919, 300], [400, 100], "bf16", where="sorted", layout="slot")
    out, _ = b.attend()
    n_slots = b.pool[0].shape[0]
    k, v = (torch.zeros((1, n_slots, 4, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    cs.cs_kv4_gather(b.pool[0], b.scales[0], b.pool[1], b.scales[1], torch.arange(n_slots, dtype=torch.int32, device=DEV), n_slots, 1, 4, 128, 0, *b.stride, k, v, cs.CS_BF16)
    other = torch.empty_like(out)
    ws = torch.empty((cs.cs_window_prefill_attn_workspace(b.n_q, 2, 28, 4, 128, b.max_blocks, cs.CS_BF16),), dtype=torch.uint8, device=DEV)
    cs.cs_window_prefill_attn(b.q, k[0], v[0], b.cu_q, b.q_pos, b.kv_len, b.table, b.max_blocks, 16, other, b.n_q, 2, 28, 4, 128, 512, 128, b.scale, cs.CS_BF16, ws)
    torch.cuda.synchronize()
    b.check(out, None)
    b.check(other, None)


@pytest.mark.parametrize("n_q", [1, 40])
def test_kv4_pools_past_32_bits(cs, n_q):
    """Rows 4 KiB apart, blocks in the last of 4.5 GB of codes: write, move, read back, attention, weights."""
    say("4-bit pool of 4.5 GB, queries:", n_q)
    n_slots, stride, d, kv = 1100000, 8192, 128, 300
    rng = np.random.default_rng(11)
    codes = [torch.zeros((n_slots * stride // 2,), dtype=torch.uint8, device=DEV) for _ in range(2)]
    scales = [torch.zeros((n_slots * stride // 32,), dtype=torch.uint8, device=DEV) for _ in range(2)]
    blocks = n_slots // 16 - 1 - rng.permutation(40)[:19].astype(np.int32)
    table = blocks[None].astype(np.int32)
    slots = (blocks[np.arange(kv) // 16] * 16 + np.arange(kv) % 16).astype(np.int32)
    assert int(slots.min()) * (stride // 2) > 1 << 32
    k, v = (rng.normal(size=(kv, 1, d)).astype(np.float32) for _ in range(2))
    cs.cs_rope_refresh_scatter(None, None, dev(k), dev(v), dev(slots), None, None, codes[0], codes[1], scales[0], scales[1], kv, 0, 1, d, 0, d, d, stride, d, 1e6, 0,
                               cs.CS_F32, cs.CS_KV4)
    low = np.arange(kv, dtype=np.int32)
    cs.cs_kv4_rerotate(codes[0], scales[0], codes[1], scales[1], dev(slots), dev(low), dev(np.zeros(kv, np.int32)), None, kv, 1, 1, d, 0, stride, d, 1e6, 0)
    got = [[torch.zeros((1, kv, 1, d), device=DEV) for _ in range(2)] for _ in range(2)]
    for at, out in ((slots, got[0]), (low, got[1])):
        cs.cs_kv4_gather(codes[0], scales[0], codes[1], scales[1], dev(at), kv, 1, 1, d, 0, stride, d, *out, cs.CS_F32)
    kq, vq = ko.values(*ko.quantise(k)), ko.values(*ko.quantise(v))
    for out in got:
        assert np.array_equal(out[0][0].double().cpu().numpy(), kq) and np.array_equal(out[1][0].double().cpu().numpy(), vq)
    q64, q = single(rng.normal(size=(n_q, 4, d)), torch.bfloat16)
    pos = np.arange(kv - n_q, kv).astype(np.int32)
    out, lse = torch.zeros_like(q), torch.zeros((n_q, 4), device=DEV)
    i32 = lambda *x: dev(np.array(x, np.int32))
    nbytes = max(cs.cs_kv4_window_attn_workspace(n_q, 1, 4, 1, d, 19), cs.cs_attn_weights_workspace(n_q, 1, 4, 1, d, 19))
    ws = torch.zeros((nbytes,), dtype=torch.uint8, device=DEV)
    cs.cs_kv4_window_attn(q, codes[0], scales[0], codes[1], scales[1], i32(0, n_q), dev(pos), i32(kv), dev(table), 19, 16, out, lse, n_q, 1, 4, 1, d, stride, d, d ** -0.5,
                          cs.CS_BF16, ws)
    want, stat, p = ko.attention(q64, kq, vq, pos, d ** -0.5)
    mass = np.einsum("thj,jhc->thc", p, np.abs(np.repeat(vq, 4, 1)))
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= 3 * B * mass + B * np.abs(want))
    w = torch.zeros((1, 19 * 16), device=DEV)
    cs.cs_attn_weights(q, lse, codes[0], scales[0], i32(0, n_q), dev(pos), i32(kv), dev(table), 19, 16, None, w, 1.0, n_q, 1, 4, 1, d, stride, d, d ** -0.5, cs.CS_BF16, cs.CS_KV4, ws)
    # (sums |q k| scale below 40, on either side of the statistics: 2 (d/8 + 8) u 40)
    assert np.all(np.abs(w[0, :kv].double().cpu().numpy() - p.sum((0, 1))) <= 80 * (d / 8 + 8) * U * p.sum((0, 1)) + 1e-30)


CACHES = [("bf16", "kv4"), ("f32", "kv4"), ("bf16", "bf16"), ("f32", "f32")]


@pytest.mark.parametrize("dtype,cache", CACHES)
@pytest.mark.parametrize("i", [0, 1, 3, 4, 5, 6, 7, 9, 10, 12])
def test_attn_weights(cs, i, dtype, cache):
    hq, hkv, d, kv, nq, where, layout = SHAPES[i]
    say("attention weights", dtype, cache, SHAPES[i])
    b = Batch(cs, 100 + i, hq, hkv, d, kv, nq, dtype, cache=cache, layout=layout, where=where, extra=i % 2)
    before = torch.rand((len(kv), 16 * b.max_blocks), device=DEV)
    got = b.weights(before, 0.75)
    b.check_weights(got, before, 0.75)
    assert torch.equal(got, b.weights(before, 0.75))                       # the same bits again
    b.check_weights(b.weights(None, 1.0), None, 1.0)
    rotten = torch.full_like(before, math.nan)
    b.check_weights(b.weights(rotten, 0.0), None, 0.0)
    lse = np.full((b.n_q, hq), np.nan, np.float32)
    for s in range(len(kv)):
        rows, _, stat, _, _ = b.oracle(s)
        lse[rows] = stat
    given = b.weights(before, 1.0, lse=dev(lse))
    b.check_weights(given, before, 1.0)
    same = before.clone()
    b.weights(same, 1.0, lse=dev(lse), in_place=True)
    for s, n in enumerate(kv):
        assert torch.equal(same[s, :n], given[s, :n]) and torch.equal(same[s, n:], before[s, n:])


def test_attn_weights_of_no_queries_fade(cs):
    say("attention weights, no queries")
    kv = dev(np.array([5, 0, 40], np.int32))
    before = torch.rand((3, 48), device=DEV)
    out = torch.full_like(before, 9.0)
    ws = torch.empty((1024,), dtype=torch.uint8, device=DEV)
    cs.cs_attn_weights(None, None, None, None, None, None, kv, None, 3, 16, before, out, 0.5, 0, 3, 4, 2, 64, 64, 64, 0.1, cs.CS_BF16, cs.CS_KV4, ws)
    for s, n in enumerate((5, 0, 40)):
        assert torch.equal(out[s, :n], before[s, :n] * 0.5) and bool((out[s, n:] == 9).all())


def test_attn_weights_sum_to_the_number_of_rows(cs):
    say("attention weights, total")
    b = Batch(cs, 140, 28, 4, 128, [1500, 900], [300, 500], "bf16", where="sorted")
    out, lse = b.attend()
    got = b.weights(None, 1.0, lse=lse)
    for s, n in enumerate(b.kv):
        assert abs(float(got[s, :n].double().sum()) - b.nq[s] * 28) <= 1e-5 * b.nq[s] * 28


# ------------------------------------------------------------------------------------------ eviction

@pytest.mark.parametrize("kv,budget,first,last", [
    ([1], 1, 0, 0), ([5, 0, 33, 16], 7, 1, 2), ([919], 460, 4, 64), ([3000, 1024, 1025, 1, 2048], 1000, 0, 0), ([300, 20], 16, 10, 10), ([300], 8, 20, 20),
    ([64, 10], 64, 3, 3), ([17000, 16383], 4096, 4, 64), ([100] * 70, 31, 0, 1),
    ([9000, 50, 4097], 3001, 3, 9), ([30001, 24577, 2], 7000, 4, 64), ([40000], 33000, 0, 0)])
@pytest.mark.parametrize("values", ["spread", "ties", "odd"])
def test_plan_evict(cs, kv, budget, first, last, values):
    say("evict", kv[:5], budget, first, last, values)
    rng = np.random.default_rng(len(kv) + budget)
    b, mbo = len(kv), -(-max(kv) // 16) + 1
    mbn = -(-min(budget, 16 * mbo) // 16) + 1
    ids = rng.permutation(b * (mbo + mbn)).astype(np.int32)
    old, new = ids[:b * mbo].reshape(b, mbo), ids[b * mbo:].reshape(b, mbn)
    w = np.exp(rng.normal(size=(b, 16 * mbo)) * 3).astype(np.float32)
    if values == "ties":
        w = np.floor(w).clip(0, 3).astype(np.float32)
    if values == "odd":
        w[rng.random(w.shape) < 0.3] = np.nan
        w[rng.random(w.shape) < 0.1] = np.inf
        w[rng.random(w.shape) < 0.1] = -np.inf
        w[rng.random(w.shape) < 0.1] = -0.0
        w[rng.random(w.shape) < 0.1] = 0.0
        w[rng.random(w.shape) < 0.1] *= -1
        w[rng.random(w.shape) < 0.1] = 1e-42
    for renumber in (True, False):
        lists = [torch.full((b, budget), -7, dtype=torch.int32, device=DEV) for _ in range(4)]
        kv_new = torch.full((b,), -7, dtype=torch.int32, device=DEV)
        w_new = torch.full((b, 16 * mbn), -7.0, device=DEV) if renumber else None
        cs.cs_plan_evict(dev(w), dev(np.array(kv, np.int32)), dev(old), mbo, dev(new), mbn, b, budget, first, last, renumber, *lists, kv_new, w_new)
        kept, src, dst, delta = (t.cpu().numpy() for t in lists)
        for s, n in enumerate(kv):
            want = np.array(ko.evict(w[s], n, budget, first, last), int)
            m = len(want)
            i = np.arange(m)
            assert int(kv_new[s]) == m
            assert kept[s, :m].tolist() == want.tolist() and np.all(kept[s, m:] == -1)
            assert src[s, :m].tolist() == (old[s, want // 16] * 16 + want % 16).tolist() and np.all(src[s, m:] == -1)
            assert dst[s, :m].tolist() == (new[s, i // 16] * 16 + i % 16).tolist() and np.all(dst[s, m:] == -1)
            assert delta[s, :m].tolist() == ((i - want) * int(renumber)).tolist() and np.all(delta[s, m:] == 0)
            if w_new is not None:
                assert np.array_equal(w_new[s, :m].cpu().numpy(), w[s, want], equal_nan=True) and bool((w_new[s, m:] == -7).all())


def test_plan_evict_clamps_lengths_past_the_table(cs):
    say("evict, kv_len past the table and negative")
    w = torch.rand((2, 32), device=DEV)
    lists = [torch.full((2, 20), -7, dtype=torch.int32, device=DEV) for _ in range(4)]
    kv_new = torch.zeros((2,), dtype=torch.int32, device=DEV)
    cs.cs_plan_evict(w, dev(np.array([90, -3], np.int32)), dev(np.arange(4, dtype=np.int32)), 2, dev(np.arange(4, 8, dtype=np.int32)), 2, 2, 20, 1, 1, True, *lists, kv_new, None)
    assert kv_new.tolist() == [20, 0]
    assert lists[0][0].tolist() == ko.evict(w[0].cpu().numpy(), 32, 20, 1, 1) and bool((lists[0][1] == -1).all())


# ------------------------------------------------------------------------------------------ captured, on other streams

def test_calls_in_a_graph_and_on_a_stream_of_their_own(cs):
    say("graph of write, attention, weights, eviction, move; replayed between eager runs")
    rng = np.random.default_rng(9)
    b = Batch(cs, 150, 8, 2, 128, [500, 77], [60, 20], "bf16", where="tail")
    budget = 64
    mbn = 5
    ids = dev(np.arange(int(b.table.max()) + 1, int(b.table.max()) + 1 + 2 * mbn).astype(np.int32)).view(2, mbn)
    big = lambda t: torch.cat([t, torch.zeros((16 * 2 * mbn,) + tuple(t.shape[1:]), dtype=t.dtype, device=DEV)]).contiguous()
    kc, vc, ks, vs = (big(t) for t in (*b.pool, *b.scales))
    sl, sh = 2 * kc.stride(0), 2 * kc.stride(1)
    out, lse = torch.zeros_like(b.q), torch.zeros((b.n_q, 8), device=DEV)
    w_in, w_out = torch.rand((2, 16 * b.max_blocks), device=DEV), torch.zeros((2, 16 * b.max_blocks), device=DEV)
    lists = [torch.zeros((2, budget), dtype=torch.int32, device=DEV) for _ in range(4)]
    kv_new, w_new = torch.zeros((2,), dtype=torch.int32, device=DEV), torch.zeros((2, 16 * mbn), device=DEV)
    new = dev(rng.normal(size=(80, 8 + 4, 128)).astype(np.float32)).bfloat16()
    pos = dev(rng.integers(0, 500, 80).astype(np.int32))
    slot = dev(np.concatenate([[int(b.table[s, p // 16]) * 16 + p % 16 for p in b.pos[s]] for s in range(2)]).astype(np.int32))
    nbytes = cs.cs_kv4_window_attn_workspace(b.n_q, 2, 8, 2, 128, b.max_blocks)
    ws = torch.zeros((nbytes,), dtype=torch.uint8, device=DEV) if nbytes else None
    ww = torch.zeros((cs.cs_attn_weights_workspace(b.n_q, 2, 8, 2, 128, b.max_blocks),), dtype=torch.uint8, device=DEV)
    q = torch.zeros((80, 8, 128), dtype=torch.bfloat16, device=DEV)

    def run():
        cs.cs_rope_refresh_scatter(new, q, new[:, 8:], new[:, 10:], slot, pos, None, kc, vc, ks, vs, 80, 8, 2, 128, new.stride(0), new.stride(0), new.stride(0), sl, sh, 1e6, 0,
                                   cs.CS_BF16, cs.CS_KV4)
        cs.cs_kv4_window_attn(q, kc, ks, vc, vs, b.cu_q, b.q_pos, b.kv_len, b.table, b.max_blocks, 16, out, lse, b.n_q, 2, 8, 2, 128, sl, sh, b.scale, cs.CS_BF16, ws)
        cs.cs_attn_weights(q, lse, kc, ks, b.cu_q, b.q_pos, b.kv_len, b.table, b.max_blocks, 16, w_in, w_out, 0.5, b.n_q, 2, 8, 2, 128, sl, sh, b.scale, cs.CS_BF16, cs.CS_KV4, ww)
        cs.cs_plan_evict(w_out, b.kv_len, b.table, b.max_blocks, ids, mbn, 2, budget, 2, 8, True, *lists, kv_new, w_new)
        cs.cs_kv4_rerotate(kc, ks, vc, vs, lists[1], lists[2], lists[3], None, 2 * budget, 1, 2, 128, 0, sl, sh, 1e6, 0)

    results = (q, out, lse, w_out, *lists, kv_new, w_new, kc, vc, ks, vs)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    want = [t.clone() for t in results]
    assert all(bool(torch.isfinite(t.float()).all()) for t in want[:4])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        for t in (q, out, lse, *lists, kv_new):
            t.fill_(1)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(results, want))
        run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(results, want))


# ------------------------------------------------------------------------------------------ a step over a 4-bit cache

@pytest.mark.parametrize("axes", ["one", "sections"])
def test_step_over_a_4bit_cache(cs, axes):
    """engine.Kv4Step (scoring, plan, position correction, rotary embedding with the write, attention, weights; then an eviction)
    against the oracles, twice eagerly and replayed from a graph."""
    from dataclasses import replace

    from paper_2604_06036_amd import engine, synth
    from tests import helpers as hp
    say("Kv4Step", axes)
    w = replace(synth.CFG2, n_streams=2, n_layers=2, n_q_heads=8, n_kv_heads=2, head_dim=64)
    data = engine.assemble_step(w, engine.hip_scorer, device="cpu")
    n_q, cap = data.info["n_q"], data.info["n_q"] + 37
    rng = np.random.default_rng(5)
    axis = AXES[axes](32)
    pos = rng.integers(0, 2500, (cap, 3) if axis is not None else (cap,)).astype(np.int32)
    plan = hp.OraclePlan(data)
    pools = [ko.quantise(t.float().numpy()) for t in (data.k_pool, data.v_pool)]
    step = engine.Kv4Step(data, pos, axis, reuse_cap=data.info["n_reuse"] + 11, q_cap=cap, weigh=True)
    codes = [t.clone() for t in (step.k_codes, step.k_scales, step.v_codes, step.v_scales)]
    for (c, s), got_c, got_s in ((pools[0], step.k_codes, step.k_scales), (pools[1], step.v_codes, step.v_scales)):
        assert np.array_equal(got_s.cpu().numpy(), s) and np.array_equal(ko.values(got_c.cpu().numpy(), s), ko.values(c, s))
    step.run()
    torch.cuda.synchronize()
    assert step.scoring_status() == 0
    hp.assert_device_plan(step, plan)
    # reused rows corrected, executed rows turned and written, then attention over them
    delta = plan.delta if axis is None else np.tile(np.array([-w.stride, 0, 0], np.int32), (len(plan.delta), 1))
    u, total = U, [np.zeros(int(n)) for n in plan.kv_len]
    slack = [np.zeros(int(n)) for n in plan.kv_len]
    for l in range(2):
        k, v = (ko.values(c[l], s[l]) for c, s in pools)
        k[plan.dst_slot] = ko.values(*ko.quantise(ko.rope_single(k[plan.src_slot].astype(np.float32), delta, axis, w.rope_base, 0)))
        v[plan.dst_slot] = v[plan.src_slot]
        k[plan.q_slot] = ko.values(*ko.quantise(ko.rope_single(data.k_new[l].float().numpy(), pos[:n_q], axis, w.rope_base, 0)))
        v[plan.q_slot] = ko.values(*ko.quantise(data.v_new[l].double().numpy()))
        q = single(ko.rope_single(data.q[l].float().numpy(), pos[:n_q], axis, w.rope_base, 0), torch.bfloat16)[0]
        for s in range(2):
            rows = slice(int(plan.cu_q[s]), int(plan.cu_q[s + 1]))
            n = int(plan.kv_len[s])
            slots = np.array([plan.block_table[s, j // 16] * 16 + j % 16 for j in range(n)])
            out, lse, p = ko.attention(q[rows], k[slots], v[slots], plan.q_pos[rows], data.softmax_scale)
            mass = np.einsum("thj,jhc->thc", p, np.abs(np.repeat(v[slots], 4, 1)))
            score = data.softmax_scale * max(float((np.abs(q[rows][:, h]) @ np.abs(k[slots][:, h // 4]).T).max()) for h in range(8))
            e = (64 / 8 + 8) * u * score + 4 * u * 2 * score
            got = step.out[l][rows].double().cpu().numpy()
            assert np.all(np.abs(got - out) <= (2 * e + 2 * B + (8 + n / 8) * u) * mass + B * np.abs(out))
            total[s] += p.sum((0, 1))
            slack[s] += (2 * e + 16 * u) * p.sum((0, 1)) + (len(q[rows]) / 2 + 80) * u * p.sum((0, 1))
    for s in range(2):
        n = int(plan.kv_len[s])
        assert np.all(np.abs(step.weight[s, :n].double().cpu().numpy() - total[s]) <= slack[s] + 1e-30)
    # once more, and from a graph, from the same cached windows
    first = step.out.clone()
    weight = step.weight.clone()

    def restore():
        for t, c in zip((step.k_codes, step.k_scales, step.v_codes, step.v_scales), codes):
            t.copy_(c)

    restore()
    step.run()
    torch.cuda.synchronize()
    assert torch.equal(step.out, first) and torch.equal(step.weight, weight)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.run()
    for _ in range(3):
        restore()
        step.out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(step.out, first) and torch.equal(step.weight, weight)
    # the windows cut to half, into the blocks of the window before
    budget = int(plan.kv_len.max()) // 2
    table = step.bt_old[:, :-(-budget // 16)].contiguous()
    before = [step.k_codes.cpu().numpy(), step.v_codes.cpu().numpy(), step.k_scales.cpu().numpy(), step.v_scales.cpu().numpy()]
    kept, kv_new, w_new = step.evict(budget, table, n_first=2, n_last=16)
    torch.cuda.synchronize()
    after = [step.k_codes.cpu().numpy(), step.v_codes.cpu().numpy(), step.k_scales.cpu().numpy(), step.v_scales.cpu().numpy()]
    for s in range(2):
        n = int(plan.kv_len[s])
        want = np.array(ko.evict(weight[s].cpu().numpy(), n, budget, 2, 16))
        assert int(kv_new[s]) == len(want) and kept[s, :len(want)].tolist() == want.tolist()
        assert np.array_equal(w_new[s, :len(want)].cpu().numpy(), weight[s].cpu().numpy()[want])
        t = table.cpu().numpy()
        src = plan.block_table[s, want // 16] * 16 + want % 16
        dst = t[s, np.arange(len(want)) // 16] * 16 + np.arange(len(want)) % 16
        for i in range(2):
            assert np.array_equal(ko.values(after[i][:, dst], after[i + 2][:, dst]), ko.values(before[i][:, src], before[i + 2][:, src]))


def test_step_over_a_4bit_cache_refuses_what_does_not_fit(cs):
    from paper_2604_06036_amd import engine, synth
    say("Kv4Step refusals")
    w = synth.small_variant(synth.CFG1, n_layers=1)
    data = engine.assemble_step(w, engine.hip_scorer, device="cpu")
    with pytest.raises(ValueError, match="positions"):
        engine.Kv4Step(data, np.zeros(data.info["n_q"] - 1, np.int32))
    with pytest.raises(ValueError, match="positions"):
        engine.Kv4Step(data, np.zeros(data.info["n_q"], np.int32), AXES["sections"](64))
    step = engine.Kv4Step(data, np.zeros(data.info["n_q"], np.int32))
    with pytest.raises(ValueError, match="weigh"):
        step.evict(100, step.bt_old)
