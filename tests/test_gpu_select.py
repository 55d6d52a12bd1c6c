"""Operators of long windows (norms with rotation and the cache write, corrections by a table of frequencies, block bounds, selection,
attention over selected blocks) against oracle/select_oracle.py, through the C ABI (needs an MI355X).

Tolerances.  u = 2^-24 (half a step of fp32), b = 2^-8 (of bf16).
Norm: the sum of squares is off by at most 20 u of itself (16 terms of a lane, four exchanges), its mean with eps by 22 u, the inverse root by half
of that and its own 2 u, the two products by u each: 16 u of the element in all.  Rotation: cosine and sine are off by 2 u (their own rounding and
the amplitude's), products and their sum by 3 u of |a| + |b|; so 21 u amplitude (|a| + |b|) before the last rounding.
Attention: a score is a sum of d products, each addition off by u of what is summed: e = (d + 8) u scale sum_c |q_c k_c|.  The exponent's argument
is off by that and by 4 u |argument|, a weight by 4 u more from the exponential, and by b where it is rounded to bf16; a sum of n weighted
values by n u of its terms."""
import math
import sys

import numpy as np
import pytest
import torch

from oracle import select_oracle as so

pytestmark = pytest.mark.gpu
DEV = "cuda"
U, B = 2.0 ** -24, 2.0 ** -8
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


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


def single(x, t):
    """float64 of numbers rounded to the torch type, and the tensor."""
    r = torch.from_numpy(np.asarray(x, np.float32)).to(t)
    return r.to(torch.float32).numpy().astype(np.float64), r.to(DEV)


def f64(t):
    return t.detach().cpu().to(torch.float32).numpy().astype(np.float64)


def pool(layout, layers, n_slots, heads, width, t, fill=0.0):
    shape = (layers, n_slots, heads, width) if layout == "slot" else (layers, heads, n_slots, width)
    x = torch.full(shape, fill, dtype=t, device=DEV)
    return x if layout == "slot" else x.transpose(1, 2)


AXES = {"one": lambda n: None, "sections": lambda n: np.repeat([0, 1, 2], [n // 4, 3 * n // 8, n - n // 4 - 3 * n // 8]).astype(np.uint8),
        "interleaved": lambda n: (np.arange(n) % 3).astype(np.uint8), "past": lambda n: (np.arange(n) % 5).astype(np.uint8)}


def freqs(rng, rotary):
    f = 1e6 ** (-2.0 * np.arange(rotary // 2) / max(1, rotary)) * np.where(rng.random(rotary // 2) < 0.5, 0.25, 1.0)
    return f.astype(np.float32)


def pair_sum(x, rotary, style):
    """|a| + |b| of every element's pair; past the rotated part 0."""
    y = np.zeros_like(x)
    for i in range(rotary // 2):
        a, b = (i, i + rotary // 2) if style == 0 else (2 * i, 2 * i + 1)
        y[..., a] = y[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return y


# ------------------------------------------------------------------------------------------ norms, rotation, write

def run_write(cs, seed, n, hq, hkv, d, rotary, dtype, axes, style, layout, q_normed=True, k_normed=True, fused=True, pos=True, in_place=False, amplitude=1.0, eps=1e-6, x=None):
    rng = np.random.default_rng(seed)
    t, code = TORCH[dtype], cs.CS_BF16 if dtype == "bf16" else cs.CS_F32
    axis = AXES[axes](rotary // 2)
    where = rng.integers(-70000, 70000, (n, 3) if axis is not None else (n,)).astype(np.int32)
    where[0] = 0
    f = freqs(rng, rotary)
    x64, x = single(rng.normal(size=(n, (hq + 2 * hkv) * d)) * np.exp(rng.normal(size=(n, 1)) * 3) if x is None else x, t)
    parts = (x[:, :hq * d], x[:, hq * d:(hq + hkv) * d], x[:, (hq + hkv) * d:])
    q, k, v = parts if fused else (p.contiguous() for p in parts)
    qw64, qw = single(rng.normal(size=d) + 1, t)
    kw64, kw = single(rng.normal(size=d) + 1, t)
    n_slots = n + 19
    slot = rng.permutation(n_slots)[:n].astype(np.int32)
    if n > 3:
        slot[rng.random(n) < 0.1] = -1
    kc, vc = (pool(layout, 1, n_slots, max(1, hkv), d, t, 7.0) for _ in range(2))
    out = q if in_place else torch.full((n, max(1, hq), d), 5.0, dtype=t, device=DEV)
    none = lambda c, v_: v_ if c else None
    cs.cs_norm_rope_refresh_scatter(none(hq, q), none(hq, out), none(hkv, k), none(hkv, v), none(hq and q_normed, qw), none(hkv and k_normed, kw), none(hkv, dev(slot)),
                                    none(pos, dev(where)), None if axis is None else dev(axis), none(pos and rotary, dev(f)), none(hkv, kc), none(hkv, vc), n, hq, hkv, d, rotary,
                                    q.stride(0) if hq else 0, k.stride(0) if hkv else 0, v.stride(0) if hkv else 0, kc.stride(1), kc.stride(2), eps, amplitude, style, code)
    torch.cuda.synchronize()
    q64, k64, v64 = (p.reshape(n, -1, d) for p in (x64[:, :hq * d], x64[:, hq * d:(hq + hkv) * d], x64[:, (hq + hkv) * d:]))

    def near(got, x_, w, what):
        y = so.norm(x_, w, eps)
        want = so.turn(y, where, axis, f, rotary, style, amplitude) if pos else y
        fresh = 16 * U * np.abs(y) if w is not None else 0.0 * np.abs(y)
        if pos and rotary:
            pair = pair_sum(y, rotary, style) * abs(amplitude)
            fresh = np.where(pair_sum(np.ones_like(y), rotary, style) > 0, (16 * (w is not None) + 5) * U * pair, fresh)
        tol = fresh + (B if dtype == "bf16" else U) * (np.abs(want) + fresh)
        # Below 2^-126 numbers are multiples of 2^-133 (bf16) and 2^-149 (fp32), so a rounding is off by half of that whatever the number:
        # one to bf16, and up to seven single-precision steps before it (a scaling, three products of the norm, products and sum of the turn).
        tol = tol + (2.0 ** -134 if dtype == "bf16" else 0.0) + 7 * 2.0 ** -150
        got = f64(got)
        assert np.array_equal(np.isfinite(got), np.isfinite(want)), what
        fine = np.isfinite(want)
        assert np.all(np.abs(got - want)[fine] <= tol[fine]), (what, float((np.abs(got - want) - tol)[fine].max()))

    if hq:
        near(out.reshape(n, hq, d) if not in_place else out.reshape(n, hq, d), q64, qw64 if q_normed else None, "q")
    if hkv:
        live = np.flatnonzero(slot >= 0)
        at = slot[live]
        other = np.setdiff1d(np.arange(n_slots), at)
        full = torch.zeros((n, hkv, d), dtype=t, device=DEV)
        full[live] = kc[0][at]
        whole = k64.copy()
        whole[slot < 0] = 0
        near(full, whole, kw64 if k_normed else None, "k")
        assert torch.equal(vc[0][at].view(torch.int16 if dtype == "bf16" else torch.int32), v.reshape(n, hkv, d)[live].contiguous().view(torch.int16 if dtype == "bf16" else torch.int32))
        assert bool((kc[0][other] == 7).all()) and bool((vc[0][other] == 7).all())


@pytest.mark.parametrize("n,hq,hkv,d,rotary,dtype,axes,style,layout,more", [
    (1, 28, 4, 128, 128, "bf16", "sections", 0, "slot", {}),
    (37, 4, 2, 64, 32, "bf16", "interleaved", 0, "slot", dict(amplitude=1.1386)),
    (37, 4, 2, 64, 64, "bf16", "past", 1, "head", dict(fused=False)),
    (130, 2, 1, 64, 16, "f32", "one", 0, "slot", {}),
    (65, 3, 3, 128, 64, "f32", "sections", 1, "slot", dict(amplitude=-0.5)),
    (9, 2, 2, 192, 96, "f32", "interleaved", 0, "head", {}),
    (9, 1, 2, 256, 256, "bf16", "one", 1, "slot", {}),
    (9, 2, 1, 256, 48, "f32", "one", 0, "slot", {}),
    (50, 5, 1, 80, 80, "f32", "interleaved", 1, "head", dict(fused=False)),
    (51, 5, 2, 80, 32, "bf16", "one", 0, "head", {}),
    (51, 3, 2, 48, 16, "f32", "one", 1, "slot", {}),
    (3, 2, 2, 16, 16, "bf16", "one", 0, "slot", {}),
    (21, 4, 2, 32, 0, "bf16", "one", 0, "slot", {}),                           # nothing is rotated
    (21, 4, 2, 128, 64, "bf16", "one", 0, "slot", dict(pos=False)),            # no positions
    (33, 0, 2, 64, 32, "bf16", "sections", 0, "slot", {}),                     # keys and values only
    (33, 4, 0, 64, 32, "f32", "sections", 0, "slot", {}),                      # queries only
    (33, 4, 2, 128, 128, "f32", "one", 0, "slot", dict(q_normed=False)),
    (33, 4, 2, 128, 128, "bf16", "one", 1, "slot", dict(k_normed=False)),
    (33, 4, 2, 128, 64, "bf16", "one", 0, "slot", dict(q_normed=False, k_normed=False, amplitude=1.25)),
    (33, 4, 2, 128, 64, "bf16", "one", 0, "slot", dict(in_place=True)),
    (33, 4, 2, 80, 32, "f32", "one", 1, "slot", dict(in_place=True)),
    (2500, 8, 2, 128, 128, "bf16", "sections", 0, "head", {}),
    (9000, 5, 1, 64, 32, "bf16", "one", 0, "slot", {}),
    (5, 2, 2, 64, 64, "f32", "one", 0, "slot", dict(eps=1e-30)),
    (5, 2, 2, 64, 64, "f32", "one", 0, "slot", dict(eps=0.5)),
])
def test_write(cs, n, hq, hkv, d, rotary, dtype, axes, style, layout, more):
    say("write", n, hq, hkv, d, rotary, dtype, axes, style, layout, more)
    run_write(cs, n + d + rotary, n, hq, hkv, d, rotary, dtype, axes, style, layout, **more)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64), ("f32", 80)])
def test_write_of_large_small_and_no_numbers(cs, dtype, d):
    """Heads whose squares pass the largest number, heads of zeros, and what is no number: it stays in its head."""
    say("write, odd numbers", dtype, d)
    rng = np.random.default_rng(3)
    n, hq, hkv = 12, 2, 1
    x = rng.normal(size=(n, hq + 2 * hkv, d))
    x[1] *= 1e30
    x[2, 0, 5] = 3e38
    x[3] = 0
    x[4] *= 1e-30
    x[5, 1] *= 1e19
    x[6, 2, 7], x[7, 0, 3], x[8, 1, 0] = np.nan, np.nan, np.nan
    x[9, 3, 2] = np.nan                    # (a value: copied)
    run_write(cs, 5, n, hq, hkv, d, 32, dtype, "one", 0, "slot", x=x.reshape(n, -1))


def test_write_infinities(cs):
    """An infinite element makes the others of its head 0 and itself no number, as the formula does."""
    say("write, infinities")
    d = 64
    x = np.ones((2, 1, d), np.float32)
    x[0, 0, 40] = np.inf
    out = torch.zeros((2, 1, d), device=DEV)
    cs.cs_norm_rope_refresh_scatter(dev(x), out, None, None, torch.ones((d,), device=DEV), None, None, None, None, None, None, None, 2, 1, 0, d, 0, d, 0, 0, 0, 0, 1e-6, 1.0, 0, cs.CS_F32)
    got = out[:, 0].cpu().numpy()
    assert np.isnan(got[0, 40]) and np.all(np.delete(got[0], 40) == 0) and np.allclose(got[1], 1.0, atol=1e-5)


# ------------------------------------------------------------------------------------------ correction by a table of frequencies

@pytest.mark.parametrize("n,layers,hkv,d,rotary,dtype,axes,style,layout,in_place", [
    (1, 1, 1, 64, 64, "bf16", "one", 0, "slot", False), (300, 3, 4, 128, 64, "bf16", "one", 0, "head", False), (77, 2, 2, 128, 128, "f32", "sections", 1, "slot", False),
    (77, 5, 3, 64, 16, "bf16", "interleaved", 0, "slot", True), (33, 2, 1, 192, 96, "f32", "past", 0, "head", False), (33, 2, 2, 256, 32, "f32", "one", 1, "slot", True),
    (33, 6, 2, 80, 48, "bf16", "one", 1, "slot", False), (5, 2, 1, 16, 16, "bf16", "one", 0, "slot", True), (5000, 2, 8, 128, 32, "bf16", "one", 0, "slot", False)])
def test_rerotate_freqs(cs, n, layers, hkv, d, rotary, dtype, axes, style, layout, in_place):
    say("rerotate", n, layers, hkv, d, rotary, dtype, axes, style, layout, in_place)
    rng = np.random.default_rng(n + d)
    t = TORCH[dtype]
    n_slots = 2 * n + 3
    axis, f = AXES[axes](rotary // 2), freqs(rng, rotary)
    k, v = (pool(layout, layers, n_slots, hkv, d, t) for _ in range(2))
    for x in (k, v):
        x.copy_(dev(rng.normal(size=tuple(x.shape)).astype(np.float32)))
    k[0, 0, 0, d - 1] = float("nan")       # (past the rotated part, or its partner's)
    v[0, 0, 0, 0] = float("nan")
    before, v_before = f64(k), v.clone()
    perm = rng.permutation(n_slots).astype(np.int32)
    src, dst = perm[:n].copy(), perm[n:2 * n].copy()
    if n > 5:
        src[3] = -1
        dst[4] = -1
    delta = rng.integers(-4000, 4000, (n, 3) if axis is not None else (n,)).astype(np.int32)
    cs.cs_kv_rerotate_freqs(k, None if in_place else v, dev(src), None if in_place else dev(dst), dev(delta), None if axis is None else dev(axis), dev(f), n, layers, hkv, d, rotary,
                            k.stride(0), k.stride(1), k.stride(2), style, cs.CS_BF16 if dtype == "bf16" else cs.CS_F32)
    to = src if in_place else dst
    live = (src >= 0) & (to >= 0)
    after = f64(k)
    rest = np.setdiff1d(np.arange(n_slots), to[live])
    bits = torch.int16 if dtype == "bf16" else torch.int32
    want_v = v_before.clone()
    if not in_place:
        want_v[:, dst[live]] = v_before[:, src[live]]
    assert torch.equal(v.contiguous().view(bits), want_v.contiguous().view(bits))
    for l in range(layers):
        assert np.array_equal(after[l, rest], before[l, rest], equal_nan=True)
        x = before[l, src[live]]
        want = so.turn(x, delta[live], axis, f, rotary, style)
        got = after[l, to[live]]
        assert np.array_equal(np.isnan(got), np.isnan(want))
        # cosines and sines within 4 u (polynomials in single precision), products and sum 3 u, storage
        fresh = 7 * U * pair_sum(x, rotary, style)
        tol = fresh + (B if dtype == "bf16" else U) * (np.abs(want) + fresh)
        fine = ~np.isnan(want)
        assert np.all(np.abs(got - want)[fine] <= tol[fine]), float((np.abs(got - want) - tol)[fine].max())
        assert np.array_equal(got[..., rotary:], x[..., rotary:], equal_nan=True)


# ------------------------------------------------------------------------------------------ caches

class Cache:
    """A paged cache of streams of these lengths.  Rows that no window holds, and rows past a window's end in its last block, are NaN."""

    def __init__(self, cs, seed, hkv, d, kv, dtype, layout="slot", gain=1.0, wide=0):
        rng = np.random.default_rng(seed)
        self.cs, self.rng, self.hkv, self.d, self.kv, self.dtype = cs, rng, hkv, d, kv, dtype
        self.t, self.code = TORCH[dtype], cs.CS_BF16 if dtype == "bf16" else cs.CS_F32
        need = [max(0, -(-n // 16)) for n in kv]
        self.max_blocks = max(1, max(need)) + 1 + wide
        n_slots = 16 * (sum(need) + 2)
        ids = rng.permutation(sum(need) + 2)
        table = np.full((len(kv), self.max_blocks), ids[-1], np.int32)       # a block of NaN
        at = 0
        for s, m in enumerate(need):
            table[s, :m] = ids[at:at + m]
            at += m
        self.slots = [np.array([table[s, j // 16] * 16 + j % 16 for j in range(max(0, n))], np.int64) for s, n in enumerate(kv)]
        used = np.concatenate(self.slots).astype(int)
        self.x64, self.pool = [], []
        for _ in range(2):
            x = rng.normal(size=(n_slots, hkv, d)) * gain
            x[np.setdiff1d(np.arange(n_slots), used)] = np.nan
            r64, r = single(x, self.t)
            p = pool(layout, 1, n_slots, hkv, d, self.t)[0]
            p.copy_(r)
            self.x64.append(r64)
            self.pool.append(p)
        self.table, self.kv_len = dev(table), dev(np.array(kv, np.int32))
        self.stride = (self.pool[0].stride(0), self.pool[0].stride(1))

    def put(self, which, s, j, h, c, value):
        """Entry j of stream s: keys (which 0) or values (1)."""
        at = self.slots[s][j]
        self.x64[which][at, h, c] = value
        self.pool[which][int(at), h, c] = value

    def n_sel(self, size):
        return -(-self.max_blocks // (size // 16))

    def bounds(self, size, since=None, fill=(77, 99)):
        b = torch.full((len(self.kv), self.hkv, self.n_sel(size), 2, self.d), fill[0], dtype=torch.int8, device=DEV)
        sc = torch.full((len(self.kv), self.hkv, self.n_sel(size)), fill[1], dtype=torch.uint8, device=DEV)
        self.cs.cs_key_bounds(self.pool[0], None if since is None else dev(np.array(since, np.int32)), self.kv_len, self.table, self.max_blocks, 16, size, b, sc, len(self.kv), self.hkv,
                              self.d, *self.stride, self.code)
        torch.cuda.synchronize()
        return b, sc

    def want_bounds(self, size, since=None, fill=(77, 99)):
        b = np.full((len(self.kv), self.hkv, self.n_sel(size), 2, self.d), fill[0], np.int64)
        sc = np.full((len(self.kv), self.hkv, self.n_sel(size)), fill[1], np.int64)
        for s, n in enumerate(self.kv):
            first = 0 if since is None else max(0, since[s]) // size
            for i in range(first, -(-max(0, n) // size)):
                rows = self.slots[s][i * size:(i + 1) * size]
                for h in range(self.hkv):
                    b[s, h, i, 0], b[s, h, i, 1], sc[s, h, i] = so.block_bounds(self.x64[0][rows, h])
        return b, sc

    def queries(self, nq, hq, gain=1.0, where="any", extra=0):
        """Tokens a stream, their positions, rows past the last stream."""
        rng = self.rng
        pos = []
        for n, m in zip(self.kv, nq):
            if where == "tail":
                pos.append(np.arange(n - m, n))
            else:
                pos.append(rng.integers(-2 if where == "any" else 0, max(1, n + 3), m))
        n_q = sum(nq) + extra
        q64, q = single(rng.normal(size=(n_q, hq, self.d)) * gain, self.t)
        pos = np.concatenate(pos + [np.full(extra, 1 << 30)]).astype(np.int32)
        return dict(hq=hq, nq=nq, n_q=n_q, q64=q64, q=q, pos=pos, q_pos=dev(pos), cu_q=dev(np.concatenate([[0], np.cumsum(nq)]).astype(np.int32)),
                    stream=np.repeat(np.arange(len(nq)), nq))

    def select(self, qs, size, n_select, n_first, n_last, bounds=None):
        b, sc = bounds or self.bounds(size)
        out = torch.full((qs["n_q"], self.hkv, n_select), -7, dtype=torch.int32, device=DEV)
        nbytes = self.cs.cs_select_blocks_workspace(qs["n_q"], len(self.kv), qs["hq"], self.hkv, self.d, self.max_blocks, size)
        ws = torch.full((max(16, nbytes),), 171, dtype=torch.uint8, device=DEV)
        self.cs.cs_select_blocks(qs["q"], b, sc, qs["cu_q"], qs["q_pos"], self.kv_len, self.max_blocks, size, n_select, n_first, n_last, out, qs["n_q"], len(self.kv), qs["hq"], self.hkv,
                                 self.d, self.code, ws)
        torch.cuda.synchronize()
        return out

    def want_selected(self, qs, size, n_select, n_first, n_last):
        b, sc = self.want_bounds(size)
        out = np.full((qs["n_q"], self.hkv, n_select), -7, np.int64)
        group = qs["hq"] // self.hkv
        for t, s in enumerate(qs["stream"]):
            n = so.candidates(int(qs["pos"][t]), min(self.kv[s], 16 * self.max_blocks), size)
            for g in range(self.hkv):
                codes = so.query_codes(qs["q64"][t, g * group:(g + 1) * group])
                scores = [so.block_score(codes, b[s, g, i, 0], b[s, g, i, 1], sc[s, g, i]) for i in range(n)]
                if not np.isfinite(qs["q64"][t, g * group:(g + 1) * group]).all():
                    scores = [math.inf if sc[s, g, i] == 255 else 0.0 for i in range(n)]
                out[t, g] = so.select(scores, n, n_select, n_first, n_last)
        return out

    def attend(self, qs, listed, size, scale=None, lse=True, stream=None):
        n_select = listed.shape[-1]
        scale = 1.0 / math.sqrt(self.d) if scale is None else scale
        out = torch.full((qs["n_q"], qs["hq"], self.d), 9.0, dtype=self.t, device=DEV)
        stat = torch.full((qs["n_q"], qs["hq"]), 9.0, device=DEV) if lse else None
        nbytes = self.cs.cs_selected_attn_workspace(qs["n_q"], len(self.kv), qs["hq"], self.hkv, self.d, size, n_select)
        ws = torch.full((max(16, nbytes),), 255, dtype=torch.uint8, device=DEV)
        self.cs.cs_selected_attn(qs["q"], self.pool[0], self.pool[1], qs["cu_q"], qs["q_pos"], self.kv_len, self.table, self.max_blocks, 16, listed, size, n_select, out, stat, qs["n_q"],
                                 len(self.kv), qs["hq"], self.hkv, self.d, *self.stride, scale, self.code, ws)
        torch.cuda.synchronize()
        return out, stat

    def check_attention(self, qs, listed, size, out, stat, scale=None):
        """Every row against the oracle."""
        scale = 1.0 / math.sqrt(self.d) if scale is None else scale
        listed = listed.cpu().numpy() if isinstance(listed, torch.Tensor) else listed
        got, lse = f64(out), None if stat is None else f64(stat)
        group, n_rows = qs["hq"] // self.hkv, len(qs["stream"])
        assert np.all(got[n_rows:] == 9.0) and (lse is None or np.all(lse[n_rows:] == 9.0))
        for t, s in enumerate(qs["stream"]):
            n = min(self.kv[s], 16 * self.max_blocks)
            if n <= 0:
                assert np.all(got[t] == 9.0) and (lse is None or np.all(lse[t] == 9.0))
                continue
            for g in range(self.hkv):
                rows = self.slots[s][so.seen(listed[t, g], int(qs["pos"][t]), n, size)] if n else []
                heads = slice(g * group, (g + 1) * group)
                q, k, v = qs["q64"][t, heads], self.x64[0][rows, g], self.x64[1][rows, g]
                want, wl = so.attend(q, k, v, scale)
                if len(rows) == 0:
                    assert np.all(got[t, heads] == 0) and (lse is None or np.all(lse[t, heads] == -np.inf))
                    continue
                with np.errstate(invalid="ignore", over="ignore"):
                    x = scale * (q @ k.T)
                    p = np.exp(x - wl[:, None])
                    e = (self.d + 8) * U * scale * (np.abs(q) @ np.abs(k).T)
                    weight = e + 4 * U * np.abs(x - x.max(-1, keepdims=True)) + 8 * U
                    spread = (p * weight).sum(-1, keepdims=True)                 # how far the sum of the weights is off
                    each = p * (weight + (B if self.dtype == "bf16" else 0.0) + len(rows) * U + spread)
                    tol = each @ np.abs(v) + 1e-30
                    tol += (B if self.dtype == "bf16" else U) * (np.abs(want) + tol)
                    tol_l = spread[:, 0] + 8 * U * (1 + np.abs(wl) + len(rows) / 8)
                same = np.isfinite(want) == np.isfinite(got[t, heads])
                assert same.all(), ("finite", t, g)
                fine = np.isfinite(want)
                err = np.abs(got[t, heads] - want)
                assert np.all(err[fine] <= tol[fine]), ("out", t, g, float((err - tol)[fine].max()))
                odd = np.isinf(want)
                assert np.array_equal(got[t, heads][odd], want[odd])
                if lse is not None:
                    fine = np.isfinite(wl)
                    assert np.array_equal(fine, np.isfinite(lse[t, heads])), ("lse", t, g)
                    assert np.all(np.abs(lse[t, heads] - wl)[fine] <= tol_l[fine]), ("lse", t, g, float((np.abs(lse[t, heads] - wl) - tol_l)[fine].max()))


# ------------------------------------------------------------------------------------------ bounds

@pytest.mark.parametrize("kv,hkv,d,dtype,layout,size", [
    ([1], 1, 64, "bf16", "slot", 16), ([0, 5, 16, 17, 63], 2, 128, "bf16", "slot", 64), ([64, 65, 200], 4, 128, "bf16", "head", 64), ([130, 33], 3, 64, "f32", "slot", 32),
    ([257], 2, 128, "f32", "head", 128), ([100, 3], 1, 64, "bf16", "head", 48), ([300], 8, 128, "bf16", "slot", 16), ([81, 97], 2, 64, "f32", "head", 112), ([1000], 2, 128, "bf16", "slot", 64)])
def test_bounds(cs, kv, hkv, d, dtype, layout, size):
    say("bounds", kv, hkv, d, dtype, layout, size)
    c = Cache(cs, sum(kv) + d + size, hkv, d, kv, dtype, layout, gain=3.0, wide=2)
    for since in (None, [max(0, n - 1) for n in kv], [n // 2 for n in kv], [-5] * len(kv), [n + 100 for n in kv]):
        (b, sc), (wb, ws) = c.bounds(size, since), c.want_bounds(size, since)
        assert np.array_equal(sc.cpu().numpy(), ws) and np.array_equal(b.cpu().numpy(), wb), since


def test_bounds_of_odd_numbers(cs):
    """Tiny, huge and mixed keys, a zero block, and blocks that hold what is no number."""
    say("bounds, odd numbers")
    for dtype in ("bf16", "f32"):
        c = Cache(cs, 4, 2, 64, [160, 40], dtype)
        for j in range(16):
            for h in range(2):
                for col in range(64):
                    c.put(0, 0, j, h, col, 0.0)
                    c.put(0, 0, 16 + j, h, col, float(c.x64[0][c.slots[0][16 + j], h, col]) * 2.0 ** -100)
        c.put(0, 0, 16, 0, 3, 1e-38)
        c.put(0, 0, 35, 0, 9, 3e38)
        c.put(0, 0, 36, 0, 10, -1e-37)
        c.put(0, 0, 50, 1, 0, float("nan"))
        c.put(0, 0, 70, 0, 63, float("inf"))
        c.put(0, 0, 90, 1, 5, float("-inf"))
        for x in (127.0, -127.0, 127.5, 126.5):
            c.put(0, 1, 20, 0, 0, x)
            (b, sc), (wb, ws) = c.bounds(16), c.want_bounds(16)
            assert np.array_equal(sc.cpu().numpy(), ws) and np.array_equal(b.cpu().numpy(), wb)
        assert (ws == 255).sum() == 3


def test_bounds_table_shorter_than_said(cs):
    """kv_len past the table's rows is clamped to them."""
    say("bounds, clamped length")
    c = Cache(cs, 9, 2, 64, [64], "bf16")
    c.max_blocks = 4
    c.table = c.table[:, :4].contiguous()
    want = c.want_bounds(32)
    c.kv_len.fill_(1000)
    b, sc = c.bounds(32)
    assert np.array_equal(b.cpu().numpy(), want[0]) and np.array_equal(sc.cpu().numpy(), want[1])


# ------------------------------------------------------------------------------------------ selection

@pytest.mark.parametrize("kv,nq,hq,hkv,d,dtype,size,n_select,n_first,n_last,where", [
    ([1], [1], 1, 1, 64, "bf16", 16, 1, 0, 0, "tail"),
    ([300], [1], 28, 4, 128, "bf16", 16, 5, 1, 2, "tail"),
    ([0, 17, 700, 333], [0, 3, 9, 20], 7, 1, 128, "bf16", 16, 8, 1, 1, "any"),
    ([700, 80], [40, 7], 8, 8, 64, "bf16", 16, 3, 0, 1, "any"),                  # group 1
    ([500, 80], [30, 7], 4, 2, 64, "f32", 32, 4, 2, 2, "any"),                   # group 2, all of the list fixed
    ([900], [33], 16, 4, 128, "f32", 64, 6, 0, 0, "any"),                        # group 4
    ([450, 450, 450], [5, 1, 11], 32, 2, 64, "bf16", 48, 2, 0, 0, "any"),        # group 16
    ([600], [13], 15, 3, 128, "bf16", 16, 33, 3, 5, "any"),                      # group 5
    ([2000], [4], 12, 1, 64, "bf16", 16, 64, 1, 2, "any"),
    ([5000], [3], 6, 2, 64, "bf16", 16, 256, 0, 7, "tail"),                      # past 256 blocks
    ([12000], [2], 4, 1, 64, "bf16", 16, 20, 1, 2, "tail"),                      # past 512 blocks
    ([100] * 70, [1] * 70, 7, 1, 64, "bf16", 16, 4, 1, 1, "any"),                # more streams than lanes
    ([15000], [9], 2, 1, 64, "bf16", 16, 30, 1, 2, "tail"),                      # past 512 blocks, many tokens
    ([20000], [1], 2, 1, 64, "bf16", 16, 12, 1, 2, "tail"),                      # past 1,024
])
def test_selection(cs, kv, nq, hq, hkv, d, dtype, size, n_select, n_first, n_last, where):
    say("select", len(kv), sum(nq), hq, hkv, d, dtype, size, n_select, n_first, n_last, where)
    c = Cache(cs, sum(kv) + d, hkv, d, kv, dtype)
    qs = c.queries(nq, hq, where=where, extra=3)
    got = c.select(qs, size, n_select, n_first, n_last).cpu().numpy()
    assert np.array_equal(got, c.want_selected(qs, size, n_select, n_first, n_last))


@pytest.mark.parametrize("n_blocks,nq", [(2500, 1), (2500, 11), (32768, 2)])
def test_selection_among_thousands_of_blocks(cs, n_blocks, nq):
    """The longest tables: scores by whole numbers in float64 (all below 2^24), sorted."""
    say("select, thousands of blocks", n_blocks, nq)
    d, hq, want = 64, 4, 20
    gen = torch.Generator(device="cuda").manual_seed(n_blocks)
    hi = torch.randint(-100, 128, (n_blocks, d), generator=gen, device=DEV)
    lo = hi - torch.randint(0, 28, hi.shape, generator=gen, device=DEV)
    bounds = torch.stack([hi, lo], 1).to(torch.int8).contiguous()
    scales = torch.randint(118, 123, (n_blocks,), generator=gen, device=DEV).to(torch.uint8)
    q = torch.randn((nq, hq, d), generator=gen, device=DEV).to(torch.bfloat16)
    last = 16 * n_blocks - 1
    pos = torch.tensor([last - 700 * i for i in range(nq)], dtype=torch.int32, device=DEV)
    out = torch.full((nq, 1, want), -7, dtype=torch.int32, device=DEV)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
    cs.cs_select_blocks(q, bounds, scales, i32(0, nq), pos, i32(16 * n_blocks), n_blocks, 16, want, 2, 3, out, nq, 1, hq, 1, d, cs.CS_BF16)
    for t in range(nq):
        codes = so.query_codes(f64(q[t]))
        c = torch.from_numpy(codes).double().to(DEV)
        score = (torch.maximum(c[:, None] * hi.double(), c[:, None] * lo.double()).sum(-1).amax(0) * torch.exp2(scales.double() - 127)).cpu().numpy()
        n = int(pos[t]) // 16 + 1
        assert out[t, 0].tolist() == so.select(score.tolist(), n, want, 2, 3)


@pytest.mark.parametrize("kv,nq,hq,hkv,d,dtype,size,n_select,n_first,n_last", [
    ([3000, 0, 1700], [300, 0, 260], 28, 4, 128, "bf16", 16, 12, 1, 2), ([900], [300], 64, 4, 64, "bf16", 32, 5, 0, 1), ([2000], [280], 16, 16, 64, "f32", 16, 20, 1, 0),
    ([16000], [520], 28, 4, 64, "bf16", 16, 30, 1, 2), ([700, 40, 1], [400, 130, 1], 8, 4, 128, "f32", 48, 3, 0, 0), ([8500], [515], 12, 4, 128, "bf16", 16, 256, 1, 2)])
def test_selection_of_many_tokens(cs, kv, nq, hq, hkv, d, dtype, size, n_select, n_first, n_last):
    """So many tokens that waves have rows of their own: the lists of calls of few tokens, and for some of them the oracle's."""
    say("select, many tokens", kv, nq, hq, hkv, d, dtype, size, n_select, n_first, n_last)
    c = Cache(cs, sum(kv) + d, hkv, d, kv, dtype)
    qs = c.queries(nq, hq, where="any", extra=3)
    bounds = c.bounds(size)
    got = c.select(qs, size, n_select, n_first, n_last, bounds)
    assert torch.all(got[sum(nq):] == -7)
    at = 0
    for s, n in enumerate(nq):
        for a in range(at, at + n, 50):
            m = min(50, at + n - a)
            few = dict(hq=hq, n_q=m, q=qs["q"][a:a + m].contiguous(), q_pos=qs["q_pos"][a:a + m].contiguous(), cu_q=dev(np.array([0] * (s + 1) + [m] * (len(kv) - s), np.int32)))
            assert torch.equal(c.select(few, size, n_select, n_first, n_last, bounds), got[a:a + m]), (s, a)
        at += n
    some = np.random.default_rng(1).permutation(sum(nq))[:12]
    part = dict(hq=hq, n_q=len(some), q64=qs["q64"][some], pos=qs["pos"][some], stream=qs["stream"][some])
    assert np.array_equal(got.cpu().numpy()[some], c.want_selected(part, size, n_select, n_first, n_last))


def test_selection_of_equal_scores_and_odd_numbers(cs):
    """Equal blocks go by index; blocks without numbers come first; a query without numbers has equal scores; negative scores have an order."""
    say("select, ties and odd numbers")
    c = Cache(cs, 31, 2, 64, [400, 400], "bf16", gain=0.5)
    for j in range(400):                    # stream 1: all blocks alike
        for h in range(2):
            for col in range(64):
                c.put(0, 1, j, h, col, float((col % 5) - 2))
    c.put(0, 0, 100, 0, 3, float("nan"))
    c.put(0, 0, 200, 1, 3, float("inf"))
    qs = c.queries([6, 6], 4, where="tail")
    qs["q"][2, 1, 5] = float("nan")
    qs["q64"][2, 1, 5] = np.nan
    qs["q"][3, 3, 5] = float("-inf")
    qs["q64"][3, 3, 5] = -np.inf
    qs["q"][4] = 0.0
    qs["q64"][4] = 0.0
    for n_select, first, last in ((1, 0, 0), (4, 0, 0), (5, 1, 2), (24, 0, 1)):
        got = c.select(qs, 16, n_select, first, last).cpu().numpy()
        assert np.array_equal(got, c.want_selected(qs, 16, n_select, first, last))
    # keys all on one side: every score is negative
    c = Cache(cs, 32, 1, 64, [400], "f32")
    for j in range(400):
        for col in range(64):
            c.put(0, 0, j, 0, col, 1.0 + j / 100.0 + col / 64.0)
    qs = c.queries([3], 2, where="tail")
    qs["q"].copy_(-qs["q"].abs())
    qs["q64"] = -np.abs(qs["q64"])
    got = c.select(qs, 16, 3, 0, 0).cpu().numpy()
    assert np.array_equal(got, c.want_selected(qs, 16, 3, 0, 0))


# ------------------------------------------------------------------------------------------ attention

def any_lists(rng, c, qs, size, n_select, kind):
    """Lists that a caller may hand over: in no order, with repeats, holes, indexes past the window and none at all."""
    top = -(-max(max(c.kv), 1) // size)
    if kind == "sorted":
        x = np.sort(rng.integers(0, top, (qs["n_q"], c.hkv, n_select)), -1)
        x[rng.random(x.shape) < 0.1] = -1
    else:
        x = rng.integers(-2, top + 3, (qs["n_q"], c.hkv, n_select))
        x[rng.random(x.shape) < 0.02] = 0x7fffffff
    x[rng.random((qs["n_q"], c.hkv)) < 0.1] = -1
    return x.astype(np.int32)


ATTENTION = [
    ([1], [1], 1, 1, 64, "bf16", 16, 1, "tail", "slot"),
    ([700], [1], 28, 4, 128, "bf16", 64, 4, "tail", "slot"),
    ([0, 17, 300, 333], [0, 3, 9, 20], 7, 1, 128, "bf16", 64, 3, "any", "head"),
    ([300, 80], [40, 7], 8, 8, 64, "bf16", 16, 5, "any", "slot"),
    ([500, 80], [30, 7], 4, 2, 64, "f32", 32, 4, "any", "slot"),
    ([400], [33], 16, 4, 128, "f32", 64, 3, "any", "head"),
    ([450, 450, 1], [5, 1, 1], 32, 2, 64, "bf16", 48, 4, "any", "slot"),
    ([600], [13], 15, 3, 128, "bf16", 16, 33, "any", "slot"),
    ([2000], [4], 12, 1, 64, "f32", 16, 100, "any", "slot"),
    ([900], [3], 6, 2, 128, "bf16", 128, 7, "any", "head"),
    ([5000], [2], 2, 2, 64, "bf16", 16, 256, "tail", "slot"),
    ([100] * 70, [1] * 70, 7, 1, 64, "bf16", 16, 4, "any", "slot"),
]


@pytest.mark.parametrize("kv,nq,hq,hkv,d,dtype,size,n_select,where,layout", ATTENTION)
@pytest.mark.parametrize("kind", ["sorted", "wild"])
def test_attention(cs, kv, nq, hq, hkv, d, dtype, size, n_select, where, layout, kind):
    say("attention", len(kv), sum(nq), hq, hkv, d, dtype, size, n_select, where, layout, kind)
    c = Cache(cs, sum(kv) + d, hkv, d, kv, dtype, layout)
    qs = c.queries(nq, hq, where=where, extra=2, gain=2.0)
    listed = any_lists(c.rng, c, qs, size, n_select, kind)
    out, stat = c.attend(qs, dev(listed), size)
    c.check_attention(qs, listed, size, out, stat)
    again, none = c.attend(qs, dev(listed), size, lse=False)
    assert none is None and torch.equal(out.view(torch.int16 if dtype == "bf16" else torch.int32), again.view(torch.int16 if dtype == "bf16" else torch.int32))


@pytest.mark.parametrize("kv,nq,hq,hkv,d,dtype,size,n_select,layout", [
    ([2000], [132], 256, 16, 64, "bf16", 16, 48, "slot"),           # one piece a tile, more places than are looked up at once
    ([1500, 0, 300], [90, 0, 44], 256, 16, 128, "bf16", 32, 20, "head"),
    ([1500, 600], [70, 70], 32, 4, 128, "bf16", 64, 8, "slot"),      # pieces
    ([900], [20], 7, 1, 64, "bf16", 16, 90, "slot"),
    ([300, 80, 5, 1, 20], [4, 0, 1, 1, 0], 7, 1, 128, "bf16", 16, 6, "slot"),      # several tokens in the kernel of few rows
    ([900, 80, 5, 1, 20], [5, 0, 1, 0, 1], 8, 4, 64, "bf16", 64, 8, "head"),
])
@pytest.mark.parametrize("kind", ["sorted", "wild"])
def test_attention_whole_and_in_pieces(cs, kv, nq, hq, hkv, d, dtype, size, n_select, layout, kind):
    say("attention, pieces", kv, nq, hq, hkv, d, dtype, size, n_select, layout, kind)
    c = Cache(cs, sum(kv) + d, hkv, d, kv, dtype, layout)
    qs = c.queries(nq, hq, where="any", extra=2, gain=2.0)
    listed = any_lists(c.rng, c, qs, size, n_select, kind)
    out, stat = c.attend(qs, dev(listed), size)
    c.check_attention(qs, listed, size, out, stat)
    again, _ = c.attend(qs, dev(listed), size)
    assert torch.equal(out.view(torch.int16), again.view(torch.int16))


@pytest.mark.parametrize("nq", [[12, 3], [12, 0, 0, 0, 0, 0, 0, 0]])
@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (7, 1, 128), (16, 16, 64)])
def test_what_is_no_number_in_one_piece(cs, hq, hkv, d, nq):
    """Blocks of 64 keys, so that the sweep is in pieces, of which some hold what is no number, before and behind the queries."""
    say("attention, odd numbers in pieces", hq, hkv, d, nq)
    c = Cache(cs, 7, hkv, d, [900] + [64] * (len(nq) - 1), "bf16")
    for which, j, h, col, x in ((1, 40, 0, 3, np.nan), (1, 300, 0, 0, np.inf), (1, 301, 0, 1, -np.inf), (0, 500, 0, 5, np.nan), (1, 700, 0, d - 1, np.nan), (1, 899, 0, 2, np.inf)):
        c.put(which, 0, j, h, col, x)
    qs = c.queries(nq, hq, where="tail")
    qs["pos"][:12] = [899, 39, 40, 299, 300, 498, 699, 898, 899, 450, 5, -1]
    qs["q_pos"].copy_(dev(qs["pos"]))
    listed = np.stack([np.stack([np.sort(c.rng.permutation(15)[:9]) for _ in range(hkv)]) for _ in range(sum(nq))]).astype(np.int32)
    out, stat = c.attend(qs, dev(listed), 64)
    c.check_attention(qs, listed, 64, out, stat)
    assert np.isnan(f64(out)).any() and np.isinf(f64(out)).any()


def test_all_blocks_are_the_window_attention(cs):
    """Every block listed: the framework's attention over whole windows."""
    say("attention, all blocks")
    c = Cache(cs, 5, 4, 128, [300, 90], "bf16")
    qs = c.queries([20, 5], 28, where="tail")
    listed = c.select(qs, 16, 32, 0, 0)
    out, _ = c.attend(qs, listed, 16)
    want = torch.zeros_like(out)
    nbytes = cs.cs_window_prefill_attn_workspace(qs["n_q"], 2, 28, 4, 128, c.max_blocks, cs.CS_BF16)
    ws = torch.zeros((max(16, nbytes),), dtype=torch.uint8, device=DEV)
    cs.cs_window_prefill_attn(qs["q"], c.pool[0], c.pool[1], qs["cu_q"], qs["q_pos"], c.kv_len, c.table, c.max_blocks, 16, want, qs["n_q"], 2, 28, 4, 128, *c.stride,
                              1 / math.sqrt(128), cs.CS_BF16, ws)
    # both are within b of their weighted values, and each is rounded
    assert float((out.float() - want.float()).abs().max()) <= 4 * B * float(c.pool[1][c.slots[0]].float().abs().max())


@pytest.mark.parametrize("hq,hkv,d,dtype", [(4, 2, 64, "bf16"), (7, 1, 128, "bf16"), (4, 4, 128, "f32"), (3, 1, 64, "f32")])
def test_what_is_no_number_reaches_only_its_readers(cs, hq, hkv, d, dtype):
    """Keys and values that are no numbers, in blocks that neighbours of the same tile read and this query does not, or behind it."""
    say("attention, odd numbers", hq, hkv, d, dtype)
    c = Cache(cs, 6, hkv, d, [200, 64], dtype)
    for which, j, h, col, x in ((1, 20, 0, 3, np.nan), (1, 70, 0, 0, np.inf), (1, 71, 0, 1, -np.inf), (0, 100, 0, 5, np.nan), (1, 150, 0, d - 1, np.nan), (1, 199, 0, 2, np.inf)):
        c.put(which, 0, j, h, col, x)
    qs = c.queries([12, 3], hq, where="tail")
    qs["pos"][:12] = [199, 19, 20, 69, 70, 98, 150, 149, 199, 110, 5, -1]
    qs["q_pos"].copy_(dev(qs["pos"]))
    listed = np.full((15, hkv, 4), -1, np.int32)
    for t in range(15):
        for g in range(hkv):
            listed[t, g] = c.rng.permutation(13)[:4]
    listed[0] = [0, 2, 3, 5]
    listed[1] = [0, 1, 4, 9]
    listed[8] = [1, 4, 6, 12]
    out, stat = c.attend(qs, dev(listed), 16)
    c.check_attention(qs, listed, 16, out, stat)
    assert np.isnan(f64(out)).any() and np.isinf(f64(out)).any()


@pytest.mark.parametrize("dtype,gain,scale", [("bf16", 40.0, None), ("f32", 40.0, None), ("f32", 1.0, 1e-6), ("bf16", 1.0, 30.0)])
def test_attention_of_large_and_small_scores(cs, dtype, gain, scale):
    say("attention, score sizes", dtype, gain, scale)
    c = Cache(cs, 8, 2, 64, [500], dtype)
    qs = c.queries([9], 6, where="tail", gain=gain)
    listed = any_lists(c.rng, c, qs, 32, 9, "sorted")
    out, stat = c.attend(qs, dev(listed), 32, scale=scale)
    c.check_attention(qs, listed, 32, out, stat, scale)


def test_a_query_without_numbers_keeps_to_its_heads(cs):
    say("attention, odd queries")
    for dtype in ("bf16", "f32"):
        c = Cache(cs, 9, 1, 64, [200], dtype)
        qs = c.queries([5], 4, where="tail")
        for t, h, x in ((1, 2, np.nan), (3, 0, np.nan)):
            qs["q"][t, h, 7] = x
            qs["q64"][t, h, 7] = x
        listed = any_lists(c.rng, c, qs, 16, 5, "sorted")
        listed[1], listed[3] = [0, 3, 5, 6, 9], [1, 2, 3, 4, 5]
        out, stat = c.attend(qs, dev(listed), 16)
        assert bool(torch.isnan(out[1, 2]).all()) and bool(torch.isnan(stat[1, 2])) and bool(torch.isnan(out[3, 0]).all())
        c.check_attention(qs, listed, 16, out, stat)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq", [[1, 1], [3, 9]])
def test_scores_of_minus_infinity_alone(cs, dtype, nq):
    """An infinite key that all of a query's heads meet with the other sign: weight 0 beside others, and nothing seen where it is alone."""
    say("attention, scores of -inf", dtype, nq)
    c = Cache(cs, 10, 1, 64, [40, 90], dtype)
    c.put(0, 0, 0, 0, 5, float("inf"))
    qs = c.queries(nq, 4, where="tail")
    qs["q"][:, :, 5] = -1.0
    qs["q64"][:, :, 5] = -1.0
    qs["pos"][: nq[0]] = 0 if nq[0] == 1 else [0, 7, 39]
    qs["q_pos"].copy_(dev(qs["pos"]))
    listed = np.tile(np.array([0, 1, 2], np.int32), (sum(nq), 1, 1))
    out, stat = c.attend(qs, dev(listed), 16)
    assert bool((out[0] == 0).all()) and bool((stat[0] == float("-inf")).all())
    for t in range(1, sum(nq)):
        s = int(qs["stream"][t])
        rows = c.slots[s][so.seen(listed[t, 0], int(qs["pos"][t]), c.kv[s], 16)]
        want, _ = so.attend(qs["q64"][t], np.where(np.isinf(c.x64[0][rows, 0]), 1e6, c.x64[0][rows, 0]), c.x64[1][rows, 0], 0.125)
        # (scores below 2^6: weights off by under 2^-15; bf16 weights and results by b each)
        tol = (2.0 ** -14 + 2 * (B if dtype == "bf16" else U)) * np.abs(c.x64[1][rows, 0]).max()
        assert np.all(np.abs(f64(out)[t] - want) <= tol)


# ------------------------------------------------------------------------------------------ how calls are made

def test_rows_past_32_bits(cs):
    """Cache blocks whose offsets pass 2^32 elements: a pool of more than 2^32 elements in bf16, of which few rows are touched."""
    say("offsets past 32 bits")
    hkv, d, kv = 4, 128, [200, 90]
    n_slots = 16 * (-(-(1 << 32) // (16 * hkv * d)) + 40)
    k, v = (torch.empty((n_slots, hkv, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    small = Cache(cs, 12, hkv, d, kv, "bf16")
    ids = small.table.cpu().numpy()
    top = n_slots // 16
    far = np.where(ids % 2 == 0, ids, top - 1 - ids).astype(np.int32)          # half of the blocks at the pool's end
    for old, new in {int(a): int(b) for a, b in zip(ids.ravel(), far.ravel())}.items():
        for src, dst in ((small.pool[0], k), (small.pool[1], v)):
            dst[16 * new:16 * new + 16] = src[16 * old:16 * old + 16]
    want = {}
    for pools, table in ((small.pool, small.table), ([k, v], dev(far))):
        small.pool, small.table = pools, table
        for nq, where in (([1, 1], "tail"), ([40, 20], "any")):
            small.rng = np.random.default_rng(3)
            qs = small.queries(nq, 28, where=where)
            listed = small.select(qs, 16, 5, 1, 1)
            got = [small.bounds(16), listed, small.attend(qs, listed, 16)]
            if nq[0] in want:
                b0, l0, a0 = want[nq[0]]
                assert torch.equal(got[0][0], b0[0]) and torch.equal(got[0][1], b0[1]) and torch.equal(listed, l0)
                assert torch.equal(got[2][0], a0[0]) and torch.equal(got[2][1], a0[1])
            want[nq[0]] = got
    # writes and corrections there
    n = 7
    slot = dev(np.array([0, 16 * top - 1, 5, 16 * top - 17, -1, 33, 16 * top - 40], np.int32))
    x = torch.randn((n, hkv, d), device=DEV).to(torch.bfloat16)
    w = torch.ones((d,), dtype=torch.bfloat16, device=DEV)
    f = torch.full((d // 2,), 0.01, device=DEV)
    pos = torch.arange(n, dtype=torch.int32, device=DEV)
    cs.cs_norm_rope_refresh_scatter(None, None, x, x, None, w, slot, pos, None, f, k, v, n, 0, hkv, d, d, 0, hkv * d, hkv * d, hkv * d, d, 1e-6, 1.0, 0, cs.CS_BF16)
    near = torch.zeros((40, hkv, d), dtype=torch.bfloat16, device=DEV), torch.zeros((40, hkv, d), dtype=torch.bfloat16, device=DEV)
    cs.cs_norm_rope_refresh_scatter(None, None, x, x, None, w, pos, pos, None, f, near[0], near[1], n, 0, hkv, d, d, 0, hkv * d, hkv * d, hkv * d, d, 1e-6, 1.0, 0, cs.CS_BF16)
    live = [0, 1, 2, 3, 5, 6]
    assert torch.equal(k[slot[live].long()], near[0][live]) and torch.equal(v[slot[live].long()], x[live])
    src, dst, delta = dev(np.array([16 * top - 1, 0], np.int32)), dev(np.array([7, 16 * top - 3], np.int32)), dev(np.array([5, -9], np.int32))
    cs.cs_kv_rerotate_freqs(k, v, src, dst, delta, None, f, 2, 1, hkv, d, d, 0, hkv * d, d, 0, cs.CS_BF16)
    cs.cs_kv_rerotate_freqs(near[0], near[1], dev(np.array([1, 0], np.int32)), dev(np.array([20, 21], np.int32)), delta, None, f, 2, 1, hkv, d, d, 0, hkv * d, d, 0, cs.CS_BF16)
    assert torch.equal(k[dst.long()], near[0][20:22]) and torch.equal(v[dst.long()], x[[1, 0]])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_graphs_replayed_beside_eager_calls(cs, dtype):
    """Captured chains of different shapes that share a workspace, replayed in turn with eager calls and changed inputs between: each gives
    what eager calls give, bit for bit."""
    say("graphs", dtype)
    c = Cache(cs, 21, 4, 128, [700, 333, 90], dtype)
    shapes = []
    for nq, size, n_select in (([1, 1, 1], 64, 6), ([30, 11, 20], 16, 9), ([620, 300, 70], 16, 12)):
        qs = c.queries(nq, 28, where="tail")
        n_sel = c.n_sel(size)
        b, sc = torch.zeros((3, 4, n_sel, 2, 128), dtype=torch.int8, device=DEV), torch.zeros((3, 4, n_sel), dtype=torch.uint8, device=DEV)
        listed = torch.zeros((qs["n_q"], 4, n_select), dtype=torch.int32, device=DEV)
        out, stat = torch.zeros_like(qs["q"]), torch.zeros((qs["n_q"], 28), device=DEV)
        shapes.append((qs, size, n_select, b, sc, listed, out, stat))
    nbytes = max(max(cs.cs_selected_attn_workspace(s[0]["n_q"], 3, 28, 4, 128, s[1], s[2]), cs.cs_select_blocks_workspace(s[0]["n_q"], 3, 28, 4, 128, c.max_blocks, s[1])) for s in shapes)
    ws = torch.full((max(16, nbytes),), 255, dtype=torch.uint8, device=DEV)

    def chain(s):
        qs, size, n_select, b, sc, listed, out, stat = s
        cs.cs_key_bounds(c.pool[0], None, c.kv_len, c.table, c.max_blocks, 16, size, b, sc, 3, 4, 128, *c.stride, c.code)
        cs.cs_select_blocks(qs["q"], b, sc, qs["cu_q"], qs["q_pos"], c.kv_len, c.max_blocks, size, n_select, 1, 1, listed, qs["n_q"], 3, 28, 4, 128, c.code, ws)
        cs.cs_selected_attn(qs["q"], c.pool[0], c.pool[1], qs["cu_q"], qs["q_pos"], c.kv_len, c.table, c.max_blocks, 16, listed, size, n_select, out, stat, qs["n_q"], 3, 28, 4, 128,
                            *c.stride, 0.09, c.code, ws)

    side = torch.cuda.Stream()
    graphs = []
    with torch.cuda.stream(side):
        for s in shapes:
            chain(s)
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                chain(s)
            graphs.append(g)
    torch.cuda.synchronize()
    gen = torch.Generator(device="cuda").manual_seed(1)
    for i in range(5):
        for s in shapes:
            s[0]["q"].copy_(torch.randn(s[0]["q"].shape, generator=gen, device=DEV))
        want = []
        for s in shapes:
            chain(s)
            torch.cuda.synchronize()
            want.append([x.clone() for x in s[3:]])
        for s in shapes:
            for x in s[5:]:
                x.zero_()
        for g in (graphs if i % 2 else graphs[::-1]):
            g.replay()
        torch.cuda.synchronize()
        for s, w in zip(shapes, want):
            for x, y in zip(s[3:], w):
                assert bool((x.view(torch.uint8) == y.view(torch.uint8)).all())


def test_work_goes_to_the_current_stream(cs):
    """Calls on a side stream whose inputs a long kernel there is still making."""
    say("side stream")
    c = Cache(cs, 22, 4, 128, [600, 50], "bf16")
    qs = c.queries([40, 9], 28, where="tail")
    listed = c.select(qs, 32, 5, 1, 1)
    want, _ = c.attend(qs, listed, 32)
    side = torch.cuda.Stream()
    keep = c.pool[1].clone()
    c.pool[1].zero_()
    torch.cuda.synchronize()
    big = torch.randn((4096, 4096), device=DEV)
    with torch.cuda.stream(side):
        for _ in range(10):
            big = big @ big * 1e-2
        c.pool[1].copy_(keep)
        out = torch.zeros_like(want)
        nbytes = cs.cs_selected_attn_workspace(qs["n_q"], 2, 28, 4, 128, 32, 5)
        ws = torch.empty((max(16, nbytes),), dtype=torch.uint8, device=DEV)
        cs.cs_selected_attn(qs["q"], c.pool[0], c.pool[1], qs["cu_q"], qs["q_pos"], c.kv_len, c.table, c.max_blocks, 16, listed, 32, 5, out, None, qs["n_q"], 2, 28, 4, 128, *c.stride,
                            1 / math.sqrt(128), cs.CS_BF16, ws)
    side.synchronize()
    assert torch.equal(out, want)


def test_two_calls_at_once_with_workspaces_of_their_own(cs):
    say("two streams at once")
    c = Cache(cs, 23, 4, 128, [900] * 3, "bf16")
    work = []
    for seed, nq in ((1, [1, 1, 1]), (2, [50, 60, 70]), (3, [1, 0, 1])):
        c.rng = np.random.default_rng(seed)
        qs = c.queries(nq, 28, where="tail")
        listed = c.select(qs, 64, 6, 1, 1)
        work.append((qs, listed, c.attend(qs, listed, 64)))
    streams = [torch.cuda.Stream() for _ in work]
    outs = [[torch.zeros_like(w[2][0]), torch.zeros_like(w[2][1])] for w in work]
    ws = [torch.full((max(16, cs.cs_selected_attn_workspace(w[0]["n_q"], 3, 28, 4, 128, 64, 6)),), 255, dtype=torch.uint8, device=DEV) for w in work]
    torch.cuda.synchronize()
    for _ in range(5):
        for (qs, listed, _), (out, stat), st, one in zip(work, outs, streams, ws):
            with torch.cuda.stream(st):
                cs.cs_selected_attn(qs["q"], c.pool[0], c.pool[1], qs["cu_q"], qs["q_pos"], c.kv_len, c.table, c.max_blocks, 16, listed, 64, 6, out, stat, qs["n_q"], 3, 28, 4, 128,
                                    *c.stride, 1 / math.sqrt(128), cs.CS_BF16, one)
    torch.cuda.synchronize()
    for (_, _, (want, lse)), (out, stat) in zip(work, outs):
        assert torch.equal(out, want) and torch.equal(stat, lse)


def test_strides_wider_than_the_rows(cs):
    """Pools whose slots and heads lie further apart than they have to: the same bits."""
    say("wide strides")
    for dtype in ("bf16", "f32"):
        c = Cache(cs, 24, 3, 64, [300, 77], dtype)
        for nq in ([1, 1], [40, 12]):
            qs = c.queries(nq, 12, where="tail")
            b, sc = c.bounds(48)
            listed = c.select(qs, 48, 4, 1, 1, (b, sc))
            want = c.attend(qs, listed, 48)
            pools, stride = c.pool, c.stride
            wide = []
            for x in pools:
                y = torch.full((x.shape[0], 5, 96), float("nan"), dtype=x.dtype, device=DEV)
                y[:, :3, :64] = x
                wide.append(y[:, :3, :64])
            c.pool, c.stride = wide, (480, 96)
            b2, sc2 = c.bounds(48)
            got = c.attend(qs, listed, 48)
            c.pool, c.stride = pools, stride
            assert torch.equal(b, b2) and torch.equal(sc, sc2) and torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


def test_lengths_that_the_table_does_not_hold(cs):
    """kv_len past the table's rows is clamped to them, for selection and attention alike; positions past it see all of it."""
    say("clamped lengths")
    for dtype in ("bf16", "f32"):
        c = Cache(cs, 25, 2, 64, [64, 64], dtype)
        c.max_blocks, c.table = 4, c.table[:, :4].contiguous()
        for nq in ([1, 1], [20, 30]):
            qs = c.queries(nq, 4, where="tail")
            qs["pos"][:] = 1 << 30
            qs["q_pos"].copy_(dev(qs["pos"]))
            listed = c.select(qs, 16, 3, 1, 1)
            want = c.attend(qs, listed, 16)
            c.kv_len.fill_(0x7fffffff)
            assert torch.equal(c.select(qs, 16, 3, 1, 1), listed)
            got = c.attend(qs, listed, 16)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
            c.kv_len.fill_(64)
            c.check_attention(qs, listed, 16, *got)


def test_more_tokens_than_said(cs):
    """cu_q past n_q: tokens from n_q on do not exist."""
    say("n_q below cu_q")
    c = Cache(cs, 26, 2, 64, [300, 200], "bf16")
    qs = c.queries([9, 14], 6, where="tail")
    listed = c.select(qs, 16, 4, 1, 1)
    want = c.attend(qs, listed, 16)
    for n in (3, 9, 17):
        out, sel = torch.full_like(want[0], 9.0), torch.full_like(listed, -7)
        cs.cs_selected_attn(qs["q"], c.pool[0], c.pool[1], qs["cu_q"], qs["q_pos"], c.kv_len, c.table, c.max_blocks, 16, listed, 16, 4, out, None, n, 2, 6, 2, 64, *c.stride, 0.125,
                            cs.CS_BF16, torch.empty((max(16, cs.cs_selected_attn_workspace(n, 2, 6, 2, 64, 16, 4)),), dtype=torch.uint8, device=DEV))
        b, sc = c.bounds(16)
        cs.cs_select_blocks(qs["q"], b, sc, qs["cu_q"], qs["q_pos"], c.kv_len, c.max_blocks, 16, 4, 1, 1, sel, n, 2, 6, 2, 64, cs.CS_BF16)
        assert torch.equal(sel[:n], listed[:n]) and bool((sel[n:] == -7).all()) and bool((out[n:] == 9).all())
        # (fewer tokens may take the other kernel: the same precision)
        assert float((out[:n].float() - want[0][:n].float()).abs().max()) <= 4 * B * float(c.pool[1][c.slots[0]].float().abs().max())
