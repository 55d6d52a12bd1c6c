"""Corners of the operators of long windows (needs an MI355X): the largest epsilon of a norm beside squares that overflow, every bit pattern of a
value, a workspace that calls of all sizes share, calls from several threads, lists of as many blocks as registers hold, more blocks than are
collected at once, rows that lie far apart."""
import math
import threading

import numpy as np
import pytest
import torch

from oracle import select_oracle as so
from tests.test_gpu_select import Cache, any_lists, cs, dev, f64, pool, run_write, say  # noqa: F401 (cs: the fixture)

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64), ("f32", 80), ("f32", 16)])
@pytest.mark.parametrize("eps", [3e38, 1e38, 2.0 ** 100, 1e-30])
def test_write_of_an_epsilon_beside_squares_past_the_largest_number(cs, dtype, d, eps):
    """Heads whose sum of squares is past single precision, just below it, and small, with an epsilon as large as their mean square: all of
    them within the bounds of test_gpu_select (an epsilon that is scaled by a power of two brings no rounding)."""
    say("write, large epsilon", dtype, d, eps)
    rng = np.random.default_rng(7)
    n, hq, hkv = 12, 2, 1
    x = rng.choice([-1.0, 1.0], (n, hq + 2 * hkv, d)) * rng.uniform(0.5, 1.0, (n, hq + 2 * hkv, d))
    x *= np.array([2e19, 1e20, 5e20, 1e22, 1e30, 2e38, 1e19, 3e18, 1e17, 1e10, 1.0, 4e19])[:, None, None]
    run_write(cs, 11, n, hq, hkv, d, 16, dtype, "one", 0, "slot", x=x.reshape(n, -1), eps=eps)


@pytest.mark.parametrize("layout", ["slot", "head"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_are_copied_bit_for_bit(cs, dtype, layout):
    """Every pattern of 16 bits (in fp32: as the upper half, the lower one drawn), signalling NaN and the smallest numbers among them."""
    say("write, value bits", dtype, layout)
    hkv, d, n = 4, 64, 256
    bits = np.arange(1 << 16, dtype=np.uint32)
    if dtype == "f32":
        bits = (bits << 16 | np.random.default_rng(2).integers(0, 1 << 16, bits.size, dtype=np.uint32)).view(np.int32)
    else:
        bits = bits.astype(np.uint16).view(np.int16)
    t, as_bits = (torch.bfloat16, torch.int16) if dtype == "bf16" else (torch.float32, torch.int32)
    v = dev(bits.reshape(n, hkv * d)).view(t)
    k = torch.ones_like(v)
    slot = dev(np.random.default_rng(3).permutation(n).astype(np.int32))
    kc, vc = (pool(layout, 1, n, hkv, d, t) for _ in range(2))
    f = torch.full((d // 2,), 0.01, device=DEV)
    for weight, pos in ((None, None), (torch.ones((d,), dtype=t, device=DEV), torch.arange(n, dtype=torch.int32, device=DEV))):
        vc.zero_()
        cs.cs_norm_rope_refresh_scatter(None, None, k, v, None, weight, slot, pos, None, f, kc, vc, n, 0, hkv, d, d, 0, hkv * d, hkv * d, kc.stride(1), kc.stride(2), 1e-6, 1.0, 0,
                                        cs.CS_BF16 if dtype == "bf16" else cs.CS_F32)
        got = vc[0].contiguous().view(as_bits)[slot.long()]
        assert torch.equal(got, v.view(as_bits).reshape(n, hkv, d))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_workspace_for_the_most_tokens_serves_fewer(cs, dtype):
    """Sized once, for a whole window: shorter questions, single tokens and fewer streams after it use the same bytes, and get what they get with
    bytes of their own."""
    say("workspace of the largest call", dtype)
    hq, hkv, d, size, n_select, kv = 28, 4, 128, 16, 12, [900, 700, 300]
    c = Cache(cs, 41, hkv, d, kv, dtype)
    most = cs.cs_selected_attn_workspace(2100, 3, hq, hkv, d, size, n_select)
    ws = torch.full((max(16, most),), 255, dtype=torch.uint8, device=DEV)
    for nq in ([1, 1, 1], [700, 700, 700], [30, 2, 0], [1, 0, 0], [200, 60, 11]):
        for streams in (3, 1):
            qs = c.queries(nq[:streams], hq, where="any")
            listed = dev(any_lists(c.rng, c, qs, size, n_select, "sorted"))
            out, stat = torch.full_like(qs["q"], 9.0), torch.full((qs["n_q"], hq), 9.0, device=DEV)
            cs.cs_selected_attn(qs["q"], c.pool[0], c.pool[1], qs["cu_q"], qs["q_pos"], c.kv_len, c.table, c.max_blocks, 16, listed, size, n_select, out, stat, qs["n_q"], streams, hq, hkv,
                                d, *c.stride, 0.1, c.code, ws if most else None)
            own = cs.cs_selected_attn_workspace(qs["n_q"], streams, hq, hkv, d, size, n_select)
            want, lse = torch.full_like(out, 9.0), torch.full_like(stat, 9.0)
            cs.cs_selected_attn(qs["q"], c.pool[0], c.pool[1], qs["cu_q"], qs["q_pos"], c.kv_len, c.table, c.max_blocks, 16, listed, size, n_select, want, lse, qs["n_q"], streams, hq, hkv,
                                d, *c.stride, 0.1, c.code, torch.full((max(16, own),), 255, dtype=torch.uint8, device=DEV))
            torch.cuda.synchronize()
            assert torch.equal(out, want) and torch.equal(stat, lse)


def lists_by_sorting(q, bounds, scales, n, want, first, last):
    """Lists of one stream and kv head from whole numbers in float64 (all below 2^24) by a stable sort.  q [nq][hq][d], n [nq] candidates."""
    codes = torch.from_numpy(np.stack([so.query_codes(x) for x in f64(q)])).to(DEV, torch.float64)
    nq, hq, d = codes.shape
    hi, lo = bounds[:, 0].to(torch.float64), bounds[:, 1].to(torch.float64)
    flat = codes.reshape(nq * hq, d)
    score = (flat.clamp(min=0) @ hi.t().contiguous() + flat.clamp(max=0) @ lo.t().contiguous()).reshape(nq, hq, -1).amax(1) * torch.exp2(scales.to(torch.float64) - 127)
    block = torch.arange(bounds.shape[0], device=DEV)[None]
    score = torch.where((block < first) | (block >= n[:, None] - last), math.inf, score)
    score = torch.where(block < n[:, None], score, -math.inf)
    best = torch.sort(score, dim=1, descending=True, stable=True).indices[:, :want]
    if best.shape[1] < want:
        best = torch.cat([best, torch.full((nq, want - best.shape[1]), 1 << 30, device=DEV)], 1)
    best = torch.where(torch.gather(torch.cat([score, torch.full((nq, 1), -math.inf, device=DEV, dtype=score.dtype)], 1), 1, best.clamp(max=score.shape[1])) == -math.inf, 1 << 30, best)
    best = best.sort(1).values
    return torch.where(best == 1 << 30, -1, best).to(torch.int32)


def test_two_threads_choose_among_tables_of_different_lengths(cs):
    """Launches of one kernel that ask for 40 and for 128 KB of LDS, from two threads at once: no call is refused, and every list is right."""
    say("select, two threads")
    d, hq, want = 64, 4, 20
    work = []
    for n_blocks in (32768, 10000, 9000):
        gen = torch.Generator(device="cuda").manual_seed(n_blocks)
        hi = torch.randint(-100, 128, (n_blocks, d), generator=gen, device=DEV)
        bounds = torch.stack([hi, hi - 9], 1).to(torch.int8).contiguous()
        scales = torch.full((n_blocks,), 120, dtype=torch.uint8, device=DEV)
        q = torch.randn((1, hq, d), generator=gen, device=DEV).to(torch.bfloat16)
        last = torch.tensor([16 * n_blocks - 1], dtype=torch.int32, device=DEV)
        work.append((n_blocks, q, bounds, scales, torch.tensor([0, 1], dtype=torch.int32, device=DEV), last, last + 1))
    torch.cuda.synchronize()
    errors, lists = [], [[] for _ in work]

    def calls(i):
        n_blocks, q, bounds, scales, cu, last, kv = work[i]
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(60):
                    out = torch.full((1, 1, want), -7, dtype=torch.int32, device=DEV)
                    cs.cs_select_blocks(q, bounds, scales, cu, last, kv, n_blocks, 16, want, 2, 3, out, 1, 1, hq, 1, d, cs.CS_BF16)
                    lists[i].append(out)
                torch.cuda.current_stream().synchronize()
        except Exception as e:      # noqa: BLE001 (shown by the test's own thread)
            errors.append((i, e))

    threads = [threading.Thread(target=calls, args=(i,)) for i in range(len(work))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors
    for (n_blocks, q, bounds, scales, _, last, _), got in zip(work, lists):
        want_list = lists_by_sorting(q, bounds, scales, last // 16 + 1, want, 2, 3)
        assert all(torch.equal(x[:, 0], want_list) for x in got)


@pytest.mark.parametrize("n_blocks", [127, 128, 129, 192, 193, 256, 257, 320, 321, 384, 385, 448, 449, 512, 513, 768, 769, 1024, 1025, 1536, 1537, 2048, 2049])
@pytest.mark.parametrize("nq,want,first,last", [(3, 16, 1, 2), (4200, 7, 1, 1), (3, 90, 0, 0)])
def test_selection_at_the_edges_of_lists_held(cs, n_blocks, nq, want, first, last):
    """As many blocks as a wave's registers of a list hold, one more and one fewer, for few and for many tokens."""
    say("select, lists held", n_blocks, nq, want)
    d, hq = 64, 4
    gen = torch.Generator(device="cuda").manual_seed(n_blocks)
    hi = torch.randint(-100, 128, (n_blocks, d), generator=gen, device=DEV)
    lo = hi - torch.randint(0, 28, hi.shape, generator=gen, device=DEV)
    bounds = torch.stack([hi, lo], 1).to(torch.int8).contiguous()
    scales = torch.randint(118, 123, (n_blocks,), generator=gen, device=DEV).to(torch.uint8)
    bounds[n_blocks // 3] = bounds[n_blocks // 2]              # (equal scores)
    scales[n_blocks // 3] = scales[n_blocks // 2]
    q = torch.randn((nq, hq, d), generator=gen, device=DEV).to(torch.bfloat16)
    pos = (16 * n_blocks - 1 - 16 * (torch.arange(nq, device=DEV) % (n_blocks // 2))).to(torch.int32)
    out = torch.full((nq, 1, want), -7, dtype=torch.int32, device=DEV)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
    cs.cs_select_blocks(q, bounds, scales, i32(0, nq), pos, i32(16 * n_blocks), n_blocks, 16, want, first, last, out, nq, 1, hq, 1, d, cs.CS_BF16)
    assert torch.equal(out[:, 0], lists_by_sorting(q, bounds, scales, pos // 16 + 1, want, first, last))


@pytest.mark.parametrize("kv,nq,hq,hkv,d,size,n_select", [([40000, 17000], [37, 5], 7, 1, 128, 16, 24), ([40000], [40], 8, 4, 64, 16, 20), ([33000, 20], [9, 1], 4, 2, 64, 16, 128),
                                                          ([35000], [700], 16, 16, 64, 16, 9)])
def test_attention_over_more_blocks_than_are_collected_at_once(cs, kv, nq, hq, hkv, d, size, n_select):
    """Windows of up to 2,500 blocks, whose readers are collected 1,024 at a time: lists in no order, with repeats, on both sides of every 1,024."""
    say("attention, many candidates", kv, nq, hq, hkv, d, size, n_select)
    c = Cache(cs, sum(kv) + d, hkv, d, kv, "bf16")
    qs = c.queries(nq, hq, where="any", extra=2, gain=2.0)
    listed = any_lists(c.rng, c, qs, size, n_select, "wild")
    edges = np.array([1023, 1024, 1023, 2047, 2048, 0, 1025, 2048], np.int32)
    for t in range(0, sum(nq), 2):
        listed[t, :, :len(edges)] = c.rng.permutation(edges)
    qs["pos"][: nq[0]: 3] = kv[0] - 1              # (the whole window in sight)
    qs["pos"][1: nq[0]: 7] = [16 * 1024 - 1, 16 * 1024, 16 * 2048 + 3][: 3][c.rng.integers(0, 3)]
    qs["q_pos"].copy_(dev(qs["pos"]))
    out, stat = c.attend(qs, dev(listed), size)
    some = np.unique(np.concatenate([np.arange(0, min(sum(nq), 40)), c.rng.integers(0, sum(nq), 20)]))
    part = dict(qs, nq=None, n_q=len(some), q64=qs["q64"][some], pos=qs["pos"][some], stream=qs["stream"][some])
    c.check_attention(part, listed[some], size, out[some], stat[some])
    again, lse = c.attend(qs, dev(listed), size)
    assert torch.equal(out.view(torch.int16), again.view(torch.int16)) and torch.equal(stat, lse)
    assert bool((out[sum(nq):] == 9).all()) and bool((stat[sum(nq):] == 9).all())


@pytest.mark.parametrize("stride", [(1 << 26) - 8, 1 << 26, (1 << 26) + 64])
def test_attention_over_rows_that_lie_far_apart(cs, stride):
    """Slots 2^26 elements apart, and a little less: both sides of what the many-token kernel's 32-bit offsets inside a cache block reach."""
    say("attention, far rows", stride)
    hkv, d = 2, 64
    c = Cache(cs, 43, hkv, d, [33, 5], "bf16")
    near, near_stride = c.pool, c.stride
    n_slots = near[0].shape[0]
    flat = torch.empty(((n_slots - 1) * stride + 2 * hkv * d,), dtype=torch.bfloat16, device=DEV)
    far = [flat[i * hkv * d:].as_strided((n_slots, hkv, d), (stride, d, 1)) for i in range(2)]
    for x, y in zip(far, near):
        x.copy_(y)
    for nq in ([1, 1], [30, 11]):
        qs = c.queries(nq, 6, where="any")
        listed = any_lists(c.rng, c, qs, 16, 5, "wild")
        c.pool, c.stride = far, (stride, d)
        bounds = c.bounds(16)
        out, stat = c.attend(qs, dev(listed), 16)
        c.pool, c.stride = near, near_stride
        c.check_attention(qs, listed, 16, out, stat)
        want = c.bounds(16)
        assert torch.equal(bounds[0], want[0]) and torch.equal(bounds[1], want[1])


def test_a_kernels_first_call_may_be_captured(cs):
    """A choice that takes more LDS than launches do unasked, captured before its kernel has run: the limit is raised in the capture, and every
    replay gives the list of the queries that are there by then."""
    say("select, first call in a capture")
    d, hq, hkv, n_blocks, want = 128, 48, 3, 20000, 9             # (fp32, heads in groups of 16: no other test has so many blocks for them)
    gen = torch.Generator(device="cuda").manual_seed(5)
    hi = torch.randint(-100, 128, (hkv, n_blocks, d), generator=gen, device=DEV)
    bounds = torch.stack([hi, hi - 9], 2).to(torch.int8).contiguous()
    scales = torch.randint(118, 123, (hkv, n_blocks), generator=gen, device=DEV).to(torch.uint8)
    q, out = torch.zeros((2, hq, d), device=DEV), torch.zeros((2, hkv, want), dtype=torch.int32, device=DEV)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
    cu, pos, kv = i32(0, 2), i32(16 * n_blocks - 1, 16 * n_blocks - 700), i32(16 * n_blocks)
    call = lambda: cs.cs_select_blocks(q, bounds, scales, cu, pos, kv, n_blocks, 16, want, 1, 1, out, 2, 1, hq, hkv, d, cs.CS_F32)
    torch.cuda.synchronize()
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        call()
    for _ in range(3):
        q.copy_(torch.randn(q.shape, generator=gen, device=DEV))
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        for h in range(hkv):
            heads = q[:, h * 16:(h + 1) * 16].contiguous()
            assert torch.equal(got[:, h], lists_by_sorting(heads, bounds[h], scales[h], pos // 16 + 1, want, 1, 1))
        call()
        torch.cuda.synchronize()
        assert torch.equal(out, got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("top", [2.0 ** 20, 2.0 ** 24, 2.0 ** 28 - 16])
def test_attention_of_scores_up_to_the_documented_size(cs, dtype, sign, top):
    """One key of every window leads all others by a half of its score: the answer is its value, though a score is only known to a multiple of up
    to 16 and the reference that it is compared with is rounded too."""
    say("attention, largest scores", dtype, sign, top)
    d, kv = 64, [700, 90]
    c = Cache(cs, 51, 2, d, kv, dtype)
    keys = np.zeros((c.pool[0].shape[0], 2, d))
    for s, n in enumerate(kv):
        # (of the first channel alone, so that a score is one product)
        lead, rest = (1.0, 0.5) if sign > 0 else (0.5, 1.0)
        keys[c.slots[s], :, 0] = c.rng.uniform(0.7, 0.99, (n, 2)) * rest
        keys[c.slots[s][n // 3], :, 0] = lead * c.rng.uniform(0.98, 0.999, 2) * (1 if sign > 0 else 0.65)
    k64 = torch.from_numpy(keys.astype(np.float32)).to(c.t)
    c.pool[0].copy_(k64)
    keys = f64(k64)
    for nq in ([1, 1], [23, 9]):
        qs = c.queries(nq, 6, where="tail")
        qs["pos"][:] = np.repeat(np.array(kv) - 1, nq)
        qs["q_pos"].copy_(dev(qs["pos"]))
        qs["q"].zero_()
        qs["q"][..., 0] = sign * 8 * top * torch.from_numpy(c.rng.uniform(0.9, 0.99, (sum(nq), 6)).astype(np.float32)).to(DEV)
        q = f64(qs["q"])
        listed = np.tile(np.arange(44, dtype=np.int32), (sum(nq), 2, 1))
        out, lse = c.attend(qs, dev(listed), 16, scale=0.125)
        got, stat = f64(out), f64(lse)
        for t, s in enumerate(qs["stream"]):
            for g in range(2):
                heads, best = slice(3 * g, 3 * g + 3), c.slots[s][kv[s] // 3]
                scores = 0.125 * np.outer(q[t, heads, 0], keys[c.slots[s], g, 0])
                assert np.all(scores.argmax(1) == kv[s] // 3) and np.all(np.abs(scores) < 2.0 ** 28)
                want = c.x64[1][best, g]
                # the weight is rounded before the product but not in the sum, and the result: half a step each, and three of fp32
                half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
                assert np.all(np.abs(got[t, heads] - want) <= (2 * half + 3 * 2.0 ** -24) * 1.01 * np.abs(want))
                # the score's product, the reference, its logarithm and their sum are rounded
                assert np.all(np.abs(stat[t, heads] - scores.max(1)) <= 6 * 2.0 ** -24 * np.abs(scores.max(1)))
