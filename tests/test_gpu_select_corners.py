"""Corners of the operators of long windows: the largest epsilon of a norm beside squares that overflow, every bit pattern of a value, a
workspace that calls of all sizes share, calls from several threads, lists of
as many blocks as registers hold (needs an MI355X)."""
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
