"""engine.SelectStep: the operators of long windows in a row, as a slide step and as single tokens behind it, against the oracles (needs an
MI355X).  Every link is checked on what the device has handed it: the rows that were written, the bounds of the cache as it is, the choice from
those bounds, attention over that choice."""
import math
import sys

import numpy as np
import pytest
import torch

from oracle import select_oracle as so
from tests import helpers as hp

pytestmark = pytest.mark.gpu
U, B = 2.0 ** -24, 2.0 ** -8


@pytest.fixture(scope="module")
def cs():
    from paper_2604_06036_amd import binding
    binding.lib()
    return binding


def f64(t):
    return t.detach().cpu().to(torch.float32).numpy().astype(np.float64)


def build(workload, axes, **kw):
    from paper_2604_06036_amd import engine
    data = engine.assemble_step(workload, hp.oracle_scorer, device="cpu")
    rng = np.random.default_rng(5)
    w, n_q = data.workload, data.info["n_q"]
    rotary = kw.get("rotary_dim", w.head_dim)
    t = torch.bfloat16 if w.dtype == "bf16" else torch.float32
    freq = (1e6 ** (-2.0 * np.arange(rotary // 2) / rotary)).astype(np.float32)
    axis = (np.arange(rotary // 2) % 3).astype(np.uint8) if axes else None
    pos = rng.integers(0, 9000, (n_q, 3) if axes else (n_q,)).astype(np.int32)
    weights = [torch.from_numpy(1 + 0.2 * rng.normal(size=(w.n_layers, w.head_dim))).to(t) for _ in range(2)]
    step = engine.SelectStep(data, pos, freq, axis, q_weight=weights[0], k_weight=weights[1], **kw)
    return data, step, dict(rng=rng, freq=freq, axis=axis, pos=pos, rotary=rotary, weights=weights, t=t)


def check_written(step, it, layer, x, got, weight, pos):
    want = so.turn(so.norm(f64(x), f64(weight[layer]), step.norm_eps), pos, it["axis"], it["freq"], it["rotary"], 0, step.amplitude)
    tol = (B if it["t"] == torch.bfloat16 else U) * np.abs(want) + 64 * U * (1 + np.abs(want).max(-1, keepdims=True))
    assert np.all(np.abs(f64(got) - want) <= tol)


def check_reading(step, it, layer, q, pos, stream, selected, out, sample):
    """Bounds, choice and attention of a layer, for some of its queries."""
    w, size = step.data.workload, step.sel_block
    table, kv = step.block_table.cpu().numpy(), step.kv_len.cpu().numpy()
    k, v, q64 = f64(step.k_pool[layer]), f64(step.v_pool[layer]), f64(q)
    bounds, scales = step.bounds[layer].cpu().numpy(), step.scales[layer].cpu().numpy()
    group = w.n_q_heads // w.n_kv_heads
    slots = [np.array([table[s, j // 16] * 16 + j % 16 for j in range(kv[s])]) for s in range(w.n_streams)]
    for s in range(w.n_streams):
        for i in range(-(-int(kv[s]) // size)):
            for h in range(w.n_kv_heads):
                hi, lo, e = so.block_bounds(k[slots[s][i * size:(i + 1) * size], h])
                assert bounds[s, h, i, 0].tolist() == hi and bounds[s, h, i, 1].tolist() == lo and scales[s, h, i] == e
    got, listed = f64(out), selected.cpu().numpy()
    for t in sample:
        s = int(stream[t])
        n = so.candidates(int(pos[t]), int(kv[s]), size)
        for g in range(w.n_kv_heads):
            heads = slice(g * group, (g + 1) * group)
            codes = so.query_codes(q64[t, heads])
            scores = [so.block_score(codes, bounds[s, g, i, 0], bounds[s, g, i, 1], scales[s, g, i]) for i in range(n)]
            assert listed[t, g].tolist() == so.select(scores, n, step.n_select, step.n_first, step.n_last)
            rows = slots[s][so.seen(listed[t, g], int(pos[t]), int(kv[s]), size)]
            want, _ = so.attend(q64[t, heads], k[rows, g], v[rows, g], step.data.softmax_scale)
            # scores, exponents and sums are off by under 2^-11 of the weights here (|score| < 60), bf16 weights and results by b each
            tol = (2.0 ** -11 + (B if it["t"] == torch.bfloat16 else 0)) * np.abs(v[rows, g]).max(0) + (B if it["t"] == torch.bfloat16 else U) * np.abs(want)
            assert np.all(np.abs(got[t, heads] - want) <= tol)


def workload(name):
    from paper_2604_06036_amd import synth
    return {"one": synth.small_variant(synth.CFG1, n_layers=2), "three": synth.small_variant(synth.CFG2, n_streams=3, n_layers=2), "f32": synth.CFG0}[name]


@pytest.mark.parametrize("name,axes,kw", [
    ("one", True, dict(n_select=5, sel_block=64)), ("three", False, dict(rotary_dim=64, amplitude=1.1386, n_select=6, sel_block=32, n_first=2, n_last=1)),
    ("f32", False, dict(rotary_dim=32, n_select=4, sel_block=16))])
def test_a_slide_and_tokens_behind_it(cs, name, axes, kw):
    print("[case] select step", name, flush=True)
    sys.stdout.flush()
    data, step, it = build(workload(name), axes, answer_blocks=1, **kw)
    w, rng = data.workload, it["rng"]
    before = step.k_pool.clone()
    step.run()
    torch.cuda.synchronize()
    plan = hp.OraclePlan(step.data)
    hp.assert_device_plan(step, plan)
    n_q = plan.q_pos.size
    stream = np.repeat(np.arange(w.n_streams), np.diff(plan.cu_q))
    last = w.n_layers - 1
    # reused rows, turned by the shift; fresh rows, normed and turned
    shift = plan.delta if not axes else np.tile([-w.stride, 0, 0], (plan.delta.size, 1))
    for layer in range(w.n_layers):
        x = f64(before[layer])[plan.src_slot]
        want = so.turn(x, shift, it["axis"], it["freq"], it["rotary"], 0)
        got = f64(step.k_pool[layer])[plan.dst_slot]
        assert np.all(np.abs(got - want) <= (B if w.dtype == "bf16" else U) * np.abs(want) + 16 * U * np.abs(x).max(-1, keepdims=True))
        check_written(step, it, layer, step.k_new[layer][:n_q], step.k_pool[layer][torch.from_numpy(plan.q_slot).long().to("cuda")], it["weights"][1], it["pos"])
        assert torch.equal(step.v_pool[layer][torch.from_numpy(plan.q_slot).long().to("cuda")], step.v_new[layer][:n_q])
    check_written(step, it, last, step.q[last][:n_q], step.q_turned[:n_q], it["weights"][0], it["pos"])
    sample = sorted(set(rng.integers(0, n_q, 24).tolist() + [0, n_q - 1]))
    check_reading(step, it, last, step.q_turned, plan.q_pos, stream, step.selected, step.out[last], sample)

    # a token a stream, until the answer block is full, and one past it
    kv0 = step.kv_len.cpu().numpy().copy()
    room = step.room.cpu().numpy()
    for i in range(18):
        shape = lambda heads: (w.n_layers, w.n_streams, heads, w.head_dim)
        q, k, v = (torch.from_numpy(rng.normal(size=shape(h)).astype(np.float32)).to(it["t"]).cuda() for h in (w.n_q_heads, w.n_kv_heads, w.n_kv_heads))
        pos = rng.integers(9000, 9100, (w.n_streams, 3) if axes else (w.n_streams,)).astype(np.int32)
        out = torch.full_like(q, 7.0)
        step.token(q, k, v, torch.from_numpy(pos).cuda(), out)
        torch.cuda.synchronize()
        kv = step.kv_len.cpu().numpy()
        assert np.array_equal(kv, np.minimum(kv0 + i + 1, room))
        if i in (0, 9, 17):
            check_written(step, it, last, q[last], step.one_q, it["weights"][0], pos)
            check_reading(step, it, last, step.one_q, kv - 1, np.arange(w.n_streams), step.one_selected, out[last], range(w.n_streams))
    # all other rows are as they were (the tokens' lie in what their stream's last own block leaves, then in its answer block)
    table = step.block_table.cpu().numpy()
    answers = [table[s, j // 16] * 16 + j % 16 for s in range(w.n_streams) for j in range(kv0[s], room[s])]
    untouched = torch.from_numpy(np.setdiff1d(np.arange(before.shape[1]), np.concatenate([plan.dst_slot, plan.q_slot, answers]))).cuda()
    bits = torch.int16 if w.dtype == "bf16" else torch.int32
    same = torch.equal(step.k_pool[:, untouched].view(bits), before[:, untouched].view(bits))
    assert same


def test_step_and_tokens_in_graphs(cs):
    """A captured step and a captured token, replayed several times with eager work between: the eager results, bit for bit."""
    print("[case] select step, graphs", flush=True)
    data, step, it = build(workload("three"), False, answer_blocks=1, n_select=5, sel_block=32)
    w = data.workload
    pool = step.k_pool.clone(), step.v_pool.clone()
    gen = torch.Generator(device="cuda").manual_seed(3)
    draw = lambda heads: torch.randn((w.n_layers, w.n_streams, heads, w.head_dim), generator=gen, device="cuda").to(it["t"])
    q, k, v = draw(w.n_q_heads), draw(w.n_kv_heads), draw(w.n_kv_heads)
    pos, out = torch.full((w.n_streams,), 9000, dtype=torch.int32, device="cuda"), torch.zeros_like(q)

    def eager():
        step.k_pool.copy_(pool[0])
        step.v_pool.copy_(pool[1])
        step.run()
        step.token(q, k, v, pos, out)
        torch.cuda.synchronize()
        return [x.clone() for x in (step.out, step.selected, step.lse[:step.n_q_true], out, step.k_pool, step.v_pool, step.bounds, step.kv_len)]

    want = eager()
    side = torch.cuda.Stream()
    graphs = []
    with torch.cuda.stream(side):
        eager()
        for body in (step.run, lambda: step.token(q, k, v, pos, out)):
            g = torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(g, stream=side):
                body()
            graphs.append(g)
    for _ in range(4):
        step.k_pool.copy_(pool[0])
        step.v_pool.copy_(pool[1])
        out.zero_()
        step.out.zero_()
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        got = [step.out, step.selected, step.lse[:step.n_q_true], out, step.k_pool, step.v_pool, step.bounds, step.kv_len]
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        eager()                                                # (its own work between the replays)
