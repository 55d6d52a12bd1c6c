"""engine.SelectStep's single tokens as a model calls them, layer by layer, and streams whose blocks are full (needs an MI355X)."""
import numpy as np
import pytest
import torch

from tests.test_gpu_select_step import build, cs, workload  # noqa: F401 (cs: the fixture)

pytestmark = pytest.mark.gpu


def draw(step, it, axes):
    w, rng = step.data.workload, it["rng"]
    q, k, v = (torch.from_numpy(rng.normal(size=(w.n_layers, w.n_streams, h, w.head_dim)).astype(np.float32)).to(it["t"]).cuda() for h in (w.n_q_heads, w.n_kv_heads, w.n_kv_heads))
    pos = torch.from_numpy(rng.integers(9000, 9100, (w.n_streams, 3) if axes else (w.n_streams,)).astype(np.int32)).cuda()
    return q, k, v, pos


@pytest.mark.parametrize("name,axes,kw", [("three", False, dict(n_select=6, sel_block=32)), ("one", True, dict(n_select=5)), ("f32", False, dict(n_select=4, sel_block=16))])
def test_layer_by_layer_is_all_layers_at_once(cs, name, axes, kw):
    """Until every stream is full, and past it: the same rows, windows and answers, bit for bit; `token_slot` names the rows that were written."""
    print("[case] select token, layer by layer", name, flush=True)
    data, step, it = build(workload(name), axes, answer_blocks=1, **kw)
    w = data.workload
    step.run()
    room, table = step.room.cpu().numpy(), step.block_table.cpu().numpy()
    dropped = 0
    for i in range(34):
        q, k, v, pos = draw(step, it, axes)
        kept = step.k_pool.clone(), step.v_pool.clone(), step.kv_len.clone(), step.bounds.clone(), step.scales.clone()
        once, by_layer = torch.full_like(q, 7.0), torch.full_like(q, 7.0)
        step.token(q, k, v, pos, once)
        want = [x.clone() for x in (step.k_pool, step.v_pool, step.kv_len, step.token_slot)]
        for x, y in zip((step.k_pool, step.v_pool, step.kv_len, step.bounds, step.scales), kept):
            x.copy_(y)
        step.begin_token()
        for layer in range(w.n_layers):
            # (one projection's output, as a model has it)
            fused = torch.cat([q[layer], k[layer], v[layer]], 1)
            step.token_layer(layer, *fused.split([w.n_q_heads, w.n_kv_heads, w.n_kv_heads], 1), pos, by_layer[layer])
        torch.cuda.synchronize()
        for x, y in zip((step.k_pool, step.v_pool, step.kv_len, step.token_slot), want):
            assert torch.equal(x, y)
        assert torch.equal(once, by_layer)
        before, slot = kept[2].cpu().numpy(), step.token_slot.cpu().numpy()
        full = before >= room
        assert np.array_equal(slot, [-1 if full[s] else table[s, before[s] // 16] * 16 + before[s] % 16 for s in range(w.n_streams)])
        assert np.array_equal(step.kv_len.cpu().numpy(), before + ~full)
        assert torch.equal(step.v_pool[:, torch.from_numpy(slot[~full]).long().cuda()], v[:, torch.from_numpy(~full).cuda()])
        if full.all():
            assert torch.equal(step.k_pool, kept[0]) and torch.equal(step.v_pool, kept[1])
        dropped += int(full.sum())
    assert dropped > 0


def test_a_token_before_any_step(cs):
    """There is no window yet: nothing is written or read, and the rows of `out` are left as they were."""
    print("[case] select token, no window yet", flush=True)
    data, step, it = build(workload("three"), False, answer_blocks=1, n_select=6, sel_block=32)
    q, k, v, pos = draw(step, it, False)
    before, out = (step.k_pool.clone(), step.v_pool.clone()), torch.full_like(q, 7.0)
    step.token(q, k, v, pos, out)
    torch.cuda.synchronize()
    assert torch.equal(step.k_pool, before[0]) and torch.equal(step.v_pool, before[1])
    assert bool((out == 7).all()) and step.token_slot.tolist() == [-1] * 3
    step.run()
    step.token(q, k, v, pos, out)
    torch.cuda.synchronize()
    assert min(step.token_slot.tolist()) >= 0 and not bool((out == 7).all())
