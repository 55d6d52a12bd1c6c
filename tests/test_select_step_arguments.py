"""Arguments that engine.SelectStep refuses before it touches a device, and the layout of its answer blocks."""
import numpy as np
import pytest
import torch

from paper_2604_06036_amd import engine, planner, synth
from tests import helpers as hp


@pytest.fixture(scope="module")
def data():
    return engine.assemble_step(synth.small_variant(synth.CFG1, n_layers=2), hp.oracle_scorer, device="cpu")


F = np.ones(64, np.float32)


@pytest.mark.parametrize("what,change", [
    ("rotary_dim", dict(rotary_dim=8)), ("rotary_dim", dict(rotary_dim=72)), ("rotary_dim", dict(rotary_dim=144)), ("inv_freq", dict(inv_freq=F.astype(np.float64))),
    ("inv_freq", dict(inv_freq=F[:32])), ("inv_freq", dict(rotary_dim=64)), ("inv_freq", dict(inv_freq=torch.ones(128)[::2])), ("axis_of_pair", dict(axis_of_pair=np.zeros(64, np.int32))),
    ("axis_of_pair", dict(axis_of_pair=np.zeros(32, np.uint8))), ("positions", dict(axis_of_pair=np.zeros(64, np.uint8))), ("positions", dict(positions=np.zeros(3, np.int32))),
    ("positions", dict(positions=np.zeros(5000, np.int64))), ("positions", dict(positions=torch.zeros((5000, 2), dtype=torch.int32)[:, 0])), ("q_weight", dict(q_weight=torch.ones((2, 128)))),
    ("k_weight", dict(k_weight=torch.ones((128,), dtype=torch.bfloat16))), ("selection", dict(sel_block=40)), ("selection", dict(sel_block=144)), ("selection", dict(n_select=0)),
    ("selection", dict(n_select=257)), ("selection", dict(n_first=9, n_last=8)), ("selection", dict(n_first=-1))])
def test_refused(data, what, change):
    with pytest.raises(ValueError, match=what):
        engine.SelectStep(data, **dict(dict(positions=np.zeros(data.info["n_q"], np.int32), inv_freq=F), **change))


def test_answer_blocks_lie_behind_the_windows_own(data):
    more = engine._with_answer_blocks(data, 3)
    new, old = more["new_layout"], data.new_layout
    need = planner.blocks_needed(old.seq_len)
    assert more["n_slots"] == data.n_slots + 3 * 16 * len(need) and more["k_pool"].shape[1] == more["n_slots"] == more["v_pool"].shape[1]
    assert torch.equal(more["k_pool"][:, :data.n_slots], data.k_pool)
    seen = []
    for s, n in enumerate(need):
        assert np.array_equal(new.block_table[s, :n], old.block_table[s, :n])
        seen += new.block_table[s, n:n + 3].tolist()
    assert sorted(seen) == list(range(data.n_slots // 16, more["n_slots"] // 16))
