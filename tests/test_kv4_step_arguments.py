"""Arguments that engine.Kv4Step and the 4-bit calls refuse before they touch a device."""
import numpy as np
import pytest
import torch

from paper_2604_06036_amd import binding as cs
from paper_2604_06036_amd import engine, synth
from tests import helpers as hp


@pytest.fixture(scope="module")
def data():
    return engine.assemble_step(synth.small_variant(synth.CFG1, n_layers=1), hp.oracle_scorer, device="cpu")


@pytest.mark.parametrize("axis", [np.zeros(64, np.int64), [0] * 64, np.zeros(64, np.int32), torch.zeros((64,), dtype=torch.int64), torch.zeros((64,)), np.zeros(63, np.uint8),
                                  np.zeros(128, np.uint8), torch.zeros((128,), dtype=torch.uint8)[::2]])
def test_axes_of_another_type_or_number_are_refused(data, axis):
    """(wider integers would be read byte by byte, and turn the wrong pairs)"""
    with pytest.raises(ValueError, match="axis_of_pair"):
        engine.Kv4Step(data, np.zeros((data.info["n_q"], 3), np.int32), axis)


@pytest.mark.parametrize("axis", [torch.zeros((32,), dtype=torch.int64), torch.zeros((32,), dtype=torch.int32), torch.zeros((64,), dtype=torch.uint8)[::2],
                                  torch.zeros((31,), dtype=torch.uint8)])
def test_calls_refuse_axes_of_another_type(axis):
    z = lambda n, dt=torch.int32: torch.zeros((n,), dtype=dt)
    with pytest.raises(ValueError, match="axis_of_pair"):
        cs.cs_kv4_rerotate(None, None, None, None, z(3), z(3), z(9), axis, 3, 1, 1, 64, 0, 64, 64, 1e6, 0)
    with pytest.raises(ValueError, match="axis_of_pair"):
        cs.cs_rope_refresh_scatter(z(192, torch.bfloat16), z(192, torch.bfloat16), None, None, None, z(9), axis, None, None, None, None, 3, 1, 0, 64, 64, 0, 0, 0, 0, 1e6, 0,
                                   cs.CS_BF16, cs.CS_KV4)


def test_positions_in_another_order_are_refused(data):
    """(time, height, width) lie behind one another, a row at a time."""
    n = data.info["n_q"]
    axis = np.zeros(64, np.uint8)
    for positions in (torch.zeros((3, n), dtype=torch.int32), torch.zeros((3, n), dtype=torch.int32).T, np.zeros((3, n), np.int32), torch.zeros((n, 4), dtype=torch.int32)[:, :3],
                      torch.zeros((n, 3), dtype=torch.int64), np.zeros((n - 1, 3), np.int32)):
        with pytest.raises(ValueError, match="positions"):
            engine.Kv4Step(data, positions, axis)
    for positions in (torch.zeros((2 * n,), dtype=torch.int32)[::2], np.zeros((n, 3), np.int32), np.zeros((n,), np.int64)):
        with pytest.raises(ValueError, match="positions"):
            engine.Kv4Step(data, positions)


def test_eviction_refuses_tables_that_would_name_other_blocks(data):
    step = engine.Kv4Step.__new__(engine.Kv4Step)          # (a step lives on a device; this check comes before that)
    step.data, step.cs, step.dev, step.weight = data, cs, torch.device("cpu"), torch.zeros((1, 32))
    good = torch.arange(40, dtype=torch.int32).view(1, 40)
    for table in (good.long(), good[:, ::2], good.view(2, 20), good[0], torch.zeros((1, 40))):
        with pytest.raises(ValueError, match="block_table"):
            step.evict(100, table)
    with pytest.raises(ValueError, match="device tensor"):
        step.weight, step.kv_len, step.block_table, step.max_blocks = torch.zeros((1, 32)), torch.zeros((1,), dtype=torch.int32), torch.zeros((1, 2), dtype=torch.int32), 2
        step.evict(100, good)
