"""Queries, keys and values that are no numbers, or infinite, and calls at the edges of what is accepted, over the 4-bit window cache,
against oracle/kv4_oracle.py (needs an MI355X).  Tolerances as in tests/test_gpu_kv4.py."""
import math

import numpy as np
import pytest
import torch

from tests.test_gpu_kv4 import CACHES, DEV, U, Batch, cs, dev, say  # noqa: F401 (cs: fixture)

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
