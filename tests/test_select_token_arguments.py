"""Where engine.SelectStep puts a token's rows, and the tensors of a token that it refuses (no device is needed)."""
import pytest
import torch

from paper_2604_06036_amd import engine

i32 = lambda *x: torch.tensor(x, dtype=torch.int32)


def test_places_of_a_token():
    """Streams with room in the block at hand, at a block's first row, full, with a full table, empty, and without a window yet."""
    table = torch.arange(100, 118, dtype=torch.int32).reshape(6, 3)
    slot, there = engine._token_places(i32(17, 32, 32, 48, 0, -9), i32(32, 48, 32, 48, 16, 48), table)
    assert slot.dtype == torch.int32
    assert slot.tolist() == [101 * 16 + 1, 105 * 16, -1, -1, 112 * 16, -1]
    assert there.tolist() == [True, True, False, False, True, False]


Q, K = torch.zeros((3, 4, 64)), torch.zeros((3, 2, 64))


def test_tensors_that_are_read():
    engine._check_token(Q, K, K, i32(1, 2, 3), (3,), 4, 2, 64, 1)
    engine._check_token(Q, K, K, torch.zeros((3, 3), dtype=torch.int32), (3,), 4, 2, 64, 3)
    engine._check_token(torch.zeros((5, 4, 64)), K, torch.zeros((4, 2, 64)), i32(1, 2, 3, 4), (3,), 4, 2, 64, 1)      # (more rows than are read)
    fused = torch.zeros((2, 3, 8, 64))
    engine._check_token(fused[:, :, :4], fused[:, :, 4:6], fused[:, :, 6:], i32(1, 2, 3), (2, 3), 4, 2, 64, 1)


@pytest.mark.parametrize("what,change", [
    ("q", dict(q=Q[:2])), ("q", dict(q=Q[None])), ("q", dict(q=torch.zeros((3, 64, 4)).transpose(1, 2))), ("q", dict(q=torch.zeros((4, 3, 64)).transpose(0, 1))), ("k_new", dict(k=Q)),
    ("v_new", dict(v=torch.zeros((3, 2, 128))[..., ::2])), ("positions", dict(pos=i32(1, 2))), ("positions", dict(width=3)),
    ("positions", dict(pos=torch.zeros((3, 4), dtype=torch.int32), rows=(4,), q=torch.zeros((4, 4, 64)), k=torch.zeros((4, 2, 64)), v=torch.zeros((4, 2, 64)), width=3))])
def test_tensors_that_are_refused(what, change):
    a = dict(dict(q=Q, k=K, v=K, pos=i32(1, 2, 3), rows=(3,), width=1), **change)
    with pytest.raises(ValueError, match=f"token: {what}"):
        engine._check_token(a["q"], a["k"], a["v"], a["pos"], a["rows"], 4, 2, 64, a["width"])
