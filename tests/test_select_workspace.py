"""The workspace of attention over selected blocks: its size over numbers of tokens and streams, and what is refused (no device is needed)."""
import pytest

from paper_2604_06036_amd import binding as cs
from tests.test_select_abi import ATTN

TOKENS = sorted(set(list(range(1, 140)) + [2 ** i + d for i in range(7, 16) for d in (-1, 0, 1)] + [200, 300, 389, 700, 1011, 1500, 2082, 22804]))


@pytest.mark.parametrize("heads,d,sel_block,n_select", [((28, 4), 128, 64, 16), ((32, 8), 128, 64, 16), ((16, 4), 64, 16, 24), ((8, 8), 64, 16, 256), ((7, 1), 128, 128, 1), ((64, 4), 64, 16, 2),
                                                        ((256, 16), 128, 48, 100), ((2000, 1000), 64, 64, 16)])
def test_more_tokens_or_streams_never_need_less(heads, d, sel_block, n_select):
    """A workspace that was sized for the largest call serves every smaller one, though fewer tokens are swept in more pieces."""
    streams = (1, 2, 3, 7, 32, 64, 500)
    need = {(n, s): cs.cs_selected_attn_workspace(n, s, *heads, d, sel_block, n_select) for n in TOKENS for s in streams}
    for s in streams:
        for a, b in zip(TOKENS, TOKENS[1:]):
            assert need[a, s] <= need[b, s], (a, b, s)
    for n in TOKENS:
        for s, more in zip(streams, streams[1:]):
            assert need[n, s] <= need[n, more], (n, s, more)
    # the results of a card's workgroups at most: 1,024 times 64 rows of sums and two statistics
    assert max(need.values()) <= 1024 * 64 * (d + 2) * 4


@pytest.mark.parametrize("shape", [dict(), dict(n=64, s=1), dict(n=64, s=1, dt=cs.CS_F32), dict(n=2, s=2, want=256), dict(ss=1 << 26, n=64, s=1)])
@pytest.mark.parametrize("ws", [dict(ws=None), dict(wsb=0), dict(wsb=2048), dict(ws=ATTN["ws"] + 8)])
def test_workspaces_that_do_not_hold_the_pieces_are_refused(shape, ws):
    assert cs.lib().cs_selected_attn(*dict(ATTN, **shape, **ws).values()) == cs.CS_EWORKSPACE
