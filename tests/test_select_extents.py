"""What the tensors of a write have to hold, whatever their shapes say (no device is needed)."""
import pytest
import torch

from paper_2604_06036_amd import binding as cs
from tests.test_select_abi import BF, P_WRITE, z


@pytest.mark.parametrize("name,row", [("q", 256), ("k", 128), ("v", 128)])
def test_tokens_that_are_one_row_seen_several_times_are_refused(name, row):
    """An expanded tensor has the elements that the call asks for, but its memory is one row."""
    with pytest.raises(ValueError, match=f"{name}.* holds fewer than 3 tokens"):
        cs.cs_norm_rope_refresh_scatter(*dict(P_WRITE, **{name: z(row, BF).expand(3, row)}).values())


@pytest.mark.parametrize("name,value", [("q", z(1024, BF)[256:]), ("q", z(3 * 512, BF).view(3, 512)[:, 256:]), ("k", z(384, BF)), ("v", z(3 * 512, BF).view(3, 512)[:, 384:])])
def test_tokens_that_are_all_there_pass(name, value):
    """Rows behind one another, at an offset, and parts of wider rows: refused only for lying on the host."""
    stride = {"q": "sq", "k": "sk", "v": "sv"}[name]
    row = P_WRITE["hq" if name == "q" else "hkv"] * P_WRITE["d"]
    with pytest.raises(ValueError, match="device tensor"):
        cs.cs_norm_rope_refresh_scatter(*dict(P_WRITE, **{name: value, stride: value.stride(0) if value.dim() > 1 else row}).values())
    with pytest.raises(ValueError, match="holds fewer"):
        short = torch.as_strided(value, value.shape[:-1] + (value.shape[-1] - 8,), value.stride(), value.storage_offset() + 8) if value.dim() > 1 else value[8:]
        cs.cs_norm_rope_refresh_scatter(*dict(P_WRITE, **{name: short, stride: value.stride(0) if value.dim() > 1 else row}).values())
