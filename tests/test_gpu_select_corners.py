"""Corners of the operators of long windows: the largest epsilon of a norm beside squares that overflow (needs an MI355X)."""
import numpy as np
import pytest

from tests.test_gpu_select import cs, run_write, say  # noqa: F401 (cs: the fixture)

pytestmark = pytest.mark.gpu


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
