"""Attention of a step's new tokens: windows wider than any request, and the ways of choosing and ordering pieces that need many KV
heads or many row blocks."""
import pytest

from test_gpu_chunk_attn import HEADS, Step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 40, 2 ** 30, 411, 410])
@pytest.mark.parametrize("heads,dtype", [("gqa", "bf16"), ("small", "f16")])
def test_windows_wider_than_any_request(heads, dtype, window):
    """Also for tokens that stand before the first row, whose place less the window is the least number there is."""
    Step(dtype, HEADS[heads], [40], [37], seed=1).check(window=window)
    Step(dtype, HEADS[heads], [9, 1, 2, 70, 1], [5, 3, 1, 411, 0], seed=2).check(window=window)
    Step(dtype, HEADS[heads], [300, 1], [100, 410], seed=3).check(window=window)
