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


# 256 compute units, and two workgroups on each at head_dim 64: with 32 KV heads 8 and 16 pieces of a head run at a time, with 16 twice as many.
MANY = {"mha128": (32, 32, 128), "mha64": (32, 32, 64), "gqa64": (32, 16, 64)}


@pytest.mark.parametrize("heads,dtype", [("mha128", "bf16"), ("mha64", "f16"), ("gqa64", "bf16")])
@pytest.mark.parametrize("window", [0, 90])
def test_more_row_blocks_than_run_at_a_time(heads, dtype, window):
    """Prompts of unlike lengths, some with rows before them, and single tokens: pieces go out longest first."""
    news = [40, 333, 1, 270, 90, 1, 512, 33, 64, 140, 257, 1, 35]
    lens = [40, 333, 900, 400, 700, 31, 512, 600, 64, 141, 300, 1, 1500]
    Step(dtype, MANY[heads], news, lens, seed=4).check(window=window, times=2)


@pytest.mark.parametrize("heads,dtype,short", [("mha128", "bf16", 30), ("mha64", "f16", 56), ("mha128", "f16", 64), ("mha64", "bf16", 70)])
def test_three_blocks_and_more_for_each_place_and_long_ones_among_them(heads, dtype, short):
    """Beyond that only blocks of more than 1.25 times a place's share of the work are cut: a single token after 6000 rows and a piece of
    a prompt after 2800, next to short requests (up to 64 requests, and more, which are listed first)."""
    news, lens = [34 + i % 9 for i in range(short)], [50 + 7 * (i % 11) for i in range(short)]
    news[5:5], lens[5:5] = [1, 0], [6000, 700]
    news[-3:-3], lens[-3:-3] = [100], [2900]
    Step(dtype, MANY[heads], news, lens, seed=5).check(times=2)


def test_single_tokens_of_many_heads():
    """No row blocks possible, and three pieces and more for each place."""
    Step("bf16", MANY["mha128"], [1] * 40, [20 + 13 * i for i in range(39)] + [5000], seed=6).check(times=2)
    Step("f16", MANY["mha64"], [1] * 90, [20 + 5 * i for i in range(89)] + [6000], seed=7).check(times=2)
