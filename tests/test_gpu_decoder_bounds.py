"""Arguments at the ends of their ranges, on the GPU against the 64-bit oracle.  Tolerances as in test_gpu_decoder.py."""
import pytest

from tests import test_gpu_decoder as tg

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 30, 2 ** 30, 300])
@pytest.mark.parametrize("rows,lens", [([130, 33, 80], [130, 33, 200]), ([100, 60], [50, 61]), ([1, 1], [1, 300]), ([3, 8], [3, 5])])
def test_windows_that_hide_nothing(window, rows, lens):
    """Fresh prompts, prompts with rows below position 0 and single rows: the window of any length is as none."""
    got = tg._check_attention(rows, lens, 4, 2, 64, 32, window=window, seed=800)
    none = tg._check_attention(rows, lens, 4, 2, 64, 32, window=0, seed=800)
    assert (got == none).all()


@pytest.mark.parametrize("rows,lens", [([130, 40], [130, 200]), ([2, 1], [40, 300])])
def test_prefixes_at_the_ends_of_their_range(rows, lens):
    """A prefix below 0 is none, one past the last token is all of them."""
    for window in (0, 20):
        for prefix in (-2 ** 31, -2 ** 31 + 20, -1, 2 ** 31 - 1):
            tg._check_attention(rows, lens, 4, 2, 64, 32, window=window, prefix=[prefix] * 2, seed=801)
