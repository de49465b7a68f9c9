"""Windows at the end of their range: as good as none, also for rows ahead of the first token, whose positions are negative."""
import pytest
import torch

import test_gpu_kv4_attention as base

pytestmark = pytest.mark.gpu
NO_LIMIT = (1 << 31) - 1


@pytest.mark.parametrize("window", [NO_LIMIT, NO_LIMIT - 1, 1 << 30])
@pytest.mark.parametrize("D", [64, 128])
def test_rows_ahead_of_the_first_token(D, window):
    """Up to 16 rows a sequence, up to 32, more in contexts of a few pages and of more, in parts."""
    base.run(1, [5], [2], 2, 1, D, window=window)
    base.run(3, [5, 3, 1], [2, 0, 70], 2, 1, D, window=window)
    base.run(2, [20, 4], [3, 4], 1, 1, D, window=window)
    base.run(1, [5], [2], 2, 1, D, window=window, cols=80)
    base.run(2, [40, 3], [7, 3], 2, 2, D, window=window)
    for max_kv in (500, 1000):
        base.run(2, [300, 40], [100, 7], 1, 1, D, window=window, max_kv=max_kv)


def test_rows_ahead_of_the_first_token_in_tall_tiles():
    base.run(2, [300, 300], [100, 290], 64, 64, 128, window=NO_LIMIT, max_kv=500)


@pytest.mark.parametrize("window", [NO_LIMIT, 4951, 4901])
@pytest.mark.parametrize("qs", [[3], [40]])
def test_windows_of_contexts_longer_than_their_bound(qs, window):
    """Positions go by the length, tokens by the bound."""
    base.run(1, qs, [5000], 2, 1, 64, window=window, max_kv=100)


@pytest.mark.parametrize("window", [0, 1, NO_LIMIT])
@pytest.mark.parametrize("qs", [[1, 1], [5, 5], [40, 40]])
def test_lengths_below_zero(qs, window):
    base.run(2, qs, [-(1 << 31), 3], 2, 1, 64, window=window, cols=1)


def test_the_largest_window_is_none():
    q, pool, table, cu, out, lse = base.run(2, [70, 5], [300, 64], 4, 2, 128)
    again = base.run(2, [70, 5], [300, 64], 4, 2, 128, window=NO_LIMIT)
    assert torch.equal(out, again[4]) and torch.equal(lse, again[5])
