"""The number of visible (query, key) pairs that FLOP counts use, against the mask itself."""
import numpy as np
import pytest

from paper_2609_13645_b200.flops import visible_pairs


@pytest.mark.parametrize("S", [1, 2, 7, 64, 129])
def test_visible_pairs_are_those_of_the_mask(S):
    i, j = np.arange(S)[:, None], np.arange(S)[None, :]
    assert visible_pairs(S) == S * (S + 1) // 2
    for window in (1, 2, 5, 63, 64, 200):
        for sinks in (0, 1, 4, 60, 300):
            assert visible_pairs(S, window, sinks) == int(((j <= i) & ((i - j < window) | (j < sinks))).sum()), (window, sinks)
