"""The bound of the 4-bit products' test is tight enough to see a mistake: planted
ones, in the oracle, fall outside it at every width."""
import numpy as np
import pytest

import w4_reference as W


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("K", [1000, 4096, 25088])
def test_planted_mistakes_are_seen(K, group):
    g = np.random.default_rng(K + group)
    weights = g.integers(-8, 8, (48, K)).astype(np.float64)
    scales = (g.random((48, -(-K // group))) + 0.5) * 0.1
    x = g.standard_normal((2, K))
    for parts, offset in ((1, 0), (3, 0)):
        y, bound = W.product(x, weights, scales, group, parts, offset)
        assert np.allclose(y, x @ (weights * np.repeat(scales, group, 1)[:, :K]).T)
        short = x.copy()
        short[:, -128:] = 0                                       # a tile of columns is left out
        wrong = W.product(short, weights, scales, group, parts, offset)[0]
        assert (np.abs(wrong - y) > bound).mean() > 0.9
        one = x.copy()
        one[:, K // 2] = 0                                        # a single column
        wrong = W.product(one, weights, scales, group, parts, offset)[0]
        assert (np.abs(wrong - y) > bound).any(0).mean() > 0.5
        moved = np.roll(scales, 1, 1)                             # the neighbouring group's scale
        wrong = W.product(x, weights, moved, group, parts, offset)[0]
        assert (np.abs(wrong - y) > bound).mean() > 0.9
