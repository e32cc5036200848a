"""Pins of the oracle's block selection: bounds that hold, scores that are at least each
key's product but for the rounding, and the order of the selection."""
import numpy as np

from oracle import cache_ops as co


def test_scores_are_bounds():
    rng = np.random.default_rng(0)
    k, q = rng.standard_normal((70, 2, 64)), rng.standard_normal((6, 64))
    codes, step = co.block_bounds(k)
    assert codes.shape == (5, 2, 2, 64) and np.abs(codes).max() == 127
    s = co.block_scores(q, codes, step)
    for h in range(2):
        for j in range(5):
            top = max(float((k[16 * j:16 * j + 16, h] @ q[g]).max()) for g in range(3 * h, 3 * h + 3))
            # half a step of a bound against |q|, and of q against the largest bound
            slack = max(np.abs(q[g]).sum() for g in range(3 * h, 3 * h + 3)) * step[j, h] / 2 + 64 * 127 * step[j, h] * np.abs(q).max() / 254
            assert s[h, j] >= top - slack


def test_one_key_is_its_own_bounds():
    k = np.array([[[1.0, -2.0, 0.5, 4.0]]])
    codes, step = co.block_bounds(k)
    assert step[0, 0] == np.float32(4) / np.float32(127)
    assert codes[0, 0, 0].tolist() == codes[0, 0, 1].tolist() == [32, -64, 16, 127]    # 31.75, -63.5 (even), 15.875


def test_selection():
    scores = np.array([[5, 1, 7, 7, np.nan, 2, 7, 0]], dtype=np.float32)
    assert co.select_blocks(scores, 3, 0, 1) == [[2, 4, 7]]       # the last, the NaN, the first of the sevens
    assert co.select_blocks(scores, 4, 1, 2) == [[0, 4, 6, 7]]
    assert co.select_blocks(scores, 5, 0, 0) == [[0, 2, 3, 4, 6]]
    assert co.select_blocks(scores, 8, 0, 1) == [list(range(8))]
    assert co.select_blocks(scores, 2, 2, 0) == [[0, 1]]


def test_odd_values():
    k = np.zeros((33, 1, 8))
    k[3, 0, 2], k[20, 0, 1] = np.inf, np.nan
    codes, step = co.block_bounds(k)
    assert np.isnan(step[:2]).all() and step[2] == 0 and not codes.any()
    assert co.steps(np.array([[2.0 ** -101, 0]]))[1][0] == 0
