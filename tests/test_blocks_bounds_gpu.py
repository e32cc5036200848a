"""Bounds of sequences that reach past their table, and of pages that sequences share."""
import numpy as np
import pytest
import torch

from helpers import ensure_lib
from oracle import cache_ops as co
from test_blocks_gpu import DEV, FORMATS, Cache

pytestmark = pytest.mark.gpu
PAGE, LENGTH = 1, 4


@pytest.fixture(scope="module")
def P():
    return ensure_lib()


# start, length, max_new, flags; a table of four pages beside it
BEYOND = [
    (0, 64, 64, 0), (0, 64, 1000, 0), (15, 64, 49, 0), (63, 64, 1, 0), (-1, 65, 66, 0), (65, 65, 1, 0), (80, 70, 1, 0),
    (0, 65, 65, PAGE), (0, 200, 200, PAGE), (0, 1 << 30, 1 << 30, PAGE), (1, 65, 64, PAGE), (15, 200, 185, PAGE), (16, 65, 49, PAGE),
    (16, 200, 184, PAGE), (63, 65, 2, PAGE), (64, 65, 1, PAGE), (500, 501, 1, PAGE), (0, (1 << 31) - 1, (1 << 31) - 1, PAGE),
    # more positions than max_new, of whose blocks those that it allows are within the table, or not
    (0, 200, 20, LENGTH), (0, 200, 34, LENGTH), (0, 200, 49, LENGTH), (0, 200, 50, LENGTH | PAGE), (16, 200, 33, LENGTH),
    (16, 200, 34, LENGTH | PAGE), (40, 200, 10, LENGTH), (40, 200, 17, LENGTH), (40, 200, 18, LENGTH | PAGE),
]


@pytest.mark.parametrize("start,length,max_new,flags", BEYOND)
def test_blocks_beyond_the_table(P, start, length, max_new, flags):
    """Are skipped and flagged from every start; blocks of the table are written, and nothing else."""
    for fmt, hkv, d in (("bf16", 3, 64), ("e2m1", 2, 128)):
        cache = Cache(fmt, hkv, d, [64], seed=1)
        err = torch.zeros(1, dtype=torch.int32, device=DEV)
        cache.update(P, [start], lengths=torch.tensor([length], dtype=torch.int32, device=DEV), max_new=max_new, err=err)
        assert int(err.item()) == flags
        c, s = co.block_bounds(cache.kv[0][0])
        want, steps = np.full(cache.bounds.shape, -128, dtype=np.int8), np.full(cache.bound_scales.shape, -7.0, dtype=np.float32)
        if 0 <= start < length:
            for j in range(start // 16, min(4, start // 16 + (max_new + 30) // 16, -(-length // 16))):
                want[1, cache.table[0, j]], steps[1, cache.table[0, j]] = c[j], s[j]
        assert np.array_equal(cache.bounds.cpu().numpy(), want) and np.array_equal(cache.bound_scales.cpu().numpy(), steps)


def test_one_of_many_reaches_beyond(P):
    """A row behind others, over a table whose width its neighbours fill."""
    cache = Cache("int8", 2, 64, [64] * 5, seed=2)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    for at, n, flags in ((None, 0, 0), (4, 65, PAGE), (2, 300, PAGE)):
        lens = torch.tensor([n if i == at else 64 for i in range(5)], dtype=torch.int32, device=DEV)
        err.zero_()
        cache.update(P, [0] * 5, lengths=lens, max_new=512, err=err)
        assert int(err.item()) == flags


@pytest.mark.parametrize("fmt", FORMATS)
def test_shared_pages(P, fmt):
    """Sequences of one call share full pages, and a page that they end in at the same length; at different lengths,
    in calls of their own, the last one's bounds stay."""
    cache = Cache(fmt, 2, 64, [500], seed=3)

    def call(lens, start):
        cache.bounds.fill_(-128)
        for l, s in zip(lens, start):
            cache.update(P, s, lengths=torch.tensor(l, dtype=torch.int32, device=DEV), max_new=500,
                         bt=cache.bt.expand(len(l), -1).contiguous())
        return cache.bounds.cpu().numpy()[1, cache.table[0]], cache.bound_scales.cpu().numpy()[1, cache.table[0]]

    for last, lens, start in ((500, [[500, 500, 160, 496, 500] * 40], [[0, 480, 0, 100, 499] * 40]),
                              (500, [[490], [500]], [[0], [490]]), (490, [[500], [490]], [[0], [0]])):
        c, s = co.block_bounds(cache.kv[0][0][:last])
        codes, steps = call(lens, start)
        assert np.array_equal(codes[:len(s)], c) and np.array_equal(steps[:len(s)], s)      # (490 keys: one block fewer)
