"""Selection from bounds that are written here, block by block, against the oracle: lists are equal to the last entry."""
import numpy as np
import pytest
import torch

from helpers import ensure_lib, to_np64
from oracle import cache_ops as co
from test_blocks_gpu import DEV, equal_lists, queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    return ensure_lib()


class Bounds:
    """Layer 1 of two: bounds of `lens` keys per sequence, on shuffled pages.  `coarse`: few values, so that many scores are
    equal."""

    def __init__(self, hkv, d, lens, seed, coarse=False):
        rng = np.random.default_rng(seed)
        blocks = [-(-n // 16) for n in lens]
        self.hkv, self.d, self.lens = hkv, d, list(lens)
        order = rng.permutation(sum(blocks) + 3).astype(np.int32)
        self.table = np.full((len(lens), max(1, *blocks)), -1, dtype=np.int32)
        self.codes, self.steps = [], []
        for i, n in enumerate(blocks):
            self.table[i, :n] = order[sum(blocks[:i]):sum(blocks[:i + 1])]
            if coarse:
                codes = np.zeros((n, hkv, 2, d), dtype=np.int64)
                codes[..., :2] = rng.integers(-1, 2, (n, hkv, 2, 2))
                step = np.ones((n, hkv), dtype=np.float32)
            else:
                codes = np.sort(rng.integers(-127, 128, (n, hkv, 2, d)), axis=2)[:, :, ::-1]
                step = np.exp(rng.normal(0, 1, (n, hkv))).astype(np.float32)
            self.codes.append(codes)
            self.steps.append(step)
        self.pages = len(order)

    def select(self, P, q, budget, first, last, max_length=None):
        codes = np.full((2, self.pages, self.hkv, 2, self.d), -128, dtype=np.int8)
        steps = np.full((2, self.pages, self.hkv), np.nan, dtype=np.float32)
        for i, (c, s) in enumerate(zip(self.codes, self.steps)):
            codes[1, self.table[i, :len(s)]], steps[1, self.table[i, :len(s)]] = c, s
        max_length = max(1, *self.lens) if max_length is None else max_length
        blocks = torch.full((len(self.lens), self.hkv, budget), 77, dtype=torch.int32, device=DEV)
        ws = torch.full((P.pallas_select_workspace_size(len(self.lens), self.hkv, max_length),), 0xA5, dtype=torch.uint8, device=DEV)
        err = torch.zeros(1, dtype=torch.int32, device=DEV)
        P.pallas_select_blocks(torch.from_numpy(codes).to(DEV), torch.from_numpy(steps).to(DEV), 1, q,
                               torch.tensor(self.lens, dtype=torch.int32, device=DEV), max_length,
                               torch.from_numpy(self.table).to(DEV), blocks, ws, first=first, last=last, err=err)
        assert int(err.item()) == 0
        return blocks

    def lists(self, q, budget, first, last):
        qn = to_np64(q)
        return [co.select_blocks(co.block_scores(qn[i], c, s), budget, first, last) if len(s) else [[]] * self.hkv
                for i, (c, s) in enumerate(zip(self.codes, self.steps))]


# blocks of a row: scored where they are selected; in a launch of their own; with the wide workgroup
@pytest.mark.parametrize("blocks", [62, 128, 129, 700, 2049, 5000])
@pytest.mark.parametrize("budget,first,last", [(12, 1, 2), (4, 1, 2), (9, 0, 0), (40, 3, 5), (3, 1, 2)])
def test_nan_above_all(P, blocks, budget, first, last):
    """Fewer blocks that score NaN than open places, as many, more, and all; the rest by their scores."""
    places = budget - first - last
    rng = np.random.default_rng(blocks + budget)
    lens = [16 * blocks - 5] * 6
    b = Bounds(2, 64, lens, seed=budget)
    for i, n in enumerate((0, max(places - 1, 0), places, places + 1, blocks - 1, blocks)):
        for h in range(2):
            b.steps[i][rng.permutation(blocks)[:n], h] = np.nan
    q = queries(6, 6, 64, seed=3)
    lists = b.lists(q, budget, first, last)
    # (at the last open place lies a NaN, and something else behind it)
    scores = co.block_scores(to_np64(q)[3], b.codes[3], b.steps[3])
    assert np.isnan(scores).sum() == 2 * (places + 1) and (~np.isnan(scores)).any()
    equal_lists(b.select(P, q, budget, first, last), lists)


# A workgroup takes 8192 blocks at a time, 131,072 keys.
@pytest.mark.parametrize("lens,hkv,d,group,budget,first,last", [
    ([131073], 1, 64, 2, 50, 1, 2),                       # one block in the second pass, always listed
    ([131073 + 16 * 60, 3000, 0], 2, 64, 3, 200, 0, 0),   # a short row and an empty one beside it
    ([140001, 131072, 40], 1, 128, 1, 33, 4, 8),
    ([300007, 290000], 1, 64, 4, 700, 2, 3),              # three passes
    ([140001], 2, 64, 2, 9, 4, 5),                        # nothing but the first and the last ones
    ([300007], 1, 64, 1, 9000, 1, 2),                     # a list longer than a pass
    ([300007], 1, 64, 1, 18000, 8500, 9000),              # first and last ones reach into other passes
])
@pytest.mark.parametrize("coarse", [False, True])
def test_more_blocks_than_a_pass_takes(P, lens, hkv, d, group, budget, first, last, coarse):
    """coarse: hundreds of scores equal the last that is listed, on both sides of the passes' border."""
    b = Bounds(hkv, d, lens, seed=budget, coarse=coarse)
    q = queries(len(lens), hkv * group, d, seed=6)
    if coarse:
        q = q.clamp(-1, 1).round()
        scores = co.block_scores(to_np64(q)[0], b.codes[0], b.steps[0])
        assert len(np.unique(scores)) < 60 * hkv
    lists = b.lists(q, budget, first, last)
    blocks = b.select(P, q, budget, first, last)
    equal_lists(blocks, lists)
    # room for longer rows
    b.table = np.pad(b.table, ((0, 0), (0, 9000)), constant_values=-1)
    assert torch.equal(b.select(P, q, budget, first, last, max_length=16 * b.table.shape[1]), blocks)


def test_equal_scores_around_a_border_of_passes(P):
    """All scores equal but some of the second pass: the earliest, up to the border, on it and behind it."""
    b = Bounds(1, 64, [16 * 20000], seed=7, coarse=True)
    b.codes[0][...] = 0
    b.codes[0][9000:9010, 0, :, 0] = 1
    q = queries(1, 1, 64, seed=8).abs()
    for budget in (8191, 8192, 8193, 8203, 8204, 16384, 16394, 16395, 19999):
        lists = b.lists(q, budget, 0, 1)
        assert lists[0][0][-1] == 19999 and set(range(9000, 9010)) <= set(lists[0][0])
        equal_lists(b.select(P, q, budget, 0, 1), lists)


@pytest.mark.parametrize("nan", [46, 47, 48, 20000])
def test_nan_in_every_pass(P, nan):
    b = Bounds(1, 64, [16 * 20000 - 3], seed=9)
    b.steps[0][np.random.default_rng(nan).permutation(20000)[:nan]] = np.nan
    q = queries(1, 2, 64, seed=10)
    equal_lists(b.select(P, q, 50, 1, 2), b.lists(q, 50, 1, 2))


@pytest.mark.parametrize("room", [16 * 9, 16 * 200])
def test_rows_that_are_listed_whole_ask_no_table(P, room):
    """Rows of as many blocks as are listed, or fewer, beside a longer one: pages outside the pool are flagged in that one alone."""
    b = Bounds(2, 64, [16 * 9, 16 * 8, 5], seed=11)
    q = queries(3, 4, 64, seed=12)
    b.table = np.pad(b.table, ((0, 0), (0, room // 16 - 9)), constant_values=-1)
    lists = b.lists(q, 8, 1, 1)
    b.table[1:], keep = 1 << 20, b.table[1:].copy()
    codes = torch.zeros((1, b.pages, 2, 2, 64), dtype=torch.int8, device=DEV)
    steps = torch.zeros((1, b.pages, 2), device=DEV)
    for i, (c, s) in enumerate(zip(b.codes, b.steps)):
        at = torch.from_numpy(b.table[0, :9] if i == 0 else keep[i - 1][:len(s)]).long()
        codes[0, at], steps[0, at] = torch.from_numpy(c.astype(np.int8)).to(DEV), torch.from_numpy(s).to(DEV)
    ws = torch.empty(P.pallas_select_workspace_size(3, 2, room), dtype=torch.uint8, device=DEV)
    for bad in (None, 4):
        table = b.table.copy()
        if bad is not None:
            table[0, bad] = -1
        err, blocks = torch.zeros(1, dtype=torch.int32, device=DEV), torch.full((3, 2, 8), 77, dtype=torch.int32, device=DEV)
        P.pallas_select_blocks(codes, steps, 0, q, torch.tensor(b.lens, dtype=torch.int32, device=DEV), room,
                               torch.from_numpy(table).to(DEV), blocks, ws, first=1, last=1, err=err)
        assert int(err.item()) == (0 if bad is None else 1)
        if bad is not None:
            lists[0] = [[j for j in range(9) if j != bad]] * 2
        equal_lists(blocks, lists)
