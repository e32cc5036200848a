"""Bounds, selection and attention over blocks against the oracle.  Bounds and lists are equal
bit for bit (their arithmetic is stated); attention over lists is held to the tolerance of
attention over the whole cache, derived in test_attend_gpu.py and test_attend_e2m1_gpu.py:
  |out - ref| <= 2^-8 |ref| + (2 delta + 2^-13) sum_j p_j |v_j| + n 2^-126 max |v|
  |lse - ref| <= delta + 2^-13,  delta = (d + 8) 2^-24 scale sum |q_i k_i|"""
import math

import numpy as np
import pytest
import torch

from helpers import ensure_lib, to_np64
from oracle import cache_ops as co

pytestmark = pytest.mark.gpu
DEV = "cuda"
FORMATS = ["bf16", "e4m3", "int8", "e2m1"]
TYPES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8, "e2m1": torch.float4_e2m1fn_x2}


@pytest.fixture(scope="module")
def P():
    return ensure_lib()


class Cache:
    """Layer 1 of two holds `lens` keys per sequence in shuffled pages (the rest reads as NaN); bounds start as a
    pattern that no call leaves."""

    def __init__(self, fmt, hkv, d, lens, seed, coarse=False, edit=None):
        g = torch.Generator().manual_seed(seed)
        pages = [(n + 15) // 16 for n in lens]
        self.max_pages = max(1, *pages)
        order = np.random.default_rng(seed).permutation(sum(pages) + 3)
        self.table = np.full((len(lens), self.max_pages), -1, dtype=np.int32)
        at = 0
        for i, n in enumerate(pages):
            self.table[i, :n] = order[at:at + n]
            at += n
        self.fmt, self.lens, self.d, self.hkv, self.pages = fmt, list(lens), d, hkv, len(order)
        self.kv = ([], [])
        shape = (2, 2, len(order), 16, hkv)
        if fmt == "bf16":
            pool = torch.full(shape + (d,), float("nan"), dtype=torch.bfloat16)
        else:
            codes = np.full(shape + (d // 2 if fmt == "e2m1" else d,), 0x77, dtype=np.uint8)
            scales = np.full(shape + (4,), 255, dtype=np.uint8) if fmt == "e2m1" else np.full(shape, np.nan, dtype=np.float32)
        for i, n in enumerate(lens):
            t = np.arange(n)
            pg, slot = self.table[i, t // 16], t % 16
            for kv, keep in enumerate(self.kv):
                x = torch.randn((n, hkv, d), generator=g) + torch.randn((-(-n // 16), hkv, d), generator=g).repeat_interleave(16, 0)[:n]
                if coarse:                  # many equal scores
                    x = x.clamp(-1, 1).round()
                x = x.to(torch.bfloat16)
                if edit is not None and kv == 0:
                    edit(i, x)
                if fmt == "bf16":
                    pool[1, kv, torch.as_tensor(pg, dtype=torch.long), torch.as_tensor(slot)] = x
                    keep.append(to_np64(x))
                elif fmt == "e2m1":
                    c, s = co.quantise4(to_np64(x))
                    codes[1, kv, pg, slot], scales[1, kv, pg, slot] = c, s
                    keep.append(co.dequantise4(c, s))
                else:
                    c, s = co.quantise(to_np64(x), fmt)
                    codes[1, kv, pg, slot], scales[1, kv, pg, slot] = c, s
                    # (a code times its scale is a float32 product)
                    with np.errstate(invalid="ignore"):
                        keep.append((co.dequantise(c, np.ones_like(s), fmt).astype(np.float32) * s[..., None]).astype(np.float64))
        if fmt == "bf16":
            self.rows = (pool.to(DEV),)
        else:
            scales = torch.from_numpy(scales).to(DEV)
            self.rows = (torch.from_numpy(codes).to(DEV).view(TYPES[fmt]), scales.view(torch.float8_e8m0fnu) if fmt == "e2m1" else scales)
        self.bt = torch.from_numpy(self.table).to(DEV)
        self.lengths = torch.tensor(self.lens, dtype=torch.int32, device=DEV)
        self.bounds = torch.full((2, len(order), hkv, 2, d), -128, dtype=torch.int8, device=DEV)
        self.bound_scales = torch.full((2, len(order), hkv), -7.0, device=DEV)

    def update(self, P, start, lengths=None, max_new=None, **kw):
        call = P.pallas_bounds_kv if self.fmt == "bf16" else P.pallas_bounds_quant
        start = torch.as_tensor(start, dtype=torch.int32).to(DEV)
        call(*self.rows, 1, self.bounds, self.bound_scales, start, self.lengths if lengths is None else lengths,
             max(1, *self.lens) if max_new is None else max_new, kw.pop("bt", self.bt), **kw)

    def select(self, P, q, budget, first, last, max_length=None, lengths=None, bt=None, **kw):
        blocks = torch.full((len(self.lens), self.hkv, budget), 77, dtype=torch.int32, device=DEV)
        max_length = max(1, *self.lens) if max_length is None else max_length
        ws = torch.full((P.pallas_select_workspace_size(len(self.lens), self.hkv, max_length),), 0xA5, dtype=torch.uint8, device=DEV)
        P.pallas_select_blocks(self.bounds, self.bound_scales, 1, q, self.lengths if lengths is None else lengths, max_length,
                               self.bt if bt is None else bt, blocks, ws, first=first, last=last, **kw)
        return blocks

    def attend(self, P, q, blocks, scale, max_length=None, lengths=None, bt=None, **kw):
        call = P.pallas_attend_blocks_kv if self.fmt == "bf16" else P.pallas_attend_blocks_quant
        max_length = max(1, *self.lens) if max_length is None else max_length
        room = P.pallas_attend_workspace_size(len(self.lens), q.shape[1], self.hkv, self.d, min(max_length, 16 * blocks.shape[2]))
        ws = torch.full((room,), 0xFF, dtype=torch.uint8, device=DEV)
        out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 9.0, device=DEV)
        call(*self.rows, 1, q, self.lengths if lengths is None else lengths, max_length, self.bt if bt is None else bt, blocks,
             scale, out, ws, lse=lse, **kw)
        return out, lse

    def lists(self, q, budget, first, last):
        """The oracle's lists [S][hkv]."""
        out = []
        for i, n in enumerate(self.lens):
            if n == 0:
                out.append([[]] * self.hkv)
                continue
            out.append(co.select_blocks(co.block_scores(to_np64(q)[i], *co.block_bounds(self.kv[0][i])), budget, first, last))
        return out

    def check_attend(self, q, lists, scale, out, lse):
        qn, on, ln = to_np64(q), to_np64(out), lse.double().cpu().numpy()
        group = q.shape[1] // self.hkv
        for i, n in enumerate(self.lens):
            for h in range(self.hkv):
                pos = np.array([t for j in lists[i][h] for t in range(16 * j, min(16 * j + 16, n))], dtype=int)
                hs = slice(h * group, (h + 1) * group)
                k, v = (self.kv[kv][i][pos, h:h + 1] for kv in (0, 1))
                ref, rl, mag, terms = co.attend(qn[i, hs], k, v, scale)
                delta = ((self.d + 8) * 2.0 ** -24 * terms)[:, None]
                tol = 2.0 ** -8 * np.abs(ref) + (2 * delta + 2.0 ** -13) * mag + len(pos) * 2.0 ** -126 * max(1.0, np.abs(v).max(initial=0.0))
                assert np.all(np.abs(on[i, hs] - ref) <= tol), (i, h, n)
                if len(pos) == 0:
                    assert np.all(ln[i, hs] == -np.inf) and not on[i, hs].any()
                else:
                    assert np.all(np.abs(ln[i, hs] - rl) <= delta[:, 0] + 2.0 ** -13), (i, h, n)


def queries(S, hq, d, seed):
    return torch.randn((S, hq, d), generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).to(DEV)


def equal_lists(got, want):
    got = got.cpu().numpy()
    for i, heads in enumerate(want):
        for h, l in enumerate(heads):
            assert got[i, h].tolist() == list(l) + [-1] * (got.shape[2] - len(l)), (i, h)


def check_bounds(cache, pages_of, start=None):
    """Bounds of the blocks [start / 16, ..) of each sequence are the oracle's, all others as they were."""
    want = np.full(cache.bounds.shape, -128, dtype=np.int8)
    scales = np.full(cache.bound_scales.shape, -7.0, dtype=np.float32)
    for i, n in enumerate(cache.lens):
        first = 0 if start is None else start[i]
        if n == 0 or first < 0 or first >= n:
            continue
        c, s = co.block_bounds(cache.kv[0][i])
        for j in range(first // 16, len(s)):
            want[1, cache.table[i, j]], scales[1, cache.table[i, j]] = c[j], s[j]
    assert np.array_equal(cache.bounds.cpu().numpy(), want)
    assert np.array_equal(cache.bound_scales.cpu().numpy(), scales, equal_nan=True)


CASES = [
    # head_dim, group, KV heads, lengths, budget, first, last
    (128, 8, 2, [0, 1, 16, 17, 100, 500, 1000], 8, 1, 2),
    (64, 4, 8, [3000, 64, 65, 0], 4, 0, 1),
    (128, 1, 4, [5000, 40], 33, 2, 5),
    (64, 3, 5, [700, 2049, 31], 17, 0, 0),
    (128, 16, 1, [4000], 64, 1, 8),
    (128, 20, 2, [900, 1], 1, 0, 1),             # more query heads than a pass takes; one block
    (64, 40, 1, [600], 5, 5, 0),
    (128, 4, 16, [330] * 40, 3, 1, 1),
    (128, 2, 2, [40000, 20], 100, 1, 4),         # more than 2048 blocks; ranges
    (64, 8, 8, [9000, 3000, 0, 8000, 500, 12000], 250, 3, 2),
    (128, 2, 8, [2000, 1100, 0, 1, 900, 1024, 1040, 1023, 1500, 17, 1600], 64, 1, 2),      # a workgroup a row of 1024 keys
    (64, 1, 8, [700, 1100, 600] * 24, 37, 0, 2),
]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d,group,hkv,lens,budget,first,last", CASES)
def test_against_oracle(P, fmt, d, group, hkv, lens, budget, first, last):
    cache = Cache(fmt, hkv, d, lens, seed=d + group)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    cache.update(P, [0] * len(lens), err=err)
    check_bounds(cache, cache.pages)
    q = queries(len(lens), hkv * group, d, seed=1)
    lists = cache.lists(q, budget, first, last)
    blocks = cache.select(P, q, budget, first, last, err=err)
    equal_lists(blocks, lists)
    out, lse = cache.attend(P, q, blocks, 1 / math.sqrt(d), err=err)
    cache.check_attend(q, lists, 1 / math.sqrt(d), out, lse)
    assert int(err.item()) == 0
    # room for longer rows: the same lists
    bt = torch.nn.functional.pad(cache.bt, (0, 4000), value=-1).contiguous()
    assert torch.equal(cache.select(P, q, budget, first, last, bt=bt, max_length=16 * bt.shape[1]), blocks)
    far, _ = cache.attend(P, q, blocks, 1 / math.sqrt(d), bt=bt, max_length=16 * bt.shape[1])
    cache.check_attend(q, lists, 1 / math.sqrt(d), far, lse)


@pytest.mark.parametrize("fmt", ["bf16", "e2m1"])
def test_equal_scores_go_to_the_earliest(P, fmt):
    cache = Cache(fmt, 2, 64, [3000, 1700], seed=3, coarse=True)
    cache.update(P, [0, 0])
    q = queries(2, 4, 64, seed=2).clamp(-1, 1).round()
    q[1] = 0                                          # every score 0
    lists = cache.lists(q, 20, 1, 2)
    assert lists[1][0] == list(range(18)) + [105, 106]
    scores = co.block_scores(to_np64(q)[0], *co.block_bounds(cache.kv[0][0]))
    assert len(np.unique(scores[0])) < 60             # of 188
    equal_lists(cache.select(P, q, 20, 1, 2), lists)


@pytest.mark.parametrize("fmt", FORMATS)
def test_new_tokens_and_padding(P, fmt):
    """Blocks that hold [start, length) alone are written: one new token, chunks from the middle of a block, padding,
    nothing due, and more than the call has room for."""
    lens = [40, 33, 200, 64, 0, 500]
    start = [39, 32, 37, -1, 0, 500]
    cache = Cache(fmt, 3, 128, lens, seed=4)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    cache.update(P, start, max_new=163, err=err)
    check_bounds(cache, cache.pages, start)
    assert int(err.item()) == 0
    cache = Cache(fmt, 3, 128, lens, seed=4)
    cache.update(P, start, max_new=1, err=err)        # one block of each: [37, 200) has eleven
    assert int(err.item()) == 4
    written = (cache.bound_scales[1] != -7.0).any(dim=-1).nonzero()[:, 0].tolist()
    assert sorted(written) == sorted([cache.table[0, 2], cache.table[1, 2], cache.table[2, 2]])


def test_bad_pages(P):
    cache = Cache("bf16", 2, 64, [1000, 700], seed=5)
    cache.update(P, [0, 0])
    q = queries(2, 4, 64, seed=6)
    bt = cache.bt.clone()
    bt[0, 5], bt[0, 62], bt[1, 20] = -3, cache.pages, 1 << 30
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    blocks = cache.select(P, q, 30, 1, 2, bt=bt, err=err)
    assert int(err.item()) == 1
    lists = []
    for i, n in enumerate(cache.lens):
        scores = co.block_scores(to_np64(q)[i], *co.block_bounds(cache.kv[0][i]))
        for j in ([5, 62], [20])[i]:
            scores[:, j] = -np.inf
        lists.append(co.select_blocks(scores, 30, 1, 2))
    equal_lists(blocks, lists)
    err.zero_()
    out, lse = cache.attend(P, q, blocks, 0.1, bt=bt, err=err)
    assert int(err.item()) == 1                      # block 62 is one of the last two
    cache.check_attend(q, [[[j for j in l if j != 62] for l in lists[0]], lists[1]], 0.1, out, lse)
    err.zero_()
    fresh = Cache("bf16", 2, 64, [1000, 700], seed=5)
    fresh.update(P, [0, 0], bt=bt, err=err)
    assert int(err.item()) == 1
    assert bool((fresh.bound_scales[1, cache.table[0, 5]] == -7.0).all())
    ok = [p for p in range(cache.pages) if p not in (cache.table[0, 5], cache.table[0, 62], cache.table[1, 20])]
    assert torch.equal(fresh.bounds[1, ok], cache.bounds[1, ok])


@pytest.mark.parametrize("fmt", FORMATS)
def test_infinities_and_nan(P, fmt):
    """A block with an infinity or a NaN has a scale of NaN, scores above all others and is selected; a query that has
    one selects the earliest blocks."""
    def edit(i, x):
        if i == 0:
            x[100, 0, 3], x[333, 1, 60] = float("inf"), float("nan")
    cache = Cache(fmt, 2, 64, [1000, 800], seed=7, edit=edit)
    # (the oracle's rows of the 8- and 4-bit caches read the row, or the quarter, as NaN)
    cache.update(P, [0, 0])
    check_bounds(cache, cache.pages)
    q = queries(2, 4, 64, seed=8)
    q[1, 0, 5], q[1, 2, 9] = float("nan"), float("-inf")
    lists = cache.lists(q, 10, 1, 2)
    assert 6 in lists[0][0] and 20 in lists[0][1] and lists[1][0] == [0, 1, 2, 3, 4, 5, 6, 7, 48, 49]
    equal_lists(cache.select(P, q, 10, 1, 2), lists)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_bounds_of_any_8_bit_rows(P, fmt, d):
    """Scales that are no powers of two, and codes that no store writes, an E4M3 NaN among them."""
    hkv, lens = 3, [16, 100, 1, 33]
    rng = np.random.default_rng(d)
    pages = sum(-(-n // 16) for n in lens)
    codes = rng.integers(0, 256, (1, 2, pages, 16, hkv, d)).astype(np.uint8)
    if fmt == "e4m3":
        codes[codes % 128 == 127] = 0
        codes[0, 0, 3, 5, 1, d - 1] = 0xFF              # of the second row of lengths; its block 2
    scales = np.exp(rng.normal(0, 2, (1, 2, pages, 16, hkv))).astype(np.float32)
    table = np.full((4, 7), -1, dtype=np.int32)
    at = 0
    for i, n in enumerate(lens):
        table[i, :-(-n // 16)] = np.arange(at, at - (-n // 16))
        at -= -n // 16
    bounds, steps = torch.full((1, pages, hkv, 2, d), -128, dtype=torch.int8, device=DEV), torch.full((1, pages, hkv), -7.0, device=DEV)
    kind = torch.float8_e4m3fn if fmt == "e4m3" else torch.int8
    P.pallas_bounds_quant(torch.from_numpy(codes).to(DEV).view(kind), torch.from_numpy(scales).to(DEV), 0, bounds, steps,
                          torch.zeros(4, dtype=torch.int32, device=DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), 100,
                          torch.from_numpy(table).to(DEV))
    nans = 0
    for i, n in enumerate(lens):
        t = np.arange(n)
        rows = codes[0, 0, table[i, t // 16], t % 16], scales[0, 0, table[i, t // 16], t % 16]
        c, s = co.block_bounds(co.dequantise(*rows, fmt))
        pg = torch.from_numpy(table[i, :len(s)]).long()
        assert np.array_equal(bounds[0, pg].cpu().numpy(), c) and np.array_equal(steps[0, pg].cpu().numpy(), s, equal_nan=True)
        nans += int(np.isnan(s).sum())
    assert nans == (fmt == "e4m3")


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("lens,n", [([300, 20, 0, 90], 12), ([3000, 2000, 900, 0], 90), ([9000] * 3, 300)])
def test_any_lists(P, fmt, lens, n):
    """Lists in any order, with blocks named twice, entries that name nothing and others that are not read."""
    hkv, d = 2, 128
    cache = Cache(fmt, hkv, d, lens, seed=9)
    rng = np.random.default_rng(1)
    q = queries(len(lens), 6, d, seed=10)
    blocks = np.full((len(lens), hkv, n), 1 << 30, dtype=np.int32)
    want = []
    for i, m in enumerate(lens):
        have = -(-m // 16)
        heads = []
        for h in range(hkv):
            l = rng.integers(-2, have + 2, size=n) if have else rng.integers(0, 3, size=n)
            if h == 1 and i == 1:
                l[:] = rng.choice([-1, -(1 << 31), have, 1 << 27, (1 << 31) - 1], size=n)      # no block at all
            blocks[i, h] = l
            heads.append([int(j) for j in l[:min(n, have)] if 0 <= j < have])
        want.append(heads)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    out, lse = cache.attend(P, q, torch.from_numpy(blocks).to(DEV), 0.1, err=err)
    cache.check_attend(q, want, 0.1, out, lse)
    assert int(err.item()) == 0


@pytest.mark.parametrize("fmt", FORMATS)
def test_every_block_is_attention_over_the_cache(P, fmt):
    """Lists of all blocks in order give the dense call's bits."""
    lens = [500, 33, 0, 16]
    cache = Cache(fmt, 2, 64, lens, seed=11)
    q = queries(4, 8, 64, seed=12)
    blocks = torch.full((4, 2, 32), -1, dtype=torch.int32)
    for i, m in enumerate(lens):
        blocks[i, :, :-(-m // 16)] = torch.arange(-(-m // 16))
    out, lse = cache.attend(P, q, blocks.to(DEV), 0.2)
    call = P.pallas_attend_kv if fmt == "bf16" else P.pallas_attend_quant
    ws = torch.empty(P.pallas_attend_workspace_size(4, 8, 2, 64, 500), dtype=torch.uint8, device=DEV)
    dense, dl = torch.zeros_like(q), torch.zeros_like(lse)
    call(*cache.rows, 1, q, cache.lengths, 500, cache.bt, 0.2, dense, ws, lse=dl)
    assert torch.equal(out, dense) and torch.equal(lse, dl)


def test_lengths_outside_the_bound(P):
    cache = Cache("bf16", 2, 64, [300, 200], seed=13)
    cache.update(P, [0, 0])
    q = queries(2, 4, 64, seed=14)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    odd = torch.tensor([1000, -7], dtype=torch.int32, device=DEV)
    blocks = cache.select(P, q, 6, 1, 1, lengths=odd, max_length=300, err=err)
    assert int(err.item()) == 4
    cache.lens = [300, 0]
    lists = cache.lists(q, 6, 1, 1)
    equal_lists(blocks, lists)
    err.zero_()
    out, lse = cache.attend(P, q, blocks, 0.1, lengths=odd, max_length=300, err=err)
    assert int(err.item()) == 4
    cache.check_attend(q, lists, 0.1, out, lse)


def test_pages_beyond_4_gib(P):
    """Bounds of the last pages of planes past 32 bits, and scores from them."""
    hkv, d, n = 16, 128, 700
    small = Cache("e2m1", hkv, d, [n], seed=15)
    pages = (1 << 32) // (hkv * 2 * d) + 60
    bounds = torch.zeros((2, pages, hkv, 2, d), dtype=torch.int8, device=DEV)
    scales = torch.zeros((2, pages, hkv), device=DEV)
    codes = torch.zeros((2, 2, pages, 16, hkv, d // 2), dtype=torch.uint8, device=DEV)
    units = torch.zeros((2, 2, pages, 16, hkv, 4), dtype=torch.uint8, device=DEV)
    place = torch.arange(pages - 1, pages - 1 - small.max_pages, -1, dtype=torch.int32, device=DEV)[None].contiguous()
    codes[1, :, place[0].long()] = small.rows[0].view(torch.uint8)[1][:, small.bt[0].long()]
    units[1, :, place[0].long()] = small.rows[1].view(torch.uint8)[1][:, small.bt[0].long()]
    start = torch.zeros(1, dtype=torch.int32, device=DEV)
    P.pallas_bounds_quant(codes.view(torch.float4_e2m1fn_x2), units.view(torch.float8_e8m0fnu), 1, bounds, scales, start,
                          small.lengths, n, place)
    small.update(P, [0])
    assert torch.equal(bounds[1, place[0].long()], small.bounds[1, small.bt[0].long()])
    assert torch.equal(scales[1, place[0].long()], small.bound_scales[1, small.bt[0].long()])
    q = queries(1, 32, d, seed=16)
    blocks = torch.zeros((1, hkv, 9), dtype=torch.int32, device=DEV)
    ws = torch.empty(P.pallas_select_workspace_size(1, hkv, n), dtype=torch.uint8, device=DEV)
    P.pallas_select_blocks(bounds, scales, 1, q, small.lengths, n, place, blocks, ws, first=1, last=1)
    assert torch.equal(blocks, small.select(P, q, 9, 1, 1))
    del bounds, codes, units
    torch.cuda.empty_cache()


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
def test_a_decode_step_captured_and_replayed(P, fmt):
    """Append, bounds, selection and attention of one new token per sequence, as a graph, while positions and lengths
    grow and one row becomes padding; each replay equals the eager calls, the last also the oracle."""
    S, hq, hkv, d, room, budget = 3, 8, 2, 128, 400, 6
    plan = P.pallas_rope_init(d, 1e6)
    lens0 = [200, 15, 370]

    class Layer:
        def __init__(self):
            self.c = Cache(fmt, hkv, d, [room] * S, seed=17)
            self.qkv = torch.zeros((S, hq + 2 * hkv, d), dtype=torch.bfloat16, device=DEV)
            self.pos = torch.zeros(S, dtype=torch.int32, device=DEV)
            self.lengths = torch.zeros(S, dtype=torch.int32, device=DEV)
            self.blocks = torch.zeros((S, hkv, budget), dtype=torch.int32, device=DEV)
            self.out = torch.zeros((S, hq, d), dtype=torch.bfloat16, device=DEV)
            self.lse = torch.zeros((S, hq), device=DEV)
            self.err = torch.zeros(1, dtype=torch.int32, device=DEV)
            self.ws = torch.empty(P.pallas_attend_workspace_size(S, hq, hkv, d, room), dtype=torch.uint8, device=DEV)
            self.ws2 = torch.empty(P.pallas_select_workspace_size(S, hkv, room), dtype=torch.uint8, device=DEV)
            self.c.update(P, [0] * S, lengths=torch.tensor(lens0, dtype=torch.int32, device=DEV))

        def step(self):
            c, q = self.c, self.qkv[:, :hq]
            P.pallas_append_quant(plan, *c.rows, 1, self.qkv[:, hq:hq + hkv], self.qkv[:, hq + hkv:], self.pos, c.bt, q=q, err=self.err)
            P.pallas_bounds_quant(*c.rows, 1, c.bounds, c.bound_scales, self.pos, self.lengths, 1, c.bt, err=self.err)
            P.pallas_select_blocks(c.bounds, c.bound_scales, 1, q, self.lengths, room, c.bt, self.blocks, self.ws2, first=1,
                                   last=2, err=self.err)
            P.pallas_attend_blocks_quant(*c.rows, 1, q, self.lengths, room, c.bt, self.blocks, 0.1, self.out, self.ws,
                                         lse=self.lse, err=self.err)

    a, b = Layer(), Layer()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        b.step()
    torch.cuda.synchronize()
    for t in range(25):
        rows = torch.randn(a.qkv.shape, generator=torch.Generator().manual_seed(t)).to(torch.bfloat16)
        pos = [n + t for n in lens0]
        if t % 7 == 3:
            pos[1] = -1
        for l in (a, b):
            l.qkv.copy_(rows)
            l.pos.copy_(torch.tensor(pos, dtype=torch.int32))
            l.lengths.copy_((l.pos + 1).clamp(min=0))
        a.step()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in ((a.out, b.out), (a.lse, b.lse), (a.blocks, b.blocks), (a.c.bounds, b.c.bounds),
                     (a.c.rows[0].view(torch.uint8), b.c.rows[0].view(torch.uint8))):
            assert torch.equal(x, y), t
        assert int(a.err.item()) == int(b.err.item()) == 0
    # The oracle over what the cache holds now, read back through the library.
    lens = [n + 25 for n in lens0]
    c = a.c
    for i, n in enumerate(lens):
        pos = torch.arange(n, dtype=torch.int32, device=DEV)
        k, v = (torch.empty((n, hkv, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        P.pallas_quant_load(*c.rows, 1, k, v, pos, c.bt, seq_ids=torch.full_like(pos, i))
        c.kv[0][i], c.kv[1][i] = to_np64(k), to_np64(v)       # (E4M3 and E2M1 values are bf16 values)
    # sequence 1 skipped steps 3, 10, 17 and 24: those positions hold the rows they were made with
    c.lens = lens
    c.lens[1] = 0                                              # its last step was padding
    lists = c.lists(a.qkv[:, :hq], budget, 1, 2)
    equal_lists(a.blocks, lists)
    c.check_attend(a.qkv[:, :hq], lists, 0.1, a.out, a.lse)


def test_many_rows_and_many_blocks(P):
    """A long context beside short ones; more blocks than a workgroup has threads, scores from several passes."""
    hkv, d = 1, 64
    lens = [70001] + [100 + 13 * i for i in range(60)]
    cache = Cache("int8", hkv, d, lens, seed=18)
    cache.update(P, [0] * len(lens))
    q = queries(len(lens), 33, d, seed=19)
    lists = cache.lists(q, 40, 1, 3)
    equal_lists(cache.select(P, q, 40, 1, 3), lists)


def test_strided_queries_and_other_streams(P):
    cache = Cache("e4m3", 2, 128, [900, 50], seed=20)
    cache.update(P, [0, 0])
    wide = queries(2, 12, 128, seed=21)
    q = wide[:, :8]
    blocks = cache.select(P, q.contiguous(), 9, 1, 2)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = cache.select(P, q, 9, 1, 2, stream=side)
    side.synchronize()
    assert torch.equal(got, blocks)
    out, lse = cache.attend(P, q.contiguous(), blocks, 0.1)
    torch.cuda.synchronize()
    o2, l2 = cache.attend(P, q, blocks, 0.1, stream=side)
    side.synchronize()
    assert torch.equal(out, o2) and torch.equal(lse, l2)


@pytest.mark.parametrize("room", [900, 9000])
def test_two_graphs_share_the_workspaces(P, room):
    """Selection and attention of two batches, replayed in turn with eager calls between them and over changing lengths."""
    hq, hkv, d, budget = 8, 4, 64, 12
    ws = torch.empty(P.pallas_attend_workspace_size(3, hq, hkv, d, 16 * budget), dtype=torch.uint8, device=DEV)
    ws2 = torch.empty(P.pallas_select_workspace_size(3, hkv, room), dtype=torch.uint8, device=DEV)

    class Batch:
        def __init__(self, seed):
            self.c = Cache("int8", hkv, d, [room, room // 2, room // 3], seed=seed)
            self.c.update(P, [0] * 3)
            self.q = queries(3, hq, d, seed)
            self.lengths = self.c.lengths.clone()

        def __call__(self):
            blocks = torch.full((3, hkv, budget), -9, dtype=torch.int32, device=DEV)
            out, lse = torch.zeros_like(self.q), torch.zeros((3, hq), device=DEV)
            P.pallas_select_blocks(self.c.bounds, self.c.bound_scales, 1, self.q, self.lengths, room, self.c.bt, blocks, ws2)
            P.pallas_attend_blocks_quant(*self.c.rows, 1, self.q, self.lengths, room, self.c.bt, blocks, 0.1, out, ws, lse=lse)
            return blocks, out, lse

    batches, graphs, results = [Batch(5), Batch(6)], [], []
    for b in batches:
        b()
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=side):
            results.append(b())
        torch.cuda.current_stream().wait_stream(side)
        graphs.append(graph)
    for cut in (1.0, 0.2, 0.0, 0.6, 1.0):
        for b in batches:
            b.lengths.copy_((b.c.lengths.double() * cut).to(torch.int32))
        for graph in graphs:
            graph.replay()
        batches[0]()
        for b, kept in zip(batches, results):
            for x, y in zip(b(), kept):
                assert torch.equal(x, y), cut
