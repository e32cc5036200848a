"""pallas_attend_kv and pallas_attend_quant against the oracle over the same caches:
lengths from none to several splits, page and split edges, head_dim 64 and 128, groups
of 1 to 20 query heads, bf16 and 8-bit rows, pages outside the pool, unwritten slots
full of NaN.

Tolerance.  A score is a float32 sum of d products: with T = scale sum |q_i k_i|, the
kernel's is within delta = (d + 8) 2^-24 T of the exact one (the additions, the scale of
the row, the product with scale log2 e, which itself is rounded, and the difference from
the running maximum).  So weights are within 2 delta relative, exp2 and the float32 sums
add at most 2^-14 (2^-22 an exponential, 2^-24 an addition in runs of a few hundred, the
weights as two bf16 parts 2^-16); out rounds to bf16 once, 2^-8 of the value:
  |out - ref| <= 2^-8 |ref| + (2 delta + 2^-13) sum_j p_j |v_j| + n 2^-126 max |v|
The last term: exp2 of less than -126 is below float32's normal range and may be 0, so
each of the n weights is off by up to 2^-126 of the largest besides (which matters where
the key of all the weight has a 0).
  |lse - ref| <= delta + 2^-13"""
import math

import numpy as np
import pytest
import torch

from helpers import ensure_lib, to_np64
from oracle import cache_ops as co
from workloads import gen

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


@pytest.fixture(scope="module")
def P():
    return ensure_lib()


class Cache:
    """A pool of two layers whose layer 1 holds `lens` keys per sequence in shuffled pages; every other
    slot holds NaN (of the rows, or of their scales)."""

    def __init__(self, fmt, hkv, d, lens, seed, spare_pages=3, sigma=1.0):
        g = torch.Generator().manual_seed(seed)
        pages = [(n + 15) // 16 for n in lens]
        self.max_pages = max(1, *pages)
        P_ = sum(pages) + spare_pages
        order = np.random.default_rng(seed).permutation(P_)
        self.table = np.full((len(lens), self.max_pages), -1, dtype=np.int32)
        at = 0
        for i, n in enumerate(pages):
            self.table[i, :n] = order[at:at + n]
            at += n
        self.fmt, self.lens, self.d, self.hkv = fmt, list(lens), d, hkv
        self.k, self.v = [], []
        shape = (2, 2, P_, 16, hkv, d)
        if fmt == "bf16":
            pool = torch.full(shape, float("nan"), dtype=torch.bfloat16)
        else:
            codes = np.full(shape, 0x7F, dtype=np.uint8)
            scales = np.full(shape[:-1], np.nan, dtype=np.float32)
        for i, n in enumerate(lens):
            t = np.arange(n)
            pg, slot = self.table[i, t // 16], t % 16
            for kv, keep in ((0, self.k), (1, self.v)):
                x = (sigma * torch.randn((n, hkv, d), generator=g)).to(torch.bfloat16)
                if fmt == "bf16":
                    pool[1, kv, torch.as_tensor(pg, dtype=torch.long), torch.as_tensor(slot)] = x
                    keep.append(to_np64(x))
                else:
                    c, s = co.quantise(to_np64(x), fmt)
                    codes[1, kv, pg, slot], scales[1, kv, pg, slot] = c, s
                    keep.append(co.dequantise(c, s, fmt))
        if fmt == "bf16":
            self.pool = pool.to(DEV)
        else:
            self.codes = torch.from_numpy(codes).to(DEV).view(TYPES[fmt])
            self.scales = torch.from_numpy(scales).to(DEV)
        self.bt = torch.from_numpy(self.table).to(DEV)
        self.lengths = torch.tensor(self.lens, dtype=torch.int32, device=DEV)

    def attend(self, P, q, scale, out=None, lse=None, max_length=None, ws=None, err=None, lengths=None, bt=None, stream=None):
        max_length = max(1, *self.lens) if max_length is None else max_length
        if ws is None:
            ws = torch.full((P.pallas_attend_workspace_size(len(self.lens), q.shape[1], self.hkv, self.d, max_length),), 0xFF,
                            dtype=torch.uint8, device=DEV)
        out = torch.full_like(q, 7.0) if out is None else out
        lengths = self.lengths if lengths is None else lengths
        bt = self.bt if bt is None else bt
        if self.fmt == "bf16":
            P.pallas_attend_kv(self.pool, 1, q, lengths, max_length, bt, scale, out, ws, lse=lse, err=err, stream=stream)
        else:
            P.pallas_attend_quant(self.codes, self.scales, 1, q, lengths, max_length, bt, scale, out, ws, lse=lse, err=err,
                                  stream=stream)
        return out


def queries(S, hq, d, seed):
    return torch.randn((S, hq, d), generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).to(DEV)


def check(cache, q, scale, out, lse, drop=None):
    """`drop[i]`: key positions of sequence i that are masked."""
    qn, on = to_np64(q), to_np64(out)
    ln = lse.double().cpu().numpy()
    for i, n in enumerate(cache.lens):
        keep = np.setdiff1d(np.arange(n), [] if drop is None else drop.get(i, []))
        ref, rl, mag, terms = co.attend(qn[i], cache.k[i][keep], cache.v[i][keep], scale)
        delta = ((cache.d + 8) * 2.0 ** -24 * terms)[:, None]
        diff, tol = np.abs(on[i] - ref), 2.0 ** -8 * np.abs(ref) + (2 * delta + 2.0 ** -13) * mag
        tol = tol + n * 2.0 ** -126 * max(1.0, np.abs(cache.v[i]).max(initial=0.0))
        assert np.all(diff <= tol), (i, n, float((diff - tol).max()))
        if len(keep) == 0:
            assert np.all(ln[i] == -np.inf) and not on[i].any()
        else:
            assert np.all(np.abs(ln[i] - rl) <= delta[:, 0] + 2.0 ** -13), (i, n)


CASES = [
    # head_dim, group, KV heads, lengths
    (128, 8, 2, [0, 1, 15, 16, 17, 31, 32, 33, 127, 128, 129]),
    (128, 4, 8, [255, 256, 257, 1000, 0, 64, 65]),
    (128, 1, 4, [63, 300, 900, 4000]),
    (64, 2, 2, [0, 31, 64, 127, 128, 1100, 0]),
    (64, 8, 1, [500, 2048, 5000]),
    (64, 3, 4, [1, 2, 2049, 640]),
    (128, 12, 1, [700, 129]),
    (128, 16, 2, [383, 1]),
    (128, 20, 1, [130, 511]),
    (64, 37, 1, [260]),
    (128, 7, 5, [1025, 12, 96]),
    (128, 8, 8, [9001]),
    (64, 4, 16, [97 * i for i in range(33)]),
    (128, 2, 4, [0] * 70 + [33] + [0] * 64 + [1, 500] + [0] * 30),   # few keys in many rows
    (64, 1, 2, [1 + i % 3 for i in range(300)]),                     # a block a row
    (128, 4, 2, [0, 0, 0]),
    (128, 8, 8, [7 * i for i in range(73)]),                         # short rows, several to a CU
    (64, 4, 4, [14 * i for i in range(36)]),
    (64, 2, 8, [i % 40 for i in range(200)]),                        # too many of them for a workgroup each
    (128, 20, 8, [512, 511, 1]),                                     # the longest short rows
    (64, 1, 1, [512, 0, 33]),
    (64, 1, 1, [513, 0, 33]),
    (128, 8, 8, [4001]),                                             # splits of one block a wave (bf16: of two)
    (128, 4, 4, [3000, 1, 0, 257]),
    (128, 8, 1, [7000, 5000]),
    (64, 4, 2, [9000]),
    (128, 5, 3, [2500, 600, 2047]),
]


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("d,group,hkv,lens", CASES)
def test_against_oracle(P, d, group, hkv, lens, fmt):
    cache = Cache(fmt, hkv, d, lens, seed=d + group)
    q = queries(len(lens), group * hkv, d, 3)
    lse = torch.full((len(lens), group * hkv), 9.0, dtype=torch.float32, device=DEV)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    scale = 1 / math.sqrt(d)
    out = cache.attend(P, q, scale, lse=lse, err=err)
    assert int(err.item()) == 0
    check(cache, q, scale, out, lse)
    # Without lse: the same bits.
    assert torch.equal(cache.attend(P, q, scale), out)
    # With a larger bound on the lengths (short rows are then divided as long ones are) and a table wider than
    # they need.
    bt = torch.full((len(lens), cache.max_pages + 300), -1, dtype=torch.int32, device=DEV)
    bt[:, :cache.max_pages] = cache.bt
    lse.fill_(9.0)
    check(cache, q, scale, cache.attend(P, q, scale, max_length=max(lens) + 4000, bt=bt, lse=lse, err=err), lse)
    assert int(err.item()) == 0


@pytest.mark.parametrize("fmt,d,hkv,n", [("bf16", 128, 2, 400000), ("e4m3", 64, 32, 100000), ("int8", 128, 16, 100000)])
def test_more_blocks_than_one_round(P, fmt, d, hkv, n):
    """Ranges at their longest, several of them a wave: against torch in float64 on the GPU, head by head."""
    lens = [n, 0, 777, n // 2]
    pages = [(x + 15) // 16 for x in lens]
    rng = np.random.default_rng(3)
    spare = 50
    bt = np.full((4, max(pages)), -1, dtype=np.int32)
    for i, x in enumerate(pages):       # the rows share the pool's pages
        bt[i, :x] = rng.permutation(max(pages) + spare)[:x]
    bt = torch.from_numpy(bt).to(DEV)
    g = torch.Generator(DEV).manual_seed(1)
    shape = (1, 2, max(pages) + spare, 16, hkv, d)
    q = queries(4, hkv, d, 4)
    lengths = torch.tensor(lens, dtype=torch.int32, device=DEV)
    out, lse = torch.empty_like(q), torch.empty((4, hkv), dtype=torch.float32, device=DEV)
    ws = torch.empty(P.pallas_attend_workspace_size(4, hkv, hkv, d, n), dtype=torch.uint8, device=DEV)
    if fmt == "bf16":
        pool = torch.randn(shape, device=DEV, generator=g).to(torch.bfloat16)
        P.pallas_attend_kv(pool, 0, q, lengths, n, bt, 0.1, out, ws, lse=lse)
    else:
        codes = torch.randint(0, 120, shape, dtype=torch.uint8, device=DEV, generator=g).view(TYPES[fmt])
        scales = torch.rand(shape[:-1], device=DEV, generator=g) * 0.01
        P.pallas_attend_quant(codes, scales, 0, q, lengths, n, bt, 0.1, out, ws, lse=lse)
    for i, x in enumerate(lens):
        t = torch.arange(x, device=DEV)
        pg, slot = bt[i].long()[t // 16], t % 16
        for h in range(0, hkv, 5):
            if fmt == "bf16":
                k, v = (pool[0, kv, pg, slot, h].double() for kv in range(2))
            else:
                k, v = (codes.view(torch.uint8)[0, kv, pg, slot, h].view(TYPES[fmt]).double() *
                        scales[0, kv, pg, slot, h].double()[:, None] for kv in range(2))
            if x == 0:
                assert not out[i, h].any() and float(lse[i, h]) == -math.inf
                continue
            qd = q[i, h].double()
            z = (k * qd).sum(1) * 0.1
            ref_lse = torch.logsumexp(z, 0)
            p = torch.exp(z - ref_lse)
            ref, mag = (p[:, None] * v).sum(0), (p[:, None] * v.abs()).sum(0)
            delta = (d + 8) * 2.0 ** -24 * float(((k * qd).abs().sum(1) * 0.1).max())
            # sums run over thousands of keys a range, and hundreds of ranges: 2^-12 in place of 2^-13
            tol = 2.0 ** -8 * ref.abs() + (2 * delta + 2.0 ** -12) * mag
            assert bool(((out[i, h].double() - ref).abs() <= tol).all()), (i, h)
            assert abs(float(lse[i, h]) - float(ref_lse)) <= delta + 2.0 ** -12


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
def test_many_sequences_and_long_ones(P, fmt):
    """Splits of the largest length, and more workgroups than fit at once."""
    lens = [17000, 3, 9000] + [40 + 61 * i for i in range(60)]
    cache = Cache(fmt, 2, 128, lens, seed=8)
    q = queries(len(lens), 8, 128, 4)
    lse = torch.empty((len(lens), 8), dtype=torch.float32, device=DEV)
    check(cache, q, 0.09, cache.attend(P, q, 0.09, lse=lse), lse)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_thousands_of_rows(P, fmt):
    """More rows than 64 partial sums of 64 lengths, most of them short or empty: a sample against the oracle."""
    rng = np.random.default_rng(4)
    lens = [int(n) for n in rng.choice([0, 1, 5, 31, 32, 33, 70], size=4500)]
    lens[2222] = 3000
    cache = Cache(fmt, 1, 64, lens, seed=14)
    q = queries(len(lens), 2, 64, 7)
    lse = torch.empty((len(lens), 2), dtype=torch.float32, device=DEV)
    out = cache.attend(P, q, 0.125, lse=lse)
    some = sorted({0, 1, 63, 64, 65, 2221, 2222, 2223, 4498, 4499, *rng.integers(0, 4500, 150).tolist()})
    cache.lens, cache.k, cache.v = [lens[i] for i in some], [cache.k[i] for i in some], [cache.v[i] for i in some]
    check(cache, q[some], 0.125, out[some], lse[some])


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
def test_pages_beyond_4_gib(P, fmt):
    """Pages at the end of planes of more than 4 GiB; nothing else of the pool is read."""
    hkv, d, lens = 8, 128, [600, 33, 1100]
    cache = Cache(fmt, hkv, d, lens, seed=15)
    page_bytes = 16 * hkv * d * (2 if fmt == "bf16" else 1)
    pages = (1 << 32) // page_bytes + 500
    small = cache.pool if fmt == "bf16" else cache.codes.view(torch.uint8)
    held = small.shape[2]
    big = torch.empty((1, 2, pages, 16, hkv, d), dtype=small.dtype, device=DEV)
    big[0, :, pages - held:] = small[1]
    bt = torch.where(cache.bt >= 0, cache.bt + (pages - held), cache.bt)
    q = queries(3, 16, d, 9)
    out, lse = torch.empty_like(q), torch.empty((3, 16), dtype=torch.float32, device=DEV)
    ws = torch.empty(P.pallas_attend_workspace_size(3, 16, hkv, d, 1100), dtype=torch.uint8, device=DEV)
    if fmt == "bf16":
        P.pallas_attend_kv(big, 0, q, cache.lengths, 1100, bt, 0.09, out, ws, lse=lse)
    else:
        scales = torch.empty((1, 2, pages, 16, hkv), dtype=torch.float32, device=DEV)
        scales[0, :, pages - held:] = cache.scales[1]
        P.pallas_attend_quant(big.view(TYPES[fmt]), scales, 0, q, cache.lengths, 1100, bt, 0.09, out, ws, lse=lse)
    check(cache, q, 0.09, out, lse)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
def test_steep_scores(P, fmt):
    """Scores of hundreds: the running maximum moves by more than the exponent's range."""
    cache = Cache(fmt, 2, 64, [700, 33], seed=5, sigma=20.0)
    q = queries(2, 8, 64, 6) * 8
    lse = torch.empty((2, 8), dtype=torch.float32, device=DEV)
    for scale in (1.0, -1.0, 0.0):
        check(cache, q, scale, cache.attend(P, q, scale, lse=lse), lse)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_strided_rows(P, fmt):
    """q inside projection rows, out inside wider rows; nothing beside them is written."""
    lens = [100, 45, 300]
    cache = Cache(fmt, 2, 128, lens, seed=6)
    S, hq, d = len(lens), 8, 128
    wide = torch.randn((S, (hq + 4) * d), device=DEV).to(torch.bfloat16)
    q = wide[:, :hq * d].view(S, hq, d)
    outs = torch.full((S, (hq + 2) * d), 5.0, dtype=torch.bfloat16, device=DEV)
    out = outs[:, d:(hq + 1) * d].view(S, hq, d)
    lse = torch.empty((S, hq), dtype=torch.float32, device=DEV)
    cache.attend(P, q, 0.1, out=out, lse=lse)
    check(cache, q, 0.1, out, lse)
    assert bool((outs[:, :d] == 5.0).all()) and bool((outs[:, (hq + 1) * d:] == 5.0).all())


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
def test_pages_outside_the_pool(P, fmt):
    """Keys on such pages are masked; a row of them alone counts as empty."""
    lens = [400, 90, 20, 33, 1500]
    cache = Cache(fmt, 2, 128, lens, seed=7)
    pages = cache.pool.shape[2] if fmt == "bf16" else cache.codes.shape[2]
    bt = cache.table.copy()
    drop = {0: [0, 7, 24], 1: [5], 2: [0, 1], 3: [1], 4: list(range(0, 94, 3))}
    for i, ps in drop.items():
        for n, p in enumerate(ps):
            bt[i, p] = (-1, pages, 2 ** 31 - 1, -2 ** 31)[n % 4]
    gone = {i: np.concatenate([np.arange(16 * p, 16 * p + 16) for p in ps]) for i, ps in drop.items()}
    q = queries(len(lens), 6, 128, 8)
    lse = torch.empty((len(lens), 6), dtype=torch.float32, device=DEV)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = cache.attend(P, q, 0.09, lse=lse, err=err, bt=torch.from_numpy(bt).to(DEV))
    assert int(err.item()) == 1
    check(cache, q, 0.09, out, lse, gone)
    # short rows alone
    cache.lens[-1] = 17
    cache.k[-1], cache.v[-1] = cache.k[-1][:17], cache.v[-1][:17]
    lengths = torch.tensor(cache.lens, dtype=torch.int32, device=DEV)
    err.zero_()
    out = cache.attend(P, q, 0.09, lse=lse, err=err, bt=torch.from_numpy(bt).to(DEV), lengths=lengths)
    assert int(err.item()) == 1
    check(cache, q, 0.09, out, lse, gone)


@pytest.mark.parametrize("fmt", ["bf16", "int8"])
def test_lengths_outside_the_bound(P, fmt):
    cache = Cache(fmt, 1, 64, [200, 200, 50], seed=9)
    q = queries(3, 4, 64, 1)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    lengths = torch.tensor([2 ** 31 - 1, -3, 50], dtype=torch.int32, device=DEV)
    lse = torch.empty((3, 4), dtype=torch.float32, device=DEV)
    out = cache.attend(P, q, 0.1, lse=lse, max_length=150, err=err, lengths=lengths)
    assert int(err.item()) == 4
    cache.lens = [150, 0, 50]
    for i, n in enumerate(cache.lens):
        cache.k[i], cache.v[i] = cache.k[i][:n], cache.v[i][:n]
    check(cache, q, 0.1, out, lse)
    # the same where long rows are possible
    bt = torch.nn.functional.pad(cache.bt, (0, 200), value=-1).contiguous()
    lengths[0] = 150
    err.zero_()
    out = cache.attend(P, q, 0.1, lse=lse, max_length=3000, err=err, lengths=lengths, bt=bt)
    assert int(err.item()) == 4
    check(cache, q, 0.1, out, lse)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
def test_a_row_does_not_depend_on_the_others(P, fmt):
    """Whatever the others ask and hold, at the same lengths: to the bit."""
    lens = [1300, 77, 500, 0]
    cache = Cache(fmt, 4, 128, lens, seed=10)
    q = queries(4, 16, 128, 2)
    lse = torch.empty((4, 16), dtype=torch.float32, device=DEV)
    out = cache.attend(P, q, 0.1, lse=lse)
    q2 = q.clone()
    q2[1:] = 100.0
    bt = cache.bt.clone()
    bt[1, :5], bt[2, 3] = -1, bt[0, 7]
    lse2 = torch.empty_like(lse)
    out2 = cache.attend(P, q2, 0.1, lse=lse2, bt=bt)
    assert torch.equal(out[0], out2[0]) and torch.equal(lse[0], lse2[0]) and not torch.equal(out[2], out2[2])


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
def test_nan_reaches_its_own_rows_alone(P, fmt):
    """A NaN key is a NaN result for the heads that read it; an infinite query too."""
    lens = [200, 300]
    cache = Cache(fmt, 2, 128, lens, seed=11)
    pg, slot = int(cache.table[0, 150 // 16]), 150 % 16
    if fmt == "bf16":
        cache.pool[1, 0, pg, slot, 1, 5] = float("nan")
    else:
        cache.scales[1, 0, pg, slot, 1] = float("nan")
    q = queries(2, 4, 128, 3)
    lse = torch.empty((2, 4), dtype=torch.float32, device=DEV)
    out = cache.attend(P, q, 0.1, lse=lse)
    assert bool(torch.isnan(out[0, 2:]).all()) and bool(torch.isnan(lse[0, 2:]).all())
    assert bool(torch.isfinite(out[0, :2]).all()) and bool(torch.isfinite(out[1]).all())
    # a NaN value among finite weights: its dimension alone (8-bit: the row)
    cache = Cache(fmt, 2, 128, lens, seed=11)
    if fmt == "bf16":
        cache.pool[1, 1, pg, slot, 1, 5] = float("nan")
    else:
        cache.scales[1, 1, pg, slot, 1] = float("nan")
    out = cache.attend(P, q, 0.1, lse=lse)
    assert bool(torch.isnan(out[0, 2:, 5]).all()) and bool(torch.isfinite(lse).all())
    assert bool(torch.isfinite(out[0, :2]).all()) and bool(torch.isfinite(out[1]).all())
    # nothing but NaN
    cache = Cache(fmt, 2, 128, [1, 40], seed=12)
    q[0] = float("nan")
    out = cache.attend(P, q, 0.1, lse=lse)
    assert bool(torch.isnan(out[0]).all()) and bool(torch.isnan(lse[0]).all()) and bool(torch.isfinite(out[1]).all())


def test_parts_join_through_lse(P):
    """Attention over a cache's two halves, joined, is attention over all of it."""
    n, half = 96 * 16, 40 * 16
    cache = Cache("bf16", 2, 128, [n], seed=13)
    q = queries(1, 8, 128, 5)
    lse = torch.empty((3, 8), dtype=torch.float32, device=DEV)
    whole = cache.attend(P, q, 0.09, lse=lse[0:1])
    a = cache.attend(P, q, 0.09, lse=lse[1:2], lengths=torch.tensor([half], dtype=torch.int32, device=DEV), max_length=n)
    b = cache.attend(P, q, 0.09, lse=lse[2:3], lengths=torch.tensor([n - half], dtype=torch.int32, device=DEV), max_length=n,
                     bt=torch.cat([cache.bt[:, 40:], cache.bt[:, :40]], dim=1).contiguous())
    wa, wb = (torch.exp(lse[i] - torch.logaddexp(lse[1], lse[2]))[None, :, None] for i in (1, 2))
    joined = wa * a.float() + wb * b.float()
    # each part and the whole round to bf16 once
    tol = 2.0 ** -8 * (whole.float().abs() + wa * a.float().abs() + wb * b.float().abs()) + 2.0 ** -12
    assert bool(((joined - whole.float()).abs() <= tol).all())
    assert bool(((torch.logaddexp(lse[1], lse[2]) - lse[0]).abs() <= 2.0 ** -12).all())
