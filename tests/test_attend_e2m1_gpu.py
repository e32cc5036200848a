"""pallas_attend_quant over a 4-bit cache against the oracle over the same values: each way
of running (one workgroup a row, splits, ranges), lengths from none to long ones, page and
block edges, head_dim 64 and 128, groups of 1 to 40 query heads, pages outside the pool,
unwritten slots full of NaN.

Tolerance.  K and V times their scales are bf16 values, so scores are float32 sums of d exact
products: with T = scale sum |q_i k_i| within delta = (d + 8) 2^-24 T of the exact ones (the
additions, the product with scale log2 e, which itself is rounded, and the difference from the
running maximum).  Weights are within 2 delta relative, exp2 and the float32 sums add at most
2^-14 (2^-22 an exponential, 2^-24 an addition in runs of a few hundred), out rounds to bf16
once, 2^-8 of the value:
  |out - ref| <= 2^-8 |ref| + (2 delta + 2^-13) sum_j p_j |v_j| + n 2^-126 max |v|
  |lse - ref| <= delta + 2^-13"""
import math

import numpy as np
import pytest
import torch

from helpers import ensure_lib, to_np64
from oracle import cache_ops as co

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def P():
    return ensure_lib()


class Cache:
    """A pool of two layers whose layer 1 holds `lens` keys per sequence in shuffled pages; every other slot
    reads as NaN."""

    def __init__(self, hkv, d, lens, seed, spare_pages=3, sigma=1.0):
        g = torch.Generator().manual_seed(seed)
        pages = [(n + 15) // 16 for n in lens]
        self.max_pages = max(1, *pages)
        order = np.random.default_rng(seed).permutation(sum(pages) + spare_pages)
        self.table = np.full((len(lens), self.max_pages), -1, dtype=np.int32)
        at = 0
        for i, n in enumerate(pages):
            self.table[i, :n] = order[at:at + n]
            at += n
        self.lens, self.d, self.hkv = list(lens), d, hkv
        codes = np.full((2, 2, len(order), 16, hkv, d // 2), 0x77, dtype=np.uint8)
        scales = np.full((2, 2, len(order), 16, hkv, 4), 255, dtype=np.uint8)
        self.kv = ([], [])
        for i, n in enumerate(lens):
            t = np.arange(n)
            pg, slot = self.table[i, t // 16], t % 16
            for kv, keep in enumerate(self.kv):
                # channels of several magnitudes, rows too
                x = sigma * torch.randn((n, hkv, d), generator=g) * torch.exp(0.7 * torch.randn((1, hkv, d), generator=g))
                c, s = co.quantise4(to_np64((x * torch.exp(0.3 * torch.randn((n, hkv, 1), generator=g))).to(torch.bfloat16)))
                codes[1, kv, pg, slot], scales[1, kv, pg, slot] = c, s
                keep.append(co.dequantise4(c, s))
        self.codes = torch.from_numpy(codes).to(DEV).view(torch.float4_e2m1fn_x2)
        self.scales = torch.from_numpy(scales).to(DEV).view(torch.float8_e8m0fnu)
        self.bt = torch.from_numpy(self.table).to(DEV)
        self.lengths = torch.tensor(self.lens, dtype=torch.int32, device=DEV)

    def attend(self, P, q, scale, lse=None, max_length=None, ws=None, err=None, lengths=None, bt=None, stream=None):
        max_length = max(1, *self.lens) if max_length is None else max_length
        if ws is None:
            ws = torch.full((P.pallas_attend_workspace_size(len(self.lens), q.shape[1], self.hkv, self.d, max_length),), 0xFF,
                            dtype=torch.uint8, device=DEV)
        out = torch.full_like(q, 7.0)
        P.pallas_attend_quant(self.codes, self.scales, 1, q, self.lengths if lengths is None else lengths, max_length,
                              self.bt if bt is None else bt, scale, out, ws, lse=lse, err=err, stream=stream)
        return out


def queries(S, hq, d, seed):
    return torch.randn((S, hq, d), generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).to(DEV)


def check(cache, q, scale, out, lse, drop=None):
    """`drop[i]`: key positions of sequence i that are masked."""
    qn, on, ln = to_np64(q), to_np64(out), lse.double().cpu().numpy()
    for i, n in enumerate(cache.lens):
        keep = np.setdiff1d(np.arange(n), [] if drop is None else drop.get(i, []))
        k, v = cache.kv[0][i][keep], cache.kv[1][i][keep]
        ref, rl, mag, terms = co.attend(qn[i], k, v, scale)
        delta = ((cache.d + 8) * 2.0 ** -24 * terms)[:, None]
        tol = 2.0 ** -8 * np.abs(ref) + (2 * delta + 2.0 ** -13) * mag + n * 2.0 ** -126 * max(1.0, np.abs(v).max(initial=0.0))
        diff = np.abs(on[i] - ref)
        assert np.all(diff <= tol), (i, n, float((diff - tol).max()))
        if len(keep) == 0:
            assert np.all(ln[i] == -np.inf) and not on[i].any()
        else:
            assert np.all(np.abs(ln[i] - rl) <= delta[:, 0] + 2.0 ** -13), (i, n)


CASES = [
    # head_dim, group, KV heads, lengths, max_length (None: the longest)
    (128, 8, 2, [0, 1, 15, 16, 17, 31, 32, 33, 127, 128, 129], None),          # a workgroup each
    (128, 4, 8, [255, 256, 257, 1000, 0, 64, 65], None),
    (128, 1, 4, [63, 300, 900, 4000], None),
    (64, 2, 2, [0, 31, 64, 127, 128, 1100, 0], None),
    (64, 8, 1, [500, 2048, 5000], None),
    (64, 3, 4, [1, 2, 2049, 640], None),
    (128, 12, 1, [700, 129], None),
    (128, 16, 2, [383, 1], None),
    (128, 20, 1, [130, 511], None),
    (64, 40, 1, [260], None),
    (128, 7, 5, [1025, 12, 96], None),
    (128, 8, 8, [9001], None),
    (64, 8, 8, [9001, 7], None),
    (128, 3, 2, [1500, 90, 20, 33, 0, 700], 20000),                             # ranges of one block
    (64, 3, 2, [3000, 1500, 0, 33], 20000),                                     # of two
    (128, 3, 8, [9000, 90, 20, 33, 0, 700, 8000, 4000, 300], None),             # of more
    (64, 3, 8, [20000, 90, 20, 33, 0, 700, 18000, 4000, 300, 15000], None),
]


@pytest.mark.parametrize("d,group,hkv,lens,max_length", CASES)
def test_matches_oracle(P, d, group, hkv, lens, max_length):
    room = max(1, *lens) if max_length is None else max_length
    cache = Cache(hkv, d, lens, seed=d + group)
    bt = torch.nn.functional.pad(cache.bt, (0, -(-room // 16) - cache.max_pages), value=-1).contiguous()
    q = queries(len(lens), hkv * group, d, seed=5)
    lse = torch.full(q.shape[:2], 9.0, device=DEV)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    scale = 1 / math.sqrt(d)
    out = cache.attend(P, q, scale, lse=lse, err=err, bt=bt, max_length=room)
    check(cache, q, scale, out, lse)
    assert int(err.item()) == 0
    again = cache.attend(P, q, scale, bt=bt, max_length=room)            # no flag, no log-sum-exp, the same bits
    assert torch.equal(out, again)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", [[40, 0, 200], [1500, 700, 100], [9000, 3, 0, 8000]])
def test_peaked_scores(P, d, lens):
    """Scores that leave one key nearly all weight, positive and negative scales."""
    cache = Cache(2, d, lens, seed=3, sigma=4.0)
    q = queries(len(lens), 6, d, seed=6) * 4
    for scale in (1.0, -0.5, 0.0):
        lse = torch.empty(q.shape[:2], device=DEV)
        out = cache.attend(P, q, scale, lse=lse)
        check(cache, q, scale, out, lse)


@pytest.mark.parametrize("d", [64, 128])
def test_pages_outside_the_pool_and_lengths_outside(P, d):
    lens = [100, 40, 5000, 20]
    cache = Cache(2, d, lens, seed=4)
    bt = cache.bt.clone()
    pages = cache.codes.shape[2]
    bt[0, 2], bt[2, 17], bt[3, 0], bt[3, 1] = pages, -5, 1 << 30, -1
    q = queries(4, 8, d, seed=7)
    lse, err = torch.empty((4, 8), device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    out = cache.attend(P, q, 0.1, lse=lse, err=err, bt=bt)
    check(cache, q, 0.1, out, lse, drop={0: np.arange(32, 48), 2: np.arange(17 * 16, 18 * 16), 3: np.arange(20)})
    assert int(err.item()) == 1
    err.zero_()
    out = cache.attend(P, q, 0.1, lse=lse, err=err, max_length=5000,
                       lengths=torch.tensor([-3, 40, 6000, 20], dtype=torch.int32, device=DEV))
    cache.lens[0] = 0
    cache.kv[0][0], cache.kv[1][0] = cache.kv[0][0][:0], cache.kv[1][0][:0]
    check(cache, q, 0.1, out, lse)
    assert int(err.item()) == 4


def test_nan_reaches_the_heads_that_read_it_alone(P):
    lens = [70, 900]
    cache = Cache(4, 128, lens, seed=8)
    q = queries(2, 8, 128, seed=9)
    lse = torch.empty((2, 8), device=DEV)
    clean = cache.attend(P, q, 0.1, lse=lse)
    raw = cache.scales.view(torch.uint8)
    raw[1, 0, cache.table[0, 3], 2, 1, 0] = 255          # a K quarter of position 50, KV head 1
    raw[1, 1, cache.table[1, 10], 0, 2, 3] = 255         # a V quarter of position 160, KV head 2
    out = cache.attend(P, q, 0.1, lse=lse)
    assert bool(torch.isnan(out[0, 2:4]).all()) and bool(torch.isnan(out[1, 4:6, 96:]).all())
    same = torch.ones_like(out, dtype=torch.bool)
    same[0, 2:4] = same[1, 4:6] = False
    assert torch.equal(out[same], clean[same])


def test_long_cache_with_offsets_past_32_bits(P):
    """Codes of more than 4 GiB a layer: keys on the last pages of the second layer."""
    hkv, d, n = 16, 128, 333
    pages = (1 << 32) // (2 * 16 * hkv * d // 2) + 40
    codes = torch.zeros((2, 2, pages, 16, hkv, d // 2), dtype=torch.uint8, device=DEV)
    scales = torch.zeros((2, 2, pages, 16, hkv, 4), dtype=torch.uint8, device=DEV)
    small = Cache(hkv, d, [n], seed=10)
    place = torch.arange(pages - 1, pages - 1 - small.max_pages, -1, dtype=torch.int32, device=DEV)[None]
    codes[1, :, place[0].long()] = small.codes.view(torch.uint8)[1][:, small.bt[0].long()]
    scales[1, :, place[0].long()] = small.scales.view(torch.uint8)[1][:, small.bt[0].long()]
    q = queries(1, 32, d, seed=11)
    a, la = torch.empty_like(q), torch.empty((1, 32), device=DEV)
    ws = torch.empty(P.pallas_attend_workspace_size(1, 32, hkv, d, n), dtype=torch.uint8, device=DEV)
    P.pallas_attend_quant(codes.view(torch.float4_e2m1fn_x2), scales.view(torch.float8_e8m0fnu), 1, q, small.lengths, n,
                          place.contiguous(), 0.1, a, ws, lse=la)
    check(small, q, 0.1, a, la)
    del codes, scales


@pytest.mark.parametrize("d", [64, 128])
def test_captured_and_replayed(P, d):
    """Replays after the lengths changed equal the eager call to the bit; eager work and synchronisation between."""
    cache = Cache(2, d, [3000, 40, 700], seed=12)
    q = queries(3, 8, d, seed=13)
    out, lse = torch.zeros_like(q), torch.zeros((3, 8), device=DEV)
    ws = torch.empty(P.pallas_attend_workspace_size(3, 8, 2, d, 3000), dtype=torch.uint8, device=DEV)
    lengths = cache.lengths.clone()

    def call():
        P.pallas_attend_quant(cache.codes, cache.scales, 1, q, lengths, 3000, cache.bt, 0.1, out, ws, lse=lse)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    torch.cuda.synchronize()
    for lens in ([3000, 40, 700], [1, 0, 650], [2999, 33, 0], [3000, 40, 700]):
        lengths.copy_(torch.tensor(lens, dtype=torch.int32))
        out.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        call()
        torch.cuda.synchronize()
        assert torch.equal(got[0], out) and torch.equal(got[1], lse)
