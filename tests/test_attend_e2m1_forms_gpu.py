"""Attention over a 4-bit cache in each of the ways in which it is run (one workgroup a row, splits
and a join, ranges of one KV head and of two neighbouring ones and a join), read back from the
workspace of a call: masked pages, NaN, strided rows, rows that do not depend on the others, weights
that cancel, many rows, more than one round of ranges, replays and shared workspaces.

Tolerances: those of test_attend_e2m1_gpu, 2^-12 in place of 2^-13 for the sums of long rows."""
import functools
import math

import numpy as np
import pytest
import torch

from helpers import ensure_lib, to_np64
from oracle import cache_ops as co
from test_attend_e2m1_gpu import DEV, Cache, check, queries

pytestmark = pytest.mark.gpu

#: form -> (KV heads, query heads of each, lengths, max_length, blocks of a range)
FORMS = {
    "short": (2, 3, [400, 90, 20, 33, 0, 500], 500, None),
    "split": (2, 3, [1500, 90, 20, 33, 0, 700], 1500, None),
    "heads": (3, 3, [9000, 90, 20, 33, 0, 700, 8000, 4000, 300], 9000, 2),
    "heads-20": (2, 20, [9000, 90, 20, 33, 0, 700, 18000, 4000, 300], 18000, 2),
    "pairs-1": (2, 3, [1500, 90, 20, 33, 0, 700], 20000, 1),
    "pairs-2": (2, 8, [3000, 1500, 0, 33], 20000, 2),
    "pairs-4": (8, 3, [9000, 90, 20, 33, 0, 700, 8000, 4000, 300], 9000, 4),
}
KINDS = [pytest.param(form, d, id=f"{form}-{d}") for form in FORMS for d in (64, 128)]


def blocks(n):
    return -(-int(n) // 32)


def range_blocks(hkv, group, lens):
    """Blocks of a range, restated."""
    pair = hkv % 2 == 0 and 2 * group <= 16
    ranges = max((256 * 3 // (hkv // 2) if pair else 256 * 12 // (hkv * -(-group // 16))) // 8 * 8, 8)
    total = sum(map(blocks, lens))
    if 2 * total <= ranges and total <= 32 * len(lens):
        return 1
    if total <= 2 * ranges:
        return 2
    rounds = max(-(-total // ((128 if pair else 32) * ranges)), 1)
    return -(-total // (rounds * ranges))


def check_form(form, ws, hkv, group, lens, max_length):
    """`ws`: the call's workspace, all 0xFF before it; a row's first record and their number are at its head."""
    if form == "short":
        assert bool((ws == 0xFF).all())
        return
    got = ws[:8 * len(lens)].cpu().numpy().view(np.int32).reshape(-1, 2).tolist()
    if form == "split":
        splits = -(-blocks(max_length) // 8)
        assert got == [[s * splits - s, 0 if blocks(n) <= 8 else -(-blocks(n) // 8)] for s, n in enumerate(lens)]
        return
    each, at, total = range_blocks(hkv, group, lens), 0, sum(map(blocks, lens))
    for s, n in enumerate(lens):
        end, r = at + blocks(n), at // each
        want = [-1, -1] if n == 0 else [r, 0 if end <= min((r + 1) * each, total) else (end - 1) // each - r + 1]
        assert got[s] == want, (form, s)
        at = end


@pytest.fixture(scope="module")
def P():
    return ensure_lib()


@functools.lru_cache(maxsize=None)
def cache_of(form, d):
    return Cache(FORMS[form][0], d, FORMS[form][2], seed=d + 1)


class Call:
    """A cache of a form's lengths (one for all tests, which leave it as it was), and calls of that form over it."""

    def __init__(self, P, form, d, seed):
        self.P, self.form, self.d = P, form, d
        self.hkv, self.group, self.lens, self.max_length, each = FORMS[form]
        assert each is None or each == range_blocks(self.hkv, self.group, self.lens)
        self.S, self.hq = len(self.lens), self.group * self.hkv
        self.cache = cache_of(form, d)
        self.bt = torch.full((self.S, -(-self.max_length // 16)), -1, dtype=torch.int32, device=DEV)
        self.bt[:, :self.cache.max_pages] = self.cache.bt
        self.q = queries(self.S, self.hq, d, seed)

    def workspace(self):
        return torch.full((self.P.pallas_attend_workspace_size(self.S, self.hq, self.hkv, self.d, self.max_length),), 0xFF,
                          dtype=torch.uint8, device=DEV)

    def __call__(self, q=None, scale=0.09, lens=None, out=None, **kw):
        """(out, lse)"""
        q = self.q if q is None else q
        lse = torch.full((self.S, self.hq), 9.0, dtype=torch.float32, device=DEV)
        ws = self.workspace()
        out = torch.full((self.S, self.hq, self.d), 7.0, dtype=torch.bfloat16, device=DEV) if out is None else out
        self.P.pallas_attend_quant(self.cache.codes, self.cache.scales, 1, q, kw.pop("lengths", self.cache.lengths), self.max_length,
                                   kw.pop("bt", self.bt), scale, out, ws, lse=lse, **kw)
        check_form(self.form, ws, self.hkv, self.group, self.lens if lens is None else lens, self.max_length)
        return out, lse


@pytest.mark.parametrize("form,d", KINDS)
def test_against_oracle_and_pages_outside_the_pool(P, form, d):
    """Keys on such pages are masked and raise the flag; a row of them alone counts as empty."""
    c = Call(P, form, d, 31)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    out, lse = c(err=err)
    check(c.cache, c.q, 0.09, out, lse)
    assert int(err.item()) == 0
    pages, bt, drop = c.cache.codes.shape[2], c.bt.cpu().numpy().copy(), {}
    rng = np.random.default_rng(1)
    for i, n in enumerate(c.lens):
        have = -(-n // 16)
        gone = np.arange(have) if n == 33 else np.unique(np.concatenate([[0, have - 1], rng.integers(0, have, have // 5)])) if have > 3 else []
        for m, p in enumerate(gone):
            bt[i, p] = (-1, pages, 2 ** 31 - 1, -2 ** 31)[m % 4]
        drop[i] = np.concatenate([np.arange(16 * p, 16 * p + 16) for p in gone] or [np.zeros(0, int)])
    out, lse = c(err=err, bt=torch.from_numpy(bt).to(DEV))
    assert int(err.item()) == 1
    check(c.cache, c.q, 0.09, out, lse, drop=drop)
    assert not out[c.lens.index(33)].any()


@pytest.mark.parametrize("form,d", KINDS)
def test_lengths_outside_the_bound(P, form, d):
    c = Call(P, form, d, 32)
    i = c.lens.index(33)
    lengths, lens, err = c.cache.lengths.clone(), list(c.lens), torch.zeros(1, dtype=torch.int32, device=DEV)
    lengths[i], lens[i] = -2 ** 31, 0
    if c.max_length in lens:
        lengths[lens.index(c.max_length)] = 2 ** 31 - 1
    want, want_lse = c(lengths=torch.tensor(lens, dtype=torch.int32, device=DEV), lens=lens)
    out, lse = c(err=err, lengths=lengths, lens=lens)
    assert int(err.item()) == 4 and torch.equal(out, want) and torch.equal(lse, want_lse)
    assert not out[i].any() and bool(torch.isneginf(lse[i]).all())


@pytest.mark.parametrize("form,d", KINDS)
def test_nan_reaches_its_own_heads_alone(P, form, d):
    """A NaN in a quarter of K, of V, in a query: all else to the bit as without it."""
    c = Call(P, form, d, 33)
    clean, clean_lse = c()
    assert not torch.isnan(clean).any()
    raw = c.cache.scales.view(torch.uint8)
    G = c.group
    for head in {0, 1, c.hkv - 1}:
        heads = slice(head * G, (head + 1) * G)
        for kv in (0, 1):
            for i, at, quarter in ((0, c.lens[0] - 7, 0), (c.S - 1, 0, 3), (0, 0, 2)):
                place = (1, kv, int(c.cache.table[i, at // 16]), at % 16, head, quarter)
                old = raw[place].item()
                raw[place] = 255
                out, lse = c()
                raw[place] = old
                bad = torch.zeros_like(out, dtype=torch.bool)
                if kv == 0:
                    bad[i, heads] = True
                else:
                    bad[i, heads, quarter * d // 4:(quarter + 1) * d // 4] = True
                assert torch.equal(torch.isnan(out), bad), (head, kv, i, quarter)
                assert torch.equal(out[~bad], clean[~bad])
                assert torch.equal(torch.isnan(lse), bad.all(dim=2)) and torch.equal(lse[~bad.all(dim=2)], clean_lse[~bad.all(dim=2)])
    q = c.q.clone()
    q[0, 1], q[-1, -1] = float("nan"), float("inf")
    out, lse = c(q)
    bad = torch.zeros((c.S, c.hq), dtype=torch.bool, device=DEV)
    bad[0, 1] = bad[-1, -1] = True
    assert torch.equal(torch.isnan(out).all(dim=2), bad) and torch.equal(out[~bad], clean[~bad])
    assert torch.equal(torch.isnan(lse), bad) and torch.equal(lse[~bad], clean_lse[~bad])


@pytest.mark.parametrize("form,d", KINDS)
def test_scales_that_overflow_stay_in_their_head(P, form, d):
    """A V quarter whose scale no store writes (2^126 and 2^127, values beyond bf16): its head's dimensions alone."""
    c = Call(P, form, d, 34)
    clean, _ = c()
    raw, codes = c.cache.scales.view(torch.uint8), c.cache.codes.view(torch.uint8)
    for head, byte in ((0, 254), (1, 253)):
        pg = int(c.cache.table[0, 2])
        old = raw[1, 1, pg, 3, head, 1].item(), codes[1, 1, pg, 3, head].clone()
        raw[1, 1, pg, 3, head, 1] = byte
        codes[1, 1, pg, 3, head, d // 8:d // 4] = 0x77
        out, _ = c()
        raw[1, 1, pg, 3, head, 1] = old[0]
        codes[1, 1, pg, 3, head] = old[1]
        bad = torch.zeros_like(out, dtype=torch.bool)
        bad[0, head * c.group:(head + 1) * c.group, d // 4:d // 2] = True
        assert not torch.isfinite(out[bad]).any() and torch.equal(out[~bad], clean[~bad])


@pytest.mark.parametrize("form,d", KINDS)
def test_strided_rows_that_do_not_depend_on_the_others(P, form, d):
    """q inside projection rows, out inside wider rows, nothing beside them written; whatever the other rows ask and
    hold, at the same lengths: to the bit."""
    c = Call(P, form, d, 35)
    want, want_lse = c()
    wide = torch.randn((c.S, (c.hq + 4) * d), device=DEV).to(torch.bfloat16)
    q = wide[:, 2 * d:(c.hq + 2) * d].view(c.S, c.hq, d)
    q.copy_(c.q)
    outs = torch.full((c.S + 2, (c.hq + 2) * d), 5.0, dtype=torch.bfloat16, device=DEV)
    out = outs[1:c.S + 1, d:(c.hq + 1) * d].view(c.S, c.hq, d)
    _, lse = c(q, out=out)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    out.fill_(5.0)
    assert bool((outs == 5.0).all())
    keep = [0, c.S - 1]
    bt = c.bt.clone()
    for i in range(c.S):
        if i not in keep:
            q[i] = float("nan") if i % 2 else 100.0
            bt[i, :-(-c.lens[i] // 32)] = -1
    out, lse = c(q, bt=bt)
    for i in keep:
        assert torch.equal(out[i], want[i]) and torch.equal(lse[i], want_lse[i])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("form,S,hkv,max_length", [("short", 64, 8, 512), ("split", 4, 8, 600), ("heads", 64, 7, 20000), ("pairs", 64, 8, 20000)])
def test_weights_that_cancel(P, form, S, hkv, max_length, d):
    """Weights keep their 24 bits on the way into the second product.  Two keys whose weighted values cancel: scores of
    single products of at most 0.55 (in log2 units 0.8), each off by the two roundings of its product and of the factor,
    2^-24 of 0.8 each, and their difference by one of 1.6: 2^-21.8, in the weight 2^-22.3; exp2 2^-23, two additions
    2^-24 each: below 2^-21 of sum p |v|, out 2^-8 of itself.  (Weights of 16 bits would be up to 2^-17 off.)"""
    rng = np.random.default_rng(d)
    pairs = [(a, b) for a in co.E2M1[1:] for b in co.E2M1[1:] if 1 < a / b <= 3]
    take = rng.integers(0, len(pairs), (S, hkv))
    a, b = np.array(pairs)[take].transpose(2, 0, 1)
    t = rng.choice(co.E2M1[1:], (S, hkv))
    scale = 0.125
    # exp(2 scale q t) = a / b but for q's rounding: 2^-9 of at most ln 3, half of it beside either weight
    q1 = torch.from_numpy(np.log(a / b) / (2 * scale * t)).to(torch.bfloat16)
    q = torch.zeros((S, hkv, d), dtype=torch.bfloat16)
    q[:, :, 1] = q1
    z = scale * to_np64(q1) * t
    p = np.stack([np.exp(z), np.exp(-z)])
    p /= p.sum(axis=0)
    up = rng.integers(-9, 10, (S, hkv, 4))                  # a power of two for each quarter of V
    code = {float(x): i for i, x in enumerate(co.E2M1)}
    of = np.vectorize(lambda x: code[float(x)])
    codes = np.full((1, 2, S, 16, hkv, d // 2), 0x77, dtype=np.uint8)
    scales = np.full((1, 2, S, 16, hkv, 4), 255, dtype=np.uint8)
    codes[0, 0, :, :2] = 0
    scales[0, 0, :, :2] = 127
    codes[0, 0, :, 0, :, 0], codes[0, 0, :, 1, :, 0] = of(t) << 4, (of(t) | 8) << 4
    codes[0, 1, :, 0] = (of(b) * 17)[..., None]
    codes[0, 1, :, 1] = ((of(a) | 8) * 17)[..., None]
    scales[0, 1, :, :2] = (127 + up)[:, None]
    v = np.ldexp(np.stack([b, -a])[..., None], up).repeat(d // 4, axis=-1)
    table = torch.arange(S, dtype=torch.int32, device=DEV)[:, None].repeat(1, -(-max_length // 16)).contiguous()
    lengths = torch.full((S,), 2, dtype=torch.int32, device=DEV)
    ws = torch.full((P.pallas_attend_workspace_size(S, hkv, hkv, d, max_length),), 0xFF, dtype=torch.uint8, device=DEV)
    q = q.to(DEV)
    out = torch.empty_like(q)
    P.pallas_attend_quant(torch.from_numpy(codes).to(DEV).view(torch.float4_e2m1fn_x2), torch.from_numpy(scales).to(DEV).view(torch.float8_e8m0fnu),
                          0, q, lengths, max_length, table, scale, out, ws)
    check_form(form, ws, hkv, 1, [2] * S, max_length)
    ref, mag = (p[..., None] * v).sum(axis=0), (p[..., None] * np.abs(v)).sum(axis=0)
    assert np.all(np.abs(ref) <= 2.0 ** -9 * mag)
    worst = (np.abs(to_np64(out) - ref) - 2.0 ** -8 * np.abs(ref)) / mag
    assert worst.max() <= 2.0 ** -20, float(np.log2(worst.max()))


def check_on_gpu(codes, scales, bt, q, lens, scale, out, lse, step):
    """Against torch in float64, every `step`th KV head of each row."""
    table = torch.from_numpy(np.concatenate([co.E2M1, -co.E2M1])).to(DEV)
    group, d = q.shape[1] // codes.shape[4], q.shape[2]

    def values(kv, pg, slot, h):
        c = codes.view(torch.uint8)[0, kv, pg, slot, h].long()
        unit = torch.exp2(scales.view(torch.uint8)[0, kv, pg, slot, h].double() - 127)
        return torch.stack([table[c & 15], table[c >> 4]], dim=-1).view(len(c), d) * unit.repeat_interleave(d // 4, dim=1)

    for i, n in enumerate(lens):
        if n == 0:
            assert not out[i].any() and bool(torch.isneginf(lse[i]).all())
            continue
        t = torch.arange(n, device=DEV)
        pg, slot = bt[i].long()[t // 16], t % 16
        for h in range(0, codes.shape[4], step):
            k, v = (values(kv, pg, slot, h) for kv in (0, 1))
            for j in range(h * group, (h + 1) * group):
                qd = q[i, j].double()
                z = (k * qd).sum(1) * scale
                rl = torch.logsumexp(z, 0)
                p = torch.exp(z - rl)[:, None]
                ref, mag = (p * v).sum(0), (p * v.abs()).sum(0)
                delta = (d + 8) * 2.0 ** -24 * float(((k * qd).abs().sum(1) * scale).max())
                assert bool(((out[i, j].double() - ref).abs() <= 2.0 ** -8 * ref.abs() + (2 * delta + 2.0 ** -12) * mag).all()), (i, j, n)
                assert abs(float(lse[i, j]) - float(rl)) <= delta + 2.0 ** -12, (i, j, n)


def random_pool(pages, hkv, d, seed):
    g = torch.Generator(DEV).manual_seed(seed)
    codes = torch.randint(0, 256, (1, 2, pages, 16, hkv, d // 2), dtype=torch.uint8, device=DEV, generator=g)
    scales = torch.randint(122, 128, (1, 2, pages, 16, hkv, 4), dtype=torch.uint8, device=DEV, generator=g)
    return codes.view(torch.float4_e2m1fn_x2), scales.view(torch.float8_e8m0fnu)


@pytest.mark.parametrize("d,hkv,group,n", [(128, 16, 1, 300000), (64, 16, 2, 300000), (64, 17, 1, 150000)])
def test_more_blocks_than_one_round(P, d, hkv, group, n):
    """Ranges at their longest, several of them a workgroup."""
    lens = [n, 0, 777, n // 2]
    pages = -(-n // 16)
    assert range_blocks(hkv, group, lens) > (64 if hkv % 2 == 0 else 16)
    assert sum(map(blocks, lens)) > (128 * 96 if hkv % 2 == 0 else 32 * 176)
    rng = np.random.default_rng(3)
    bt = np.full((4, pages), -1, dtype=np.int32)
    for i, x in enumerate(lens):       # the rows share the pool's pages
        bt[i, :-(-x // 16)] = rng.permutation(pages + 50)[:-(-x // 16)]
    bt = torch.from_numpy(bt).to(DEV)
    codes, scales = random_pool(pages + 50, hkv, d, 1)
    q = queries(4, hkv * group, d, 4)
    out, lse = torch.empty_like(q), torch.empty((4, hkv * group), device=DEV)
    ws = torch.empty(P.pallas_attend_workspace_size(4, hkv * group, hkv, d, n), dtype=torch.uint8, device=DEV)
    P.pallas_attend_quant(codes, scales, 0, q, torch.tensor(lens, dtype=torch.int32, device=DEV), n, bt, 0.1, out, ws, lse=lse)
    check_on_gpu(codes, scales, bt, q, lens, 0.1, out, lse, 5)


@pytest.mark.parametrize("hkv,group", [(2, 2), (3, 2)])
def test_thousands_of_rows(P, hkv, group):
    """Most of them short or empty, some long, in ranges."""
    rng = np.random.default_rng(5)
    lens = rng.integers(0, 70, 3000) * (rng.random(3000) < 0.4)
    lens[[0, 700, 1500, 2999]] = 600, 1, 900, 33
    cache = Cache(hkv, 64, lens.tolist(), seed=12)
    q = queries(3000, hkv * group, 64, seed=13)
    lse = torch.empty((3000, hkv * group), device=DEV)
    ws = torch.full((P.pallas_attend_workspace_size(3000, hkv * group, hkv, 64, 900),), 0xFF, dtype=torch.uint8, device=DEV)
    out = cache.attend(P, q, 0.12, lse=lse, ws=ws)
    check_form("ranges", ws, hkv, group, cache.lens, 900)
    check(cache, q, 0.12, out, lse)


@pytest.mark.parametrize("form", ["split", "heads", "pairs-4"])
def test_replays_and_shared_workspaces(P, form):
    """Two graphs over one workspace, replayed in turn with eager calls between them and over changing lengths."""
    calls = [Call(P, form, 128, seed) for seed in (36, 37)]
    ws, lengths = calls[0].workspace(), calls[0].cache.lengths.clone()
    outs = [torch.empty_like(c.q) for c in calls]

    def run(c, out, ws):
        P.pallas_attend_quant(c.cache.codes, c.cache.scales, 1, c.q, lengths, c.max_length, c.bt, 0.09, out, ws)

    graphs = []
    for c, out in zip(calls, outs):
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=stream):
            run(c, out, ws)
        torch.cuda.current_stream().wait_stream(stream)
        graphs.append(graph)
    for cut in (1.0, 0.3, 0.0, 0.7, 1.0):
        lengths.copy_((calls[0].cache.lengths.double() * cut).to(torch.int32))
        for c, out, graph in zip(calls, outs, graphs):
            out.fill_(7.0)
            graph.replay()
            own = torch.empty_like(out)
            run(calls[0], own, ws)              # the same workspace, in order
            run(c, own, c.workspace())
            torch.cuda.synchronize()
            assert torch.equal(out, own), (form, cut)
