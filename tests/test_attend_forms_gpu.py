"""What attention of one new token promises beside plain accuracy, in each of the ways in
which it is run (attend_forms.FORMS; which one a call took is read back from its
workspace): masked pages, lengths outside the bound, steep scores, strided rows, rows that
do not depend on the others, NaN, parts joined through lse, planes of more than 4 GiB.

Tolerances: those of test_attend_gpu (`check`)."""
import functools

import numpy as np
import pytest
import torch

from attend_forms import FORMS, blocks_per_range, check_form, fresh_workspace
from helpers import ensure_lib
from test_attend_gpu import DEV, TYPES, Cache, check, queries

pytestmark = pytest.mark.gpu
D, GROUP = 128, 3
KINDS = [pytest.param(form, fmt, id=f"{form}-{fmt}") for form in FORMS for fmt in ("bf16", "e4m3", "int8")]


@pytest.fixture(scope="module")
def P():
    return ensure_lib()


@functools.lru_cache(maxsize=None)
def cache_of(form, fmt):
    hkv, lens, _, _ = FORMS[form]
    return Cache(fmt, hkv, D, lens, seed=21)


class Call:
    """A cache of a form's lengths (one for all tests, which leave it as it was), and calls of that form over it."""

    def __init__(self, P, form, fmt, seed):
        self.P, self.form, self.fmt = P, form, fmt
        self.hkv, self.lens, self.max_length, each = FORMS[form]
        self.S, self.hq = len(self.lens), GROUP * self.hkv
        self.cache = cache_of(form, fmt)
        self.bt = torch.full((self.S, -(-self.max_length // 16)), -1, dtype=torch.int32, device=DEV)
        self.bt[:, :self.cache.max_pages] = self.cache.bt
        self.q = queries(self.S, self.hq, D, seed + 1)
        if each is not None:
            got = blocks_per_range(fmt, D, self.hq, self.hkv, self.lens)
            assert got == each or (each > 2 and got > 2)

    def __call__(self, q=None, scale=0.09, lens=None, **kw):
        """(out, lse); `lens`: the lengths as the call cuts them (None: not looked at)."""
        q = self.q if q is None else q
        lse = torch.full((self.S, self.hq), 9.0, dtype=torch.float32, device=DEV)
        ws = fresh_workspace(self.P, self.S, self.hq, self.hkv, D, self.max_length)
        kw.setdefault("bt", self.bt)
        out = self.cache.attend(self.P, q, scale, lse=lse, max_length=self.max_length, ws=ws, **kw)
        if lens is not None:
            check_form(self.form, ws, self.fmt, D, self.hq, self.hkv, lens, self.max_length)
        return out, lse

    def check(self, out, lse, q=None, scale=0.09, drop=None):
        check(self.cache, self.q if q is None else q, scale, out, lse, drop)


@pytest.mark.parametrize("form,fmt", KINDS)
def test_pages_outside_the_pool(P, form, fmt):
    """Keys on such pages are masked and raise the flag; a row of them alone counts as empty."""
    c = Call(P, form, fmt, 21)
    pages = c.cache.pool.shape[2] if fmt == "bf16" else c.cache.codes.shape[2]
    bt, drop = c.bt.cpu().numpy().copy(), {}
    rng = np.random.default_rng(1)
    for i, n in enumerate(c.lens):
        have = -(-n // 16)
        gone = np.arange(have) if n == 33 else np.unique(np.concatenate([[0, have - 1], rng.integers(0, have, have // 5)])) if have > 3 else []
        for m, p in enumerate(gone):
            bt[i, p] = (-1, pages, 2 ** 31 - 1, -2 ** 31)[m % 4]
        drop[i] = np.concatenate([np.arange(16 * p, 16 * p + 16) for p in gone] or [np.zeros(0, int)])
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    out, lse = c(err=err, bt=torch.from_numpy(bt).to(DEV), lens=c.lens)
    assert int(err.item()) == 1
    c.check(out, lse, drop=drop)
    assert not out[c.lens.index(33)].any()
    # one bad page in the whole call, at the end of its longest row
    bt = c.bt.clone()
    i = int(np.argmax(c.lens))
    last = -(-c.lens[i] // 16) - 1
    bt[i, last] = pages
    err.zero_()
    out, lse = c(err=err, bt=bt, lens=c.lens)
    assert int(err.item()) == 1
    c.check(out, lse, drop={i: np.arange(16 * last, 16 * last + 16)})
    err.zero_()
    c(err=err)
    assert int(err.item()) == 0


@pytest.mark.parametrize("form,fmt", KINDS)
def test_lengths_outside_the_bound(P, form, fmt):
    """Cut, and flagged: below zero in a row of its own, above where the longest row has all of max_length."""
    c = Call(P, form, fmt, 22)
    lens = list(c.lens)
    i = lens.index(33) if 33 in lens else 0
    for j, bad in [(i, -3), (i, -2 ** 31)] + ([(lens.index(c.max_length), 2 ** 31 - 1)] if c.max_length in lens else []):
        lengths, cut = c.cache.lengths.clone(), list(lens)
        lengths[j] = bad
        cut[j] = min(max(bad, 0), c.max_length)
        err = torch.zeros(1, dtype=torch.int32, device=DEV)
        out, lse = c(err=err, lengths=lengths, lens=cut)
        assert int(err.item()) == 4
        full = c.cache.k[j], c.cache.v[j]
        c.cache.lens[j] = cut[j]
        c.cache.k[j], c.cache.v[j] = full[0][:cut[j]], full[1][:cut[j]]
        c.check(out, lse)
        c.cache.lens[j], c.cache.k[j], c.cache.v[j] = lens[j], *full


@pytest.mark.parametrize("form,fmt", KINDS)
def test_steep_scores(P, form, fmt):
    """Scores of hundreds: maxima move by more than the exponent's range within a part and between parts."""
    c = Call(P, form, fmt, 23)
    q = c.q * 160
    for scale in (1.0, -1.0, 0.0):
        out, lse = c(q, scale, lens=c.lens)
        c.check(out, lse, q, scale)


@pytest.mark.parametrize("form,fmt", KINDS)
def test_strided_rows(P, form, fmt):
    """q inside projection rows, out inside wider rows; nothing beside them is written."""
    c = Call(P, form, fmt, 24)
    wide = torch.randn((c.S, (c.hq + 4) * D), device=DEV).to(torch.bfloat16)
    q = wide[:, 2 * D:(c.hq + 2) * D].view(c.S, c.hq, D)
    outs = torch.full((c.S + 2, (c.hq + 2) * D), 5.0, dtype=torch.bfloat16, device=DEV)
    out = outs[1:c.S + 1, D:(c.hq + 1) * D].view(c.S, c.hq, D)
    _, lse = c(q, out=out, lens=c.lens)
    c.check(out, lse, q)
    rest = outs.clone()
    rest[1:c.S + 1, D:(c.hq + 1) * D] = 5.0
    assert bool((rest == 5.0).all())


@pytest.mark.parametrize("form,fmt", KINDS)
def test_a_row_does_not_depend_on_the_others(P, form, fmt):
    """Whatever the others ask and hold, at the same lengths: to the bit."""
    c = Call(P, form, fmt, 25)
    out, lse = c(lens=c.lens)
    keep = [0, c.S - 1]
    q2, bt = c.q.clone(), c.bt.clone()
    for i in range(c.S):
        if i not in keep:
            q2[i] = float("nan") if i % 2 else 100.0
            bt[i, :-(-c.lens[i] // 32)] = -1
    out2, lse2 = c(q2, bt=bt, lens=c.lens)
    for i in keep:
        assert torch.equal(out[i], out2[i]) and torch.equal(lse[i], lse2[i])
    assert not torch.equal(out[1:-1], out2[1:-1])


@pytest.mark.parametrize("form,fmt", KINDS)
def test_nan_reaches_its_own_heads_alone(P, form, fmt):
    """A NaN in K, in V, in a query; rows of nothing but NaN, whole and in parts."""
    c = Call(P, form, fmt, 26)
    where = [(0, c.lens[0] - 7), (c.S - 1, 0)]            # the end of the first row, the start of the last
    for kv in (0, 1):
        for i, at in where:
            pg, slot = int(c.cache.table[i, at // 16]), at % 16
            hold = c.cache.pool if fmt == "bf16" else c.cache.scales
            place = (1, kv, pg, slot, 1, 5) if fmt == "bf16" else (1, kv, pg, slot, 1)
            old = hold[place].item()
            hold[place] = float("nan")
            out, lse = c(lens=c.lens)
            hold[place] = old
            bad = torch.zeros_like(out, dtype=torch.bool)
            heads = slice(GROUP, 2 * GROUP)
            if kv == 0 or fmt != "bf16":
                bad[i, heads] = True
            else:
                bad[i, heads, 5] = True
            assert torch.equal(torch.isnan(out), bad)
            assert torch.equal(torch.isnan(lse), bad.all(dim=2) & (kv == 0))
            assert bool((torch.isneginf(lse) == (torch.tensor(c.lens, device=DEV) == 0)[:, None]).all())
    q = c.q.clone()
    q[0], q[c.S - 1, 1] = float("nan"), float("inf")
    out, lse = c(q, lens=c.lens)
    assert bool(torch.isnan(out[0]).all()) and bool(torch.isnan(lse[0]).all())
    assert bool(torch.isnan(out[-1, 1]).all()) and bool(torch.isnan(lse[-1, 1]).all())
    q[0], q[c.S - 1, 1] = c.q[0], c.q[-1, 1]
    fine, fine_lse = c(q, lens=c.lens)
    out[0], out[-1, 1], lse[0], lse[-1, 1] = fine[0], fine[-1, 1], fine_lse[0], fine_lse[-1, 1]
    assert torch.equal(out, fine) and torch.equal(lse, fine_lse)


@pytest.mark.parametrize("form,fmt", KINDS)
def test_parts_join_through_lse(P, form, fmt):
    """Attention over a cache's two halves, joined, is attention over all of it."""
    c = Call(P, form, fmt, 27)
    rows = [i for i, n in enumerate(c.lens) if n > 16]
    half = torch.tensor([n // 32 * 16 if n > 16 else n for n in c.lens], dtype=torch.int32, device=DEV)
    rolled = c.bt.clone()
    for i in rows:
        h = int(half[i]) // 16
        rolled[i] = torch.cat([c.bt[i, h:], c.bt[i, :h]])
    whole, lw = c(lens=c.lens)
    a, la = c(lengths=half)
    b, lb = c(lengths=c.cache.lengths - half, bt=rolled)
    both = torch.logaddexp(la, lb)
    wa, wb = (torch.exp(x - both)[rows, :, None] for x in (la, lb))
    whole, a, b = (x[rows].float() for x in (whole, a, b))
    # each part and the whole round to bf16 once; float32 sums as in `check`, here below 2^-12 for each of parts
    # and whole, and the weights of the parts
    tol = 2.0 ** -8 * (whole.abs() + wa * a.abs() + wb * b.abs()) + 2.0 ** -10
    assert bool(((wa * a + wb * b - whole).abs() <= tol).all())
    assert bool(((both - lw)[rows].abs() <= 2.0 ** -11).all())


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
def test_ranges_over_planes_of_more_than_4_gib(P, fmt):
    """Pages at the end of the planes."""
    hkv, lens, max_length = 8, [600, 33, 1100], 20000
    cache = Cache(fmt, hkv, D, lens, seed=28)
    small = cache.pool if fmt == "bf16" else cache.codes.view(torch.uint8)
    held = small.shape[2]
    pages = (1 << 32) // (16 * hkv * D * (2 if fmt == "bf16" else 1)) + 500
    big = torch.empty((1, 2, pages, 16, hkv, D), dtype=small.dtype, device=DEV)
    big[0, :, pages - held:] = small[1]
    bt = torch.full((3, max_length // 16), -1, dtype=torch.int32, device=DEV)
    bt[:, :cache.max_pages] = torch.where(cache.bt >= 0, cache.bt + (pages - held), cache.bt)
    q = queries(3, 16, D, 9)
    out, lse = torch.empty_like(q), torch.empty((3, 16), dtype=torch.float32, device=DEV)
    ws = fresh_workspace(P, 3, 16, hkv, D, max_length)
    if fmt == "bf16":
        P.pallas_attend_kv(big, 0, q, cache.lengths, max_length, bt, 0.09, out, ws, lse=lse)
    else:
        scales = torch.empty((1, 2, pages, 16, hkv), dtype=torch.float32, device=DEV)
        scales[0, :, pages - held:] = cache.scales[1]
        P.pallas_attend_quant(big.view(TYPES[fmt]), scales, 0, q, cache.lengths, max_length, bt, 0.09, out, ws, lse=lse)
    check_form("ranges", ws, fmt, D, 16, hkv, lens, max_length)
    check(cache, q, 0.09, out, lse)


ALONE = [1, 15, 16, 17, 32, 33, 64, 65, 500, 1000, 1024, 1025, 4000, 8000, 8192]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
def test_one_short_row_under_a_large_bound(P, fmt, d):
    """A captured graph's capacity far above the row's length: ranges of one and of two blocks, whose pages are
    read before the length is known."""
    hkv, hq, max_length = 8, 16, 40000
    cache = Cache(fmt, hkv, d, [max(ALONE)], seed=29)
    pages = cache.pool.shape[2] if fmt == "bf16" else cache.codes.shape[2]
    bt = torch.full((1, max_length // 16), -1, dtype=torch.int32, device=DEV)
    bt[:, :cache.max_pages] = cache.bt
    q, k, v, seen = queries(1, hq, d, 30), cache.k[0], cache.v[0], set()
    for n in ALONE:
        for bad in (False, True):
            lens, lse, ws = [n], torch.empty((1, hq), device=DEV), fresh_workspace(P, 1, hq, hkv, d, max_length)
            err, table, drop = torch.zeros(1, dtype=torch.int32, device=DEV), bt, None
            if bad:
                gone = list(range(0, -(-n // 16), 3))
                table, drop = bt.clone(), {0: np.concatenate([np.arange(16 * p, 16 * p + 16) for p in gone])}
                table[0, gone] = pages
            out = cache.attend(P, q, 0.1, lse=lse, max_length=max_length, ws=ws, bt=table, err=err,
                               lengths=torch.tensor(lens, dtype=torch.int32, device=DEV))
            check_form("ranges", ws, fmt, d, hq, hkv, lens, max_length)
            cache.lens, cache.k, cache.v = lens, [k[:n]], [v[:n]]
            check(cache, q, 0.1, out, lse, drop)
            assert int(err.item()) == int(bad)
            seen.add(blocks_per_range(fmt, d, hq, hkv, lens))
    assert seen == {1, 2}
