"""Host side of the cache operators: rotary plans against the oracle, workspace
sizes, and refusals, which come before anything is enqueued (every pointer here is
one that no call may touch).  No GPU needed."""
import ctypes as C
import itertools
import math

import numpy as np
import pytest
import torch

from helpers import ensure_lib
from oracle import cache_ops as co
from paper_2608_16477_amd.binding import KVPoolC, QuantPoolC, RopeConfigC, RopePlan

FAKE = 0x10000


@pytest.fixture(scope="module")
def P():
    return ensure_lib()


# ------------------------------------------------------------------ rotary plans
PLANS = [dict(), dict(scaling="linear", factor=4.0), dict(scaling="ntk", factor=8.0),
         dict(scaling="yarn", factor=8.0, trained_len=4096, fast=32.0, slow=1.0),
         dict(scaling="yarn", factor=2.0, trained_len=2, fast=32.0, slow=1.0, magnitude=0.7),
         dict(scaling="bands", factor=8.0, trained_len=8192, fast=4.0, slow=1.0)]


@pytest.mark.parametrize("kw", PLANS)
@pytest.mark.parametrize("r,theta", [(2, 1e4), (54, 5e5), (128, 1e6), (256, 1e4)])
def test_plan_frequencies(P, kw, r, theta):
    plan = P.pallas_rope_init(r, theta, "interleaved", **kw)
    f, m = co.rope_frequencies(r, theta, **{"scaling": "none", **kw})
    got = np.array(plan.turns[: r // 2], dtype=np.float64) * 2.0 ** -64 * 2 * math.pi
    assert np.all(np.abs(got - f) <= 1e-13 * f + 2.0 ** -61)     # the oracle's own 53-bit powers
    assert plan.magnitude == np.float32(m) and plan.layout == 1 and plan.rotary_dim == r
    assert not any(plan.turns[r // 2:])


def test_plan_first_pair_is_a_radian(P):
    turns = P.pallas_rope_init(64, 1e4).turns[0]
    assert abs(turns - 2935890503282001226) <= 1                # 2^64 / (2 pi)


GOOD = dict(rotary_dim=64, layout=0, scaling=0, trained_len=0, theta=1e4, factor=1.0, fast=0.0, slow=0.0, magnitude=0.0)


@pytest.mark.parametrize("bad", [
    dict(rotary_dim=0), dict(rotary_dim=63), dict(rotary_dim=258), dict(layout=2), dict(layout=-1), dict(scaling=5),
    dict(scaling=-1), dict(theta=1.0), dict(theta=math.nan), dict(theta=math.inf), dict(scaling=1, factor=0.5),
    dict(scaling=2, factor=math.nan), dict(scaling=3, factor=2.0, fast=32.0, slow=1.0),
    dict(scaling=3, factor=2.0, trained_len=10, fast=1.0, slow=1.0), dict(scaling=4, factor=2.0, trained_len=10, fast=4.0),
    dict(scaling=4, factor=math.inf, trained_len=10, fast=4.0, slow=1.0), dict(magnitude=-1.0), dict(magnitude=math.nan)])
def test_plan_refusals(P, bad):
    cfg, plan = RopeConfigC(**{**GOOD, **bad}), RopePlan()
    plan.rotary_dim = 77
    assert P.lib().pallas_rope_init(C.byref(cfg), C.byref(plan)) == P.Status.INVALID_ARG
    assert plan.rotary_dim == 77 and "rope" in P.pallas_last_error()
    assert P.lib().pallas_rope_init(None, C.byref(plan)) == P.Status.INVALID_ARG


ROPE = dict(plan=None, inverse=0, tokens=4, heads=2, d=64, pos=FAKE, x=FAKE, xt=128, xh=64, y=FAKE * 2, yt=128, yh=64)


def rope_rc(P, **kw):
    a = {**ROPE, **kw}
    if a["plan"] is None:
        a["plan"] = P.pallas_rope_init(64, 1e4)
    return P.Status(P.lib().pallas_rope_apply(
        None if a["plan"] == 0 else C.byref(a["plan"]), a["inverse"], a["tokens"], a["heads"], a["d"], a["pos"], a["x"],
        a["xt"], a["xh"], a["y"], a["yt"], a["yh"], None))


@pytest.mark.parametrize("bad", [
    dict(plan=0), dict(plan=RopePlan()), dict(tokens=-1), dict(heads=0), dict(d=62), dict(pos=None), dict(x=None),
    dict(y=None), dict(x=FAKE + 1), dict(y=FAKE + 1), dict(pos=FAKE + 2), dict(xt=-1), dict(yh=-64), dict(yt=63),
    dict(yh=32), dict(yt=0), dict(x=FAKE, y=FAKE, yt=256)])
def test_rope_refusals(P, bad):
    assert rope_rc(P, **bad) == P.Status.INVALID_ARG
    assert "rope" in P.pallas_last_error()


def test_rope_limits(P):
    assert rope_rc(P, heads=(1 << 14) + 1) == P.Status.UNSUPPORTED
    assert rope_rc(P, tokens=1 << 24) == P.Status.UNSUPPORTED
    assert rope_rc(P, tokens=0) == P.Status.OK           # nothing to do: nothing is touched


@pytest.mark.parametrize("tokens,heads,yt,yh,ok", [
    (4, 2, 128, 64, True), (4, 2, 64, 256, True),            # heads of a token side by side, tokens of a head
    (4, 2, 127, 64, False), (4, 2, 64, 255, False), (4, 2, 64, 64, False), (4, 3, 96, 64, False),
    (1, 2, 0, 64, True), (4, 1, 64, 0, True), (1, 2, 0, 63, False), (2, 1, 63, 0, False),
    (2, 2, 1 << 62, 1 << 61, True), (4, 1 << 14, 1 << 20, 64, True), (4, 1 << 14, (1 << 20) - 1, 64, False)])
def test_rope_output_heads_do_not_overlap(P, tokens, heads, yt, yh, ok):
    """Strides that pass are refused by the next check (in place with other strides), so that nothing is enqueued."""
    at = sorted(t * yt + h * yh for t in range(tokens) for h in range(heads))
    assert all(b - a >= 64 for a, b in zip(at, at[1:])) == ok
    assert rope_rc(P, tokens=tokens, heads=heads, x=FAKE, y=FAKE, yt=yt, yh=yh, xt=yt + 8, xh=yh + 8) == P.Status.INVALID_ARG
    assert ("in place" if ok else "overlap") in P.pallas_last_error()


@pytest.mark.parametrize("m", [1e-300, 2.0 ** -127, 2.0 ** 127, 1e300])
def test_plan_magnitude_has_a_reciprocal(P, m):
    cfg, plan = RopeConfigC(**{**GOOD, "magnitude": m}), RopePlan()
    assert P.lib().pallas_rope_init(C.byref(cfg), C.byref(plan)) == P.Status.INVALID_ARG
    for fine in (2.0 ** -126, 2.0 ** 126):
        assert P.pallas_rope_init(64, 1e4, magnitude=fine).magnitude == fine


# ------------------------------------------------------------------ 8-bit pool
def quant_pool(**kw):
    a = dict(codes=FAKE, scales=FAKE, num_pages=8, page_size=16, n_layers=2, n_kv_heads=4, head_dim=64, format=1)
    return QuantPoolC(**{**a, **kw})


QUANT = dict(layer=1, tokens=3, seq=FAKE, pos=FAKE, k=FAKE, ks=256, v=FAKE, vs=256, seqs=2, bt=FAKE, max_pages=4)


def quant_rc(P, name, pool=None, **kw):
    a = {**QUANT, **kw}
    pool = quant_pool() if pool is None else pool
    return P.Status(getattr(P.lib(), name)(
        None if pool == 0 else C.byref(pool), a["layer"], a["tokens"], a["seq"], a["pos"], a["k"], a["ks"], a["v"],
        a["vs"], a["seqs"], a["bt"], a["max_pages"], None, None))


@pytest.mark.parametrize("name", ["pallas_quant_store", "pallas_quant_load"])
def test_quant_refusals(P, name):
    S = P.Status
    for bad in (dict(tokens=-1), dict(seqs=0), dict(max_pages=0), dict(pos=None), dict(k=None), dict(v=None),
                dict(bt=None), dict(seq=None), dict(k=FAKE + 8), dict(v=FAKE + 2), dict(ks=260), dict(vs=252),
                dict(ks=248), dict(vs=0), dict(ks=-256)):
        assert quant_rc(P, name, **bad) == S.INVALID_ARG, bad
        assert name[7:].replace("_", " ") in P.pallas_last_error()
    for bad in (dict(layer=2), dict(layer=-1)):
        assert quant_rc(P, name, **bad) == S.OUT_OF_RANGE, bad
    for bad in (dict(codes=None), dict(scales=None), dict(codes=FAKE + 8), dict(scales=FAKE + 4), dict(num_pages=0),
                dict(n_kv_heads=0), dict(head_dim=-64), dict(format=0), dict(format=3)):
        assert quant_rc(P, name, quant_pool(**bad)) == S.INVALID_ARG, bad
    for bad in (dict(head_dim=96), dict(head_dim=256), dict(page_size=32), dict(n_kv_heads=4097)):
        assert quant_rc(P, name, quant_pool(**bad)) == S.UNSUPPORTED, bad
    assert quant_rc(P, name, pool=0) == S.INVALID_ARG
    assert quant_rc(P, name, tokens=1 << 26) == S.UNSUPPORTED          # 2^35 elements
    for bad in (dict(seq=FAKE + 2), dict(pos=FAKE + 1), dict(bt=FAKE + 2)):
        assert quant_rc(P, name, **bad) == S.INVALID_ARG, bad
    assert quant_rc(P, name, tokens=0) == S.OK           # nothing to do


# ------------------------------------------------------------------ attention
ATTEND = dict(layer=0, seqs=3, heads=8, q=FAKE, qs=512, lens=FAKE, max_length=64, bt=FAKE, max_pages=4, scale=0.125,
              out=FAKE, os=512, lse=None, ws=FAKE, ws_bytes=1 << 40)


def attend_rc(P, quant, pool=None, **kw):
    a = {**ATTEND, **kw}
    if pool is None:
        pool = quant_pool() if quant else KVPoolC(FAKE, 8, 16, 2, 4, 64)
    fn = P.lib().pallas_attend_quant if quant else P.lib().pallas_attend_kv
    return P.Status(fn(None if pool == 0 else C.byref(pool), a["layer"], a["seqs"], a["heads"], a["q"], a["qs"], a["lens"],
                       a["max_length"], a["bt"], a["max_pages"], a["scale"], a["out"], a["os"], a["lse"], a["ws"],
                       a["ws_bytes"], None, None))


@pytest.mark.parametrize("quant", [False, True])
def test_attend_refusals(P, quant):
    S = P.Status
    for bad in (dict(seqs=0), dict(heads=0), dict(heads=6), dict(max_length=0), dict(q=None), dict(lens=None),
                dict(bt=None), dict(out=None), dict(max_pages=0), dict(q=FAKE + 8), dict(out=FAKE + 4), dict(qs=516),
                dict(os=508), dict(qs=504), dict(os=0), dict(scale=math.inf), dict(scale=math.nan), dict(scale=3e38), dict(ws=None),
                dict(ws=FAKE + 16), dict(lens=FAKE + 2), dict(lse=FAKE + 1)):
        assert attend_rc(P, quant, **bad) == S.INVALID_ARG, bad
        assert "attend" in P.pallas_last_error()
    for bad in (dict(layer=2), dict(layer=-1), dict(max_length=65)):
        assert attend_rc(P, quant, **bad) == S.OUT_OF_RANGE, bad
    for bad in (dict(seqs=65536), dict(heads=8192, qs=1 << 20, os=1 << 20), dict(seqs=65535, max_length=(1 << 20), max_pages=1 << 16)):
        assert attend_rc(P, quant, **bad) == S.UNSUPPORTED, bad
    assert attend_rc(P, quant, pool=0) == S.INVALID_ARG
    pools = [quant_pool(head_dim=96), quant_pool(page_size=8)] if quant else [
        KVPoolC(FAKE, 8, 16, 2, 4, 96), KVPoolC(FAKE, 8, 32, 2, 4, 64), KVPoolC(FAKE, 8, 16, 2, 4, 256)]
    for pool in pools:
        assert attend_rc(P, quant, pool, qs=4096, os=4096) == S.UNSUPPORTED
    if quant:      # a layer's scales, 2 * 16 * 4 * 4 bytes a page, from 4 GiB on
        assert attend_rc(P, quant, quant_pool(num_pages=1 << 23)) == S.UNSUPPORTED
        assert "4 GiB" in P.pallas_last_error()
        assert attend_rc(P, quant, quant_pool(num_pages=(1 << 23) - 1), ws_bytes=0) == S.WORKSPACE
    need = P.pallas_attend_workspace_size(3, 8, 4, 64, 64)
    assert attend_rc(P, quant, ws_bytes=need - 1) == S.WORKSPACE
    assert attend_rc(P, quant, ws_bytes=0) == S.WORKSPACE


def test_attend_workspace(P):
    size = P.pallas_attend_workspace_size
    for bad in ((0, 8, 4, 64, 1), (1, 6, 4, 64, 1), (1, 8, 4, 96, 1), (1, 8, 4, 64, 0), (65536, 8, 4, 64, 1)):
        assert size(*bad) == 0
    # Enough for fewer sequences and shorter ones.
    lens = [1, 127, 128, 129, 1000, 1024, 1025, 5000, 16384, 131072, 1 << 20]
    seqs = [1, 2, 3, 5, 7, 8, 31, 32, 33, 64, 100, 128, 129, 1000]
    for hq, hkv, d in ((64, 8, 128), (8, 8, 64), (40, 2, 64)):
        b = np.array([[size(s, hq, hkv, d, n) for n in lens] for s in seqs], dtype=np.int64)
        assert (b > 0).all() and (b % 256 == 0).all()
        assert (np.diff(b, axis=0) >= 0).all() and (np.diff(b, axis=1) >= 0).all()
    # Records of any lengths fit: (range, sequence) pairs of every division (the rule, restated, with each
    # cache type's number of ranges).
    rng = np.random.default_rng(0)
    for d, hq, hkv in ((128, 64, 8), (64, 8, 8), (128, 40, 1), (64, 4, 2), (128, 4096, 4096)):
        for row_bytes in (d, 2 * d):
            ranges = 256 * (1024 // row_bytes) // (hkv * -(-(hq // hkv) // 16))
            ranges = max(ranges // 8 * 8, 8)
            for s, n in itertools.product((1, 2, 5, 64, 200), (1, 31, 64, 1000, 40000, 1 << 20)):
                for _ in range(3):
                    blocks = -(-rng.integers(0, n + 1, s) // 32)
                    blocks[rng.integers(s)] = -(-n // 32)
                    total = int(blocks.sum())
                    rounds = max(-(-total // (32 * ranges)), 1)
                    each = 1 if 2 * total <= ranges and total <= 32 * s else 2 if total <= 2 * ranges else -(-total // (ranges * rounds))
                    assert each <= 32
                    last = -(-total // each) - 1 + s - 1                # the largest range + sequence
                    assert size(s, hq, hkv, d, n) >= 8 * s + (last + 1) * hq * (d + 2) * 4
                heads, waves = hkv * -(-(hq // hkv) // 16), min(1024 // row_bytes, 8)
                for each in (1, 2):                                     # splits of one or two blocks a wave
                    splits = -(-(-(-n // 32)) // (waves * each))
                    if s * heads * splits <= 256:
                        assert size(s, hq, hkv, d, n) >= 8 * s + s * splits * hq * (d + 2) * 4


# ------------------------------------------------------------------ binding
def test_binding_refuses_what_the_kernels_cannot_take(P):
    x = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    pos = torch.zeros(4, dtype=torch.int32)
    plan = P.pallas_rope_init(64, 1e4)
    codes = torch.zeros((1, 2, 3, 16, 2, 64), dtype=torch.int8)
    scales = torch.zeros((1, 2, 3, 16, 2))
    bt = torch.zeros((4, 3), dtype=torch.int32)
    pool = torch.zeros((1, 2, 3, 16, 2, 64), dtype=torch.bfloat16)
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    calls = [
        lambda: P.pallas_rope_apply(plan, x, pos),                       # host tensors
        lambda: P.pallas_rope_apply(plan, x.float(), pos),
        lambda: P.pallas_rope_apply(plan, x.transpose(1, 2), pos),
        lambda: P.pallas_rope_apply(plan, x, pos[:3]),
        lambda: P.pallas_rope_apply(plan, x, pos.long()),
        lambda: P.pallas_rope_apply(plan, x, pos, x[:, :1]),
        lambda: P.pallas_rope_init(64, 1e4, "thirds"),
        lambda: P.pallas_rope_init(64, 1e4, scaling="more"),
        lambda: P.pallas_quant_store(codes, scales, 0, x, x, pos, bt),   # host tensors
        lambda: P.pallas_quant_store(codes.to(torch.uint8), scales, 0, x, x, pos, bt),
        lambda: P.pallas_quant_store(codes, scales[..., :1], 0, x, x, pos, bt),
        lambda: P.pallas_quant_store(codes, scales, 0, x[:, :1], x, pos, bt),
        lambda: P.pallas_quant_load(codes, scales, 0, x, x[..., :32], pos, bt),
        lambda: P.pallas_quant_load(codes, scales, 0, x, x, pos, bt, seq_ids=pos[:2]),
        lambda: P.pallas_attend_kv(pool, 0, x, pos, 48, bt, 0.1, x.clone(), ws),   # host tensors
        lambda: P.pallas_attend_kv(pool, 0, x, pos[:3], 48, bt, 0.1, x.clone(), ws),
        lambda: P.pallas_attend_kv(pool, 0, x, pos, 48, bt[:3], 0.1, x.clone(), ws),
        lambda: P.pallas_attend_kv(pool, 0, x, pos, 48, bt, 0.1, x[:, :1], ws),
        lambda: P.pallas_attend_kv(pool, 0, x, pos, 48, bt, 0.1, x.clone(), ws, lse=torch.zeros((4, 3))),
        lambda: P.pallas_attend_quant(codes, scales, 0, x.float(), pos, 48, bt, 0.1, x.clone(), ws),
    ]
    for i, call in enumerate(calls):
        with pytest.raises(P.PallasError) as e:
            call()
        assert e.value.status == P.Status.INVALID_ARG, i
