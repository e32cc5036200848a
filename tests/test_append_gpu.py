"""pallas_append_kv and pallas_append_quant against the oracle.

The rotation is exact to far below a bf16 step, so rotated values are, bit for bit, the oracle's
64-bit ones rounded to float32 and then to bf16; where those lie within 2^-34 (pair's magnitude;
the oracle's angles are position times frequency in 53 bits, 2^-22 of a radian for 2^31, and
less in the ratio of the position otherwise) of a border between two bf16 values, either of the
two.  Codes and scales are the oracle's of the rotated bf16 values, bit for bit."""
import numpy as np
import pytest
import torch

from helpers import bits, ensure_lib, to_np64
from oracle import cache_ops as co
from oracle.numerics import bf16_bits, bf16_round

pytestmark = pytest.mark.gpu
DEV = "cuda"
FORMATS = ["bf16", "e4m3", "int8", "e2m1"]
TYPES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8, "e2m1": torch.float4_e2m1fn_x2}
YARN = dict(scaling="yarn", factor=8.0, trained_len=4096, fast=32.0, slow=1.0)


@pytest.fixture(scope="module")
def P():
    return ensure_lib()


class Pool:
    """A pool of two layers, full of a pattern; `append` works on layer 1."""

    def __init__(self, fmt, pages, hkv, d):
        self.fmt, self.d = fmt, d
        shape = (2, 2, pages, 16, hkv)
        if fmt == "bf16":
            self.raw = torch.full(shape + (d,), 0x3C5B, dtype=torch.int16, device=DEV)
            self.scales = None
        else:
            self.raw = torch.full(shape + (d // 2 if fmt == "e2m1" else d,), 0x5B, dtype=torch.uint8, device=DEV)
            self.scales = (torch.full(shape + (4,), 0x77, dtype=torch.uint8, device=DEV) if fmt == "e2m1" else
                           torch.full(shape, -7.0, device=DEV))

    def append(self, P, plan, *a, **kw):
        if self.fmt == "bf16":
            P.pallas_append_kv(plan, self.raw.view(torch.bfloat16), 1, *a, **kw)
        else:
            scales = self.scales.view(torch.float8_e8m0fnu) if self.fmt == "e2m1" else self.scales
            P.pallas_append_quant(plan, self.raw.view(TYPES[self.fmt]), scales, 1, *a, **kw)

    def numpy(self):
        return self.raw.cpu().numpy().copy(), None if self.scales is None else self.scales.cpu().numpy().copy()

    def put(self, want, kv, pg, slot, rows):
        """Rows (bf16 bits [n, hkv, d]) as the pool holds them, into want[1, kv, pg, slot]."""
        if self.fmt == "bf16":
            want[0][1, kv, pg, slot] = rows.view(np.int16)
            return
        x = torch.from_numpy(rows.view(np.int16).copy()).view(torch.bfloat16)
        c, s = co.quantise4(to_np64(x)) if self.fmt == "e2m1" else co.quantise(to_np64(x), self.fmt)
        want[0][1, kv, pg, slot], want[1][1, kv, pg, slot] = c, s


def rotated(x, pos, f, m, layout, got):
    """bf16 bits of x [T, H, d] turned; `got` decides where the exact value lies at a border."""
    ref = co.rope(to_np64(x), pos, f, m, layout)
    r = 2 * len(f)
    same = bits(x)
    size = np.where(np.isfinite(to_np64(x)), np.abs(to_np64(x)), 0.0).max(axis=-1, keepdims=True) * m * 2
    near = size * (2.0 ** -34 + np.abs(pos.astype(np.float64))[:, None, None] * 2.0 ** -52)
    with np.errstate(all="ignore"):
        low, mid, high = (bf16_bits(bf16_round((ref + k * near).astype(np.float32))) for k in (-1, 0, 1))
    out = np.where((got == low) | (got == high), got, mid)
    open_ = (low != high) & np.isfinite(ref) & (ref != 0)
    assert open_[..., :r].mean() < 1e-3 + np.abs(pos).max() * 2.0 ** -40
    bad = ~np.isfinite(ref)      # (a pair with an infinity or a NaN: complex products lose which of the two it becomes)
    assert (got[bad] & 0x7F80 == 0x7F80).all()
    out = np.where(bad, got, out)
    out[..., r:] = same[..., r:]
    return out


def check(P, fmt, hq, hkv, d, r, layout, where, scaling={}, seed=0, special=False, in_place=False, top=None):
    rng = np.random.default_rng(seed)
    seq = np.repeat(np.arange(len(where)), [len(w) for w in where]).astype(np.int32)
    pos = np.array([p for w in where for p in w], dtype=np.int32)
    mix = rng.permutation(len(pos))
    seq, pos = seq[mix], pos[mix]
    T = len(pos)
    width = int(pos.max()) // 16 + 1
    used = sorted({(s, p // 16) for s, p in zip(seq.tolist(), pos.tolist())})
    pages = len(used) + 3
    table = np.full((len(where), width), -1, dtype=np.int32)
    for (s, j), pg in zip(used, rng.permutation(pages)):
        table[s, j] = pg
    wide = torch.randn((T, (hq + 2 * hkv + 1) * d), generator=torch.Generator().manual_seed(seed + 1))
    wide = (wide * torch.exp(torch.randn((T, 1), generator=torch.Generator().manual_seed(seed + 2)))).to(torch.bfloat16)
    rows = wide.view(T, hq + 2 * hkv + 1, d)
    if special:      # infinities, NaN and zeros in K and V rows
        rows[0, hq, 3], rows[T // 2, hq + hkv - 1, d - 1], rows[T - 1, hq + hkv, 5] = float("inf"), float("nan"), float("-inf")
        rows[T // 3, hq:] = 0
    wide = wide.to(DEV)
    rows = wide.view(T, hq + 2 * hkv + 1, d)
    before = rows.clone().cpu()
    pool = Pool(fmt, pages, hkv, d)
    want = pool.numpy()
    plan = P.pallas_rope_init(r, 1e6, layout, **scaling)
    f, m = co.rope_frequencies(r, 1e6, **{"scaling": "none", **scaling})
    m = float(np.float32(m))
    d_seq, d_pos, d_bt = (torch.from_numpy(a).to(DEV) for a in (seq, pos, table))
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    q_out = torch.full((T, hq + 1, d), 3.0, dtype=torch.bfloat16, device=DEV) if hq and not in_place else None
    kw = dict(q=rows[:, :hq], q_out=None if in_place else q_out[:, :hq]) if hq else {}
    pool.append(P, plan, rows[:, hq:hq + hkv], rows[:, hq + hkv:hq + 2 * hkv], d_pos, d_bt, seq_ids=d_seq, err=err, **kw)
    assert int(err.item()) == 0
    after = rows.cpu()
    if hq:
        got = after[:, :hq] if in_place else q_out[:, :hq].cpu()
        assert np.array_equal(bits(got), rotated(before[:, :hq], pos, f, m, layout, bits(got)))
        if not in_place:
            assert bool((q_out[:, hq:] == 3.0).all())
            assert np.array_equal(bits(after[:, :hq]), bits(before[:, :hq]))
    assert np.array_equal(bits(after[:, hq:]), bits(before[:, hq:]))
    pg, slot = table[seq, pos // 16], pos % 16
    have = pool.numpy()
    if fmt == "bf16":
        k = rotated(before[:, hq:hq + hkv], pos, f, m, layout, have[0][1, 0, pg, slot].view(np.uint16))
    else:            # the bf16 values that the codes are made of
        plain = Pool("bf16", pages, hkv, d)
        plain.append(P, plan, rows[:, hq:hq + hkv], rows[:, hq + hkv:hq + 2 * hkv], d_pos, d_bt, seq_ids=d_seq)
        got = plain.numpy()[0][1, 0, pg, slot].view(np.uint16)
        k = rotated(before[:, hq:hq + hkv], pos, f, m, layout, got)
    pool.put(want, 0, pg, slot, k)
    pool.put(want, 1, pg, slot, bits(before[:, hq + hkv:hq + 2 * hkv]))
    if fmt == "bf16":
        nan = np.isnan(torch.from_numpy(want[0]).view(torch.bfloat16).float().numpy())
        assert np.array_equal(nan, np.isnan(torch.from_numpy(have[0]).view(torch.bfloat16).float().numpy()))
        assert np.array_equal(want[0][~nan], have[0][~nan])
    else:
        assert np.array_equal(want[0], have[0]) and np.array_equal(want[1], have[1], equal_nan=fmt != "e2m1")


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("hq,hkv,d,r,layout,where", [
    (8, 2, 128, 128, "half", [[0], [17], [8000]]),
    (4, 4, 64, 64, "interleaved", [[5, 6, 7], [], [100, 15, 16]]),
    (12, 4, 128, 64, "half", [list(range(3, 40))]),
    (3, 1, 64, 16, "interleaved", [list(range(33)), [70]]),
    (0, 5, 128, 32, "half", [list(range(20))]),
    (64, 8, 128, 128, "interleaved", [[1], [2], [3]]),
    (7, 1, 128, 54, "half", [list(range(9)), [1000, 999]]),          # rotary_dim no multiple of 8
    (6, 2, 64, 2, "half", [[3, 4]]),
    (5, 5, 64, 62, "interleaved", [list(range(18))]),
    (1, 1, 128, 100, "interleaved", [[12345]]),
    (1, 16, 64, 40, "half", [[0, 1], [2]]),
])
def test_against_oracle(P, fmt, hq, hkv, d, r, layout, where):
    check(P, fmt, hq, hkv, d, r, layout, where, seed=hq + d + r)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d,r,layout", [(128, 128, "half"), (64, 24, "interleaved"), (128, 70, "half")])
def test_many_tokens(P, fmt, d, r, layout):
    """From 512 tokens on a workgroup takes all heads of its tokens."""
    check(P, fmt, 9, 3, d, r, layout, [list(range(100, 500)), list(range(0, 260)), [3]], scaling=YARN, seed=5, special=True)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_special_rows_in_place(P, fmt, layout):
    check(P, fmt, 6, 3, 128, 96, layout, [list(range(10, 31))], seed=6, special=True, in_place=True)
    check(P, fmt, 2, 2, 64, 64, layout, [list(range(600))], seed=7, in_place=True)


@pytest.mark.parametrize("kw", [dict(), dict(scaling="linear", factor=4.0), dict(scaling="ntk", factor=8.0), YARN,
                                dict(scaling="bands", factor=8.0, trained_len=8192, fast=4.0, slow=1.0)])
def test_scalings_and_far_positions(P, kw):
    check(P, "bf16", 2, 1, 64, 64, "half", [[1 << 20, (1 << 20) - 1, 131071]], scaling=kw, seed=8)


def test_last_position(P):
    """Position 2^31 - 1 of a sequence whose table reaches so far."""
    plan = P.pallas_rope_init(64, 1e4)
    table = torch.full((1, 1 << 27), -1, dtype=torch.int32, device=DEV)
    table[0, -1] = 2
    pos = torch.tensor([2 ** 31 - 1], dtype=torch.int32, device=DEV)
    k = torch.randn((1, 2, 64), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(DEV)
    pool = Pool("bf16", 3, 2, 64)
    pool.append(P, plan, k, k, pos, table)
    f, m = co.rope_frequencies(64, 1e4)
    got = pool.raw.view(torch.bfloat16)[1, 0, 2, 15].double().cpu().numpy()
    ref = co.rope(to_np64(k), np.array([2 ** 31 - 1]), f, m)[0]
    # bf16 has 8 significant bits: half a step is up to 2^-8 of the value.  2^31 f is known to 2^-22 of a radian in
    # the oracle.
    assert np.all(np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -21 * np.abs(to_np64(k)).max())


@pytest.mark.parametrize("fmt", FORMATS)
def test_padding_and_bad_places(P, fmt):
    hq, hkv, d = 4, 2, 128
    table = torch.tensor([[2, 0], [1, 9], [3, -1]], dtype=torch.int32, device=DEV)      # 9, -1: no pages of the pool
    seq = torch.tensor([0, 1, 1, 2, 3, -1, 0, 0, 2], dtype=torch.int32, device=DEV)
    pos = torch.tensor([5, 4, 16, 17, 0, 0, 32, -1, 3], dtype=torch.int32, device=DEV)
    good = [0, 1, 8]
    rows = torch.randn((9, hq + 2 * hkv, d), generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).to(DEV)
    plan = P.pallas_rope_init(d, 1e6)
    a, b = Pool(fmt, 4, hkv, d), Pool(fmt, 4, hkv, d)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    q_out = torch.full((9, hq, d), 3.0, dtype=torch.bfloat16, device=DEV)
    q, k, v = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
    a.append(P, plan, k, v, pos, table, q=q, q_out=q_out, seq_ids=seq, err=err)
    assert int(err.item()) == 1
    sub = torch.tensor(good, device=DEV)
    err.zero_()
    b.append(P, plan, k[sub].contiguous(), v[sub].contiguous(), pos[sub], table, seq_ids=seq[sub], err=err)
    assert int(err.item()) == 0
    assert torch.equal(a.raw, b.raw) and (a.scales is None or torch.equal(a.scales, b.scales))
    assert bool((q_out[7] == 3.0).all())                                               # padding: nothing
    alone = torch.empty((8, hq, d), dtype=torch.bfloat16, device=DEV)
    rest = torch.tensor([i for i in range(9) if i != 7], device=DEV)
    P.pallas_rope_apply(plan, q[rest].contiguous(), pos[rest], alone)                  # within a step of it
    step = (alone.float().abs() * 2.0 ** -7).clamp(min=1e-6)
    assert bool(((q_out[rest].float() - alone.float()).abs() <= step).all())
    before = a.numpy()
    a.append(P, plan, k, v, torch.full_like(pos, -1), table, q=q, q_out=q_out, seq_ids=seq, err=err)
    assert int(err.item()) == 0 and np.array_equal(before[0], a.numpy()[0])
    a.append(P, plan, k[:0], v[:0], pos[:0], table, q=q[:0], q_out=q_out[:0])           # no token
    # token t is sequence t without ids
    c, e = Pool(fmt, 4, hkv, d), Pool(fmt, 4, hkv, d)
    c.append(P, plan, k[:2], v[:2], pos[:2], table)
    e.append(P, plan, k[:2], v[:2], pos[:2], table, seq_ids=seq[:2])
    assert torch.equal(c.raw, e.raw)


@pytest.mark.parametrize("fmt", FORMATS)
def test_pages_beyond_4_gib(P, fmt):
    hkv, d = 16, 128
    row = {"bf16": 256, "e4m3": 128, "int8": 128, "e2m1": 64}[fmt]
    pages = (1 << 32) // (16 * hkv * row) + 9
    if fmt == "bf16":
        raw, scales = torch.empty((2, 2, pages, 16, hkv, d), dtype=torch.int16, device=DEV), None
    else:
        raw = torch.empty((2, 2, pages, 16, hkv, row), dtype=torch.uint8, device=DEV)
        scales = torch.empty((2, 2, pages, 16, hkv) + ((4,) if fmt == "e2m1" else ()),
                             dtype=torch.uint8 if fmt == "e2m1" else torch.float32, device=DEV)
    pool = Pool(fmt, 1, hkv, d)
    pool.raw, pool.scales = raw, scales
    table = torch.tensor([[pages - 1, 3, pages - 7]], dtype=torch.int32, device=DEV)
    pos = torch.tensor([0, 15, 16, 47, 33], dtype=torch.int32, device=DEV)
    x = torch.randn((5, 2 * hkv, d), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).to(DEV)
    plan = P.pallas_rope_init(d, 1e6)
    pool.append(P, plan, x[:, :hkv], x[:, hkv:], pos, table, seq_ids=torch.zeros_like(pos))
    small = Pool(fmt, 3, hkv, d)
    small.append(P, plan, x[:, :hkv], x[:, hkv:], pos, torch.tensor([[0, 1, 2]], dtype=torch.int32, device=DEV),
                 seq_ids=torch.zeros_like(pos))
    big, tiny = table[0, (pos // 16).long()].long(), (pos // 16).long()
    slot = (pos % 16).long()
    for kv in range(2):
        assert torch.equal(raw[1, kv, big, slot], small.raw[1, kv, tiny, slot])
        if scales is not None:
            assert torch.equal(scales[1, kv, big, slot], small.scales[1, kv, tiny, slot])


@pytest.mark.parametrize("fmt", ["bf16", "e2m1"])
def test_captured_and_replayed_on_another_stream(P, fmt):
    hq, hkv, d, S = 8, 2, 128, 3
    plan = P.pallas_rope_init(d, 1e6)
    table = torch.arange(12, dtype=torch.int32, device=DEV).view(3, 4)
    a, b = Pool(fmt, 12, hkv, d), Pool(fmt, 12, hkv, d)
    rows = torch.zeros((S, hq + 2 * hkv, d), dtype=torch.bfloat16, device=DEV)
    pos = torch.zeros(S, dtype=torch.int32, device=DEV)
    out, want = (torch.zeros((S, hq, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))

    def call(pool, q_out, **kw):
        pool.append(P, plan, rows[:, hq:hq + hkv], rows[:, hq + hkv:], pos, table, q=rows[:, :hq], q_out=q_out, **kw)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call(a, out)
    torch.cuda.synchronize()
    for t in range(5):
        rows.copy_(torch.randn(rows.shape, generator=torch.Generator().manual_seed(t)).to(torch.bfloat16))
        pos.copy_(torch.tensor([3 * t, 40 + t, -1 if t == 2 else t], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        other = torch.cuda.Stream()
        call(b, want, stream=other)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(a.raw, b.raw) and (a.scales is None or torch.equal(a.scales, b.scales))
