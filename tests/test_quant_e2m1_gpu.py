"""pallas_quant_store and pallas_quant_load of a 4-bit pool: codes, scales and values read
back equal the oracle's bit for bit, whatever the rows hold, and nothing else is written."""
import numpy as np
import pytest
import torch

from helpers import bits, ensure_lib, to_np64
from oracle import cache_ops as co
from oracle.numerics import bf16_bits

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def P():
    return ensure_lib()


def make_pool(L, pages, hkv, d):
    """(codes, scales) as bytes."""
    return (torch.full((L, 2, pages, 16, hkv, d // 2), 0x5B, dtype=torch.uint8, device=DEV),
            torch.full((L, 2, pages, 16, hkv, 4), 0x77, dtype=torch.uint8, device=DEV))


def typed(codes, scales):
    return codes.view(torch.float4_e2m1fn_x2), scales.view(torch.float8_e8m0fnu)


def special_rows(T, hkv, d, seed):
    """Normal rows of many magnitudes, and among them zeros, single values, subnormals, the largest values,
    infinities and NaN, quarters whose maximum sits at a border of the scale."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((T * hkv, d), generator=g) * torch.exp(2 * torch.randn((T * hkv, 1), generator=g))
    x = x.to(torch.bfloat16)
    h = d // 4
    puts = [lambda r: r.zero_(), lambda r: r.zero_().index_fill_(0, torch.tensor([d - 1]), -3e38),
            lambda r: r.mul_(1e-37), lambda r: r.copy_(torch.full((d,), 1e-40).to(torch.bfloat16)),
            lambda r: r.index_fill_(0, torch.tensor([5]), float("inf")), lambda r: r.index_fill_(0, torch.tensor([d // 2]), float("nan")),
            lambda r: r.clamp_(-1, 1).index_fill_(0, torch.tensor([0, h, 2 * h]), 1.5), lambda r: r.clamp_(-1, 1).index_fill_(0, torch.tensor([3, d - h]), -1.5078125),
            lambda r: r.index_fill_(0, torch.tensor([d - 2]), float("-inf")), lambda r: r.zero_().neg_(),
            lambda r: r.mul_(2.0 ** -100), lambda r: r.clamp_(-1, 1).mul_(2.0 ** 127)]
    for i, put in enumerate(puts):
        if (7 * i + 3) < len(x):
            put(x[7 * i + 3])
    return x.view(T, hkv, d)


def bits_equal(got, val):
    """bf16 rows against float64 values that bf16 holds; NaN where they are."""
    fine = np.isfinite(val)
    return np.array_equal(torch.isnan(got).cpu().numpy(), ~fine) and np.array_equal(bits(got)[fine], bf16_bits(val[fine]))


CASES = [
    # heads, head_dim, positions per sequence
    (1, 64, [[0]]), (8, 128, [[0, 15, 16, 31], [7]]), (3, 128, [list(range(5, 38)), [], [100, 3]]),
    (5, 64, [list(range(40))]), (16, 64, [[47], [46], [1]]), (2, 128, [list(range(0, 129))]),
]


@pytest.mark.parametrize("hkv,d,where", CASES)
def test_round_trip(P, hkv, d, where):
    rng = np.random.default_rng(hkv + d)
    seq = np.repeat(np.arange(len(where)), [len(w) for w in where])
    pos = np.array([p for w in where for p in w])
    mix = rng.permutation(len(pos))
    seq, pos = seq[mix].astype(np.int32), pos[mix].astype(np.int32)
    pages = 9 * len(where) + 2
    table = rng.permutation(pages)[: 9 * len(where)].reshape(len(where), 9).astype(np.int32)
    T = len(pos)
    wide = torch.randn((T, 3 * hkv * d), device=DEV).to(torch.bfloat16)     # K and V inside projection rows
    k = wide[:, hkv * d:2 * hkv * d].view(T, hkv, d)
    v = wide[:, 2 * hkv * d:].view(T, hkv, d)
    k.copy_(special_rows(T, hkv, d, 1))
    v.copy_(special_rows(T, hkv, d, 2))
    codes, scales = make_pool(3, pages, hkv, d)
    want_codes, want_scales = codes.cpu().numpy().copy(), scales.cpu().numpy().copy()
    pg, slot = table[seq, pos // 16], pos % 16
    vals = []
    for kv, x in ((0, k), (1, v)):
        c, s = co.quantise4(to_np64(x))
        want_codes[1, kv, pg, slot], want_scales[1, kv, pg, slot] = c, s
        vals.append(co.dequantise4(c, s))
    d_seq, d_pos, d_bt = (torch.from_numpy(a).to(DEV) for a in (seq, pos, table))
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    P.pallas_quant_store(*typed(codes, scales), 1, k, v, d_pos, d_bt, seq_ids=d_seq, err=err)
    assert np.array_equal(scales.cpu().numpy(), want_scales)
    assert np.array_equal(codes.cpu().numpy(), want_codes)
    back = torch.full((T, 5 * hkv * d), 3.0, dtype=torch.bfloat16, device=DEV)      # read back, into strided rows
    bk, bv = back[:, :hkv * d].view(T, hkv, d), back[:, 3 * hkv * d:4 * hkv * d].view(T, hkv, d)
    P.pallas_quant_load(*typed(codes, scales), 1, bk, bv, d_pos, d_bt, seq_ids=d_seq, err=err)
    assert bits_equal(bk, vals[0]) and bits_equal(bv, vals[1])
    rest = back.clone()
    rest[:, :hkv * d], rest[:, 3 * hkv * d:4 * hkv * d] = 3.0, 3.0
    assert bool((rest == 3.0).all())
    assert int(err.item()) == 0


def test_every_bf16_value(P):
    """Each finite bf16 value beside each of a few maxima of its quarter."""
    v = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    v = v[torch.isfinite(v)]
    v = torch.cat([v, v[:(-len(v)) % 15]]).view(-1, 15)
    tops = torch.tensor([0.0, 1.0, 1.5, 1.5078125, 3.3e38, 2e-38, 2.0 ** -100, 2.0 ** -99, 6.0], dtype=torch.bfloat16)
    x = torch.cat([torch.cat([v, top.expand(len(v), 1)], dim=1) for top in tops])
    x = torch.cat([x, x[:(-len(x)) % 4]]).view(-1, 1, 64).to(DEV)
    T = len(x)
    table = torch.arange((T + 15) // 16, dtype=torch.int32, device=DEV)[None]
    codes, scales = make_pool(1, table.shape[1], 1, 64)
    pos = torch.arange(T, dtype=torch.int32, device=DEV)
    P.pallas_quant_store(*typed(codes, scales), 0, x, x, pos, table, seq_ids=torch.zeros_like(pos))
    c, s = co.quantise4(to_np64(x))
    for kv in range(2):
        assert np.array_equal(scales[0, kv].reshape(-1, 1, 4)[:T].cpu().numpy(), s)
        assert np.array_equal(codes[0, kv].reshape(-1, 1, 32)[:T].cpu().numpy(), c)


def test_every_code_and_scale_reads_back(P):
    """All 16 codes with all 256 scale bytes: exact, but for what bf16 has no value for (the greatest and the
    least scales, which the store does not write), and NaN at 255."""
    codes, scales = make_pool(1, 8, 2, 64)
    codes[:] = torch.arange(256, dtype=torch.uint8, device=DEV).view(8, 32).repeat(1, 2 * 16 // 2).view(8, 16, 1, 32)
    scales.view(-1, 4)[:] = torch.arange(256, dtype=torch.uint8, device=DEV).repeat_interleave(2)[:, None]
    T = 128
    pos, table = torch.arange(T, dtype=torch.int32, device=DEV), torch.arange(8, dtype=torch.int32, device=DEV)[None]
    bk, bv = (torch.empty((T, 2, 64), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    P.pallas_quant_load(*typed(codes, scales), 0, bk, bv, pos, table, seq_ids=torch.zeros_like(pos))
    for kv, got in ((0, bk), (1, bv)):
        c, s = codes[0, kv].cpu().numpy(), scales[0, kv].cpu().numpy()
        val = co.dequantise4(c, s).reshape(T, 2, 64)
        s = np.repeat(s.reshape(T, 2, 4), 16, axis=-1)
        held = (s >= 2) & (s <= 252)
        assert np.array_equal(bits(got)[held], bf16_bits(val[held]))
        assert np.array_equal(torch.isnan(got).cpu().numpy(), s == 255)


def test_padding_and_bad_places(P):
    """Tokens of negative position are skipped; sequences, positions and pages outside raise the flag; rows of
    skipped tokens stay as they were on reading back."""
    hkv, d = 4, 128
    table = torch.tensor([[2, 0], [1, 9], [3, -1]], dtype=torch.int32, device=DEV)      # 9, -1: no pages of the pool
    seq = torch.tensor([0, 1, 1, 2, 3, -1, 0, 0, 2], dtype=torch.int32, device=DEV)
    pos = torch.tensor([5, 4, 16, 17, 0, 0, 32, -1, 3], dtype=torch.int32, device=DEV)
    good = [0, 1, 8]
    k, v = special_rows(9, hkv, d, 3).to(DEV), special_rows(9, hkv, d, 4).to(DEV)
    codes, scales = make_pool(1, 4, hkv, d)
    want_codes, want_scales = codes.cpu().numpy().copy(), scales.cpu().numpy().copy()
    tb, sq, ps = table.cpu().numpy(), seq.cpu().numpy()[good], pos.cpu().numpy()[good]
    for kv, x in ((0, k), (1, v)):
        want_codes[0, kv, tb[sq, ps // 16], ps % 16], want_scales[0, kv, tb[sq, ps // 16], ps % 16] = co.quantise4(to_np64(x[good]))
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    P.pallas_quant_store(*typed(codes, scales), 0, k, v, pos, table, seq_ids=seq, err=err)
    assert int(err.item()) == 1
    assert np.array_equal(scales.cpu().numpy(), want_scales) and np.array_equal(codes.cpu().numpy(), want_codes)
    bk, bv = torch.full_like(k, 3.0), torch.full_like(v, 3.0)
    err.zero_()
    P.pallas_quant_load(*typed(codes, scales), 0, bk, bv, pos, table, seq_ids=seq, err=err)
    assert int(err.item()) == 1
    skipped = [i for i in range(9) if i not in good]
    assert bool((bk[skipped] == 3.0).all()) and bool((bv[skipped] == 3.0).all())
    assert not bool((bk[good] == 3.0).all())


def test_pages_beyond_4_gib(P):
    """Slots at the end of a plane of more than 4 GiB, of the second layer."""
    hkv, d = 16, 128
    pages = (1 << 32) // (16 * hkv * d // 2) + 9
    codes = torch.empty((2, 2, pages, 16, hkv, d // 2), dtype=torch.uint8, device=DEV)
    scales = torch.empty((2, 2, pages, 16, hkv, 4), dtype=torch.uint8, device=DEV)
    table = torch.tensor([[pages - 1, 3, pages - 7]], dtype=torch.int32, device=DEV)
    pos = torch.tensor([0, 15, 16, 47, 33], dtype=torch.int32, device=DEV)
    x = special_rows(5, hkv, d, 6).to(DEV)
    seq = torch.zeros_like(pos)
    P.pallas_quant_store(*typed(codes, scales), 1, x, x, pos, table, seq_ids=seq)
    c, s = co.quantise4(to_np64(x))
    pg, slot = table[0, (pos // 16).long()].long(), (pos % 16).long()
    for kv in range(2):
        assert np.array_equal(scales[1, kv, pg, slot].cpu().numpy(), s)
        assert np.array_equal(codes[1, kv, pg, slot].cpu().numpy(), c)
    bk, bv = torch.empty_like(x), torch.empty_like(x)
    P.pallas_quant_load(*typed(codes, scales), 1, bk, bv, pos, table, seq_ids=seq)
    assert bits_equal(bk, co.dequantise4(c, s)) and bits_equal(bv, co.dequantise4(c, s))


@pytest.mark.parametrize("hkv,d", [(8, 128), (3, 64)])
def test_many_rows(P, hkv, d):
    """More than 4 MiB read back, which is stored another way, in strided rows; the last workgroup is not full."""
    T = 4201 if d == 128 else 11003
    x = torch.randn((T, 2 * hkv, d), generator=torch.Generator().manual_seed(7)).to(torch.bfloat16).to(DEV)
    k, v = x[:, :hkv], x[:, hkv:]
    pages = -(-T // 16)
    table = torch.from_numpy(np.random.default_rng(3).permutation(pages).astype(np.int32)).to(DEV)[None]
    codes, scales = make_pool(1, pages, hkv, d)
    pos = torch.arange(T, dtype=torch.int32, device=DEV)
    P.pallas_quant_store(*typed(codes, scales), 0, k, v, pos, table, seq_ids=torch.zeros_like(pos))
    back = torch.full((T, 2 * hkv + 1, d), 3.0, dtype=torch.bfloat16, device=DEV)
    P.pallas_quant_load(*typed(codes, scales), 0, back[:, :hkv], back[:, hkv:2 * hkv], pos, table, seq_ids=torch.zeros_like(pos))
    for got, rows in ((back[:, :hkv], k), (back[:, hkv:2 * hkv], v)):
        assert bits_equal(got, co.dequantise4(*co.quantise4(to_np64(rows))))
    assert bool((back[:, 2 * hkv] == 3.0).all())


def test_codes_and_scales_migrate(P):
    """Pack and assemble move the codes as rows of d / 4 and the scales as rows of 2 bf16 elements."""
    L, hkv, d, n = 2, 4, 128, 75
    a, b = make_pool(L, 6, hkv, d), make_pool(L, 7, hkv, d)
    src = torch.tensor([4, 0, 3, 1, 5], dtype=torch.int32, device=DEV)
    dst = torch.tensor([6, 2, 0, 5, 1], dtype=torch.int32, device=DEV)
    pos = torch.arange(n, dtype=torch.int32, device=DEV)
    x = torch.randn((L, n, 2 * hkv, d), generator=torch.Generator().manual_seed(8)).to(torch.bfloat16).to(DEV)
    for l in range(L):
        P.pallas_quant_store(*typed(*a), l, x[l, :, :hkv], x[l, :, hkv:], pos, src[None], seq_ids=torch.zeros_like(pos))
    for s, t in zip(a, b):
        s16, t16 = (y.view(L, 2, y.shape[2], 16, hkv, -1).view(torch.bfloat16) for y in (s, t))
        width = s16.shape[-1]
        arena = torch.empty(n * 2 * L * hkv * width * 2, dtype=torch.uint8, device=DEV)
        P.pallas_pack_suffix_blocks(s16, src, [P.ChunkDesc(0, n, 0)], arena)
        P.pallas_assemble_kv(t16, dst, [P.ChunkHeader(1, 1, 0, n, 0, L, hkv, width, 2)], arena, 1, 1)
    for l in range(L):
        bk, bv = (torch.empty((n, hkv, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        P.pallas_quant_load(*typed(*b), l, bk, bv, pos, dst[None], seq_ids=torch.zeros_like(pos))
        for got, rows in ((bk, x[l, :, :hkv]), (bv, x[l, :, hkv:])):
            assert bits_equal(got, co.dequantise4(*co.quantise4(to_np64(rows))))
