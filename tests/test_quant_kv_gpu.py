"""pallas_quant_store and pallas_quant_load: codes, scales and values read back equal
the oracle's bit for bit, whatever the rows hold, and nothing else is written."""
import numpy as np
import pytest
import torch

from helpers import bits, ensure_lib, to_np64
from oracle import cache_ops as co
from oracle.numerics import bf16_bits, bf16_round

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


@pytest.fixture(scope="module")
def P():
    return ensure_lib()


def make_pool(L, pages, hkv, d, fmt):
    codes = torch.full((L, 2, pages, 16, hkv, d), 0x5B, dtype=torch.uint8, device=DEV).view(TYPES[fmt])
    return codes, torch.full((L, 2, pages, 16, hkv), -7.0, dtype=torch.float32, device=DEV)


def special_rows(T, hkv, d, seed):
    """Normal rows, and among them zeros, one non-zero value, subnormals, the largest
    values, infinities and NaN, rows whose maximum sits at a border of the scale."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((T * hkv, d), generator=g) * torch.exp(2 * torch.randn((T * hkv, 1), generator=g))
    x = x.to(torch.bfloat16)
    n = T * hkv
    puts = [lambda r: r.zero_(), lambda r: r.zero_().index_fill_(0, torch.tensor([d - 1]), -3e38),
            lambda r: r.mul_(1e-37), lambda r: r.copy_(torch.full((d,), 1e-40).to(torch.bfloat16)),
            lambda r: r.index_fill_(0, torch.tensor([5]), float("inf")), lambda r: r.index_fill_(0, torch.tensor([d // 2]), float("nan")),
            lambda r: r.clamp_(-1, 1).index_fill_(0, torch.tensor([0]), 1.75), lambda r: r.clamp_(-1, 1).index_fill_(0, torch.tensor([3]), -1.7578125),
            lambda r: r.index_fill_(0, torch.tensor([d - 2]), float("-inf")), lambda r: r.zero_().neg_()]
    for i, put in enumerate(puts):
        if (7 * i + 3) < n:
            put(x[7 * i + 3])
    return x.view(T, hkv, d)


def stored(want_codes, want_scales, codes, scales, layer, kv, table, seq, pos, x, fmt):
    c, s = co.quantise(to_np64(x), fmt)
    for t in range(len(pos)):
        pg = table[seq[t], pos[t] // 16]
        want_codes[layer, kv, pg, pos[t] % 16] = c[t]
        want_scales[layer, kv, pg, pos[t] % 16] = s[t]


CASES = [
    # heads, head_dim, positions per sequence
    (1, 64, [[0]]), (8, 128, [[0, 15, 16, 31], [7]]), (3, 128, [list(range(5, 38)), [], [100, 3]]),
    (5, 64, [list(range(40))]), (16, 64, [[47], [46], [1]]), (2, 128, [list(range(0, 129))]),
]


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("hkv,d,where", CASES)
def test_round_trip(P, hkv, d, where, fmt):
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
    codes, scales = make_pool(3, pages, hkv, d, fmt)
    want_codes, want_scales = codes.view(torch.uint8).cpu().numpy().copy(), scales.cpu().numpy().copy()
    for kv, x in ((0, k), (1, v)):
        stored(want_codes, want_scales, codes, scales, 1, kv, table, seq, pos, x, fmt)
    d_seq, d_pos, d_bt = (torch.from_numpy(a).to(DEV) for a in (seq, pos, table))
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    P.pallas_quant_store(codes, scales, 1, k, v, d_pos, d_bt, seq_ids=d_seq, err=err)
    assert np.array_equal(scales.cpu().numpy(), want_scales, equal_nan=True)
    assert np.array_equal(codes.view(torch.uint8).cpu().numpy(), want_codes)
    # read back, into strided rows
    back = torch.full((T, 5 * hkv * d), 3.0, dtype=torch.bfloat16, device=DEV)
    bk, bv = back[:, :hkv * d].view(T, hkv, d), back[:, 3 * hkv * d:4 * hkv * d].view(T, hkv, d)
    P.pallas_quant_load(codes, scales, 1, bk, bv, d_pos, d_bt, seq_ids=d_seq, err=err)
    for kv, got in ((0, bk), (1, bv)):
        pg, slot = table[seq, pos // 16], pos % 16
        c, s = want_codes[1, kv, pg, slot], want_scales[1, kv, pg, slot]
        val = (co.dequantise(c, np.ones_like(s), fmt).astype(np.float32) * s[..., None])      # float32 product
        fine = np.isfinite(val)
        assert np.array_equal(fine, torch.isfinite(got).cpu().numpy())
        assert np.array_equal(bits(got)[fine], bf16_bits(bf16_round(val.astype(np.float64)))[fine])
    rest = back.clone()
    rest[:, :hkv * d], rest[:, 3 * hkv * d:4 * hkv * d] = 3.0, 3.0
    assert bool((rest == 3.0).all())
    assert int(err.item()) == 0


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_every_bf16_value(P, fmt):
    """Each finite bf16 value beside each of a few maxima."""
    v = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    v = v[torch.isfinite(v)]
    v = torch.cat([v, v[:(-len(v)) % 56]]).view(-1, 56)
    tops = torch.tensor([0.0, 1.0, 1.75, 1.7578125, 3.3e38, 2e-38, 5e-31], dtype=torch.bfloat16)
    x = torch.cat([torch.cat([v, top.expand(len(v), 1), torch.zeros((len(v), 7), dtype=torch.bfloat16)], dim=1)
                   for top in tops]).view(-1, 1, 64).to(DEV)
    T = len(x)
    table = torch.arange((T + 15) // 16, dtype=torch.int32, device=DEV)[None]
    codes, scales = make_pool(1, table.shape[1], 1, 64, fmt)
    pos = torch.arange(T, dtype=torch.int32, device=DEV)
    P.pallas_quant_store(codes, scales, 0, x, x, pos, table, seq_ids=torch.zeros_like(pos))
    c, s = co.quantise(to_np64(x), fmt)
    for kv in range(2):
        assert np.array_equal(scales[0, kv].reshape(-1, 1)[:T].cpu().numpy(), s)
        assert np.array_equal(codes.view(torch.uint8)[0, kv].reshape(-1, 1, 64)[:T].cpu().numpy(), c)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_padding_and_bad_places(P, fmt):
    """Tokens of negative position are skipped; sequences, positions and pages outside
    raise the flag; rows of skipped tokens stay as they were on reading back."""
    hkv, d = 4, 128
    table = torch.tensor([[2, 0], [1, 9], [3, -1]], dtype=torch.int32, device=DEV)      # 9, -1: no pages of the pool
    seq = torch.tensor([0, 1, 1, 2, 3, -1, 0, 0, 2], dtype=torch.int32, device=DEV)
    pos = torch.tensor([5, 4, 16, 17, 0, 0, 32, -1, 3], dtype=torch.int32, device=DEV)
    good = [0, 1, 8]
    T = len(seq)
    k, v = special_rows(T, hkv, d, 3).to(DEV), special_rows(T, hkv, d, 4).to(DEV)
    codes, scales = make_pool(1, 4, hkv, d, fmt)
    want_codes, want_scales = codes.view(torch.uint8).cpu().numpy().copy(), scales.cpu().numpy().copy()
    tb, sq, ps = table.cpu().numpy(), seq.cpu().numpy()[good], pos.cpu().numpy()[good]
    for kv, x in ((0, k), (1, v)):
        stored(want_codes, want_scales, codes, scales, 0, kv, tb, sq, ps, x[good], fmt)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    P.pallas_quant_store(codes, scales, 0, k, v, pos, table, seq_ids=seq, err=err)
    assert int(err.item()) == 1
    assert np.array_equal(scales.cpu().numpy(), want_scales, equal_nan=True)
    assert np.array_equal(codes.view(torch.uint8).cpu().numpy(), want_codes)
    bk, bv = torch.full_like(k, 3.0), torch.full_like(v, 3.0)
    err.zero_()
    P.pallas_quant_load(codes, scales, 0, bk, bv, pos, table, seq_ids=seq, err=err)
    assert int(err.item()) == 1
    skipped = [i for i in range(T) if i not in good]
    assert bool((bk[skipped] == 3.0).all()) and bool((bv[skipped] == 3.0).all())
    assert not bool((bk[good] == 3.0).all())
    # padding alone raises nothing, and no flag is wanted
    err.zero_()
    P.pallas_quant_store(codes, scales, 0, k, v, torch.full_like(pos, -1), table, seq_ids=seq, err=err)
    P.pallas_quant_load(codes, scales, 0, bk, bv, pos, table, seq_ids=seq)
    assert int(err.item()) == 0
    assert np.array_equal(codes.view(torch.uint8).cpu().numpy(), want_codes)


def test_one_token_per_sequence(P):
    """Without sequence ids token t belongs to sequence t; spare tables are fine."""
    table = torch.tensor([[1], [0], [2]], dtype=torch.int32, device=DEV)
    pos = torch.tensor([3, 15], dtype=torch.int32, device=DEV)
    k, v = (torch.randn((2, 2, 64), device=DEV).to(torch.bfloat16) for _ in range(2))
    a, b = make_pool(1, 3, 2, 64, "e4m3"), make_pool(1, 3, 2, 64, "e4m3")
    P.pallas_quant_store(*a, 0, k, v, pos, table)
    P.pallas_quant_store(*b, 0, k, v, pos, table, seq_ids=torch.tensor([0, 1], dtype=torch.int32, device=DEV))
    assert torch.equal(a[0].view(torch.uint8), b[0].view(torch.uint8)) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_pages_beyond_4_gib(P, fmt):
    """Slots at the end of a plane of more than 4 GiB, of the second layer."""
    hkv, d = 16, 128
    pages = (1 << 32) // (16 * hkv * d) + 9
    codes = torch.empty((2, 2, pages, 16, hkv, d), dtype=torch.uint8, device=DEV).view(TYPES[fmt])
    scales = torch.empty((2, 2, pages, 16, hkv), device=DEV)
    table = torch.tensor([[pages - 1, 3, pages - 7]], dtype=torch.int32, device=DEV)
    pos = torch.tensor([0, 15, 16, 47, 33], dtype=torch.int32, device=DEV)
    x = special_rows(5, hkv, d, 6).to(DEV)
    seq = torch.zeros_like(pos)
    P.pallas_quant_store(codes, scales, 1, x, x, pos, table, seq_ids=seq)
    c, s = co.quantise(to_np64(x), fmt)
    pg, slot = table[0, (pos // 16).long()].long(), (pos % 16).long()
    for kv in range(2):
        assert np.array_equal(scales[1, kv, pg, slot].cpu().numpy(), s, equal_nan=True)
        assert np.array_equal(codes.view(torch.uint8)[1, kv, pg, slot].cpu().numpy(), c)
    bk, bv = torch.empty_like(x), torch.empty_like(x)
    P.pallas_quant_load(codes, scales, 1, bk, bv, pos, table, seq_ids=seq)
    val = co.dequantise(c, np.ones_like(s), fmt).astype(np.float32) * s[..., None]
    fine = np.isfinite(val)
    for got in (bk, bv):
        assert np.array_equal(bits(got)[fine], bf16_bits(bf16_round(val.astype(np.float64)))[fine])


def test_an_empty_err_is_refused(P):
    """An empty slice has an address that is another tensor's."""
    codes, scales = torch.zeros((1, 2, 3, 16, 2, 64), dtype=torch.int8, device=DEV), torch.zeros((1, 2, 3, 16, 2), device=DEV)
    x, ints = torch.ones((1, 2, 64), dtype=torch.bfloat16, device=DEV), torch.zeros(8, dtype=torch.int32, device=DEV)
    bt = torch.full((1, 3), 99, dtype=torch.int32, device=DEV)
    ws = torch.empty(P.pallas_attend_workspace_size(1, 2, 2, 64, 5), dtype=torch.uint8, device=DEV)
    err, pos, lens = ints[2:2], ints[4:5], ints[5:6].fill_(5)
    for call in (lambda: P.pallas_quant_store(codes, scales, 0, x, x, pos, bt, err=err),
                 lambda: P.pallas_quant_load(codes, scales, 0, x, x, pos, bt, err=err),
                 lambda: P.pallas_attend_quant(codes, scales, 0, x, lens, 5, bt, 1.0, x.clone(), ws, err=err)):
        with pytest.raises(P.PallasError) as e:
            call()
        assert e.value.status == P.Status.INVALID_ARG
    assert ints.tolist() == [0, 0, 0, 0, 0, 5, 0, 0]
