"""pallas_quant_load of 4 MiB and more, whose rows are stored past the caches, and just below:
every row's bits against the oracle's, into strided rows, with skipped tokens left as they were."""
import numpy as np
import pytest
import torch

from helpers import bits, ensure_lib
from oracle import cache_ops as co
from oracle.numerics import bf16_bits, bf16_round
from test_quant_kv_gpu import TYPES, special_rows

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def P():
    return ensure_lib()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("hkv,d,more", [(8, 128, 0), (8, 128, -1), (8, 128, 1777), (5, 64, 1), (5, 64, -1), (16, 64, 700), (1, 128, 3)])
def test_large_reads(P, fmt, hkv, d, more):
    T = -(-(4 << 20) // (2 * hkv * d * 2)) + more          # tokens whose K and V are 4 MiB, and `more`
    rng = np.random.default_rng(T)
    pages = -(-T // 16)
    table = rng.permutation(pages + 3)[:pages].astype(np.int32)[None]
    g = torch.Generator().manual_seed(T)
    codes = torch.randint(0, 256, (2, 2, pages + 3, 16, hkv, d), dtype=torch.uint8, generator=g)
    scales = torch.exp2(torch.randint(-20, 20, (2, 2, pages + 3, 16, hkv), generator=g).float())
    if fmt == "e4m3":
        codes[(codes & 0x7F) == 0x7F] = 0x3C               # (no NaN codes)
    else:
        scales *= torch.rand(scales.shape, generator=g) + 0.5
    pos = rng.permutation(T).astype(np.int32)
    skip = rng.choice(T, 40, replace=False)
    pos[skip[:20]] = -1
    d_pos, seq = torch.from_numpy(pos).to(DEV), torch.zeros(T, dtype=torch.int32, device=DEV)
    seq[torch.from_numpy(skip[20:]).to(DEV)] = 1           # no such sequence
    back = torch.full((T, (2 * hkv + 3) * d), 3.0, dtype=torch.bfloat16, device=DEV)
    k, v = back[:, d:(hkv + 1) * d].view(T, hkv, d), back[:, (hkv + 2) * d:(2 * hkv + 2) * d].view(T, hkv, d)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    P.pallas_quant_load(codes.to(DEV).view(TYPES[fmt]), scales.to(DEV), 1, k, v, d_pos, torch.from_numpy(table).to(DEV), seq_ids=seq,
                        err=err)
    assert int(err.item()) == 1
    live = np.setdiff1d(np.arange(T), skip)
    pg, slot = table[0, pos[live] // 16], pos[live] % 16
    for kv, got in ((0, k), (1, v)):
        c, s = codes.numpy()[1, kv, pg, slot], scales.numpy()[1, kv, pg, slot]
        want = co.dequantise(c, np.ones_like(s), fmt).astype(np.float32) * s[..., None]          # float32 product
        assert np.array_equal(bits(got)[live], bf16_bits(bf16_round(want.astype(np.float64))))
        assert bool((got[torch.from_numpy(skip).to(DEV)] == 3.0).all())
    k.fill_(3.0)
    v.fill_(3.0)
    assert bool((back == 3.0).all())


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_a_large_round_trip(P, fmt):
    """Rows of every kind, written and read back in one call each."""
    T, hkv, d = 1100, 8, 128
    x = special_rows(T, hkv, d, 7)
    codes = torch.zeros((1, 2, 70, 16, hkv, d), dtype=torch.uint8, device=DEV).view(TYPES[fmt])
    scales = torch.zeros(codes.shape[:-1], device=DEV)
    table = torch.arange(70, dtype=torch.int32, device=DEV).flip(0)[None].contiguous()
    pos, seq = torch.arange(T, dtype=torch.int32, device=DEV), torch.zeros(T, dtype=torch.int32, device=DEV)
    xd = x.to(DEV)
    P.pallas_quant_store(codes, scales, 0, xd, xd, pos, table, seq_ids=seq)
    k, v = torch.empty_like(xd), torch.empty_like(xd)
    P.pallas_quant_load(codes, scales, 0, k, v, pos, table, seq_ids=seq)
    c, s = co.quantise(x.double().numpy(), fmt)
    want = co.dequantise(c, np.ones_like(s), fmt).astype(np.float32) * s[..., None]
    fine = np.isfinite(want)
    assert not fine.all()
    for got in (k, v):
        assert np.array_equal(fine, torch.isfinite(got).cpu().numpy())
        assert np.array_equal(bits(got)[fine], bf16_bits(bf16_round(want.astype(np.float64)))[fine])
