"""The ends of the 8-bit formats: what reads back exactly, and what as an infinity."""
import numpy as np
import pytest
import torch

from helpers import ensure_lib, to_np64
from oracle import cache_ops as co

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


@pytest.fixture(scope="module")
def P():
    return ensure_lib()


def through(P, x, fmt):
    """(codes, scales, K read back, V read back) of rows [T, 1, 64]."""
    T = len(x)
    codes = torch.zeros((1, 2, -(-T // 16), 16, 1, 64), dtype=torch.uint8, device=DEV).view(TYPES[fmt])
    scales = torch.zeros(codes.shape[:-1], device=DEV)
    table = torch.arange(codes.shape[2], dtype=torch.int32, device=DEV)[None]
    pos = torch.arange(T, dtype=torch.int32, device=DEV)
    seq = torch.zeros_like(pos)
    P.pallas_quant_store(codes, scales, 0, x, x, pos, table, seq_ids=seq)
    k, v = torch.empty_like(x), torch.empty_like(x)
    P.pallas_quant_load(codes, scales, 0, k, v, pos, table, seq_ids=seq)
    flat = codes.view(torch.uint8)[0, 0].reshape(-1, 64)[:T].cpu().numpy()
    return flat, scales[0, 0].reshape(-1)[:T].cpu().numpy(), k[:, 0], v[:, 0]


def finite_bf16():
    v = torch.arange(32768, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    return v[torch.isfinite(v)]


def test_e4m3_reads_back_exactly_below_its_last_step(P):
    """Each bf16 magnitude as the largest of a row, with values below it: code * scale is a bf16 value, so that
    nothing is rounded but the code; from 248 * 2^120 on the code is 2^128, which reads back as an infinity."""
    a = finite_bf16()
    x = torch.zeros((len(a), 1, 64), dtype=torch.bfloat16)
    part = 2.0 ** torch.linspace(0, -20, 63)
    x[:, 0, 0] = a
    x[:, 0, 1:] = -(a.float()[:, None] * part)
    codes, scales, k, v = through(P, x.to(DEV), "e4m3")
    want = co.e4m3_value(codes) * scales.astype(np.float64)[:, None]
    over = np.abs(want) >= 2.0 ** 128
    last = to_np64(x[:, 0]) >= 248 * 2.0 ** 120
    assert np.array_equal(over, np.abs(to_np64(x[:, 0])) >= 248 * 2.0 ** 120) and last.any()
    for got in (to_np64(k), to_np64(v)):
        assert np.array_equal(np.isinf(got), over)
        assert np.array_equal(got[~over], want[~over])


def test_int8_reads_back_finite(P):
    a = finite_bf16()
    x = torch.zeros((len(a), 1, 64), dtype=torch.bfloat16)
    x[:, 0, 3] = -a
    codes, scales, k, v = through(P, x.to(DEV), "int8")
    live = to_np64(a) >= 2.0 ** -100
    # a / 127 and its 127-fold round by 2^-24 each: the row's largest value comes back
    for got in (to_np64(k), to_np64(v)):
        assert np.array_equal(got[:, 3], np.where(live, -to_np64(a), 0))
