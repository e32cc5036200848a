"""Attention's weights keep their 24 bits on the way into the second product.

Two keys per row whose weighted values cancel, so that an error of a weight is seen beside a
small output.  Scores are single products of bf16 values, |score| <= 1/2, so the score in
log2 units is off by two roundings of at most 2^-24 of 0.73, the difference of two such by one
more of 2^-24: together 2^-22.2, in the weight 2^-22.7; exp2 2^-23; the product with the row's
scale, and two additions, 2^-24 each: below 2^-21 of sum p |v|.
  |out - ref| <= 2^-8 |ref| + 2^-20 sum_j p_j |v_j|
(Weights of 16 bits would be up to 2^-17 off: 2^-18 of that sum here.)"""
import numpy as np
import pytest
import torch

from attend_forms import check_form, fresh_workspace
from helpers import ensure_lib, to_np64
from oracle import cache_ops as co

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


@pytest.fixture(scope="module")
def P():
    return ensure_lib()


def cancelling(ratio):
    """Integers (a, b) up to 255 with a ratio - b as near to zero as it gets, relative to their size."""
    a = np.arange(1, 256)
    b = np.clip(np.rint(a * ratio), 1, 255)
    i = int(np.argmin(np.abs(a * ratio - b) / (a * ratio + b)))
    return int(a[i]), int(b[i])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("form,S,max_length", [("short", 64, 512), ("split", 4, 600), ("ranges", 64, 20000)])
@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
def test_weights_that_cancel(P, fmt, form, S, max_length, d):
    hkv, scale = 8, 0.125
    if form == "split" and d == 64 and fmt != "bf16":
        max_length = 300 * 8      # (more keys to a split)
    rng = np.random.default_rng(d)
    q = torch.zeros((S, hkv, d), dtype=torch.bfloat16)
    q[:, :, 1] = torch.from_numpy(rng.uniform(0.5, 4.0, (S, hkv))).to(torch.bfloat16)
    # K: a multiple of 1/16 below 1, in every format; scores 0.125 * 4 * 1 at most
    t = rng.integers(-15, 16, (S, 2, hkv)) / 16.0
    z = scale * to_np64(q)[:, None, :, 1] * t
    p = np.exp(z - z.max(axis=1, keepdims=True))
    k, v = np.zeros((2, S, 2, hkv, d))
    k[..., 1] = t
    vs = np.ones((S, 2, hkv), dtype=np.float32)
    if fmt == "bf16":
        for s in range(S):
            for h in range(hkv):
                a, b = cancelling(p[s, 0, h] / p[s, 1, h])
                v[s, 0, h], v[s, 1, h] = a, -b
    else:
        a, b = rng.integers(8, 16, (2, S, hkv)) if fmt == "e4m3" else rng.integers(60, 128, (2, S, hkv))
        vs[:, 1] = (p[:, 0] * a / (p[:, 1] * b)).astype(np.float32)
        v[:, 0], v[:, 1] = a[..., None], -(b * vs[:, 1].astype(np.float64))[..., None]
    table = torch.arange(S, dtype=torch.int32, device=DEV)[:, None].repeat(1, -(-max_length // 16)).contiguous()
    lengths = torch.full((S,), 2, dtype=torch.int32, device=DEV)
    ws = fresh_workspace(P, S, hkv, hkv, d, max_length)
    q = q.to(DEV)
    out, lse = torch.empty_like(q), torch.empty((S, hkv), dtype=torch.float32, device=DEV)
    if fmt == "bf16":
        pool = torch.full((1, 2, S, 16, hkv, d), float("nan"), dtype=torch.bfloat16)
        pool[0, 0, :, :2], pool[0, 1, :, :2] = torch.from_numpy(k).to(torch.bfloat16), torch.from_numpy(v).to(torch.bfloat16)
        P.pallas_attend_kv(pool.to(DEV), 0, q, lengths, max_length, table, scale, out, ws, lse=lse)
    else:
        codes = np.zeros((1, 2, S, 16, hkv, d), dtype=np.uint8)
        scales = np.full((1, 2, S, 16, hkv), np.nan, dtype=np.float32)
        def code(x):
            return co.e4m3_code(x.astype(np.float64)) if fmt == "e4m3" else x.astype(np.int8).view(np.uint8)
        codes[0, 0, :, :2] = code(k * 16)
        codes[0, 1, :, 0], codes[0, 1, :, 1] = code(a)[..., None], code(-b)[..., None]
        scales[0, 0, :, :2], scales[0, 1, :, :2] = 1 / 16, vs
        P.pallas_attend_quant(torch.from_numpy(codes).to(DEV).view(TYPES[fmt]), torch.from_numpy(scales).to(DEV), 0, q, lengths,
                              max_length, table, scale, out, ws, lse=lse)
    check_form(form, ws, fmt, d, hkv, hkv, [2] * S, max_length)
    got = to_np64(out)
    w = (p / p.sum(axis=1, keepdims=True))[..., None]
    ref, mag = (w * v).sum(axis=1), (w * np.abs(v)).sum(axis=1)
    assert np.all(np.abs(ref) <= 2.0 ** -11 * mag)
    worst = (np.abs(got - ref) - 2.0 ** -8 * np.abs(ref)) / mag
    assert worst.max() <= 2.0 ** -20, float(np.log2(worst.max()))
