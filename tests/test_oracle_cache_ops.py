"""Pins of the cache operators' oracle: the 8-bit formats against every bf16 value
and torch's own cast, rotary against closed forms, attention against a plain
softmax."""
import math

import numpy as np
import pytest
import torch

from oracle import cache_ops as co


def all_bf16():
    v = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).double().numpy()
    return v[np.isfinite(v)]


def test_e4m3_codes_against_cast():
    v = all_bf16()
    v = v[np.abs(v) <= 448]
    want = torch.tensor(v).to(torch.float32).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(co.e4m3_code(v), want)
    codes = np.arange(256, dtype=np.uint8)
    vals = torch.tensor(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(co.e4m3_value(codes), vals, equal_nan=True)


def test_e4m3_scale_is_the_least_power_of_two():
    v = all_bf16()
    v = v[v > 0]
    codes, scale = co.quantise(v[:, None], "e4m3")
    s = scale.astype(np.float64)
    assert np.all(np.frexp(s)[0] == 0.5)
    assert np.all(v <= 448 * s)
    assert np.all((v > 448 * s / 2) | (s == 2.0 ** -126))
    # one code in the upper binade: within half a step, 2^-4 relative, or half the least code
    back = co.dequantise(codes, scale, "e4m3")[:, 0]
    assert np.all(np.abs(back - v) <= np.maximum(v * 2.0 ** -4, s * 2.0 ** -10))


def test_int8_rows():
    x = np.array([[1.0, -0.5, 0.25, 0.0], [0, 0, 0, 0], [2.0 ** -101, 0, 0, 0], [np.inf, 1, 2, 3], [np.nan, 0, 0, 0]])
    codes, scale = co.quantise(x, "int8")
    assert codes.view(np.int8)[0].tolist() == [127, -64, 32, 0]          # 63.5 and 31.75: ties to even, nearest
    assert scale[0] == np.float32(1) / np.float32(127)
    assert not codes[1:].any() and scale[1] == 0 and scale[2] == 0 and np.isnan(scale[3:]).all()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_turns(layout):
    rng = np.random.default_rng(0)
    x = rng.standard_normal((4, 3, 20))
    f, m = co.rope_frequencies(12, 1e4)
    pos = np.array([0, 1, 77, -5])
    y = co.rope(x, pos, f, m, layout)
    assert np.array_equal(y[0], x[0]) and np.array_equal(y[..., 12:], x[..., 12:])
    i, p, t = 2, 77, 2
    a, b = (i, i + 6) if layout == "half" else (2 * i, 2 * i + 1)
    ang = p * 1e4 ** (-2 * i / 12)
    assert np.allclose(y[t, 1, a], x[t, 1, a] * math.cos(ang) - x[t, 1, b] * math.sin(ang))
    assert np.allclose(y[t, 1, b], x[t, 1, b] * math.cos(ang) + x[t, 1, a] * math.sin(ang))
    assert np.allclose(co.rope(y, pos, f, 1.0, layout, inverse=True), x)
    # scores depend on the difference of positions alone
    u, w = rng.standard_normal((1, 1, 12)), rng.standard_normal((1, 1, 12))
    def score(p, q):
        return (co.rope(u, [p], f, 1.0, layout) * co.rope(w, [q], f, 1.0, layout)).sum()
    assert np.isclose(score(3, 10), score(103, 110))


def test_rope_scalings():
    f, _ = co.rope_frequencies(64, 1e4)
    assert np.allclose(co.rope_frequencies(64, 1e4, "linear", 4.0)[0] * 4, f)
    ntk = co.rope_frequencies(64, 1e4, "ntk", 4.0)[0]
    assert np.isclose(ntk[0], f[0]) and np.isclose(ntk[-1], f[-1] / 4)     # first kept, last as linear
    for kind, fast, slow in (("yarn", 32.0, 1.0), ("bands", 4.0, 1.0)):
        g, m = co.rope_frequencies(64, 1e4, kind, 4.0, 4096, fast, slow)
        ratio = g / f
        assert np.isclose(ratio[0], 1) and np.isclose(ratio[-1], 0.25) and np.all(np.diff(ratio) <= 1e-12)
        assert np.isclose(m, 0.1 * math.log(4) + 1 if kind == "yarn" else 1)
        turns = 4096 * f / (2 * math.pi)
        if kind == "bands":
            assert np.allclose(ratio[turns >= 4], 1) and np.allclose(ratio[turns <= 1], 0.25)
    assert co.rope_frequencies(64, 1e4, "yarn", 4.0, 4096, 32.0, 1.0, magnitude=1.5)[1] == 1.5


def test_attend_plain():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((4, 8)), rng.standard_normal((5, 2, 8)), rng.standard_normal((5, 2, 8))
    out, lse, _, _ = co.attend(q, k, v, 0.3)
    z = 0.3 * np.einsum("hd,nhd->hn", q, np.repeat(k, 2, axis=1))
    p = np.exp(z) / np.exp(z).sum(1, keepdims=True)
    assert np.allclose(out, np.einsum("hn,nhd->hd", p, np.repeat(v, 2, axis=1)))
    assert np.allclose(lse, np.log(np.exp(z).sum(1)))
    out, lse, _, _ = co.attend(q, k[:0], v[:0], 0.3)
    assert not out.any() and np.all(lse == -np.inf)
