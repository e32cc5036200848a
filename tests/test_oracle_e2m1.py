"""Pins of the oracle's 4-bit rows: the values of the codes, rounding at the halfway
points, the scale at its borders, and the error that a value may have."""
import numpy as np

from oracle import cache_ops as co


def test_codes():
    assert co.e2m1_code(co.E2M1).tolist() == list(range(8))
    assert co.e2m1_code(-co.E2M1).tolist() == list(range(8, 16))
    half = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    assert co.E2M1[co.e2m1_code(half)].tolist() == [0, 1, 1, 2, 2, 4, 4]      # the even code
    assert co.e2m1_code(np.nextafter(half, 9)).tolist() == [1, 2, 3, 4, 5, 6, 7]
    assert co.e2m1_code(np.nextafter(half, 0)).tolist() == [0, 1, 2, 3, 4, 5, 6]
    assert co.e2m1_code(np.array([7.9, -1e9, -0.0])).tolist() == [7, 15, 8]


def test_scales_and_layout():
    x = np.zeros((7, 16))
    x[0, :4] = [6, -3, 0.5, 0]                # fits at 1
    x[1, :4] = [6.03125, 0, 0, 0]             # just does not
    x[2, :4] = [2.0 ** -100, 0, 0, 0]
    x[3, :4] = [2.0 ** -101, 0, 0, 0]
    x[4, :4] = [2.0 ** 127 * 1.9921875, 2.0 ** 126, 0, 0]
    x[5, :4] = [np.inf, 1, 1, 1]
    x[6, 12:] = [0, np.nan, 0, 0]
    c, b = co.quantise4(x)
    assert b[:, 0].tolist() == [127, 128, 127 - 102, 0, 252, 255, 0] and b[6, 3] == 255
    assert c[0, :2].tolist() == [7 | (8 | 5) << 4, 1] and c[1, 0] == 5        # 3.015625 -> 3
    assert c[2, 0] == 6 and c[3, 0] == 0 and c[4, 0] == 7 | 4 << 4           # 2^-100 = 4 2^-102; 7.97 -> 6; 2^126 = 2 2^125
    assert c[5, 0] == 0 and not c[6].any()
    v = co.dequantise4(c, b)
    assert np.isnan(v[5, :4]).all() and np.isnan(v[6, 12:]).all() and np.isfinite(v[:5]).all()
    assert v[0, :4].tolist() == [6, -3, 0.5, 0] and v[4, 0] == 6 * 2.0 ** 125


def test_error_is_half_a_step():
    x = np.random.default_rng(0).standard_normal((200, 128)) * np.exp(np.random.default_rng(1).standard_normal((200, 1)))
    c, b = co.quantise4(x)
    v, unit = co.dequantise4(c, b), np.repeat(np.ldexp(1.0, b.astype(int) - 127), 32, axis=-1)
    y = np.abs(x) / unit
    step = np.where(y <= 2, 0.5, np.where(y <= 4, 1.0, 2.0))
    assert (y <= 6).all() and (np.abs(v - x) / unit <= step / 2).all()
    # the least scale that fits
    assert (np.abs(x).reshape(200, 4, 32).max(-1) > 3 * np.ldexp(1.0, b.astype(int) - 127)).all()
