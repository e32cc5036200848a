"""Operators on the cache, in float64: rotary positions (layouts, partial heads,
long-context scaling), the 8-bit row formats, attention of one new token.

Written from the formulas that ``include/pallas.h`` states.
"""
import math

import numpy as np


# ------------------------------------------------------------------ rotary
def rope_frequencies(r, theta, scaling="none", factor=1.0, trained_len=0, fast=0.0, slow=0.0, magnitude=0.0):
    """Radians per position of the r / 2 pairs, and the factor on the rotated values."""
    f = np.array([theta ** (-2.0 * i / r) for i in range(r // 2)])
    m = 1.0
    if scaling == "linear":
        f = f / factor
    elif scaling == "ntk" and r > 2:
        f = np.array([(theta * factor ** (r / (r - 2.0))) ** (-2.0 * i / r) for i in range(r // 2)])
    elif scaling == "yarn":
        def pair(t):
            return r * math.log(trained_len / (t * 2 * math.pi)) / (2 * math.log(theta))
        a, b = max(math.floor(pair(fast)), 0), min(math.ceil(pair(slow)), r - 1)
        w = np.clip((np.arange(r // 2) - a) / max(b - a, 0.001), 0, 1)
        f = (1 - w) * f + w * f / factor
        m = 0.1 * math.log(factor) + 1
    elif scaling == "bands":
        w = np.clip((trained_len * f / (2 * math.pi) - slow) / (fast - slow), 0, 1)
        f = w * f + (1 - w) * f / factor
    return f, magnitude or m


def rope(x, positions, f, m=1.0, layout="half", inverse=False):
    """x [T, heads, d]; the first 2 len(f) elements of a head turn, as complex numbers."""
    x = np.asarray(x, dtype=np.float64)
    r = 2 * len(f)
    lo, hi = (np.arange(0, r // 2), np.arange(r // 2, r)) if layout == "half" else (np.arange(0, r, 2), np.arange(1, r, 2))
    turn = np.exp(1j * np.asarray(positions, dtype=np.float64)[:, None] * f[None])[:, None]
    turn = turn.conj() / m if inverse else turn * m
    z = (x[..., lo] + 1j * x[..., hi]) * turn
    y = x.copy()
    y[..., lo], y[..., hi] = z.real, z.imag
    return y


# ------------------------------------------------------------------ 8-bit rows
def e4m3_value(code):
    """Value of an OCP E4M3 code: sign, 4 exponent bits (bias 7), 3 mantissa bits; no infinities."""
    code = np.asarray(code).astype(np.int64)
    e, man = (code >> 3) & 15, code & 7
    v = np.where(e == 0, man * 2.0 ** -9, (8 + man) * 2.0 ** (e - 10.0))
    v = np.where((code & 0x7F) == 0x7F, np.nan, v)
    return np.where(code & 0x80, -v, v)


_E4M3 = e4m3_value(np.arange(0x7F))      # ascending, 0 .. 448


def e4m3_code(y):
    """Nearest E4M3 code of |y| <= 448, ties to the even code."""
    a = np.abs(y)
    hi = np.clip(np.searchsorted(_E4M3, a), 0, 0x7E)
    lo = np.maximum(hi - 1, 0)
    below, above = a - _E4M3[lo], _E4M3[hi] - a
    code = np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    return (code | np.where(np.signbit(y), 0x80, 0)).astype(np.uint8)


def quantise(x, fmt):
    """(codes uint8, scales float32) of the rows of x (float64 values of bf16)."""
    x = np.asarray(x, dtype=np.float64)
    bad = ~np.isfinite(x).all(axis=-1)
    x = np.where(bad[..., None], 0.0, x)
    a = np.abs(x).max(axis=-1)
    if fmt == "int8":
        live = a >= 2.0 ** -100
        a32 = np.where(live, a, 1.0).astype(np.float32)
        up = np.float32(127) / a32                                  # float32, as stated
        y = x.astype(np.float32) * up[..., None]
        codes = np.where(live[..., None], np.clip(np.rint(y), -127, 127), 0).astype(np.int8).view(np.uint8)
        scale = np.where(live, a32 / np.float32(127), np.float32(0))
    else:
        live = a > 0
        e = np.maximum(np.ceil(np.log2(np.where(live, a, 1.0) / 448.0)), -126)
        e = np.where(np.ldexp(448.0, e.astype(int) - 1) >= np.where(live, a, np.inf), e - 1, e)   # (log2 rounded up)
        e = np.maximum(e, -126).astype(int)
        codes = np.where(live[..., None], e4m3_code(np.ldexp(x, -e[..., None])), 0).astype(np.uint8)
        scale = np.where(live, np.ldexp(1.0, e), 0.0)
    return codes, np.where(bad, np.nan, scale).astype(np.float32)


def dequantise(codes, scales, fmt):
    v = codes.view(np.int8).astype(np.float64) if fmt == "int8" else e4m3_value(codes)
    return v * np.asarray(scales, dtype=np.float64)[..., None]


# ------------------------------------------------------------------ attention
def attend(q, k, v, scale):
    """One query per head over keys [n, Hkv, d]: (out [Hq, d], lse [Hq], sum of p |v|, largest
    scale sum |q_i k_i| of a key)."""
    hq, d = q.shape
    n, hkv, _ = k.shape
    out, mag = np.zeros((hq, d)), np.zeros((hq, d))
    lse, terms = np.full(hq, -np.inf), np.zeros(hq)
    if n == 0:
        return out, lse, mag, terms
    for h in range(hq):
        kh = h // (hq // hkv)
        z = scale * (k[:, kh] @ q[h])
        top = z.max()
        p = np.exp(z - top)
        lse[h] = top + math.log(p.sum())
        p /= p.sum()
        out[h], mag[h] = p @ v[:, kh], p @ np.abs(v[:, kh])
        terms[h] = abs(scale) * (np.abs(k[:, kh]) @ np.abs(q[h])).max()
    return out, lse, mag, terms
