"""Operators on the cache, in float64: rotary positions (layouts, partial heads,
long-context scaling), the 8- and 4-bit row formats, attention of one new token, the
selection of blocks.

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


# ------------------------------------------------------------------ 4-bit rows
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])      # sign apart: 2 exponent bits (bias 1), 1 mantissa bit


def e2m1_code(y):
    """Nearest E2M1 code (4 bits), ties to the even code; |y| beyond 6 is 6."""
    away = np.abs(np.abs(y)[..., None] - E2M1)
    best = away == away.min(axis=-1, keepdims=True)                # one, or two neighbours
    even = best & (np.arange(8) % 2 == 0)
    return np.where(even.any(axis=-1), even.argmax(axis=-1), best.argmax(axis=-1)) | np.where(np.signbit(y), 8, 0)


def quantise4(x):
    """(codes uint8 [.., d / 2], bytes uint8 [.., 4]) of the rows of x (float64 values of bf16): element 2 i in the low
    half of byte i, a power of two 2^(byte - 127) per quarter of the row."""
    x = np.asarray(x, dtype=np.float64)
    d = x.shape[-1]
    x = x.reshape(x.shape[:-1] + (4, d // 4))
    bad = ~np.isfinite(x).all(axis=-1)
    x = np.where(bad[..., None], 0.0, x)
    a = np.abs(x).max(axis=-1)
    live = a >= 2.0 ** -100
    e = np.full(a.shape, 125)
    for k in range(124, -104, -1):                                # the least that fits
        e = np.where((e == k + 1) & (a <= np.ldexp(6.0, k)), k, e)
    codes = np.where(live[..., None], e2m1_code(np.ldexp(x, -e[..., None])), 0).reshape(x.shape[:-2] + (d,))
    unit = np.where(bad, 255, np.where(live, e + 127, 0)).astype(np.uint8)
    return (codes[..., 0::2] | codes[..., 1::2] << 4).astype(np.uint8), unit


def dequantise4(codes, unit):
    d = 2 * codes.shape[-1]
    both = np.stack([codes & 15, codes >> 4], axis=-1).reshape(codes.shape[:-1] + (4, d // 4)).astype(np.int64)
    v = np.where(both & 8, -E2M1[both & 7], E2M1[both & 7])
    scale = np.where(unit == 255, np.nan, np.ldexp(1.0, unit.astype(np.int64) - 127))
    return (v * scale[..., None]).reshape(codes.shape[:-1] + (d,))


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


# ------------------------------------------------------------------ blocks
def steps(x):
    """(whole numbers of at most 127, float32 step) of the rows of x, which float32 holds; the products are float32
    ones, as stated."""
    x = np.asarray(x, dtype=np.float64)
    bad = ~np.isfinite(x).all(axis=-1)
    x = np.where(bad[..., None], 0.0, x)
    a = np.abs(x).max(axis=-1).astype(np.float32)
    live = a >= np.float32(2.0 ** -100)
    a = np.where(live, a, np.float32(1))
    with np.errstate(under="ignore"):
        y = x.astype(np.float32) * (np.float32(127) / a)[..., None]
    codes = np.where(live[..., None], np.clip(np.rint(y), -127, 127), 0).astype(np.int64)
    return codes, np.where(bad, np.float32(np.nan), np.where(live, a / np.float32(127), np.float32(0)))


def block_bounds(k):
    """(codes [blocks, Hkv, 2, d], steps [blocks, Hkv]) of keys k [n, Hkv, d] by blocks of 16."""
    n, hkv, d = k.shape
    both = np.zeros((-(-n // 16), hkv, 2, d))
    for j in range(len(both)):
        part = k[16 * j:16 * j + 16]
        both[j, :, 0], both[j, :, 1] = part.max(axis=0), part.min(axis=0)      # (NaN stays)
    codes, step = steps(both.reshape(len(both), hkv, 2 * d))
    return codes.reshape(both.shape), step


def block_scores(q, codes, step):
    """float32 [Hkv, blocks]: q [Hq, d] against bounds."""
    blocks, hkv = step.shape
    c, t = steps(q)
    group = len(q) // hkv
    out = np.empty((hkv, blocks), dtype=np.float32)
    for h in range(hkv):
        per = []
        for g in range(h * group, (h + 1) * group):
            dot = np.where(c[g] > 0, c[g] * codes[:, h, 0], c[g] * codes[:, h, 1]).sum(axis=-1)
            per.append(dot.astype(np.float32) * step[:, h] * t[g])
        out[h] = np.max(per, axis=0)                                            # (NaN stays)
    return out


def select_blocks(scores, budget, first, last):
    """Ascending lists [Hkv][<= budget] of the blocks: `first` first and `last` last ones, then the highest scores (NaN
    above all), of equal ones the earliest."""
    lists = []
    for row in scores:
        n = len(row)
        always = [j for j in range(n) if j < first or j >= n - last]
        key = np.where(np.isnan(row), np.inf, row)
        rest = sorted((j for j in range(n) if j not in set(always)), key=lambda j: (not np.isnan(row[j]), -key[j], j))
        lists.append(sorted((always + rest)[:budget]) if n > budget else list(range(n)))
    return lists
