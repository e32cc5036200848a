"""How near appended rotations come to the exact ones, where the two products of a pair cancel.

y = m (x0 cos a - x1 sin a), a = 2 pi p f: the plan holds f in units of 2^-64 of a turn, rounded down, so a is off by up
to p 2^-64 turns < p 2^-61; the kernel's sine and cosine add less than 2^-49, its products and their sum
in 64 bits 2^-51.  With p 2^-61 + 2^-48 of m (|x0| + |x1|) for all of these, float32 and bf16 add half a step each:
2^-24 and 2^-8 of the result."""
import math

import numpy as np
import pytest
import torch

from helpers import ensure_lib, to_np64

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def P():
    return ensure_lib()


def inverse_of_two_pi(bits):
    """floor(2^bits / (2 pi)), pi = 16 atan(1/5) - 4 atan(1/239) in whole numbers."""
    one = 1 << (bits + 40)

    def atan_inverse(n):
        total = term = one // n
        k = 1
        while term:
            term //= -n * n
            k += 2
            total += term // k
        return total

    pi = 16 * atan_inverse(5) - 4 * atan_inverse(239)
    return (1 << bits) * one // (2 * pi)


def cancelling(high, count, seed):
    """Positions below `high` and bf16 pairs (x0, x1), frequency 1, whose turned first element nearly vanishes:
    (position, x0, x1, exact first element), the nearest `count` of many tried."""
    rng = np.random.default_rng(seed)
    pos = rng.integers(high // 2, high, 400000)
    unit = inverse_of_two_pi(160)
    angle = np.array([math.ldexp(((int(p) * unit) & ((1 << 160) - 1)) >> 96, -64) for p in pos]) * (2 * math.pi)
    # x0 cos a = x1 sin a: the bf16 ratio nearest to tan a, of 8-bit whole numbers
    tan = np.tan(angle)
    best = np.full(len(pos), np.inf)
    x0, x1 = np.zeros(len(pos)), np.zeros(len(pos))
    for m in range(128, 256):
        n = np.clip(np.rint(m * np.abs(tan)), 128, 255)
        y = np.abs(n * np.cos(angle) - np.copysign(m, tan) * np.sin(angle))
        at = y < best
        best, x0, x1 = np.where(at, y, best), np.where(at, n, x0), np.where(at, np.copysign(m, tan), x1)
    near = np.argsort(best)[:count]
    # (In 64 bits: angles to 2^-50, so this value to 2^-40 for pairs of 2^8.)
    return pos[near], x0[near], x1[near], (x0 * np.cos(angle) - x1 * np.sin(angle))[near]


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("high", [1 << 31, 1 << 24, 1 << 17])
def test_where_a_pair_cancels(P, layout, high):
    d, n = 64, 512
    pos, x0, x1, exact = cancelling(high, n, seed=1)
    first, second = (0, 32) if layout == "half" else (0, 1)
    q = torch.zeros((n, 1, d), dtype=torch.bfloat16)
    q[:, 0, first], q[:, 0, second] = torch.from_numpy(x0).to(torch.bfloat16), torch.from_numpy(x1).to(torch.bfloat16)
    assert np.array_equal(to_np64(q)[:, 0, first], x0) and np.array_equal(to_np64(q)[:, 0, second], x1)
    q = q.to(DEV)
    out, kv = torch.empty_like(q), torch.zeros_like(q)
    pool = torch.zeros((1, 2, 1, 16, 1, d), dtype=torch.bfloat16, device=DEV)
    table = torch.zeros((1, 1), dtype=torch.int32, device=DEV)
    # (The positions lie beyond the table: queries alone are written.)
    P.pallas_append_kv(P.pallas_rope_init(d, 1e4, layout=layout), pool, 0, kv, kv, torch.from_numpy(pos).to(torch.int32).to(DEV),
                       table, q=q, q_out=out, seq_ids=torch.zeros(n, dtype=torch.int32, device=DEV))
    off = np.abs(to_np64(out)[:, 0, first] - exact)
    pair = np.abs(x0) + np.abs(x1)
    assert np.all(off <= (2.0 ** -8 + 2.0 ** -24) * np.abs(exact) + (pos * 2.0 ** -61 + 2.0 ** -48) * pair + 2.0 ** -40)
    # the nearest pairs are such that a term in the pair's magnitudes is needed at far positions
    assert high < 1 << 31 or np.any(off > 2.0 ** -7 * np.abs(exact))
