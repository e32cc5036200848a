"""Sine and cosine of pallas_rope_apply are within 2^-23 of those of the exact angle, at every
position: pairs (x0, x1) whose first result nearly cancels, so that bf16 hides nothing.

  |y0 - (x0 cos a - x1 sin a)| <= 2^-8 |y0| + 2^-22 (|x0| + |x1|)
(2^-23 of the sum for the sine and the cosine, 2^-24 of each product and of their difference,
each at most that sum's larger part.)  The angle p turns_i 2^-64 is taken in integers, and its
last turn in 53 bits."""
import numpy as np
import pytest
import torch

from helpers import ensure_lib, to_np64

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def P():
    return ensure_lib()


def angles(plan, positions):
    """Radians, [positions, pairs], within 2^-50."""
    part = [[(int(p) * int(t)) % (1 << 64) for t in plan.turns[:plan.rotary_dim // 2]] for p in positions]
    return np.array([[a / 2.0 ** 64 for a in row] for row in part]) * (2 * np.pi)


def cancelling(a):
    """bf16 integers x0, x1 up to 255 in size with x0 cos a - x1 sin a as near to zero as it gets."""
    c, s = np.abs(np.cos(a)), np.abs(np.sin(a))
    best, x0, x1 = np.full(a.shape, np.inf), np.zeros(a.shape), np.zeros(a.shape)
    for k in range(1, 256):
        for u, v in ((np.full(a.shape, float(k)), np.rint(k * c / s)), (np.rint(k * s / c), np.full(a.shape, float(k)))):
            off = np.where(np.maximum(u, v) <= 255, np.abs(u * c - v * s) / (u + v), np.inf)
            better = off < best
            best, x0, x1 = np.where(better, off, best), np.where(better, u, x0), np.where(better, v, x1)
    return x0 * np.sign(np.sin(a)), x1 * np.sign(np.cos(a))


@pytest.mark.parametrize("layout,r", [("half", 128), ("interleaved", 128), ("half", 54)])
def test_sine_and_cosine(P, layout, r):
    rng = np.random.default_rng(5)
    pos = np.concatenate([np.arange(1, 40), rng.integers(40, 1 << 20, 60), rng.integers(1 << 20, 1 << 31, 60),
                          -rng.integers(1, 1 << 31, 60), [2 ** 31 - 1, -2 ** 31, 1 << 24, (1 << 24) + 1]]).astype(np.int32)
    plan = P.pallas_rope_init(r, 1e6, layout)
    a = angles(plan, pos)
    x0, x1 = cancelling(a)
    x = np.zeros((len(pos), 1, r))
    lo, hi = (slice(0, r // 2), slice(r // 2, r)) if layout == "half" else (slice(0, r, 2), slice(1, r, 2))
    x[:, 0, lo], x[:, 0, hi] = x0, x1
    t = torch.from_numpy(x).to(torch.bfloat16).to(DEV)
    assert np.array_equal(to_np64(t), x)
    got = to_np64(P.pallas_rope_apply(plan, t, torch.from_numpy(pos).to(DEV), torch.empty_like(t)))[:, 0, lo]
    want = x0 * np.cos(a) - x1 * np.sin(a)
    size = np.abs(x0) + np.abs(x1)
    off = (np.abs(got - want) - 2.0 ** -8 * np.abs(want)) / size
    assert off.max() <= 2.0 ** -22, float(np.log2(off.max()))
    # (the inputs do cancel, where neither part is alone)
    assert np.median(np.abs(want) / size) < 2.0 ** -14
