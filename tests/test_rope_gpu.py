"""pallas_rope_apply against the oracle: layouts, partial heads, scalings, strides,
sizes around a workgroup's share, positions to the ends of int32.

Tolerance: one rounding to bf16, 2^-8 of the value, and the float32 arithmetic: the
sine and cosine are within 2^-22 (polynomials, 2^-31 turn of the angle; the oracle's
own angle within 2^-21 at the far end), each product and the sum round by 2^-24:
together below 2^-20 m (|x0| + |x1|)."""
import numpy as np
import pytest
import torch

from helpers import ensure_lib, to_np64
from oracle import cache_ops as co

pytestmark = pytest.mark.gpu
DEV = "cuda"
SCALED = {"none": dict(), "linear": dict(scaling="linear", factor=4.0), "ntk": dict(scaling="ntk", factor=8.0),
          "yarn": dict(scaling="yarn", factor=8.0, trained_len=4096, fast=32.0, slow=1.0),
          "bands": dict(scaling="bands", factor=8.0, trained_len=8192, fast=4.0, slow=1.0)}
SENTINEL = 0x7FA5


@pytest.fixture(scope="module")
def P():
    return ensure_lib()


def rows(T, H, d, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn((T, H, d), generator=g).to(torch.bfloat16).to(DEV)


def check(got, x, pos, plan_kw, r, theta, layout, inverse=False):
    f, m = co.rope_frequencies(r, theta, **{"scaling": "none", **plan_kw})
    want = co.rope(to_np64(x), pos.cpu().numpy(), f, m, layout, inverse)
    lo, hi = (np.arange(r // 2), np.arange(r // 2, r)) if layout == "half" else (np.arange(0, r, 2), np.arange(1, r, 2))
    tol = 2.0 ** -8 * np.abs(want)
    size = np.abs(to_np64(x)) * (1 / m if inverse else m)
    both = 2.0 ** -20 * (size[..., lo] + size[..., hi])
    tol[..., lo] += both
    tol[..., hi] += both
    diff = np.abs(to_np64(got) - want)
    assert np.all(diff <= tol), float((diff - tol).max())
    assert torch.equal(got[..., r:], x[..., r:])


CASES = [
    # tokens, heads, head_dim, rotary_dim, layout, scaling
    (1, 1, 64, 64, "half", "none"), (1, 72, 128, 128, "half", "yarn"), (3, 40, 128, 32, "interleaved", "bands"),
    (17, 5, 80, 54, "half", "ntk"), (17, 5, 80, 54, "interleaved", "linear"), (5, 3, 7, 2, "half", "none"),
    (5, 3, 9, 6, "interleaved", "none"), (33, 16, 96, 96, "half", "linear"), (33, 17, 256, 256, "interleaved", "yarn"),
    (2, 80, 256, 64, "half", "bands"), (513, 9, 128, 64, "half", "ntk"), (600, 70, 64, 24, "half", "none"),
    (1000, 1, 128, 128, "interleaved", "yarn"), (130, 2, 96, 24, "interleaved", "none"), (2, 3, 2050, 16, "half", "none"),
    (2, 2, 2056, 256, "half", "none"),
]


@pytest.mark.parametrize("T,H,d,r,layout,scaling", CASES)
def test_against_oracle(P, T, H, d, r, layout, scaling):
    x = rows(T, H, d, T + H + d)
    pos = torch.randint(0, 200000, (T,), dtype=torch.int32, generator=torch.Generator().manual_seed(1)).to(DEV)
    kw = SCALED[scaling]
    plan = P.pallas_rope_init(r, 1e6, layout, **kw)
    out = torch.empty_like(x)
    keep = x.clone()
    P.pallas_rope_apply(plan, x, pos, out)
    assert torch.equal(x, keep)
    check(out, x, pos, kw, r, 1e6, layout)
    # in place: the same bits
    P.pallas_rope_apply(plan, keep, pos)
    assert torch.equal(keep, out)
    # and back
    P.pallas_rope_apply(plan, keep, pos, inverse=True)
    check(keep, out, pos, kw, r, 1e6, layout, inverse=True)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("offset,width", [(0, 20), (8, 21), (1, 20), (4, 20)])
def test_strides_and_neighbours(P, layout, offset, width):
    """Heads in the middle of wider rows, aligned and not; nothing beside them is written."""
    T, H, d, r = 37, 5, 64, 48
    flat = torch.empty(T * width * d + 64, dtype=torch.bfloat16, device=DEV)
    flat.view(torch.int16).fill_(SENTINEL)
    x = torch.as_strided(flat, (T, H, d), (width * d, 2 * d, 1), offset)
    src = rows(T, H, d, 5)
    x.copy_(src)
    pos = torch.arange(T, dtype=torch.int32, device=DEV) * 991
    plan = P.pallas_rope_init(r, 1e4, layout)
    whole = flat.clone()
    P.pallas_rope_apply(plan, x, pos)
    check(x, src, pos, {}, r, 1e4, layout)
    torch.as_strided(whole, (T, H, d), (width * d, 2 * d, 1), offset).copy_(x)
    assert torch.equal(whole.view(torch.int16), flat.view(torch.int16))
    # heads-first output
    out = torch.empty((H, T, d), dtype=torch.bfloat16, device=DEV).transpose(0, 1)
    P.pallas_rope_apply(plan, src, pos, out)
    assert torch.equal(out, x)


def test_far_and_negative_positions(P):
    pos = torch.tensor([0, -1, 2 ** 31 - 1, -2 ** 31, 1 << 24, (1 << 24) + 1, 131071, -77777], dtype=torch.int32, device=DEV)
    x = rows(len(pos), 4, 128, 9)
    plan = P.pallas_rope_init(128, 1e6)
    out = P.pallas_rope_apply(plan, x, pos, torch.empty_like(x))
    check(out, x, pos, {}, 128, 1e6, "half")
    assert torch.equal(out[0], x[0])


def test_one_row_many_heads_and_broadcast(P):
    """A head stride of 0 on the input: one head to many."""
    x = rows(6, 1, 128, 3)
    out = torch.empty((6, 9, 128), dtype=torch.bfloat16, device=DEV)
    pos = torch.arange(6, dtype=torch.int32, device=DEV)
    plan = P.pallas_rope_init(128, 1e6)
    P.pallas_rope_apply(plan, x.expand(6, 9, 128), pos, out)
    one = P.pallas_rope_apply(plan, x, pos, torch.empty_like(x))
    assert torch.equal(out, one.expand(6, 9, 128))


def test_non_finite_values_stay_in_their_pairs(P):
    x = torch.ones((1, 1, 64), dtype=torch.bfloat16, device=DEV)
    x[0, 0, 3], x[0, 0, 40] = float("nan"), float("inf")
    y = P.pallas_rope_apply(P.pallas_rope_init(64, 1e4), x, torch.tensor([7], dtype=torch.int32, device=DEV),
                            torch.empty_like(x))[0, 0]
    bad = ~torch.isfinite(y)
    assert bad.nonzero().flatten().tolist() == [3, 8, 35, 40]
