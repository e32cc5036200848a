"""Attention in a workspace of what the call itself uses: over bf16 and 8-bit rows that is no more than
their own number of ranges asks for, which the size for any cache may exceed."""
import pytest
import torch

from helpers import ensure_lib
from test_blocks_gpu import DEV, Cache, queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    return ensure_lib()


def own_size(row_bytes, S, hq, hkv, d, max_length):
    """The rule, restated: two words a row, then, of each range and row that meet, d + 2 floats a query head."""
    ranges = max(256 * (1024 // row_bytes) // (hkv * -(-(hq // hkv) // 16)) // 8 * 8, 8)
    total = S * -(-max_length // 32)
    records = min(total, ranges + total // 32) + S
    at = -(-S * 8 // 256) * 256
    return -(-(at + records * hq * (d + 2) * 4) // 256) * 256


CASES = [([9000, 40, 0, 5000, 700] * 3, 16, 8, 128), ([40000], 64, 8, 128), ([2000] * 70, 8, 2, 64), ([70, 30] * 900, 4, 4, 128)]


@pytest.mark.parametrize("listed", [False, True])
@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("lens,hq,hkv,d", CASES)
def test_own_size_is_enough(P, fmt, lens, hq, hkv, d, listed):
    cache = Cache(fmt, hkv, d, lens, seed=4)
    S, n = len(lens), max(lens)
    q = queries(S, hq, d, seed=5)
    blocks = torch.arange(-(-n // 16) * 3 // 4 + 1, dtype=torch.int32, device=DEV).expand(S, hkv, -1).contiguous()
    rows = min(n, 16 * blocks.shape[2]) if listed else n

    def call(room):
        ws = torch.full((room + 4096,), 0x7F, dtype=torch.uint8, device=DEV)
        out, lse = torch.full_like(q, 7.0), torch.full((S, hq), 9.0, device=DEV)
        fn = getattr(P, f"pallas_attend{'_blocks' if listed else ''}_{'kv' if fmt == 'bf16' else 'quant'}")
        fn(*cache.rows, 1, q, cache.lengths, n, cache.bt, *((blocks,) if listed else ()), 0.1, out, ws[:room], lse=lse)
        assert bool((ws[room:] == 0x7F).all())
        return out, lse

    # (What both 8-bit types need; bf16, of twice the bytes, needs as much or less.)
    whole, own = P.pallas_attend_workspace_size(S, hq, hkv, d, rows), own_size(d, S, hq, hkv, d, rows)
    assert own <= whole
    for x, y in zip(call(whole), call(own)):
        assert torch.equal(x, y)
    least = own_size(2 * d if fmt == "bf16" else d, S, hq, hkv, d, rows)
    with pytest.raises(P.PallasError) as e:
        call(least - 256)
    assert e.value.status == P.Status.WORKSPACE


def test_cases_that_the_size_for_any_cache_exceeds(P):
    assert own_size(128, 1, 64, 8, 128, 131071) < P.pallas_attend_workspace_size(1, 64, 8, 128, 131071)
    assert sum(own_size(d, len(l), hq, hkv, d, max(l)) < P.pallas_attend_workspace_size(len(l), hq, hkv, d, max(l)) for l, hq, hkv, d in CASES) >= 2
