"""Rows without keys between rows that share a range: the answer, and that a batch does not
wait for each of them in turn."""
import numpy as np
import pytest
import torch

from attend_forms import check_form, fresh_workspace
from helpers import ensure_lib
from test_attend_gpu import DEV, Cache, check, queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    return ensure_lib()


def spread(S, rows):
    lens = [0] * S
    for i, n in rows.items():
        lens[i] = n
    return lens


LENS = {
    "two far apart": spread(700, {0: 40, 699: 33}),
    "runs at window edges": spread(400, {3: 5, 63: 70, 64: 1, 65: 40, 127: 33, 128: 32, 320: 400, 399: 1}),
    "the first rows empty": spread(300, {150: 2000, 151: 64, 299: 17}),
    "more than 4096": spread(6000, {0: 100, 93: 31, 94: 33, 187: 1, 188: 900, 4095: 64, 4096: 65, 5999: 300}),
    "every seventh": [(37 * i) % 300 if i % 7 == 3 else 0 for i in range(900)],
    "one": spread(5000, {2500: 77}),
}


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("name", LENS)
def test_against_oracle(P, name, fmt):
    lens, hkv, hq, d, max_length = LENS[name], 2, 4, 64, 20000
    cache = Cache(fmt, hkv, d, lens, seed=3)
    bt = torch.full((len(lens), max_length // 16), -1, dtype=torch.int32, device=DEV)
    bt[:, :cache.max_pages] = cache.bt
    q, lse = queries(len(lens), hq, d, 4), torch.full((len(lens), hq), 9.0, device=DEV)
    ws, err = fresh_workspace(P, len(lens), hq, hkv, d, max_length), torch.zeros(1, dtype=torch.int32, device=DEV)
    out = cache.attend(P, q, 0.125, lse=lse, max_length=max_length, ws=ws, bt=bt, err=err)
    check_form("ranges", ws, fmt, d, hq, hkv, lens, max_length)
    check(cache, q, 0.125, out, lse)
    assert int(err.item()) == 0


def test_empty_rows_cost_no_more_between_than_behind(P):
    """20,000 of them between two rows of 4000 keys: once 12 times the call with them behind both."""
    S, hq, hkv, d = 20002, 8, 8, 64
    pool = torch.zeros((1, 2, 300, 16, hkv, d), dtype=torch.bfloat16, device=DEV)
    bt = torch.from_numpy(np.random.default_rng(0).integers(0, 300, (S, 250)).astype(np.int32)).to(DEV)
    q = torch.zeros((S, hq, d), dtype=torch.bfloat16, device=DEV)
    out, ws = torch.empty_like(q), fresh_workspace(P, S, hq, hkv, d, 4000)

    def time(rows):
        lengths = torch.tensor(spread(S, rows), dtype=torch.int32, device=DEV)
        best = float("inf")
        for _ in range(6):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            P.pallas_attend_kv(pool, 0, q, lengths, 4000, bt, 0.1, out, ws)
            b.record()
            b.synchronize()
            best = min(best, a.elapsed_time(b))
        return best

    assert time({0: 4000, S - 1: 4000}) < 3 * time({0: 4000, 1: 4000})
