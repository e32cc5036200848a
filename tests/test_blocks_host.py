"""Refusals of the calls around selected blocks, before anything is enqueued (every pointer is
one that no call may touch).  No GPU needed."""
import ctypes as C
import math

import pytest
import torch

from helpers import ensure_lib
from paper_2608_16477_amd.binding import BoundsPoolC, KVPoolC
from test_cache_ops_host import FAKE, quant_pool


@pytest.fixture(scope="module")
def P():
    return ensure_lib()


def bounds_pool(**kw):
    return BoundsPoolC(**{**dict(codes=FAKE, scales=FAKE, num_pages=8, n_layers=2, n_kv_heads=4, head_dim=64), **kw})


def ref(x):
    return None if x == 0 else C.byref(x)


BOUNDS = dict(layer=1, seqs=2, start=FAKE, lens=FAKE, max_new=40, bt=FAKE, max_pages=4, err=None)


def bounds_rc(P, quant, pool=None, bounds=None, **kw):
    a = {**BOUNDS, **kw}
    pool = (quant_pool() if quant else KVPoolC(FAKE, 8, 16, 2, 4, 64)) if pool is None else pool
    fn = P.lib().pallas_bounds_quant if quant else P.lib().pallas_bounds_kv
    return P.Status(fn(ref(pool), ref(bounds_pool() if bounds is None else bounds), a["layer"], a["seqs"], a["start"], a["lens"],
                       a["max_new"], a["bt"], a["max_pages"], a["err"], None))


@pytest.mark.parametrize("quant", [False, True])
def test_bounds_refusals(P, quant):
    S = P.Status
    for bad in (dict(seqs=0), dict(max_new=0), dict(max_pages=0), dict(start=None), dict(lens=None), dict(bt=None),
                dict(start=FAKE + 2), dict(lens=FAKE + 1), dict(bt=FAKE + 2), dict(err=FAKE + 2), dict(pool=0), dict(bounds=0)):
        assert bounds_rc(P, quant, **bad) == S.INVALID_ARG, bad
        assert "bounds" in P.pallas_last_error()
    for bad in (dict(codes=None), dict(scales=None), dict(codes=FAKE + 8), dict(scales=FAKE + 4), dict(num_pages=0), dict(num_pages=9),
                dict(n_kv_heads=5), dict(n_layers=3), dict(head_dim=128), dict(n_layers=0)):
        assert bounds_rc(P, quant, bounds=bounds_pool(**bad)) == S.INVALID_ARG, bad
    assert bounds_rc(P, quant, layer=2) == S.OUT_OF_RANGE
    for bad in (dict(seqs=65536), dict(max_new=1 << 29, max_pages=1 << 26)):
        assert bounds_rc(P, quant, **bad) == S.UNSUPPORTED, bad
    pools = [quant_pool(head_dim=96), quant_pool(page_size=8)] if quant else [KVPoolC(FAKE, 8, 32, 2, 4, 64), KVPoolC(FAKE, 8, 16, 2, 4, 96)]
    for pool in pools:
        assert bounds_rc(P, quant, pool, bounds_pool(head_dim=pool.head_dim)) == S.UNSUPPORTED


SELECT = dict(layer=0, seqs=3, heads=8, q=FAKE, qs=512, lens=FAKE, max_length=64, bt=FAKE, max_pages=4, max_blocks=3, first=1, last=2,
              blocks=FAKE, ws=FAKE, ws_bytes=1 << 40, err=None)


def select_rc(P, bounds=None, **kw):
    a = {**SELECT, **kw}
    return P.Status(P.lib().pallas_select_blocks(
        ref(bounds_pool() if bounds is None else bounds), a["layer"], a["seqs"], a["heads"], a["q"], a["qs"], a["lens"],
        a["max_length"], a["bt"], a["max_pages"], a["max_blocks"], a["first"], a["last"], a["blocks"], a["ws"], a["ws_bytes"],
        a["err"], None))


def test_select_refusals(P):
    S = P.Status
    for bad in (dict(bounds=0), dict(seqs=0), dict(heads=0), dict(heads=6), dict(q=None), dict(lens=None), dict(bt=None),
                dict(blocks=None), dict(max_pages=0), dict(max_length=0), dict(q=FAKE + 8), dict(qs=516), dict(qs=504),
                dict(lens=FAKE + 2), dict(bt=FAKE + 1), dict(blocks=FAKE + 2), dict(err=FAKE + 2), dict(max_blocks=0, first=0, last=0),
                dict(first=-1), dict(last=-1), dict(first=2, last=2), dict(first=2 ** 31 - 1, last=2 ** 31 - 1), dict(ws=None), dict(ws=FAKE + 16)):
        assert select_rc(P, **bad) == S.INVALID_ARG, bad
        assert "select" in P.pallas_last_error()
    for bad in (dict(layer=2), dict(layer=-1), dict(max_length=65)):
        assert select_rc(P, **bad) == S.OUT_OF_RANGE, bad
    for bad in (dict(seqs=65536), dict(heads=8192, qs=1 << 20), dict(seqs=65535, max_length=1 << 20, max_pages=1 << 16),
                dict(seqs=1, max_length=(1 << 30) + 1, max_pages=1 << 27)):
        assert select_rc(P, **bad) == S.UNSUPPORTED, bad
    assert select_rc(P, bounds_pool(head_dim=96), qs=4096) == S.UNSUPPORTED
    assert select_rc(P, bounds_pool(n_kv_heads=4097)) == S.UNSUPPORTED
    need = P.pallas_select_workspace_size(3, 4, 64)
    assert need >= 3 * 4 * 4 * 4 and need % 256 == 0
    assert select_rc(P, ws_bytes=need - 1) == S.WORKSPACE


def test_select_workspace(P):
    size = P.pallas_select_workspace_size
    for bad in ((0, 4, 1), (1, 0, 1), (1, 4097, 1), (1, 4, 0), (65536, 4, 1), (65535, 4, 1 << 20), (1, 4096, 1 << 30)):
        assert size(*bad) == 0, bad
    for s in (1, 3, 64, 1000):
        for n in (1, 16, 17, 1000, 131072, 1 << 20):
            assert size(s, 8, n) >= s * 8 * -(-n // 16) * 4
            assert size(s, 8, n) <= size(s + 1, 8, n) and size(s, 8, n) <= size(s, 8, n + 100) and size(s, 8, n) <= size(s, 9, n)


ATTEND = dict(layer=0, seqs=3, heads=8, q=FAKE, qs=512, lens=FAKE, max_length=64, bt=FAKE, max_pages=4, blocks=FAKE, max_blocks=2,
              scale=0.125, out=FAKE, os=512, lse=None, ws=FAKE, ws_bytes=1 << 40)


def attend_rc(P, quant, pool=None, **kw):
    a = {**ATTEND, **kw}
    pool = (quant_pool() if quant else KVPoolC(FAKE, 8, 16, 2, 4, 64)) if pool is None else pool
    fn = P.lib().pallas_attend_blocks_quant if quant else P.lib().pallas_attend_blocks_kv
    return P.Status(fn(ref(pool), a["layer"], a["seqs"], a["heads"], a["q"], a["qs"], a["lens"], a["max_length"], a["bt"],
                       a["max_pages"], a["blocks"], a["max_blocks"], a["scale"], a["out"], a["os"], a["lse"], a["ws"], a["ws_bytes"],
                       None, None))


@pytest.mark.parametrize("quant", [False, True])
def test_attend_refusals(P, quant):
    S = P.Status
    for bad in (dict(seqs=0), dict(heads=6), dict(max_length=0), dict(q=None), dict(lens=None), dict(bt=None), dict(out=None),
                dict(blocks=None), dict(blocks=FAKE + 2), dict(max_blocks=0), dict(max_blocks=-1), dict(q=FAKE + 8), dict(qs=516),
                dict(os=504), dict(scale=math.nan), dict(ws=None), dict(ws=FAKE + 16), dict(lse=FAKE + 1), dict(pool=0)):
        assert attend_rc(P, quant, **bad) == S.INVALID_ARG, bad
        assert "attend" in P.pallas_last_error()
    for bad in (dict(layer=2), dict(max_length=65)):
        assert attend_rc(P, quant, **bad) == S.OUT_OF_RANGE, bad
    assert attend_rc(P, quant, seqs=1, max_length=(1 << 30) + 1, max_pages=1 << 27) == S.UNSUPPORTED
    # room for what the lists hold is enough, and needed
    for blocks, keys in ((2, 32), (4, 64), (100, 64)):
        need = P.pallas_attend_workspace_size(3, 8, 4, 64, keys)
        assert attend_rc(P, quant, max_blocks=blocks, ws_bytes=need - 1) == S.WORKSPACE


def test_binding_refusals(P):
    bounds, scales = torch.zeros((1, 3, 2, 2, 64), dtype=torch.int8), torch.zeros((1, 3, 2))
    pool, q = torch.zeros((1, 2, 3, 16, 2, 64), dtype=torch.bfloat16), torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    lens, bt = torch.zeros(4, dtype=torch.int32), torch.zeros((4, 3), dtype=torch.int32)
    blocks, ws = torch.zeros((4, 2, 3), dtype=torch.int32), torch.zeros(1 << 16, dtype=torch.uint8)
    for call in (lambda: P.pallas_bounds_kv(pool, 0, bounds, scales, lens, lens, 1, bt),           # host tensors
                 lambda: P.pallas_bounds_kv(pool, 0, bounds, scales[0], lens, lens, 1, bt),
                 lambda: P.pallas_bounds_kv(pool.float(), 0, bounds, scales, lens, lens, 1, bt),
                 lambda: P.pallas_select_blocks(bounds, scales, 0, q, lens, 48, bt, blocks, ws),
                 lambda: P.pallas_select_blocks(bounds.float(), scales, 0, q, lens, 48, bt, blocks, ws),
                 lambda: P.pallas_attend_blocks_kv(pool, 0, q, lens, 48, bt, blocks, 0.1, q.clone(), ws),
                 lambda: P.pallas_attend_blocks_kv(pool, 0, q, lens, 48, bt, None, 0.1, q.clone(), ws)):
        with pytest.raises(P.PallasError) as e:
            call()
        assert e.value.status == P.Status.INVALID_ARG


def test_select_takes_all_that_is_below_its_limits(P):
    size = P.pallas_select_workspace_size
    for heads, n in ((4096, (1 << 22) - 1), (16, (1 << 30) - 1), (15, 1 << 30), (3000, ((1 << 34) - 1) // 3000)):
        assert heads * n < 1 << 34 and size(1, heads, n) >= heads * -(-n // 16) * 4, (heads, n)
        assert size(1, heads, min(n + 1, 1 << 30)) == 0 or heads * min(n + 1, 1 << 30) < 1 << 34
    assert size(65535, 4, (1 << 35) // 65535) > 0 and size(65535, 4, (1 << 35) // 65535 + 1) == 0
