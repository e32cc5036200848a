"""Refusals of pallas_append_kv and pallas_append_quant, before anything is enqueued (every
pointer is one that no call may touch).  No GPU needed."""
import ctypes as C

import pytest
import torch

from helpers import ensure_lib
from paper_2608_16477_amd.binding import KVPoolC, RopePlan
from test_cache_ops_host import FAKE, quant_pool


@pytest.fixture(scope="module")
def P():
    return ensure_lib()


GOOD = dict(layer=1, tokens=3, seq=FAKE, pos=FAKE, heads=8, q=FAKE, qs=512, qo=FAKE, qos=512, k=FAKE, ks=256, v=FAKE, vs=256,
            seqs=2, bt=FAKE, max_pages=4, err=None)


def append_rc(P, quant, pool=None, plan=None, **kw):
    a = {**GOOD, **kw}
    if pool is None:
        pool = quant_pool() if quant else KVPoolC(FAKE, 8, 16, 2, 4, 64)
    plan = P.pallas_rope_init(64, 1e4) if plan is None else plan
    fn = P.lib().pallas_append_quant if quant else P.lib().pallas_append_kv
    return P.Status(fn(None if plan == 0 else C.byref(plan), None if pool == 0 else C.byref(pool), a["layer"], a["tokens"],
                       a["seq"], a["pos"], a["heads"], a["q"], a["qs"], a["qo"], a["qos"], a["k"], a["ks"], a["v"], a["vs"],
                       a["seqs"], a["bt"], a["max_pages"], a["err"], None))


@pytest.mark.parametrize("quant", [False, True])
def test_refusals(P, quant):
    S = P.Status
    for bad in (dict(tokens=-1), dict(seqs=0), dict(max_pages=0), dict(pos=None), dict(k=None), dict(v=None), dict(bt=None),
                dict(seq=None), dict(k=FAKE + 8), dict(v=FAKE + 2), dict(ks=260), dict(vs=252), dict(ks=248), dict(vs=0),
                dict(seq=FAKE + 2), dict(pos=FAKE + 1), dict(bt=FAKE + 2), dict(err=FAKE + 2),
                dict(heads=-1), dict(heads=0), dict(q=None), dict(qo=None), dict(heads=0, q=None), dict(heads=0, qo=None),
                dict(q=FAKE + 8), dict(qo=FAKE + 8), dict(qs=516), dict(qos=508), dict(qs=504), dict(qos=504),
                dict(qos=520), dict(plan=RopePlan()), dict(plan=0), dict(plan=P.pallas_rope_init(66, 1e4)), dict(pool=0)):
        assert append_rc(P, quant, **bad) == S.INVALID_ARG, bad
        assert "append" in P.pallas_last_error() or "rope" in P.pallas_last_error()
    for bad in (dict(layer=2), dict(layer=-1)):
        assert append_rc(P, quant, **bad) == S.OUT_OF_RANGE, bad
    for bad in (dict(tokens=1 << 24, seqs=1 << 25), dict(heads=4097, qs=4097 * 64, qos=4097 * 64)):
        assert append_rc(P, quant, **bad) == S.UNSUPPORTED, bad
    pools = [quant_pool(head_dim=96), quant_pool(page_size=8), quant_pool(n_kv_heads=4097)] if quant else [
        KVPoolC(FAKE, 8, 16, 2, 4, 96), KVPoolC(FAKE, 8, 32, 2, 4, 64), KVPoolC(FAKE, 8, 16, 2, 4, 256), KVPoolC(FAKE, 8, 16, 2, 4097, 64)]
    for pool in pools:
        assert append_rc(P, quant, pool, ks=1 << 19, vs=1 << 19, qs=1 << 13, qos=1 << 13) == S.UNSUPPORTED
    assert append_rc(P, quant, tokens=0) == S.OK
    assert append_rc(P, quant, tokens=0, heads=0, q=None, qo=None) == S.OK


def test_binding_refusals(P):
    plan = P.pallas_rope_init(64, 1e4)
    x = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    pos, bt = torch.zeros(4, dtype=torch.int32), torch.zeros((4, 3), dtype=torch.int32)
    pool = torch.zeros((1, 2, 3, 16, 2, 64), dtype=torch.bfloat16)
    codes, scales = torch.zeros((1, 2, 3, 16, 2, 64), dtype=torch.int8), torch.zeros((1, 2, 3, 16, 2))
    for call in (lambda: P.pallas_append_kv(plan, pool, 0, x, x, pos, bt),                      # host tensors
                 lambda: P.pallas_append_kv(plan, pool.half(), 0, x, x, pos, bt),
                 lambda: P.pallas_append_quant(plan, codes, scales, 0, x, x, pos, bt),
                 lambda: P.pallas_append_quant(plan, codes, scales[..., :1], 0, x, x, pos, bt),
                 lambda: P.pallas_append_quant(plan, codes, scales, 0, x, x, pos.long(), bt, q=x)):
        with pytest.raises(P.PallasError) as e:
            call()
        assert e.value.status == P.Status.INVALID_ARG
