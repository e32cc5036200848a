"""A batch without tokens or sequences through every cache operator: checked as any other,
nothing enqueued, nothing written."""
import pytest
import torch

from helpers import ensure_lib

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def P():
    return ensure_lib()


def test_an_empty_batch(P):
    hq, hkv, d = 4, 2, 64
    q, kv = (torch.empty((0, h, d), dtype=torch.bfloat16, device=DEV) for h in (hq, hkv))
    ints, bt = torch.empty(0, dtype=torch.int32, device=DEV), torch.empty((0, 4), dtype=torch.int32, device=DEV)
    pool = torch.full((1, 2, 3, 16, hkv, d), 5.0, dtype=torch.bfloat16, device=DEV)
    codes = torch.full((1, 2, 3, 16, hkv, d), 7, dtype=torch.int8, device=DEV)
    scales = torch.full((1, 2, 3, 16, hkv), 2.0, device=DEV)
    lse, ws, err = torch.empty((0, hq), device=DEV), torch.empty(0, dtype=torch.uint8, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    P.pallas_rope_apply(P.pallas_rope_init(d, 1e4), q, ints)
    P.pallas_quant_store(codes, scales, 0, kv, kv, ints, bt, err=err)
    P.pallas_quant_load(codes, scales, 0, kv, kv, ints, bt, seq_ids=ints, err=err)
    for attend in (lambda q_, l: P.pallas_attend_kv(pool, 0, q_, l, 64, bt, 0.1, torch.empty_like(q_), ws, lse=lse, err=err),
                   lambda q_, l: P.pallas_attend_quant(codes, scales, 0, q_, l, 64, bt, 0.1, torch.empty_like(q_), ws, lse=lse, err=err)):
        attend(q, ints)
        for bad in ((q.float(), ints), (q[..., :32], ints), (q, torch.zeros(1, dtype=torch.int32, device=DEV)), (q, ints.long())):
            with pytest.raises(P.PallasError) as e:
                attend(*bad)
            assert e.value.status == P.Status.INVALID_ARG
    torch.cuda.synchronize()
    assert bool((pool == 5.0).all()) and bool((codes == 7).all()) and bool((scales == 2.0).all()) and int(err.item()) == 0
