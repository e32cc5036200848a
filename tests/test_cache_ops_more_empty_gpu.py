"""A batch without tokens or sequences through append, bounds, selection and attention over blocks:
checked as any other, nothing enqueued, nothing written."""
import pytest
import torch

from helpers import ensure_lib

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def P():
    return ensure_lib()


@pytest.mark.parametrize("fmt", ["bf16", "int8", "e2m1"])
def test_an_empty_batch(P, fmt):
    hq, hkv, d = 4, 2, 64
    q, kv = (torch.empty((0, h, d), dtype=torch.bfloat16, device=DEV) for h in (hq, hkv))
    ints, bt = torch.empty(0, dtype=torch.int32, device=DEV), torch.empty((0, 4), dtype=torch.int32, device=DEV)
    if fmt == "bf16":
        pool = (torch.full((1, 2, 3, 16, hkv, d), 5.0, dtype=torch.bfloat16, device=DEV),)
    elif fmt == "int8":
        pool = torch.full((1, 2, 3, 16, hkv, d), 7, dtype=torch.int8, device=DEV), torch.full((1, 2, 3, 16, hkv), 2.0, device=DEV)
    else:
        pool = (torch.full((1, 2, 3, 16, hkv, d // 2), 7, dtype=torch.uint8, device=DEV).view(torch.float4_e2m1fn_x2),
                torch.full((1, 2, 3, 16, hkv, 4), 127, dtype=torch.uint8, device=DEV).view(torch.float8_e8m0fnu))
    bounds, steps = torch.full((1, 3, hkv, 2, d), 3, dtype=torch.int8, device=DEV), torch.full((1, 3, hkv), 0.5, device=DEV)
    held = [x.view(torch.uint8).clone() for x in (*pool, bounds, steps)]
    name = "kv" if fmt == "bf16" else "quant"
    ws, lse, err = torch.empty(0, dtype=torch.uint8, device=DEV), torch.empty((0, hq), device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    lists = torch.empty((0, hkv, 2), dtype=torch.int32, device=DEV)
    getattr(P, "pallas_append_" + name)(P.pallas_rope_init(d, 1e4), *pool, 0, kv, kv, ints, bt, q=q, err=err)
    getattr(P, "pallas_bounds_" + name)(*pool, 0, bounds, steps, ints, ints, 1, bt, err=err)
    P.pallas_select_blocks(bounds, steps, 0, q, ints, 64, bt, lists, ws, err=err)
    out = torch.empty_like(q)
    getattr(P, "pallas_attend_blocks_" + name)(*pool, 0, q, ints, 64, bt, lists, 0.1, out, ws, lse=lse, err=err)
    torch.cuda.synchronize()
    for x, y in zip((*pool, bounds, steps), held):
        assert torch.equal(x.view(torch.uint8), y)
    assert int(err.item()) == 0
