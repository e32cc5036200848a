"""A 4-bit pool's refusals, before anything is enqueued.  No GPU needed."""
import pytest
import torch

from helpers import ensure_lib
from test_cache_ops_host import FAKE, attend_rc, quant_pool, quant_rc


@pytest.fixture(scope="module")
def P():
    return ensure_lib()


@pytest.mark.parametrize("name", ["pallas_quant_store", "pallas_quant_load"])
def test_quant_refusals(P, name):
    S = P.Status
    for bad in (dict(tokens=-1), dict(pos=None), dict(k=FAKE + 8), dict(ks=260), dict(vs=252), dict(bt=FAKE + 2)):
        assert quant_rc(P, name, quant_pool(format=4), **bad) == S.INVALID_ARG, bad
    for bad in (dict(codes=FAKE + 8), dict(scales=FAKE + 4), dict(num_pages=0), dict(format=5), dict(format=6), dict(format=-4)):
        assert quant_rc(P, name, quant_pool(**{"format": 4, **bad})) == S.INVALID_ARG, bad
    for bad in (dict(head_dim=96), dict(head_dim=32), dict(page_size=32)):
        assert quant_rc(P, name, quant_pool(format=4, **bad)) == S.UNSUPPORTED, bad
    assert quant_rc(P, name, quant_pool(format=4), tokens=0) == S.OK


def test_attend_refusals(P):
    S = P.Status
    for bad in (dict(seqs=0), dict(heads=6), dict(q=FAKE + 8), dict(ws=FAKE + 16)):
        assert attend_rc(P, True, quant_pool(format=4), **bad) == S.INVALID_ARG, bad
    assert attend_rc(P, True, quant_pool(format=4, num_pages=1 << 23)) == S.UNSUPPORTED
    assert attend_rc(P, True, quant_pool(format=4), ws_bytes=0) == S.WORKSPACE
    assert attend_rc(P, True, quant_pool(format=4), layer=2) == S.OUT_OF_RANGE


def test_workspace_has_room_for_every_range(P):
    """12 waves of 4-bit rows to a CU: the (range, sequence) pairs of divisions at their borders."""
    for hq, hkv, d in ((64, 8, 128), (8, 8, 64), (40, 1, 128), (8, 8, 128)):
        heads = hkv * -(-(hq // hkv) // 16)
        ranges = max(256 * 12 // heads // 8 * 8, 8)
        for s in (1, 2, 5, 64, 200):
            for n in (32, 1000, 40000, 1 << 20):
                total = s * -(-n // 32)
                rounds = max(-(-total // (32 * ranges)), 1)
                each = 1 if 2 * total <= ranges and total <= 32 * s else 2 if total <= 2 * ranges else -(-total // (ranges * rounds))
                last = -(-total // each) - 1 + s - 1
                assert P.pallas_attend_workspace_size(s, hq, hkv, d, n) >= 8 * s + (last + 1) * hq * (d + 2) * 4


def test_binding_refusals(P):
    codes = torch.zeros((1, 2, 3, 16, 2, 32), dtype=torch.uint8)
    scales = torch.zeros((1, 2, 3, 16, 2, 4), dtype=torch.uint8)
    x, pos, bt = torch.zeros((4, 2, 64), dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32), torch.zeros((4, 3), dtype=torch.int32)
    f4, e8 = torch.float4_e2m1fn_x2, torch.float8_e8m0fnu
    for c, s in ((codes, scales), (codes.view(f4), scales.view(e8)),               # bytes; host tensors
                 (codes.view(f4), scales), (codes.view(f4), scales[..., 0].view(e8))):
        with pytest.raises(P.PallasError) as e:
            P.pallas_quant_store(c, s, 0, x, x, pos, bt)
        assert e.value.status == P.Status.INVALID_ARG


@pytest.mark.parametrize("gone", [("float4_e2m1fn_x2",), ("float8_e8m0fnu",), ("float4_e2m1fn_x2", "float8_e8m0fnu")])
def test_a_torch_without_the_4_bit_types_has_the_8_bit_pools(P, monkeypatch, gone):
    import types
    from paper_2608_16477_amd import binding
    names = ("float8_e4m3fn", "int8", "float32", "float4_e2m1fn_x2", "float8_e8m0fnu")
    monkeypatch.setattr(binding, "_torch", types.SimpleNamespace(**{n: getattr(torch, n) for n in names if n not in gone}))
    assert binding._quant_formats() == {torch.float8_e4m3fn: (1, 1, torch.float32, 5), torch.int8: (2, 1, torch.float32, 5)}
    monkeypatch.undo()
    assert binding._quant_formats()[torch.float4_e2m1fn_x2] == (4, 2, torch.float8_e8m0fnu, 6)
