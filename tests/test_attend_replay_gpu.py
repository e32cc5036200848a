"""Captured graphs whose lengths grow and shrink in device memory, and workspaces used by
several calls, where attention leaves records in the workspace (splits and a join, ranges
and a join; attend_forms says which, from the workspace): each replay equals the eager call
to the bit, and the oracle's formula in float64 on the GPU."""
import math

import numpy as np
import pytest
import torch

from attend_forms import blocks_per_range, check_form, fresh_workspace
from helpers import ensure_lib
from test_cache_ops_chain_gpu import Layer

pytestmark = pytest.mark.gpu
DEV = "cuda"
D, GROUP, S = 128, 2, 3
TYPES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
#: form -> (KV heads, capacity, lengths of each replay)
GROWTH = {
    "split": (2, 1500, [(1, 0, 3), (128, 129, 1500), (700, 33, 256), (1500, 1500, 1499), (0, 0, 0), (257, 512, 513), (32, 1, 0)]),
    "ranges": (8, 20000, [(1, 0, 3), (40, 17, 512), (900, 1000, 1100), (5000, 3000, 1), (12000, 7000, 33),
                          (19999, 16000, 20000), (0, 0, 0), (64, 2000, 0)]),
}
KINDS = [pytest.param(form, fmt, id=f"{form}-{fmt}") for form in GROWTH for fmt in ("bf16", "e4m3", "int8")]


@pytest.fixture(scope="module")
def P():
    return ensure_lib()


class Batch:
    """S rows over one random cache (their tables share its pages)."""

    def __init__(self, P, form, fmt, seed):
        self.P, self.form, self.fmt = P, form, fmt
        self.hkv, self.room, self.steps = GROWTH[form]
        self.hq = GROUP * self.hkv
        pages = -(-self.room // 16)
        rng, g = np.random.default_rng(seed), torch.Generator(DEV).manual_seed(seed)
        self.bt = torch.from_numpy(np.stack([rng.permutation(pages + 7)[:pages] for _ in range(S)]).astype(np.int32)).to(DEV)
        shape = (1, 2, pages + 7, 16, self.hkv, D)
        if fmt == "bf16":
            self.pool = torch.randn(shape, device=DEV, generator=g).to(torch.bfloat16)
        else:
            raw = torch.randint(0, 256, shape, dtype=torch.uint8, device=DEV, generator=g)
            raw = raw & 0xF7 if fmt == "e4m3" else raw            # (no NaN codes)
            self.codes = raw.view(TYPES[fmt])
            self.scales = (0.5 + torch.rand(shape[:-1], device=DEV, generator=g)) * (0.01 if fmt == "e4m3" else 0.02)
        self.q = torch.randn((S, self.hq, D), device=DEV, generator=g).to(torch.bfloat16)
        self.lengths = torch.zeros(S, dtype=torch.int32, device=DEV)
        self.out = torch.zeros_like(self.q)
        self.lse = torch.zeros((S, self.hq), device=DEV)
        self.err = torch.zeros(1, dtype=torch.int32, device=DEV)

    def workspace(self):
        return fresh_workspace(self.P, S, self.hq, self.hkv, D, self.room)

    def attend(self, ws, out=None, lse=None):
        out, lse = self.out if out is None else out, self.lse if lse is None else lse
        args = (0, self.q, self.lengths, self.room, self.bt, 0.07, out, ws)
        if self.fmt == "bf16":
            self.P.pallas_attend_kv(self.pool, *args, lse=lse, err=self.err)
        else:
            self.P.pallas_attend_quant(self.codes, self.scales, *args, lse=lse, err=self.err)
        return out, lse

    def rows(self, i, n, h):
        t = torch.arange(n, device=DEV)
        pg, slot = self.bt[i].long()[t // 16], t % 16
        if self.fmt == "bf16":
            return [self.pool[0, kv, pg, slot, h].double() for kv in range(2)]
        return [self.codes.view(torch.uint8)[0, kv, pg, slot, h].view(TYPES[self.fmt]).double() *
                self.scales[0, kv, pg, slot, h].double()[:, None] for kv in range(2)]


def check_rows(rows, q, lens, hkv, scale, out, lse):
    """`rows(i, n, h)`: float64 K and V of n keys of KV head h.  Tolerances: those of test_attend_gpu, 2^-12 for the
    longer sums."""
    for i, n in enumerate(lens):
        if n == 0:
            assert not out[i].any() and bool(torch.isneginf(lse[i]).all())
            continue
        for h in range(0, hkv, 3):
            k, v = rows(i, n, h)
            for j in range(h * GROUP, (h + 1) * GROUP):
                qd = q[i, j].double()
                z = (k * qd).sum(1) * scale
                rl = torch.logsumexp(z, 0)
                p = torch.exp(z - rl)[:, None]
                ref, mag = (p * v).sum(0), (p * v.abs()).sum(0)
                delta = (D + 8) * 2.0 ** -24 * float(((k * qd).abs().sum(1) * scale).max())
                assert bool(((out[i, j].double() - ref).abs() <= 2.0 ** -8 * ref.abs() + (2 * delta + 2.0 ** -12) * mag).all()), (i, j, n)
                assert abs(float(lse[i, j]) - float(rl)) <= delta + 2.0 ** -12, (i, j, n)


def capture(call):
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        call()
    torch.cuda.current_stream().wait_stream(stream)
    return graph


@pytest.mark.parametrize("form,fmt", KINDS)
def test_replays_over_changing_lengths(P, form, fmt):
    b = Batch(P, form, fmt, 1)
    ws, seen = b.workspace(), set()
    graph = capture(lambda: b.attend(ws))
    out, lse = torch.empty_like(b.out), torch.empty_like(b.lse)
    for lens in b.steps + b.steps[::-1]:
        b.lengths.copy_(torch.tensor(lens, dtype=torch.int32))
        b.out.fill_(7.0)
        b.lse.fill_(7.0)
        graph.replay()
        own = b.workspace()
        b.attend(own, out, lse)
        torch.cuda.synchronize()
        assert torch.equal(b.out, out) and torch.equal(b.lse, lse), lens
        check_form(form, own, fmt, D, b.hq, b.hkv, lens, b.room)
        check_rows(b.rows, b.q, lens, b.hkv, 0.07, out, lse)
        seen.add(min(blocks_per_range(fmt, D, b.hq, b.hkv, lens), 3))
    assert int(b.err.item()) == 0
    assert form == "split" or seen == {1, 2, 3}


@pytest.mark.parametrize("form", GROWTH)
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_decode_chain_replayed_over_changing_lengths(P, form, fmt):
    """Rotary, store and attention in one graph, each row at its own position of a full cache."""
    hkv, room, steps = GROWTH[form]
    hq = GROUP * hkv
    a, b = (Layer(P, fmt, S, hq, hkv, D, room, seed=1) for _ in range(2))
    g = torch.Generator(DEV).manual_seed(4)
    pos = torch.arange(room, dtype=torch.int32, device=DEV).repeat(S)
    seq = torch.arange(S, dtype=torch.int32, device=DEV).repeat_interleave(room)
    k, v = (torch.randn((S * room, hkv, D), device=DEV, generator=g).to(torch.bfloat16) for _ in range(2))
    for l in (a, b):
        P.pallas_quant_store(l.codes, l.scales, 0, k, v, pos, l.bt, seq_ids=seq)
        l.ws.fill_(0xFF)
    del k, v
    feed = torch.randn((len(steps), *a.qkv.shape), device=DEV, generator=g).to(torch.bfloat16)
    graph = capture(b.step)

    def rows(i, n, h):
        t = torch.arange(n, device=DEV)
        pg, slot = a.bt[i].long()[t // 16], t % 16
        return [a.codes.view(torch.uint8)[0, kv, pg, slot, h].view(TYPES[fmt]).double() * a.scales[0, kv, pg, slot, h].double()[:, None]
                for kv in range(2)]

    for n, lens in enumerate(steps):
        for l in (a, b):
            l.qkv.copy_(feed[n])
            l.lengths.copy_(torch.tensor(lens, dtype=torch.int32))
            l.pos.copy_(l.lengths - 1)
        a.ws.fill_(0xFF)
        a.step()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a.qkv, b.qkv) and torch.equal(a.out, b.out) and torch.equal(a.lse, b.lse), lens
        assert torch.equal(a.codes.view(torch.uint8), b.codes.view(torch.uint8))
        assert torch.equal(a.scales.view(torch.int32), b.scales.view(torch.int32))     # (slots not written hold NaN)
        check_form(form, a.ws, fmt, D, hq, hkv, lens, room)
        check_rows(rows, a.heads(0, hq), lens, hkv, 1 / math.sqrt(D), a.out, a.lse)
    assert int(a.err.item()) == 0 and int(b.err.item()) == 0


@pytest.mark.parametrize("form,fmt", KINDS)
def test_workspaces_of_several_calls(P, form, fmt):
    """Two streams at once with a workspace each; then one workspace for two graphs and eager calls, in turn."""
    batches = [Batch(P, form, fmt, s) for s in (2, 3)]
    lens = [batches[0].steps[3], batches[0].steps[2]]
    spaces, want = [b.workspace() for b in batches], []
    for b, n, ws in zip(batches, lens, spaces):
        b.lengths.copy_(torch.tensor(n, dtype=torch.int32))
        b.attend(ws)
        check_form(form, ws, fmt, D, b.hq, b.hkv, n, b.room)
        assert any(parts[1] > 0 for parts in ws[:8 * S].cpu().numpy().view(np.int32).reshape(-1, 2))     # records
        want.append((b.out.clone(), b.lse.clone()))
        check_rows(b.rows, b.q, n, b.hkv, 0.07, b.out, b.lse)

    def check():
        torch.cuda.synchronize()
        for b, (out, lse) in zip(batches, want):
            assert torch.equal(b.out, out) and torch.equal(b.lse, lse)
            b.out.fill_(7.0)
            b.lse.fill_(7.0)
        torch.cuda.synchronize()

    check()
    streams = [torch.cuda.Stream() for _ in batches]
    for _ in range(3):
        for _ in range(10):
            for b, ws, s in zip(batches, spaces, streams):
                with torch.cuda.stream(s):
                    b.attend(ws)
        check()
    graphs = [capture(lambda b=b: b.attend(spaces[0])) for b in batches]
    for _ in range(4):
        for g in graphs:
            g.replay()
        check()
        for g, b in zip(graphs, batches[::-1]):
            g.replay()
            b.attend(spaces[0])
        check()
