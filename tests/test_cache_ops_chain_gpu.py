"""The cache operators together, as a decoder's layer calls them for one new token per
sequence: rotary on the Q and K heads inside the projection's rows, the 8-bit store,
attention; eagerly and as a captured graph that is replayed while positions and lengths
grow in device memory.  Then the cache is migrated (pack, assemble), attended at its new
place and read back."""
import math

import numpy as np
import pytest
import torch

from helpers import ensure_lib, gpu_model, to_np64
from oracle import cache_ops as co
from workloads import configs, gen

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


@pytest.fixture(scope="module")
def P():
    return ensure_lib()


class Layer:
    """Buffers of a decode batch over one layer of an 8-bit cache."""

    def __init__(self, P, fmt, S, hq, hkv, d, room, seed):
        self.P, self.hq, self.hkv, self.d, self.room = P, hq, hkv, d, room
        pages = (room + 15) // 16
        order = np.random.default_rng(seed).permutation(S * pages).reshape(S, pages)
        self.bt = torch.from_numpy(order.astype(np.int32)).to(DEV)
        self.codes = torch.full((1, 2, S * pages, 16, hkv, d), 0x7F, dtype=torch.uint8, device=DEV).view(TYPES[fmt])
        self.scales = torch.full((1, 2, S * pages, 16, hkv), float("nan"), device=DEV)
        self.qkv = torch.zeros((S, (hq + 2 * hkv) * d), dtype=torch.bfloat16, device=DEV)
        self.pos = torch.zeros(S, dtype=torch.int32, device=DEV)
        self.lengths = torch.zeros(S, dtype=torch.int32, device=DEV)
        self.out = torch.zeros((S, hq, d), dtype=torch.bfloat16, device=DEV)
        self.lse = torch.zeros((S, hq), device=DEV)
        self.err = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.ws = torch.empty(P.pallas_attend_workspace_size(S, hq, hkv, d, room), dtype=torch.uint8, device=DEV)
        self.plan = P.pallas_rope_init(d, 1e6, scaling="yarn", factor=8.0, trained_len=4096, fast=32.0, slow=1.0)
        self.scale = 1 / math.sqrt(d)

    def heads(self, a, b):
        return self.qkv[:, a * self.d:b * self.d].unflatten(1, (b - a, self.d))

    def step(self):
        P, hq, hkv = self.P, self.hq, self.hkv
        P.pallas_rope_apply(self.plan, self.heads(0, hq + hkv), self.pos)
        P.pallas_quant_store(self.codes, self.scales, 0, self.heads(hq, hq + hkv), self.heads(hq + hkv, hq + 2 * hkv), self.pos,
                             self.bt, err=self.err)
        P.pallas_attend_quant(self.codes, self.scales, 0, self.heads(0, hq), self.lengths, self.room, self.bt, self.scale,
                              self.out, self.ws, lse=self.lse, err=self.err)


def feed(layer, start, t, seed):
    """Projection rows of step t, and where they go."""
    g = torch.Generator().manual_seed(1000 * seed + t)
    layer.qkv.copy_(torch.randn(layer.qkv.shape, generator=g).to(torch.bfloat16))
    layer.pos.copy_(torch.tensor([s + t if s >= 0 else -1 for s in start], dtype=torch.int32))
    layer.lengths.copy_((layer.pos + 1).clamp(min=0))


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (6, 2, 64)])
def test_decode_steps_eager_and_replayed(P, fmt, hq, hkv, d):
    """Steps 0 .. 39 of a batch with one padded row; each replay equals the eager step to the bit, and the
    last steps the oracle."""
    start, steps = [0, 0, -1, 0], 40
    a, b = (Layer(P, fmt, len(start), hq, hkv, d, 64, seed=1) for _ in range(2))
    feed(b, start, 0, 2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            b.step()
    torch.cuda.current_stream().wait_stream(side)
    f, m = co.rope_frequencies(d, 1e6, "yarn", 8.0, 4096, 32.0, 1.0)
    ks, vs = [], []
    for t in range(steps):
        feed(a, start, t, 2)
        raw = to_np64(a.qkv).reshape(len(start), hq + 2 * hkv, d)
        a.step()
        feed(b, start, t, 2)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a.qkv, b.qkv) and torch.equal(a.out, b.out) and torch.equal(a.lse, b.lse)
        assert torch.equal(a.codes.view(torch.uint8), b.codes.view(torch.uint8))
        # the rows as rotated by the kernel (bf16) are the oracle's input from here on
        got = to_np64(a.qkv).reshape(len(start), hq + 2 * hkv, d)
        live = [i for i, s in enumerate(start) if s >= 0]
        want = co.rope(raw[live, :hq + hkv], [start[i] + t for i in live], f, m)
        assert np.all(np.abs(got[live, :hq + hkv] - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -18 * np.abs(raw[live]).max())
        ks.append(co.dequantise(*co.quantise(got[:, hq:hq + hkv], fmt), fmt))
        vs.append(co.dequantise(*co.quantise(got[:, hq + hkv:], fmt), fmt))
        assert not a.out[2].any() and bool((a.lse[2] == -math.inf).all())
        if t >= steps - 3 or t == 0:
            for i in live:
                k, v = np.stack([x[i] for x in ks]), np.stack([x[i] for x in vs])
                ref, rl, mag, terms = co.attend(got[i, :hq], k, v, a.scale)
                delta = ((d + 8) * 2.0 ** -24 * terms)[:, None]
                assert np.all(np.abs(to_np64(a.out)[i] - ref) <= 2.0 ** -8 * np.abs(ref) + (2 * delta + 2.0 ** -13) * mag)
                assert np.all(np.abs(to_np64(a.lse)[i] - rl) <= delta[:, 0] + 2.0 ** -13)
    assert int(a.err.item()) == 0 and int(b.err.item()) == 0


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_prefill_then_quantise_migrate_and_attend(P, fmt):
    """A model's prefill writes a bf16 pool; each layer is taken into an 8-bit pool, page by page; both pools are
    migrated through the chunk arena; attention over the migrated 8-bit cache is that of the source's to the bit,
    and near the bf16 cache's."""
    cfg = configs.TINY.replace(n_kv_heads=4, n_q_heads=8, name="tiny-kv4")
    n, p = 100, 40
    glob, layers = gen.model_weights(cfg, seed=3)
    model = gpu_model(P, cfg, glob, layers)
    L, hkv, d = cfg.n_layers, cfg.n_kv_heads, cfg.head_dim
    pages = (n + 15) // 16
    bt = torch.tensor(gen.block_table(pages, 12, pages, 3, 1), dtype=torch.int32, device=DEV)
    bt2 = torch.tensor(gen.block_table(pages, 12, pages, 3, 2), dtype=torch.int32, device=DEV)
    pool = torch.zeros((L, 2, 12, 16, hkv, d), dtype=torch.bfloat16, device=DEV)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    ids = torch.tensor(gen.token_ids(n, cfg.vocab, seed=3).numpy(), dtype=torch.int32, device=DEV)
    model.prefill_prefix(ids, [0, n], bt[None], pool, model.workspace(n), err)
    codes = torch.zeros((L, 2, 12, 16, hkv, d), dtype=torch.uint8, device=DEV).view(TYPES[fmt])
    scales = torch.zeros((L, 2, 12, 16, hkv), device=DEV)
    # slot by slot: the token in slot s of page g is position `of[g, s]`
    of = torch.full((12, 16), -1, dtype=torch.int32, device=DEV)
    t = torch.arange(n, device=DEV)
    of[bt[t // 16].long(), t % 16] = t.to(torch.int32)
    seq = torch.zeros(12 * 16, dtype=torch.int32, device=DEV)
    for l in range(L):
        P.pallas_quant_store(codes, scales, l, pool[l, 0].view(-1, hkv, d), pool[l, 1].view(-1, hkv, d), of.view(-1), bt[None],
                             seq_ids=seq, err=err)
    # migrate positions [0, n) in two chunks: codes as rows of d / 2 two-byte elements, scales of 2
    moved = torch.zeros_like(codes.view(torch.uint8)).view(TYPES[fmt])
    moved_scales = torch.zeros_like(scales)
    for src, dst, width in ((codes, moved, d // 2), (scales, moved_scales, 2)):
        s16, d16 = (x.view(torch.uint8).view(L, 2, 12, 16, hkv, -1).view(torch.bfloat16) for x in (src, dst))
        assert s16.shape[-1] == width
        token = L * 2 * hkv * width * 2
        arena = torch.empty(n * token, dtype=torch.uint8, device=DEV)
        P.pallas_pack_suffix_blocks(s16, bt, [P.ChunkDesc(0, p, 0), P.ChunkDesc(p, n - p, p * token)], arena, err)
        hdrs = [P.ChunkHeader(1, 1, a, c, a * token, L, hkv, width, 2) for a, c in ((0, p), (p, n - p))]
        P.pallas_assemble_kv(d16, bt2, hdrs, arena, 1, 1, err)
    q = torch.randn((1, cfg.n_q_heads, d), device=DEV, generator=torch.Generator(DEV).manual_seed(1)).to(torch.bfloat16)
    lengths = torch.tensor([n], dtype=torch.int32, device=DEV)
    ws = torch.empty(P.pallas_attend_workspace_size(1, cfg.n_q_heads, hkv, d, n), dtype=torch.uint8, device=DEV)
    outs = [torch.empty_like(q) for _ in range(3)]
    pos = torch.arange(n, dtype=torch.int32, device=DEV)
    for l in range(L):
        P.pallas_attend_quant(codes, scales, l, q, lengths, n, bt[None], 0.125, outs[0], ws, err=err)
        P.pallas_attend_quant(moved, moved_scales, l, q, lengths, n, bt2[None], 0.125, outs[1], ws, err=err)
        P.pallas_attend_kv(pool, l, q, lengths, n, bt[None], 0.125, outs[2], ws, err=err)
        assert torch.equal(outs[0], outs[1])
        k8, v8 = (torch.empty((n, hkv, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        P.pallas_quant_load(moved, moved_scales, l, k8, v8, pos, bt2[None], seq_ids=torch.zeros_like(pos), err=err)
        rows = [pool[l, kv, bt[t // 16].long(), t % 16] for kv in range(2)]
        worst = 0.0
        for got, x in ((k8, rows[0]), (v8, rows[1])):
            e = (got.double() - x.double()).abs()
            top = x.double().abs().amax(dim=-1, keepdim=True)
            # half a step of the format (E4M3: 2^-4 of the value, or of the least code's double; INT8: of a / 127), and
            # the bf16 result
            half = torch.maximum(x.double().abs() * 2.0 ** -4, top * 2.0 ** -17) if fmt == "e4m3" else top / 254 * 1.001
            assert bool((e <= half + got.double().abs() * 2.0 ** -8).all())
            worst = max(worst, float(e.max()))
        # attention: each key moves a score by at most scale |q|_1 worst, each value by at most worst
        shift = 0.125 * float(q.double().abs().sum(-1).max()) * worst
        vmax = float(rows[1].double().abs().max())
        assert float((outs[0].double() - outs[2].double()).abs().max()) <= 2 * (math.exp(2 * shift) - 1) * vmax + 2 * worst + 2.0 ** -7 * vmax
    assert int(err.item()) == 0


def test_two_streams_and_a_shared_workspace(P):
    """Calls on two streams with a workspace each, and two captured graphs that share one and run after each other."""
    layers = [Layer(P, "e4m3", 3, 8, 2, 128, 300, seed=s) for s in (1, 2)]
    rows = []
    for n, l in enumerate(layers):
        g = torch.Generator(DEV).manual_seed(n)
        pos = torch.arange(300, dtype=torch.int32, device=DEV).repeat(3)
        seq = torch.arange(3, dtype=torch.int32, device=DEV).repeat_interleave(300)
        k, v = (torch.randn((900, 2, 128), device=DEV, generator=g).to(torch.bfloat16) for _ in range(2))
        P.pallas_quant_store(l.codes, l.scales, 0, k, v, pos, l.bt, seq_ids=seq)
        l.qkv.copy_(torch.randn(l.qkv.shape, device=DEV, generator=g).to(torch.bfloat16))
        l.lengths.copy_(torch.tensor([300, 129, 256]))

    def attend(l, ws):
        P.pallas_attend_quant(l.codes, l.scales, 0, l.heads(0, 8), l.lengths, 300, l.bt, l.scale, l.out, ws, lse=l.lse)

    for l in layers:
        attend(l, l.ws)
        rows.append((l.out.clone(), l.lse.clone()))
        l.out.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in layers]
    for l, s in zip(layers, streams):
        with torch.cuda.stream(s):
            for _ in range(20):
                attend(l, l.ws)
    torch.cuda.synchronize()
    for l, (o, z) in zip(layers, rows):
        assert torch.equal(l.out, o) and torch.equal(l.lse, z)
        l.out.zero_()
    torch.cuda.synchronize()
    graphs = []
    for l, s in zip(layers, streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            attend(l, layers[0].ws)
        graphs.append(g)
    for _ in range(3):
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for l, (o, z) in zip(layers, rows):
            assert torch.equal(l.out, o) and torch.equal(l.lse, z)
            l.out.zero_()
        torch.cuda.synchronize()
