"""The cache operators as a user calls them, for timing and for comparing outputs.

Three operators around the paged KV cache:
  rope    rotary positions of Q and K rows: half and interleaved layouts, part
          of the head, scaled for long contexts
  quant   an 8-bit cache (E4M3 or INT8 codes, one float32 scale per token and
          KV head): rows are quantised as they are written, and read back
  attend  attention of one new token per sequence over a paged cache, bf16 or
          8-bit, split over the cache's length and joined

``run`` computes them in plain torch operations (``own`` false) or through the
library's entry points (``own`` true).

A case is a dict of plain values; ``kind`` names the operator.
  rope    tokens, heads, head_dim, rotary_dim, layout, scaling, span (positions
          lie below it), packed (rows are a part of wider projection rows)
  quant   format, kv_heads, head_dim, start, new (per sequence, comma-
          separated: tokens in the cache already, and tokens written), context
          (whether the whole cache is read back, or the new tokens alone)
  attend  format, q_heads, kv_heads, head_dim, lengths (comma-separated)
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
PAGE = 16
LAYERS = 2          # layers of a pool; LAYER is worked on
LAYER = 1
SPARE_PAGES = 32    # pool pages that belong to nobody
THETA = 1e6
#: scaling -> the plan's parameters: a context 8 times the trained one
SCALING = {
    "none": dict(),
    "linear": dict(factor=8.0),
    "ntk": dict(factor=8.0),
    "yarn": dict(factor=8.0, trained_len=16384, fast=32.0, slow=1.0),
    "bands": dict(factor=8.0, trained_len=16384, fast=4.0, slow=1.0),
}


def _text(values):
    return ",".join(str(int(v)) for v in values)


def _ints(text):
    return [int(v) for v in str(text).split(",")]


def _spread(seed, n, lo, hi):
    """n lengths, log-uniform in [lo, hi]."""
    r = np.random.Generator(np.random.PCG64(np.random.SeedSequence([seed, n, lo, hi])))
    return [int(v) for v in np.floor(np.exp(r.uniform(math.log(lo), math.log(hi), size=n)))]


def listed():
    ctx8 = _spread(0, 8, 1000, 8000)
    return [
        # Q and K of eight resumed requests, one token each (32 + 8 heads of 128): launch latency.
        dict(name="rope_decode_8", kind="rope", tokens=8, heads=40, head_dim=128, rotary_dim=128, layout="half",
             scaling="none", span=8000, packed=True),
        # Q and K of a 3000-token prefix at 64 + 8 heads, inside the projection's rows, for a context 8 times the trained one.
        dict(name="rope_prefix_3000", kind="rope", tokens=3000, heads=72, head_dim=128, rotary_dim=128, layout="half",
             scaling="yarn", span=131072, packed=True),
        # Rotary pairs next to each other in a quarter of the head, a long prompt, odd token count.
        dict(name="rope_part_16001", kind="rope", tokens=16001, heads=20, head_dim=128, rotary_dim=32,
             layout="interleaved", scaling="bands", span=131072, packed=False),
        # A batch of 64 new tokens: written and read back.
        dict(name="quant_decode_64", kind="quant", format="e4m3", kv_heads=8, head_dim=128,
             start=_text(_spread(1, 64, 500, 2000)), new=_text([1] * 64), context=False),
        # A 256-token chunk of a prefill: written, then the context of 3000 read back for its attention.
        dict(name="quant_chunk_256", kind="quant", format="int8", kv_heads=8, head_dim=128, start="2744", new="256",
             context=True),
        # Prefixes of eight requests taken into an 8-bit cache at once.
        dict(name="quant_prefix_8", kind="quant", format="e4m3", kv_heads=8, head_dim=128, start=_text([0] * 8),
             new=_text(_spread(2, 8, 2000, 8000)), context=True),
        # One short request over a bf16 cache: the chain of launches.
        dict(name="attend_bf16_1x500", kind="attend", format="bf16", q_heads=32, kv_heads=8, head_dim=128,
             lengths="500"),
        # Eight migrated requests resumed in one batch.
        dict(name="attend_bf16_8", kind="attend", format="bf16", q_heads=64, kv_heads=8, head_dim=128,
             lengths=_text(ctx8)),
        # A full batch of sessions over an 8-bit cache.
        dict(name="attend_e4m3_64", kind="attend", format="e4m3", q_heads=64, kv_heads=8, head_dim=128,
             lengths=_text(_spread(3, 64, 500, 8000))),
        # A padded batch: five rows have no key; three query heads per KV head of 64.
        dict(name="attend_e4m3_pad", kind="attend", format="e4m3", q_heads=12, kv_heads=4, head_dim=64,
             lengths=_text(_spread(4, 27, 30, 2000) + [0] * 5)),
        # One long context, 131,071 positions: work split over its length alone.
        dict(name="attend_int8_long", kind="attend", format="int8", q_heads=64, kv_heads=8, head_dim=128,
             lengths="131071"),
        # The same of bf16, a few long documents.
        dict(name="attend_bf16_long", kind="attend", format="bf16", q_heads=32, kv_heads=8, head_dim=128,
             lengths="60001,33333,47"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    kind = rng.choice(("rope", "quant", "attend", "attend"))
    if kind == "rope":
        d = rng.choice((64, 80, 96, 128, 128, 256))
        r = rng.choice((d, d, d // 2, d // 4, 2 * rng.randint(1, d // 2)))
        return dict(kind=kind, tokens=_log(rng, 1, 16384), heads=rng.randint(1, 80), head_dim=d, rotary_dim=r,
                    layout=rng.choice(("half", "interleaved")), scaling=rng.choice(tuple(SCALING)),
                    span=_log(rng, 16384, 1 << 20), packed=rng.random() < 0.5)
    d = rng.choice((64, 128, 128))
    kvh = rng.choice((1, 2, 4, 5, 8, 8, 16))
    if kind == "quant":
        n = _log(rng, 1, 64)
        context = rng.random() < 0.5
        start = [rng.choice((0, _log(rng, 1, 4000))) for _ in range(n)]
        new = [_log(rng, 1, 4000) if context else rng.choice((1, 1, 1, rng.randint(1, 40))) for _ in range(n)]
        return dict(kind=kind, format=rng.choice(("e4m3", "int8")), kv_heads=kvh, head_dim=d, start=_text(start),
                    new=_text(new), context=context)
    n = rng.choice((1, 1, 2, 3, _log(rng, 1, 128)))
    top = _log(rng, 16, 131072)
    lengths = [0 if rng.random() < 0.03 else _log(rng, 1, top) for _ in range(n - 1)] + [top]
    return dict(kind=kind, format=rng.choice(("bf16", "e4m3", "int8")), q_heads=kvh * rng.choice((1, 2, 3, 4, 7, 8, 12)),
                kv_heads=kvh, head_dim=d, lengths=_text(lengths))


def draw(rng):
    most = {}
    for c in listed():
        for k, v in work(c).items():
            most[k] = max(most.get(k, 0), v)
        most["padded"] = max(most.get("padded", 0), _padded(c))
    while True:
        c = _draw_once(rng)
        w = work(c)
        if all(w[k] <= most[k] for k in w) and _padded(c) <= most["padded"]:
            return c


def _padded(case):
    """Elements of K that the plain form of attention gathers."""
    if case["kind"] != "attend":
        return 0
    lens = _ints(case["lengths"])
    return len(lens) * max(lens) * case["kv_heads"] * case["head_dim"]


def work(case):
    if case["kind"] == "rope":
        n = case["tokens"] * case["heads"] * case["head_dim"]
        return {"bytes": float(4 * n + 4 * case["tokens"]),
                "flops": 3.0 * case["tokens"] * case["heads"] * case["rotary_dim"]}
    if case["kind"] == "quant":
        start, new = _ints(case["start"]), _ints(case["new"])
        row = 2 * case["kv_heads"]                       # K and V rows of a token
        back = sum(new) + (sum(start) if case["context"] else 0)
        d = case["head_dim"]
        # written: bf16 in, codes and scale out; read back: codes and scale in, bf16 out
        return {"bytes": float(row * (3 * d + 4) * (sum(new) + back)), "flops": 2.0 * row * d * (sum(new) + back)}
    lens = _ints(case["lengths"])
    d, elem, scale = case["head_dim"], 2 if case["format"] == "bf16" else 1, 0 if case["format"] == "bf16" else 4
    keys = sum(lens)
    return {"bytes": float(keys * case["kv_heads"] * 2 * (d * elem + scale) + len(lens) * case["q_heads"] * (4 * d + 4)),
            "flops": 4.0 * keys * case["q_heads"] * d}


# ------------------------------------------------------------------ inputs
def _generator(seed, tag):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1000003 + tag) & 0x7FFFFFFF)
    return g


def _rows(tokens, heads, d, seed, tag):
    """Activations: normal, some channels of a head several times larger than the others."""
    g = _generator(seed, tag)
    channel = torch.exp(0.7 * torch.randn((heads, d), generator=g, device=DEV))
    return (torch.randn((tokens, heads, d), generator=g, device=DEV) * channel).to(torch.bfloat16)


def _tables(lengths, seed):
    """Block tables of sequences with room for `lengths` tokens, in a shuffled pool, and the pool's pages."""
    pages = [(n + PAGE - 1) // PAGE for n in lengths]
    total = sum(pages) + SPARE_PAGES
    order = np.random.Generator(np.random.PCG64(np.random.SeedSequence([int(seed), 7]))).permutation(total)
    bt = np.full((len(lengths), max(1, max(pages))), -1, dtype=np.int32)
    at = 0
    for i, n in enumerate(pages):
        bt[i, :n] = order[at:at + n]
        at += n
    return torch.from_numpy(bt).to(DEV), total


def _cached_rows(pages, case, seed, tag):
    return _rows(pages * PAGE, case["kv_heads"], case["head_dim"], seed, tag).view(
        pages, PAGE, case["kv_heads"], case["head_dim"])


def _filled(case, pages, seed):
    """An 8-bit pool whose layer LAYER holds quantised rows."""
    codes = torch.zeros((LAYERS, 2, pages, PAGE, case["kv_heads"], case["head_dim"]), dtype=torch.uint8, device=DEV)
    scales = torch.zeros((LAYERS, 2, pages, PAGE, case["kv_heads"]), dtype=torch.float32, device=DEV)
    for kv in range(2):
        c, s = _quantise(_cached_rows(pages, case, seed, 20 + kv), case["format"])
        codes[LAYER, kv] = c
        scales[LAYER, kv] = s
    return codes.view(torch.int8 if case["format"] == "int8" else torch.float8_e4m3fn), scales


def prepare(case, seed):
    s = {"case": case}
    if case["kind"] == "rope":
        T, H, d = case["tokens"], case["heads"], case["head_dim"]
        extra = max(1, H // 9) if case["packed"] else 0        # V heads behind Q and K in a row
        s["x"] = _rows(T, H + extra, d, seed, 1)[:, :H]
        if T <= 64:         # new tokens of as many requests
            s["positions"] = torch.randint(0, case["span"], (T,), generator=_generator(seed, 2), device=DEV,
                                           dtype=torch.int32)
        else:               # a prompt, or a chunk of one
            first = torch.randint(0, case["span"] - T + 1, (1,), generator=_generator(seed, 2), device=DEV)
            s["positions"] = (torch.arange(T, device=DEV) + first).to(torch.int32)
        if own:
            import paper_2608_16477_amd as P
            s["plan"] = P.pallas_rope_init(case["rotary_dim"], THETA, case["layout"], case["scaling"],
                                           **SCALING[case["scaling"]])
            s["out"] = torch.empty((T, H, d), dtype=torch.bfloat16, device=DEV)
        return s
    if case["kind"] == "quant":
        start, new = _ints(case["start"]), _ints(case["new"])
        H, d = case["kv_heads"], case["head_dim"]
        s["tables"], pages = _tables([a + b for a, b in zip(start, new)], seed)
        s["codes"], s["scales"] = _filled(case, pages, seed)
        s["k"], s["v"] = _rows(sum(new), H, d, seed, 3), _rows(sum(new), H, d, seed, 4)

        def tokens(first, count):
            seq = np.repeat(np.arange(len(count)), count)
            pos = np.concatenate([np.arange(a, a + b) for a, b in zip(first, count)])
            return [torch.from_numpy(x.astype(np.int32)).to(DEV) for x in (seq, pos)]

        s["seq"], s["pos"] = tokens(start, new)
        s["back_seq"], s["back_pos"] = s["seq"], s["pos"]
        if case["context"]:
            s["back_seq"], s["back_pos"] = tokens([0] * len(new), [a + b for a, b in zip(start, new)])
        n = s["back_pos"].numel()
        s["back_k"] = torch.empty((n, H, d), dtype=torch.bfloat16, device=DEV)
        s["back_v"] = torch.empty((n, H, d), dtype=torch.bfloat16, device=DEV)
        return s
    lens = _ints(case["lengths"])
    d = case["head_dim"]
    s["tables"], pages = _tables(lens, seed)
    s["lengths"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    s["longest"] = max(lens)
    s["q"] = _rows(len(lens), case["q_heads"], d, seed, 5)
    s["scale"] = 1.0 / math.sqrt(d)
    if case["format"] == "bf16":
        s["pool"] = torch.zeros((LAYERS, 2, pages, PAGE, case["kv_heads"], d), dtype=torch.bfloat16, device=DEV)
        for kv in range(2):
            s["pool"][LAYER, kv] = _cached_rows(pages, case, seed, 20 + kv)
    else:
        s["codes"], s["scales"] = _filled(case, pages, seed)
    if own:
        import paper_2608_16477_amd as P
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(s["q"].shape[:2], dtype=torch.float32, device=DEV)
        s["ws"] = torch.empty(P.pallas_attend_workspace_size(len(lens), case["q_heads"], case["kv_heads"], d, max(lens)),
                              dtype=torch.uint8, device=DEV)
    return s


# ------------------------------------------------------------------ plain forms
def _frequencies(case):
    """Radians per position of the rotary pairs, and the factor on the rotated values."""
    r, kind = case["rotary_dim"], case["scaling"]
    p = SCALING[kind]
    i = torch.arange(r // 2, dtype=torch.float64, device=DEV)
    theta = THETA
    if kind == "ntk" and r > 2:
        theta = THETA * p["factor"] ** (r / (r - 2))
    f = theta ** (-2.0 * i / r)
    if kind == "linear":
        return f / p["factor"], 1.0
    if kind == "yarn":
        # the pair index at which a pair makes `turns` turns over the trained length
        def pair(turns):
            return r * math.log(p["trained_len"] / (turns * 2 * math.pi)) / (2 * math.log(THETA))
        lo, hi = max(math.floor(pair(p["fast"])), 0), min(math.ceil(pair(p["slow"])), r - 1)
        slow = ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        return f * (1 - slow) + f / p["factor"] * slow, 0.1 * math.log(p["factor"]) + 1.0
    if kind == "bands":
        turns = p["trained_len"] * f / (2 * math.pi)
        keep = ((turns - p["slow"]) / (p["fast"] - p["slow"])).clamp(0, 1)
        return f * keep + f / p["factor"] * (1 - keep), 1.0
    return f, 1.0


def _rope(s):
    case = s["case"]
    r = case["rotary_dim"]
    f, magnitude = _frequencies(case)
    angle = s["positions"].to(torch.float64)[:, None] * f[None]      # 64 bits: far positions
    cos, sin = (angle.cos() * magnitude).float()[:, None], (angle.sin() * magnitude).float()[:, None]
    x = s["x"].float()
    y = x.clone()
    if case["layout"] == "half":
        a, b = slice(0, r // 2), slice(r // 2, r)
    else:
        a, b = slice(0, r, 2), slice(1, r, 2)
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    return y.to(torch.bfloat16)


def _quantise(x, fmt):
    """Codes (uint8 patterns) and scales of the rows of x."""
    x = x.float()
    top = x.abs().amax(dim=-1)
    one = torch.ones_like(top)
    if fmt == "int8":
        up = torch.where(top > 0, 127.0 / torch.where(top > 0, top, one), 0 * one)
        codes = torch.round(x * up[..., None]).clamp(-127, 127).to(torch.int8)
        return codes.view(torch.uint8), top / torch.full_like(top, 127.0)
    m, e = torch.frexp(top)                     # top = m 2^e, m in [1/2, 1): at most 448 = (7/8) 2^9 after scaling
    e = torch.where(m > 0.875, e - 8, e - 9).clamp(min=-126)
    scale = torch.where(top > 0, torch.ldexp(one, e), 0 * one)
    up = torch.where(top > 0, torch.ldexp(one, -e), 0 * one)
    codes = (x * up[..., None]).to(torch.float8_e4m3fn)
    return codes.view(torch.uint8), scale


def _slots(tables, seq, pos):
    return tables[seq.long(), pos.long() // PAGE].long(), pos.long() % PAGE


def _values(codes, scales):
    return codes.float() * scales[..., None]


def _quant(s):
    case = s["case"]
    pg, slot = _slots(s["tables"], s["seq"], s["pos"])
    raw = s["codes"].view(torch.uint8)
    for kv, rows in ((0, s["k"]), (1, s["v"])):
        c, sc = _quantise(rows, case["format"])
        raw[LAYER, kv, pg, slot] = c
        s["scales"][LAYER, kv, pg, slot] = sc
    pg, slot = _slots(s["tables"], s["back_seq"], s["back_pos"])
    typed = torch.int8 if case["format"] == "int8" else torch.float8_e4m3fn
    k, v = (_values(raw[LAYER, kv, pg, slot].view(typed), s["scales"][LAYER, kv, pg, slot]).to(torch.bfloat16)
            for kv in (0, 1))
    return k, v, s["scales"]


def _attend(s):
    case = s["case"]
    S, longest, d = s["q"].shape[0], s["longest"], case["head_dim"]
    kvh, group = case["kv_heads"], case["q_heads"] // case["kv_heads"]
    j = torch.arange(longest, device=DEV)
    valid = j[None] < s["lengths"][:, None]                               # [S, longest]
    pg = s["tables"].long()[:, j // PAGE].clamp(min=0)
    slot = (j % PAGE)[None].expand(S, -1)

    def gather(kv):                                                      # [S, kvh, longest, d], float32
        if case["format"] == "bf16":
            x = s["pool"][LAYER, kv][pg, slot].float()
        else:
            raw = s["codes"].view(torch.uint8)[LAYER, kv][pg, slot]
            x = _values(raw.view(s["codes"].dtype), s["scales"][LAYER, kv][pg, slot])
        return x.masked_fill(~valid[..., None, None], 0.0).permute(0, 2, 1, 3).contiguous()

    q = s["q"].float().view(S, kvh, group, d).transpose(2, 3).contiguous()
    score = torch.matmul(gather(0), q) * s["scale"]                       # [S, kvh, longest, group]
    score = score.masked_fill(~valid[:, None, :, None], -math.inf)
    top = score.amax(dim=2, keepdim=True)
    p = torch.exp(score - top.masked_fill(top == -math.inf, 0.0))
    total = p.sum(dim=2, keepdim=True)
    lse = (top + torch.log(total)).view(S, case["q_heads"])
    p = (p / total.masked_fill(total == 0, 1.0)).transpose(2, 3).contiguous()
    out = torch.matmul(p, gather(1)).reshape(S, case["q_heads"], d)
    return out.to(torch.bfloat16), lse


def run(state):
    s = state
    kind = s["case"]["kind"]
    if own:
        import paper_2608_16477_amd as P
        if kind == "rope":
            P.pallas_rope_apply(s["plan"], s["x"], s["positions"], s["out"])
            return s["out"]
        if kind == "quant":
            P.pallas_quant_store(s["codes"], s["scales"], LAYER, s["k"], s["v"], s["pos"], s["tables"],
                                 seq_ids=s["seq"])
            P.pallas_quant_load(s["codes"], s["scales"], LAYER, s["back_k"], s["back_v"], s["back_pos"], s["tables"],
                                seq_ids=s["back_seq"])
            return s["back_k"], s["back_v"], s["scales"]
        if s["case"]["format"] == "bf16":
            P.pallas_attend_kv(s["pool"], LAYER, s["q"], s["lengths"], s["longest"], s["tables"], s["scale"], s["out"],
                               s["ws"], lse=s["lse"])
        else:
            P.pallas_attend_quant(s["codes"], s["scales"], LAYER, s["q"], s["lengths"], s["longest"], s["tables"],
                                  s["scale"], s["out"], s["ws"], lse=s["lse"])
        return s["out"], s["lse"]
    return {"rope": _rope, "quant": _quant, "attend": _attend}[kind](s)


# ------------------------------------------------------------------ 64 bits
def _row_values64(x, fmt):
    """What the rows of x stand for after quantisation, in 64 bits, and their scales."""
    x = x.double()
    top = x.abs().max(dim=-1, keepdim=True).values
    some = torch.where(top > 0, top, torch.ones_like(top))
    if fmt == "int8":
        step = top / 127.0
        return torch.round(x / (some / 127.0)).clamp(-127, 127) * step, step[..., 0]
    unit = torch.exp2(torch.ceil(torch.log2(some / 448.0)))              # the least power of two that fits
    y = x / unit
    lead = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -20))).clamp(min=-6)
    grid = torch.exp2(lead - 3)                                          # 3 bits behind the leading one
    return torch.round(y / grid) * grid * unit, torch.where(top > 0, unit, 0 * unit)[..., 0]


def _exact_rope(s):
    case = s["case"]
    r, kind = case["rotary_dim"], case["scaling"]
    p = SCALING[kind]
    pos = s["positions"].double().cpu().numpy()
    x = s["x"].double().cpu().numpy()
    y = x.copy()
    magnitude = 0.1 * math.log(p["factor"]) + 1.0 if kind == "yarn" else 1.0
    for i in range(r // 2):
        base = THETA * p["factor"] ** (r / (r - 2.0)) if kind == "ntk" and r > 2 else THETA
        f = base ** (-2.0 * i / r)
        if kind == "linear":
            f /= p["factor"]
        elif kind == "yarn":
            at = [r * math.log(p["trained_len"] / (t * 2 * math.pi)) / (2 * math.log(THETA)) for t in (p["fast"], p["slow"])]
            lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), r - 1)
            w = min(max((i - lo) / max(hi - lo, 0.001), 0.0), 1.0)
            f = f * (1 - w) + w * f / p["factor"]
        elif kind == "bands":
            w = min(max((p["trained_len"] * f / (2 * math.pi) - p["slow"]) / (p["fast"] - p["slow"]), 0.0), 1.0)
            f = w * f + (1 - w) * f / p["factor"]
        a, b = (i, i + r // 2) if case["layout"] == "half" else (2 * i, 2 * i + 1)
        c, sn = (np.cos(pos * f) * magnitude)[:, None], (np.sin(pos * f) * magnitude)[:, None]
        y[:, :, a] = x[:, :, a] * c - x[:, :, b] * sn
        y[:, :, b] = x[:, :, b] * c + x[:, :, a] * sn
    return y


def _exact_quant(s):
    case = s["case"]
    start, new = _ints(case["start"]), _ints(case["new"])
    cut = np.cumsum([0] + new)
    scales = s["scales"].double()
    stored = [_row_values64(s[n], case["format"]) for n in ("k", "v")]
    outs = []
    for kv, (values, unit) in enumerate(stored):
        parts = []
        for i in range(len(new)):
            def place(a, b):
                t = torch.arange(a, b, device=DEV)
                return s["tables"][i].long()[t // PAGE], t % PAGE
            pg, slot = place(start[i], start[i] + new[i])
            scales[LAYER, kv, pg, slot] = unit[cut[i]:cut[i + 1]]
            if case["context"] and start[i]:
                pg, slot = place(0, start[i])
                parts.append(s["codes"][LAYER, kv].view(torch.uint8)[pg, slot].view(s["codes"].dtype).to(torch.float64)
                             * s["scales"][LAYER, kv, pg, slot].double()[..., None])
            parts.append(values[cut[i]:cut[i + 1]])
        outs.append(torch.cat(parts))
    return outs[0], outs[1], scales


def _exact_attend(s):
    case = s["case"]
    d, kvh = case["head_dim"], case["kv_heads"]
    group = case["q_heads"] // kvh
    outs, lses = [], []
    for i, n in enumerate(_ints(case["lengths"])):
        if n == 0:
            outs.append(torch.zeros((case["q_heads"], d), dtype=torch.float64, device=DEV))
            lses.append(torch.full((case["q_heads"],), -math.inf, dtype=torch.float64, device=DEV))
            continue
        t = torch.arange(n, device=DEV)
        pg, slot = s["tables"][i].long()[t // PAGE], t % PAGE
        rows = []
        for kv in range(2):
            if case["format"] == "bf16":
                rows.append(s["pool"][LAYER, kv, pg, slot].double())
            else:
                c = s["codes"].view(torch.uint8)[LAYER, kv, pg, slot].view(s["codes"].dtype)
                rows.append(c.to(torch.float64) * s["scales"][LAYER, kv, pg, slot].double()[..., None])
        heads, sums = [], []
        for h in range(case["q_heads"]):
            k, v = rows[0][:, h // group], rows[1][:, h // group]
            z = (k * s["q"][i, h].double()).sum(-1) * s["scale"]
            lse = torch.logsumexp(z, 0)
            heads.append((torch.exp(z - lse)[:, None] * v).sum(0))
            sums.append(lse)
        outs.append(torch.stack(heads))
        lses.append(torch.stack(sums))
    return torch.stack(outs), torch.stack(lses)


def exact(case, seed):
    w = work(case)
    if w["bytes"] > 2e9 or w["flops"] > 2e11:
        return None                                     # too long in 64 bits
    s = prepare(case, seed)
    return {"rope": _exact_rope, "quant": _exact_quant, "attend": _exact_attend}[case["kind"]](s)
