"""The three ways in which attention of one new token is run (one workgroup a row, splits
and a join, ranges and a join), restated from the lengths, and read back from the
workspace of a call: a test that means one of them fails when a call takes another."""
import numpy as np
import torch


def _waves(fmt, d):
    return 1024 // (2 * d if fmt == "bf16" else d)


def _blocks(n):
    return -(-int(n) // 32)


def launch_form(fmt, d, hq, hkv, lens, max_length):
    """("short" | "split" | "ranges", int2 per row that the call leaves at the head of its workspace; None: as it was)."""
    heads = hkv * -(-(hq // hkv) // 16)
    rows, most = len(lens) * heads, _blocks(max_length)
    if max_length <= 512 and rows <= 1536:
        return "short", [None] * len(lens)
    for each in (1, 2):
        per = min(_waves(fmt, d), 8) * each
        splits = -(-most // per)
        if rows * splits <= 256:
            if splits == 1:
                return "short", [None] * len(lens)
            return "split", [(s * splits - s, 0 if _blocks(n) <= per else -(-_blocks(n) // per)) for s, n in enumerate(lens)]
    each = blocks_per_range(fmt, d, hq, hkv, lens)
    total, at, parts = sum(map(_blocks, lens)), 0, []
    for n in lens:
        end = at + _blocks(n)
        r = at // each
        parts.append(None if n == 0 else (r, 0 if end <= min((r + 1) * each, total) else (end - 1) // each - r + 1))
        at = end
    return "ranges", parts


def blocks_per_range(fmt, d, hq, hkv, lens):
    ranges = max(256 * _waves(fmt, d) // (hkv * -(-(hq // hkv) // 16)) // 8 * 8, 8)
    total = sum(map(_blocks, lens))
    if 2 * total <= ranges and total <= 32 * len(lens):
        return 1
    if total <= 2 * ranges:
        return 2
    rounds = max(-(-total // (32 * ranges)), 1)
    return -(-total // (rounds * ranges))


def check_form(form, ws, fmt, d, hq, hkv, lens, max_length):
    """`ws`: the call's workspace, all 0xFF before it."""
    want, parts = launch_form(fmt, d, hq, hkv, lens, max_length)
    assert want == form.split("-")[0], (want, form)
    if want == "short":      # (nothing is written)
        assert bool((ws == 0xFF).all())
        return
    got = ws[:8 * len(lens)].cpu().numpy().view(np.int32).reshape(-1, 2)
    for s, (g, w) in enumerate(zip(got.tolist(), parts)):
        assert g == list(w if w is not None else (-1, -1)), (form, s, g, w)


#: form -> (KV heads, lengths, max_length, blocks of a range or None): head_dim 128, 3 query heads per KV head
FORMS = {
    "short": (2, [400, 90, 20, 33, 0, 500], 500, None),
    "split": (2, [1500, 90, 20, 33, 0, 700], 1500, None),
    "ranges-1": (2, [1500, 90, 20, 33, 0, 700], 20000, 1),
    "ranges-2": (2, [3000, 1500, 0, 33], 20000, 2),
    "ranges-3": (8, [9000, 90, 20, 33, 0, 700, 8000, 4000, 300], 9000, 3),     # 3 of 8-bit rows, 6 of bf16 ones
}


def fresh_workspace(P, S, hq, hkv, d, max_length):
    return torch.full((P.pallas_attend_workspace_size(S, hq, hkv, d, max_length),), 0xFF, dtype=torch.uint8, device="cuda")
