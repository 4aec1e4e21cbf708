"""Four operators of a paged cache in 4 bits, in plain form and through the library, with cases to time.

    step     block tables and slots on the GPU: rows that ended give their pages back, rows with new tokens get pages
    append   new keys (normed, rotated) and values into the 4-bit pages, the step's queries on the way, and the new tokens
             read back as the values that the cache now holds for them
    load     tokens of a 4-bit cache by their slots, as dense keys and values
    attend   attention over the 4-bit pages: single tokens, drafts and chunks of prompts, behind shared prefixes or not

The cache: 16 coordinates of a head share a scale S, their largest magnitude rounded up to 4 significant bits (no finer than
2^-17); code n = floor(8 x / S) + 8, at most 15, stands for (n - 7.5) S / 8. A cell holds 16 tokens of a page and head: key codes,
key scales, value codes, value scales. Eight codes lie in 32 bits: even ones in the low half, odd ones in the high half, each
half rotated left by 2. A scale is the upper byte of the fp16's 15 bits without sign.

`own` = False computes them with elementary torch operations in 32 bits (quotients next to a border and angles in 64), True calls
paper_2402_06082_b200.binding. Lengths of a case come from the case alone (its "mix"), values from the seed.
"""
import math
import random

import numpy as np
import torch

own = False

BASE, EPS = 10000.0, 1e-6
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ---- cases --------------------------------------------------------------------------------------------------------

def _step(B, added_lo, added_hi, ctx, page, ended, mix=0):
    return {"op": "step", "B": B, "added_lo": added_lo, "added_hi": added_hi, "ctx": ctx, "page": page, "ended": ended, "mix": mix}


def _append(B, new_lo, new_hi, ctx, H, Hkv, d, dtype, page, norm, mix=0):
    return {"op": "append", "B": B, "new_lo": new_lo, "new_hi": new_hi, "ctx": ctx, "H": H, "Hkv": Hkv, "d": d, "dtype": dtype,
            "page": page, "norm": norm, "mix": mix}


def _load(n, ctx, Hkv, d, dtype, page, mix=0):
    return {"op": "load", "n": n, "ctx": ctx, "Hkv": Hkv, "d": d, "dtype": dtype, "page": page, "mix": mix}


def _attend(B, new_lo, new_hi, own_lo, own_hi, prefix, groups, H, Hkv, d, dtype, page, mix=0):
    return {"op": "attend", "B": B, "new_lo": new_lo, "new_hi": new_hi, "own_lo": own_lo, "own_hi": own_hi, "prefix": prefix,
            "groups": groups, "H": H, "Hkv": Hkv, "d": d, "dtype": dtype, "page": page, "mix": mix}


def listed():
    cases = {
        # the tables of a decoding step: 64 rows, a token each, some rows end
        "step of 64": _step(64, 1, 1, 8192, 16, 4),
        # the tables of a step that also takes prompts in: 1024 rows, over 100 K new tokens
        "step with prompts": _step(1024, 0, 255, 16384, 16, 128),
        # one step of 64 sequences into pages of 16, heads normed and rotated
        "append step": _append(64, 1, 1, 4096, 32, 8, 128, "bf16", 16, True),
        # chunks of eight prompts of odd lengths into pages of 64
        "append prompt chunks": _append(8, 1025, 4095, 8192, 32, 8, 128, "bf16", 64, False),
        # a whole context back as dense keys and values, as a prefill takes them
        "load a context": _load(32768, 32768, 8, 128, "bf16", 64),
        # some hundred tokens of a 32-bit path with heads of 64
        "load some fp32": _load(333, 5000, 8, 64, "fp32", 32),
        # one short sequence: latency
        "attend one short": _attend(1, 1, 1, 1000, 1000, 0, 0, 32, 8, 128, "bf16", 16),
        # one long sequence: the cache read once
        "attend one long": _attend(1, 1, 1, 131072, 131072, 0, 0, 32, 8, 128, "bf16", 64),
        # a step of 64 sequences of all lengths, pages of 16
        "attend batch": _attend(64, 1, 1, 17, 8191, 0, 0, 32, 8, 128, "bf16", 16),
        # drafted tokens of 16 sequences behind two system prompts of odd length
        "attend drafts": _attend(16, 1, 8, 17, 4095, 16383, 2, 32, 8, 128, "bf16", 16),
        # chunks of four prompts behind a shared document
        "attend prompt chunks": _attend(4, 513, 2047, 2048, 4096, 8192, 1, 32, 8, 128, "bf16", 128),
        # 32-bit queries, heads of 64, one key head per query head
        "attend fp32": _attend(8, 1, 3, 100, 1500, 2001, 1, 8, 8, 64, "fp32", 32),
    }
    return [dict(c, name=name) for name, c in cases.items()]


def _between(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 6.5, w["flops"] / (1700.0 if case.get("dtype") != "fp32" else 50.0))


def _most(op):
    return max(_cost(c) for c in listed() if c["op"] == op)


def draw(rng):
    op = rng.choice(["step", "append", "load", "attend", "attend", "attend"])
    while True:
        d, dtype, page = rng.choice([64, 128, 128]), rng.choice(["bf16", "bf16", "bf16", "fp32"]), rng.choice([16, 32, 64, 128])
        Hkv = rng.choice([1, 2, 4, 8, 8, 32])
        H, mix = Hkv * rng.choice([1, 2, 4, 8] if Hkv <= 8 else [1]), rng.randrange(1 << 20)
        if op == "step":
            B = _between(rng, 1, 1024)
            hi = _between(rng, 1, 2047)
            case = _step(B, rng.choice([0, 1, hi]), hi, _between(rng, 16, 32768), page, rng.randint(0, B // 4), mix)
        elif op == "append":
            hi = _between(rng, 1, 4095)
            case = _append(_between(rng, 1, 128), rng.randint(1, hi), hi, _between(rng, 64, 8192), H, Hkv, d, dtype, page, rng.random() < 0.5, mix)
        elif op == "load":
            ctx = _between(rng, 16, 65536)
            case = _load(_between(rng, 1, ctx), ctx, Hkv, d, dtype, page, mix)
        else:
            hi, own_hi = rng.choice([1, 1, _between(rng, 1, 8), _between(rng, 8, 2047)]), _between(rng, 1, 65536)
            own_hi = max(hi, own_hi)
            prefix = rng.choice([0, 0, _between(rng, 1, 65536)])
            B = _between(rng, 1, 64)
            case = _attend(B, rng.randint(1, hi), hi, rng.randint(hi, own_hi), own_hi, prefix, min(B, rng.choice([1, 1, 2, 3])) if prefix else 0,
                           H, Hkv, d, dtype, page, mix)
        if op == "attend":
            small = _shape(case)["cells"] < 2e9                          # scores that the plain form holds at once
        elif op == "step":
            small = case["B"] * (case["added_lo"] + case["added_hi"]) <= 262144
        else:
            small = op == "load" or case["B"] * (case["ctx"] + hi) * Hkv * d < 1e9
        if small and _cost(case) <= _most(op):
            return case


# ---- lengths and work ---------------------------------------------------------------------------------------------

def _shape(c):
    """The lengths of a case: new tokens, own tokens (the new ones among them), groups of sequences and their prefixes."""
    r = random.Random(c["mix"])
    if c["op"] == "load":
        return {"new": [0], "own": [c["ctx"]], "groups": 0, "edges": [], "prefix": []}
    B = c["B"]
    if c["op"] == "step":
        added = [r.randint(c["added_lo"], c["added_hi"]) for _ in range(B)]
        have = [r.randint(0, c["ctx"]) for _ in range(B)]
        ended = set(r.sample(range(B), c["ended"]))
        return {"added": [0 if b in ended else k for b, k in enumerate(added)], "have": have, "ended": [int(b in ended) for b in range(B)]}
    new = [r.randint(c["new_lo"], c["new_hi"]) for _ in range(B)]
    if c["op"] == "append":
        return {"new": new, "own": [k + r.randint(0, c["ctx"]) for k in new], "groups": 0, "edges": [], "prefix": []}
    length = [max(k, r.randint(c["own_lo"], c["own_hi"])) for k in new]
    g = c["groups"]
    edges = [0] + sorted(r.sample(range(1, B), g - 1)) + [B] if g else []
    prefix = [c["prefix"]] + [r.randint(max(1, c["prefix"] // 2), c["prefix"]) for _ in range(g - 1)] if g else []
    rows = max([sum(new[edges[i]:edges[i + 1]]) for i in range(g)] + [0])
    return {"new": new, "own": length, "groups": g, "edges": edges, "prefix": prefix,
            "cells": c["H"] * (B * max(new) * max(length) + g * rows * c["prefix"]) + 4 * B * c["Hkv"] * max(length) * c["d"]}


def _pages_of(length, page):
    return -(-length // page)


def work(c):
    s = _shape(c)
    if c["op"] == "step":
        n, page = sum(s["added"]), c["page"]
        moved = sum(_pages_of(h, page) for h, e in zip(s["have"], s["ended"]) if e)
        taken = sum(_pages_of(h + k, page) - _pages_of(h, page) for h, k, e in zip(s["have"], s["added"], s["ended"]) if not e)
        return {"bytes": 20 * c["B"] + 12 * n + 8 * (moved + taken), "flops": 4 * n + 16 * c["B"]}
    e, d, Hkv = (4 if c["dtype"] == "fp32" else 2), c["d"], c["Hkv"]
    row = 2 * (d // 2 + d // 16)                                             # a token's keys and values in one head
    if c["op"] == "load":
        return {"bytes": c["n"] * (Hkv * (row + 2 * d * e) + 8), "flops": 4 * c["n"] * Hkv * d}
    H, n = c["H"], sum(s["new"])
    if c["op"] == "append":
        return {"bytes": n * (2 * H * d * e + Hkv * (2 * d * e + row + 2 * d * e)), "flops": n * ((8 if c["norm"] else 3) * H * d + 20 * Hkv * d)}
    pairs = sum(k * m - k * (k - 1) // 2 for k, m in zip(s["new"], s["own"]))
    pairs += sum(sum(s["new"][s["edges"][g]:s["edges"][g + 1]]) * s["prefix"][g] for g in range(s["groups"]))
    return {"bytes": (sum(s["own"]) + sum(s["prefix"])) * Hkv * row + 2 * n * H * d * e, "flops": 4 * pairs * H * d}


# ---- the format ---------------------------------------------------------------------------------------------------

def _groups(x):
    """x [..., d] in 32 bits -> scales [..., d / 16] in 32 bits and codes [..., d] (int32)."""
    x = x.unflatten(-1, (-1, 16))
    a = x.abs().amax(-1)
    m, e = torch.frexp(a)                                                    # a = m 2^e, m in [1/2, 1)
    scale = torch.where(a < 2.0 ** -14, torch.ceil(a * 2.0 ** 17) * 2.0 ** -17, torch.ldexp(torch.ceil(m * 16), e - 4))
    scale = torch.where(a <= 61440.0, scale, torch.full_like(scale, math.nan))
    n = torch.floor(8 * x.double() / scale[..., None].double()).nan_to_num(0.0) + 8      # 0 / 0: the group is all 0
    return scale, n.clamp(0, 15).to(torch.int32).flatten(-2)


def _packed(scale, code):
    """Bytes of the codes [..., d / 2] and of the scales [..., d / 16]."""
    c = code.unflatten(-1, (-1, 4, 2)).transpose(-1, -2)                     # [..., d / 8, low or high half, its four codes]
    w = c[..., 0] | c[..., 1] << 4 | c[..., 2] << 8 | c[..., 3] << 12
    w = (w << 2 | w >> 14) & 0xffff
    codes = torch.stack((w & 255, w >> 8), -1).flatten(-3).to(torch.uint8)
    byte = torch.where(scale.isnan(), torch.full_like(scale, 255), (scale.to(torch.float16).view(torch.int16) >> 7).float())
    return codes, byte.to(torch.uint8)


def _values(codes, scales):
    """What the bytes stand for, in 32 bits: codes [..., d / 2], scales [..., d / 16] -> [..., d]."""
    b = codes.to(torch.int32).unflatten(-1, (-1, 2, 2))
    w = b[..., 0] | b[..., 1] << 8
    w = w >> 2 | (w & 3) << 14
    n = torch.stack((w & 15, w >> 4 & 15, w >> 8 & 15, w >> 12), -1)         # [..., d / 8, half, four]
    n = n.transpose(-1, -2).flatten(-3).float()
    s = (scales.to(torch.int16) << 7).view(torch.float16).float()
    return ((n.unflatten(-1, (-1, 16)) - 7.5) * (s / 8)[..., None]).flatten(-2)


def _parts(pool, page, d):
    """Views of a pool [pages, Hkv, bytes]: for keys and for values their codes [pages, Hkv, cells, 16, d / 2] and scales."""
    x = pool.unflatten(-1, (page // 16, 2, 16 * (d // 2 + d // 16)))
    codes, scales = x[..., : 8 * d].unflatten(-1, (16, d // 2)), x[..., 8 * d:].unflatten(-1, (16, d // 16))
    return [(codes[:, :, :, i], scales[:, :, :, i]) for i in range(2)]


# ---- inputs -------------------------------------------------------------------------------------------------------

def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _prepare_step(c, g):
    s, page, B = _shape(c), c["page"], c["B"]
    held = [_pages_of(h, page) for h in s["have"]]
    taken = sum(_pages_of(h + k, page) - n for h, k, n in zip(s["have"], s["added"], held))
    pages = sum(held) + taken + 37                                           # some stay free
    perm = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    wide = _pages_of(c["ctx"] + c["added_hi"], page) + 1
    at = np.full((B, wide), -1, np.int64)
    first = 0
    for b, k in enumerate(held):
        at[b, :k] = first + np.arange(k)
        first += k
    at = torch.from_numpy(at).cuda()
    free = torch.zeros(pages, dtype=torch.int32, device="cuda")
    free[: pages - first] = perm[first:]
    return {"case": c, "table": torch.where(at >= 0, perm[at.clamp(min=0)], torch.full((), -1, dtype=torch.int32, device="cuda")),
            "free": free, "free_count": _ints([pages - first]), "lengths": _ints(s["have"]), "added": _ints(s["added"]), "ended": _ints(s["ended"]),
            "n": max(1, sum(s["added"])) + 5}                                # the rows of the step's tensors, a few of them padding


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    if c["op"] == "step":
        return _prepare_step(c, g)
    dt, Hkv, d, page = TYPES[c["dtype"]], c["Hkv"], c["d"], c["page"]
    shape = _shape(c)
    s = {"case": c, "shape": shape}
    own_pages = [_pages_of(x, page) for x in shape["own"]]
    pre_pages = [_pages_of(x, page) for x in shape["prefix"]]
    pages, n, groups = sum(own_pages) + sum(pre_pages), sum(shape["new"]), shape["groups"]
    perm = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)     # pages lie anywhere in the pool

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda", dtype=dt)

    def weight():
        return (1 + 0.1 * torch.randn(d, generator=g, device="cuda")).to(dt)

    def tables(counts, first):
        at = np.full((len(counts), max(counts)), -1, np.int64)
        for i, k in enumerate(counts):
            at[i, :k] = first + np.arange(k)
            first += k
        at = torch.from_numpy(at).cuda()
        return torch.where(at >= 0, perm[at.clamp(min=0)], torch.zeros((), dtype=torch.int32, device="cuda"))

    # a pool that earlier calls have filled: normal keys and values, rounded into their cells a few pages at a time
    s["pool"] = torch.zeros(pages, Hkv, page * 2 * (d // 2 + d // 16), dtype=torch.uint8, device="cuda")
    some = max(1, (1 << 24) // (Hkv * page * d))
    for codes, scales in _parts(s["pool"], page, d):
        for i in range(0, pages, some):
            x = torch.randn(min(some, pages - i), Hkv, page // 16, 16, d, generator=g, device="cuda")
            codes[i:i + some], scales[i:i + some] = _packed(*_groups(x))
    s["table"] = tables(own_pages, 0)
    s["lengths"] = _ints(shape["own"])
    s["cu_q"] = _ints([0] + np.cumsum(shape["new"]).tolist())
    if groups:
        s["cu_group"], s["prefix_len"] = _ints(shape["edges"]), _ints(shape["prefix"])
        s["prefix_table"] = tables(pre_pages, sum(own_pages))
    if c["op"] == "load":
        at = torch.arange(c["ctx"] - c["n"], c["ctx"], device="cuda")
        s["slots"] = s["table"][0, at // page].long() * page + at % page
    elif c["op"] == "append":
        H = c["H"]
        qkv = randn(n, (H + 2 * Hkv) * d)                                    # the fused projection that the heads are views of
        s["q"], s["k"] = qkv[:, : H * d].view(n, H, d), qkv[:, H * d: (H + Hkv) * d].view(n, Hkv, d)
        s["v"] = qkv[:, (H + Hkv) * d:].view(n, Hkv, d)
        s["wq"], s["wk"] = (weight(), weight()) if c["norm"] else (None, None)
        seq, at = _tokens(s)
        s["slots"] = s["table"][seq, at // page].long() * page + at % page   # as the step's tables give them
    else:
        s["q"] = randn(n, c["H"], d)
    if own:
        from paper_2402_06082_b200 import binding
        s["cache"] = binding.PagedCache4(s["pool"], page, d)
        if c["op"] == "append":
            s["rope"] = binding.Rope(d, base=BASE)
        if c["op"] != "load":
            s["batch"] = binding.PagedBatch(s["cu_q"], s["lengths"], s["table"], s.get("cu_group"), s.get("prefix_len"), s.get("prefix_table"))
    return s


# ---- plain forms --------------------------------------------------------------------------------------------------

def _step_plain(s):
    page, table, free, n = s["case"]["page"], s["table"], s["free"], s["n"]
    had, added, ended = s["lengths"].long(), s["added"].long(), s["ended"] != 0
    wide, cap = table.shape[1], free.shape[0]
    k = torch.arange(wide, device="cuda")
    held = (had + page - 1) // page
    back = torch.where(ended, held, 0)                                       # pages that go back, in order of rows and places
    before = back.cumsum(0) - back
    count = s["free_count"].long()
    spot = torch.where(k < back[:, None], count + before[:, None] + k, cap)
    pushed = torch.cat((free, free.new_zeros(1))).scatter(0, spot.flatten(), table.flatten())[:cap]
    top = count + back.sum()
    kept = torch.where(ended, 0, had)
    first = (kept + page - 1) // page
    want = (kept + added + page - 1) // page - first
    fits = ((want == 0) | (want.cumsum(0) <= top)) & ((added == 0) | (added.cumsum(0) <= n)) & (first + want <= wide)
    added, want = torch.where(fits, added, 0), torch.where(fits, want, 0)
    at = want.cumsum(0) - want
    fill = (k >= first[:, None]) & (k < (first + want)[:, None])
    taken = pushed[(top - 1 - at[:, None] - (k - first[:, None])).clamp(0, cap - 1)]
    table.copy_(torch.where(fill, taken, table))
    free.copy_(pushed)
    cu = torch.cat((added.new_zeros(1), added.cumsum(0)))
    tok = torch.arange(n, device="cuda")
    row = torch.searchsorted(cu[1:].contiguous(), tok, right=True).clamp(max=table.shape[0] - 1)
    place = kept[row] + tok - cu[row]
    there = tok < cu[-1]
    slot = table[row, (place // page).clamp(0, wide - 1)].long() * page + place % page
    return {"cu_q": cu.int(), "lengths": (kept + added).int(), "free_count": (top - want.sum()).int(), "table": table, "free": free,
            "slots": torch.where(there, slot, -1), "positions": torch.where(there, place, 0).int()}


def _rotated(x, pos, w):
    """RMS norm over the head (if there is a weight), then the rotation; 32 bits, the angles in 64."""
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
    half = x.shape[-1] // 2
    angle = (pos.double()[:, None] * BASE ** (-torch.arange(half, device=x.device, dtype=torch.float64) / half))[:, None, :]
    cos, sin = angle.cos().float(), angle.sin().float()
    a, b = x[..., :half], x[..., half:]
    return torch.cat((a * cos - b * sin, b * cos + a * sin), -1)


def _tokens(s):
    """For each new token its sequence and its place among that sequence's own tokens."""
    cu, lengths = s["cu_q"].long(), s["lengths"].long()
    tok = torch.arange(s["q"].shape[0], device="cuda")
    seq = torch.searchsorted(cu[1:].contiguous(), tok, right=True)
    return seq, lengths[seq] - cu[seq + 1] + tok


def _append_plain(s):
    c = s["case"]
    seq, at = _tokens(s)
    page = c["page"]
    where, row = s["table"][seq, at // page].long(), at % page
    new = []
    for (codes, scales), x in zip(_parts(s["pool"], page, c["d"]), (_rotated(s["k"], at, s["wk"]), s["v"].float())):
        a, b = _packed(*_groups(x))
        codes[where, :, row // 16, row % 16], scales[where, :, row // 16, row % 16] = a, b
        new.append(_values(a, b).to(s["k"].dtype))
    return _rotated(s["q"], at, s["wq"]).to(s["q"].dtype), new[0], new[1]


def _load_plain(s):
    c = s["case"]
    page, row = c["page"], s["slots"] % c["page"]
    where = (s["slots"] // page, slice(None), row // 16, row % 16)
    return tuple(_values(codes[where], scales[where]).to(TYPES[c["dtype"]]) for codes, scales in _parts(s["pool"], page, c["d"]))


def _pages(codes, scales, table, length):
    """[rows of the table, Hkv, length, d] in 32 bits."""
    x = _values(codes[table.long()], scales[table.long()]).transpose(1, 2)   # [rows, pages, Hkv, cells, 16, d], pages first
    return x.reshape(x.shape[0], x.shape[1], -1, x.shape[-1])[:, :, :length]


def _part(q, K, V, limit):
    """Largest score, sum and weighted values of every query row: q [S, T, H, d], K and V [S, Hkv, L, d], limit [S, T]."""
    S, T, H, d = q.shape
    Hkv, L = K.shape[1], K.shape[2]
    q = q.reshape(S, T, Hkv, H // Hkv, d).permute(0, 2, 1, 3, 4).reshape(S, Hkv, -1, d)
    seen = torch.arange(L, device=q.device) < limit[..., None]
    scores = (q @ K.transpose(-1, -2) * d ** -0.5).view(S, Hkv, T, H // Hkv, L)
    scores = scores.masked_fill(~seen[:, None, :, None], -math.inf)
    m = scores.amax(-1, keepdim=True).clamp(min=-1e30)
    p = (scores - m).exp()
    V = torch.where((torch.arange(L, device=q.device) < limit.amax(1)[:, None])[:, None, :, None], V, 0.0)
    z = p.view(S, Hkv, -1, L) @ V
    back = lambda x: x.reshape(S, Hkv, T, H // Hkv, -1).permute(0, 2, 1, 3, 4).reshape(S, T, H, -1)  # noqa: E731
    return back(m), back(p.sum(-1)), back(z)


def _attend_plain(s):
    c, shape, cu = s["case"], s["shape"], s["cu_q"].long()
    n = s["q"].shape[0]
    seq, at = _tokens(s)
    q = s["q"].float()
    parts = _parts(s["pool"], c["page"], c["d"])
    wide, longest = max(shape["new"]), max(shape["own"])
    tok = torch.arange(n, device="cuda")
    mine = (cu[:-1, None] + torch.arange(wide, device="cuda")).clamp(max=n - 1)
    new = (cu[1:] - cu[:-1])[:, None]
    limit = (s["lengths"].long()[:, None] - new + 1 + torch.arange(wide, device="cuda")).minimum(s["lengths"].long()[:, None])
    m, l, z = (x[seq, tok - cu[seq]] for x in _part(q[mine], *(_pages(a, b, s["table"], longest) for a, b in parts), limit))
    if shape["groups"]:
        first = cu[s["cu_group"].long()]
        group = torch.searchsorted(first[1:].contiguous(), tok, right=True)
        rows = max(sum(shape["new"][a:b]) for a, b in zip(shape["edges"], shape["edges"][1:]))
        mine = (first[:-1, None] + torch.arange(rows, device="cuda")).clamp(max=n - 1)
        limit = s["prefix_len"].long()[:, None].expand(-1, rows)
        K, V = (_pages(a, b, s["prefix_table"], max(shape["prefix"])) for a, b in parts)
        m2, l2, z2 = (x[group, tok - first[group]] for x in _part(q[mine], K, V, limit))
        top = torch.maximum(m, m2)
        a, b = (m - top).exp(), (m2 - top).exp()
        l, z = l * a + l2 * b, z * a + z2 * b
    return torch.where(l > 0, z / l, 0.0).to(s["q"].dtype)


def run(state):
    s = state
    c = s["case"]
    if own:
        from paper_2402_06082_b200 import binding
        if c["op"] == "step":
            x = binding.page_step(s["lengths"], s["table"], s["free"], s["free_count"], s["added"], c["page"], s["n"], ended=s["ended"], in_place=False)
            return {"cu_q": x.cu_q, "lengths": x.lengths, "free_count": x.free_count, "table": s["table"], "free": s["free"], "slots": x.slots,
                    "positions": x.positions}
        if c["op"] == "append":
            q = s["cache"].append(s["batch"], s["k"], s["v"], rope=s["rope"], q=s["q"], wq=s["wq"], wk=s["wk"], eps=EPS)
            return (q, *s["cache"].load(s["slots"], s["k"].dtype))
        if c["op"] == "load":
            return s["cache"].load(s["slots"], TYPES[c["dtype"]])
        return s["cache"].attend(s["batch"], s["q"], scale=c["d"] ** -0.5)
    return {"step": _step_plain, "append": _append_plain, "load": _load_plain, "attend": _attend_plain}[c["op"]](s)


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def _step_by_rows(c, s):
    """One row after the other, as a host program would keep its tables."""
    page, n = c["page"], s["n"]
    table, free = s["table"].cpu().numpy().copy(), s["free"].cpu().numpy().copy()
    lengths, top = s["lengths"].tolist(), int(s["free_count"])
    for b, over in enumerate(s["ended"].tolist()):
        if over:
            for k in range(_pages_of(lengths[b], page)):
                free[top] = table[b, k]
                top += 1
            lengths[b] = 0
    cu, slots, positions, pages, tokens, whole = [0], [], [], 0, 0, top
    for b, k in enumerate(s["added"].tolist()):
        held = _pages_of(lengths[b], page)
        want = _pages_of(lengths[b] + k, page) - held
        pages, tokens = pages + want, tokens + k
        if (want and pages > whole) or (k and tokens > n) or held + want > table.shape[1]:
            k = 0
        else:
            for i in range(want):
                top -= 1
                table[b, held + i] = free[top]
        for i in range(lengths[b], lengths[b] + k):
            slots.append(int(table[b, i // page]) * page + i % page)
            positions.append(i)
        lengths[b] += k
        cu.append(cu[-1] + k)
    pad = n - len(slots)
    return {"cu_q": _ints(cu), "lengths": _ints(lengths), "free_count": _ints([top]), "table": torch.from_numpy(table).cuda(),
            "free": torch.from_numpy(free).cuda(), "slots": torch.tensor(slots + [-1] * pad, device="cuda"), "positions": _ints(positions + [0] * pad)}


def _turned(x, pos, w):
    """x [n, heads, d] as complex numbers turned by their angles."""
    x = x.double()
    if w is not None:
        x = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + EPS) * w.double()
    half = x.shape[-1] // 2
    phase = torch.outer(pos.double(), torch.exp(-torch.arange(half, dtype=torch.float64, device=x.device) / half * math.log(BASE)))
    t = torch.complex(x[..., :half].contiguous(), x[..., half:].contiguous()) * torch.polar(torch.ones_like(phase), phase)[:, None]
    return torch.cat((t.real, t.imag), -1)


def _rounded(x):
    """The nearest of the 16 values of each group, by looking at all of them; 64 bits."""
    y = x.double().unflatten(-1, (-1, 16))
    a = y.abs().amax(-1, keepdim=True)
    unit = torch.exp2((torch.floor(torch.log2(a.clamp(min=2.0 ** -14))) - 3).clamp(min=-17))     # the scales of this octave are its multiples
    scale = torch.ceil(a / unit) * unit
    out, best = torch.zeros_like(y), torch.full_like(y, math.inf)
    for n in range(16):                                                      # of two as near the upper
        value = (n - 7.5) * scale / 8
        off = (y - value).abs()
        near = off <= best
        out, best = torch.where(near, value, out), torch.where(near, off, best)
    return out.flatten(-2)


def _decoded(raw, page, d, ids):
    """Pages `ids` of a pool as 64-bit keys and values [Hkv, tokens, d]: byte by byte from the format."""
    x = raw[ids.long()].reshape(len(ids), raw.shape[1], page // 16, 2, -1)
    codes, scale = x[..., : 8 * d].reshape(*x.shape[:4], 16, d // 8, 4), x[..., 8 * d:].reshape(*x.shape[:4], 16, d // 16)
    e, f = torch.div(scale, 8, rounding_mode="floor").double(), (scale % 8).double()
    size = torch.where(e > 0, (1 + f / 8) * torch.exp2(e - 15), f / 8 * 2.0 ** -14)
    half = [codes[..., 2 * i].long() + 256 * codes[..., 2 * i + 1].long() for i in (0, 1)]
    bits = [torch.stack([torch.bitwise_right_shift(h, (j + 2) % 16) & 1 for j in range(16)], -1) for h in half]      # bit j before the rotation
    n = [sum(b[..., i:: 4] * (1 << i) for i in range(4)) for b in bits]      # [..., d / 8, 4] each
    y = (torch.stack(n, -1).flatten(-3).double() - 7.5) * size.repeat_interleave(16, -1) / 8
    y = y.permute(3, 1, 0, 2, 4, 5).reshape(2, raw.shape[1], -1, d)
    return y[0], y[1]


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["op"] == "step":
        return _step_by_rows(c, s)
    shape, page, d = s["shape"], c["page"], c["d"]
    if c["op"] == "load":
        K, V = _decoded(s["pool"], page, d, s["table"][0])
        return tuple(x[:, c["ctx"] - c["n"]: c["ctx"]].transpose(0, 1) for x in (K, V))
    starts = [0] + np.cumsum(shape["new"]).tolist()
    if c["op"] == "append":
        place = torch.tensor([m - k + i for k, m in zip(shape["new"], shape["own"]) for i in range(k)], device="cuda")
        return _turned(s["q"], place, s["wq"]), _rounded(_turned(s["k"], place, s["wk"])), _rounded(s["v"])
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    group = c["H"] // c["Hkv"]
    for b in range(c["B"]):
        rows = [(s["table"][b], shape["own"][b])]
        for g in range(shape["groups"]):
            if shape["edges"][g] <= b < shape["edges"][g + 1]:
                rows.insert(0, (s["prefix_table"][g], shape["prefix"][g]))
        both = [_decoded(s["pool"], page, d, row[: _pages_of(length, page)]) for row, length in rows]
        K, V = (torch.cat([x[i][:, :length] for x, (_, length) in zip(both, rows)], 1) for i in (0, 1))
        a, e, new = starts[b], starts[b + 1], shape["new"][b]
        L = K.shape[1]
        for t in range(a, e, 256):                                       # 256 queries at a time
            u = min(e, t + 256)
            q = s["q"][t:u].double().view(u - t, c["Hkv"], group, d)
            logits = torch.einsum("thgd,hld->thgl", q, K) / math.sqrt(d)
            last = L - new + torch.arange(t - a, u - a, device="cuda")
            logits += torch.where(torch.arange(L, device="cuda")[None] > last[:, None], -math.inf, 0.0)[:, None, None]
            out[t:u] = torch.einsum("thgl,hld->thgd", torch.softmax(logits, -1), V).reshape(u - t, c["H"], d)
    return out
