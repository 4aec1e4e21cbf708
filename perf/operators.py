"""Three operators of a serving step next to the cache kernels, in plain form and through the library, with cases to time.

    norm_rope   RMS norm of every head's query and key, and the position rotation, in one pass
                (what a prompt or a step goes through before SubGen.prefill / step or an exact cache sees it)
    append      new keys (normed, rotated) and values into a paged cache, the step's queries rotated on the way
    attend      exact attention over a paged cache for a batch whose sequences share long prefixes:
                single tokens, drafted tokens and chunks of prompts, masked causally

`own` = False computes them with elementary torch operations in 32 bits (angles in 64), True calls
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

def _norm_rope(n, H, Hkv, d, dtype, rot, interleaved=False, mix=0):
    return {"op": "norm_rope", "n": n, "H": H, "Hkv": Hkv, "d": d, "dtype": dtype, "rot": rot, "interleaved": interleaved, "mix": mix}


def _append(B, new_lo, new_hi, ctx, H, Hkv, d, dtype, page, norm, mix=0):
    return {"op": "append", "B": B, "new_lo": new_lo, "new_hi": new_hi, "ctx": ctx, "H": H, "Hkv": Hkv, "d": d, "dtype": dtype,
            "page": page, "norm": norm, "mix": mix}


def _attend(B, new_lo, new_hi, own_lo, own_hi, prefix, groups, H, Hkv, d, dtype, page, mix=0):
    return {"op": "attend", "B": B, "new_lo": new_lo, "new_hi": new_hi, "own_lo": own_lo, "own_hi": own_hi, "prefix": prefix,
            "groups": groups, "H": H, "Hkv": Hkv, "d": d, "dtype": dtype, "page": page, "mix": mix}


def listed():
    cases = {
        # one sequence's next token: nothing but latency
        "qk one token": _norm_rope(1, 32, 8, 128, "bf16", 128),
        # a partly rotated head in pairs of neighbours, 32-bit, an odd number of tokens
        "qk fp32 interleaved": _norm_rope(2047, 16, 4, 64, "fp32", 32, True),
        # a prompt of 16384 tokens with 32 key heads
        "qk prompt": _norm_rope(16384, 32, 32, 128, "bf16", 128),
        # one step of 64 sequences: a token each, queries on the way, pages of 16
        "append step": _append(64, 1, 1, 4096, 32, 8, 128, "bf16", 16, True),
        # chunks of eight prompts of odd lengths into pages of 64
        "append prompt chunks": _append(8, 1025, 4095, 8192, 32, 32, 128, "bf16", 64, False),
        # drafted tokens of a 32-bit cache
        "append fp32 drafts": _append(48, 1, 8, 1000, 8, 8, 64, "fp32", 32, True),
        # one short sequence, no shared prefix: latency
        "attend one short": _attend(1, 1, 1, 1000, 1000, 0, 0, 32, 8, 128, "bf16", 16),
        # one long sequence: the cache read once
        "attend one long": _attend(1, 1, 1, 131072, 131072, 0, 0, 32, 8, 128, "bf16", 64),
        # 64 sequences behind one prompt of 32768 tokens, each with what it has generated so far
        "attend shared prompt": _attend(64, 1, 1, 1, 2048, 32768, 1, 32, 8, 128, "bf16", 64),
        # drafted tokens of 16 sequences behind two system prompts of odd length
        "attend drafts": _attend(16, 1, 8, 17, 4095, 16383, 2, 32, 8, 128, "bf16", 16),
        # chunks of four prompts behind a shared document
        "attend prompt chunks": _attend(4, 513, 2047, 2048, 4096, 8192, 1, 32, 8, 128, "bf16", 128),
        # a 32-bit cache, heads of 64, one key head per query head
        "attend fp32": _attend(8, 1, 3, 100, 1500, 2001, 1, 8, 8, 64, "fp32", 32),
    }
    return [dict(c, name=name) for name, c in cases.items()]


def _between(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 6.5, w["flops"] / (1700.0 if case["dtype"] == "bf16" else 50.0))


def _most(op):
    return max(_cost(c) for c in listed() if c["op"] == op)


def draw(rng):
    op = rng.choice(["norm_rope", "append", "attend", "attend"])
    while True:
        d, dtype, page = rng.choice([64, 128, 128]), rng.choice(["bf16", "bf16", "bf16", "fp32"]), rng.choice([16, 32, 64, 128])
        Hkv = rng.choice([1, 2, 4, 8, 8, 32])
        H, mix = Hkv * rng.choice([1, 2, 4, 8] if Hkv <= 8 else [1]), rng.randrange(1 << 20)
        if op == "norm_rope":
            case = _norm_rope(_between(rng, 1, 16384), H, Hkv, d, dtype, rng.choice([d, d, d // 2]), rng.random() < 0.3, mix)
        elif op == "append":
            hi = _between(rng, 1, 4095)
            case = _append(_between(rng, 1, 128), rng.randint(1, hi), hi, _between(rng, 64, 8192), H, Hkv, d, dtype, page, rng.random() < 0.5, mix)
        else:
            hi, own_hi = rng.choice([1, 1, _between(rng, 1, 8), _between(rng, 8, 2047)]), _between(rng, 1, 65536)
            own_hi = max(hi, own_hi)
            prefix = rng.choice([0, _between(rng, 1, 65536), _between(rng, 1, 65536)])
            B = _between(rng, 1, 64)
            case = _attend(B, rng.randint(1, hi), hi, rng.randint(hi, own_hi), own_hi, prefix, min(B, rng.choice([1, 1, 2, 3])) if prefix else 0,
                           H, Hkv, d, dtype, page, mix)
        if op == "attend":
            small = _shape(case)["cells"] < 3e9                          # scores that the plain form holds at once
        else:
            small = op == "norm_rope" or case["B"] * (case["ctx"] + hi) * Hkv * d < 1e9      # values of one pool
        if small and _cost(case) <= _most(op):
            return case


# ---- lengths and work ---------------------------------------------------------------------------------------------

def _shape(c):
    """The lengths of a case: new tokens, own tokens (the new ones among them), groups of sequences and their prefixes."""
    r = random.Random(c["mix"])
    B = c["B"]
    new = [r.randint(c["new_lo"], c["new_hi"]) for _ in range(B)]
    if c["op"] == "append":
        return {"new": new, "own": [k + r.randint(0, c["ctx"]) for k in new], "groups": 0, "edges": [], "prefix": []}
    length = [max(k, r.randint(c["own_lo"], c["own_hi"])) for k in new]
    g = c["groups"]
    edges = [0] + sorted(r.sample(range(1, B), g - 1)) + [B] if g else []
    prefix = [c["prefix"]] + [r.randint(max(1, c["prefix"] // 2), c["prefix"]) for _ in range(g - 1)] if g else []
    rows = max([sum(new[edges[i]:edges[i + 1]]) for i in range(g)] + [0])
    return {"new": new, "own": length, "groups": g, "edges": edges, "prefix": prefix,
            "cells": c["H"] * (B * max(new) * max(length) + g * rows * c["prefix"]) + 2 * B * c["Hkv"] * max(length) * c["d"]}


def work(c):
    e, d, H, Hkv = (4 if c["dtype"] == "fp32" else 2), c["d"], c["H"], c["Hkv"]
    if c["op"] == "norm_rope":
        x = c["n"] * (H + Hkv) * d
        return {"bytes": 2 * x * e + 4 * c["n"], "flops": 8 * x}
    s = _shape(c)
    n = sum(s["new"])
    if c["op"] == "append":
        return {"bytes": 2 * n * (H + 2 * Hkv) * d * e, "flops": (8 if c["norm"] else 3) * n * (H + Hkv) * d}
    pairs = sum(k * m - k * (k - 1) // 2 for k, m in zip(s["new"], s["own"]))
    pairs += sum(sum(s["new"][s["edges"][g]:s["edges"][g + 1]]) * s["prefix"][g] for g in range(s["groups"]))
    return {"bytes": 2 * (sum(s["own"]) + sum(s["prefix"])) * Hkv * d * e + 2 * n * H * d * e, "flops": 4 * pairs * H * d}


# ---- inputs -------------------------------------------------------------------------------------------------------

def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, H, Hkv, d = TYPES[c["dtype"]], c["H"], c["Hkv"], c["d"]
    s = {"case": c}

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda", dtype=dt)

    def weight():
        return (1 + 0.1 * torch.randn(d, generator=g, device="cuda")).to(dt)

    if c["op"] == "norm_rope":
        qkv = randn(c["n"], (H + 2 * Hkv) * d)          # the fused projection that the heads are views of
        s["q"], s["k"] = qkv[:, : H * d].view(c["n"], H, d), qkv[:, H * d: (H + Hkv) * d].view(c["n"], Hkv, d)
        s["wq"], s["wk"] = weight(), weight()
        s["pos"] = torch.randint(0, 131072, (c["n"],), generator=g, device="cuda", dtype=torch.int32)
        if own:
            from paper_2402_06082_b200 import binding
            s["rope"] = binding.Rope(d, base=BASE, rotary_dim=c["rot"], interleaved=c["interleaved"])
        return s

    shape = _shape(c)
    B, n, page, groups = c["B"], sum(shape["new"]), c["page"], shape["groups"]
    s["shape"] = shape
    own_pages = [-(-x // page) for x in shape["own"]]
    pre_pages = [-(-x // page) for x in shape["prefix"]]
    pages = sum(own_pages) + sum(pre_pages)
    perm = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)     # pages lie anywhere in the pool

    def tables(counts, first):
        wide = max(counts)
        at = np.full((len(counts), wide), -1, np.int64)
        for i, k in enumerate(counts):
            at[i, :k] = first + np.arange(k)
            first += k
        at = torch.from_numpy(at).cuda()
        return torch.where(at >= 0, perm[at.clamp(min=0)], torch.zeros((), dtype=torch.int32, device="cuda"))

    s["K"], s["V"] = randn(pages, Hkv, page, d), randn(pages, Hkv, page, d)
    s["table"] = tables(own_pages, 0)
    s["lengths"] = _ints(shape["own"])
    s["cu_q"] = _ints([0] + np.cumsum(shape["new"]).tolist())
    if groups:
        s["cu_group"], s["prefix_len"] = _ints(shape["edges"]), _ints(shape["prefix"])
        s["prefix_table"] = tables(pre_pages, sum(own_pages))
    if c["op"] == "append":
        qkv = randn(n, (H + 2 * Hkv) * d)
        s["q"], s["k"] = qkv[:, : H * d].view(n, H, d), qkv[:, H * d: (H + Hkv) * d].view(n, Hkv, d)
        s["v"] = qkv[:, (H + Hkv) * d:].view(n, Hkv, d)
        s["wq"], s["wk"] = (weight(), weight()) if c["norm"] else (None, None)
    else:
        s["q"] = randn(n, H, d)
    if own:
        from paper_2402_06082_b200 import binding
        if c["op"] == "append":
            s["rope"] = binding.Rope(d, base=BASE)
        s["cache"] = binding.PagedCache(s["K"], s["V"])
        s["batch"] = binding.PagedBatch(s["cu_q"], s["lengths"], s["table"], s.get("cu_group"), s.get("prefix_len"), s.get("prefix_table"))
    return s


# ---- plain forms --------------------------------------------------------------------------------------------------

def _rotated(x, pos, w, rot, interleaved):
    """RMS norm over the head (if there is a weight), then the rotation of its first `rot` coordinates; 32 bits."""
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
    half = rot // 2
    freq = BASE ** (-torch.arange(half, device=x.device, dtype=torch.float64) / half)
    angle = (pos.double()[:, None] * freq)[:, None, :]
    cos, sin = angle.cos().float(), angle.sin().float()
    head, tail = x[..., :rot], x[..., rot:]
    if interleaved:
        a, b = head[..., 0::2], head[..., 1::2]
        head = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = head[..., :half], head[..., half:]
        head = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((head, tail), -1)


def _tokens(s):
    """For each new token its sequence and its place among that sequence's own tokens."""
    cu, lengths = s["cu_q"].long(), s["lengths"].long()
    tok = torch.arange(s["q"].shape[0], device="cuda")
    seq = torch.searchsorted(cu[1:].contiguous(), tok, right=True)
    return seq, lengths[seq] - cu[seq + 1] + tok


def _append_plain(s):
    seq, at = _tokens(s)
    page = s["case"]["page"]
    q = _rotated(s["q"], at, s["wq"], s["case"]["d"], False)
    k = _rotated(s["k"], at, s["wk"], s["case"]["d"], False)
    where = s["table"][seq, at // page].long()
    s["K"][where, :, at % page] = k.to(s["K"].dtype)
    s["V"][where, :, at % page] = s["v"]
    return q.to(s["q"].dtype), s["K"], s["V"]


def _pages(pool, table, length):
    """[rows of the table, Hkv, length, d] in 32 bits."""
    x = pool[table.long()].transpose(1, 2)
    return x.reshape(x.shape[0], x.shape[1], -1, x.shape[-1])[:, :, :length].float()


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
    wide, longest = max(shape["new"]), max(shape["own"])
    tok = torch.arange(n, device="cuda")
    mine = (cu[:-1, None] + torch.arange(wide, device="cuda")).clamp(max=n - 1)
    new = (cu[1:] - cu[:-1])[:, None]
    limit = (s["lengths"].long()[:, None] - new + 1 + torch.arange(wide, device="cuda")).minimum(s["lengths"].long()[:, None])
    m, l, z = (x[seq, tok - cu[seq]] for x in _part(q[mine], _pages(s["K"], s["table"], longest), _pages(s["V"], s["table"], longest), limit))
    if shape["groups"]:
        first = cu[s["cu_group"].long()]
        group = torch.searchsorted(first[1:].contiguous(), tok, right=True)
        rows = max(sum(shape["new"][a:b]) for a, b in zip(shape["edges"], shape["edges"][1:]))
        mine = (first[:-1, None] + torch.arange(rows, device="cuda")).clamp(max=n - 1)
        K, V = (_pages(s[x], s["prefix_table"], max(shape["prefix"])) for x in "KV")
        limit = s["prefix_len"].long()[:, None].expand(-1, rows)
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
        if c["op"] == "norm_rope":
            return binding.qk_norm_rope(s["q"], s["k"], s["pos"], s["rope"], wq=s["wq"], wk=s["wk"], eps=EPS)
        if c["op"] == "append":
            q = s["cache"].append(s["batch"], s["k"], s["v"], rope=s["rope"], q=s["q"], wq=s["wq"], wk=s["wk"], eps=EPS)
            return q, s["K"], s["V"]
        return s["cache"].attend(s["batch"], s["q"], scale=c["d"] ** -0.5)
    if c["op"] == "norm_rope":
        return tuple(_rotated(s[x], s["pos"], s["w" + x], c["rot"], c["interleaved"]).to(s[x].dtype) for x in "qk")
    return _append_plain(s) if c["op"] == "append" else _attend_plain(s)


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def _turned(x, pos, w, rot, interleaved):
    """x [n, heads, d] as complex numbers turned by their angles."""
    x = x.double()
    if w is not None:
        x = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + EPS) * w.double()
    j = torch.arange(rot // 2, dtype=torch.float64, device=x.device)
    phase = torch.outer(pos.double(), torch.exp(-2 * j / rot * math.log(BASE)))
    spin = torch.polar(torch.ones_like(phase), phase)[:, None]
    re, im = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    y = x.clone()
    t = torch.complex(x[..., re].contiguous(), x[..., im].contiguous()) * spin
    y[..., re], y[..., im] = t.real, t.imag
    return y


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["op"] == "norm_rope":
        return tuple(_turned(s[x], s["pos"], s["w" + x], c["rot"], c["interleaved"]) for x in "qk")
    shape, page, d, group = s["shape"], c["page"], c["d"], c["H"] // c["Hkv"]
    starts = [0] + np.cumsum(shape["new"]).tolist()
    if c["op"] == "append":
        place = torch.tensor([m - k + i for k, m in zip(shape["new"], shape["own"]) for i in range(k)], device="cuda")
        q, k = _turned(s["q"], place, s["wq"], d, False), _turned(s["k"], place, s["wk"], d, False)
        row = torch.tensor([b for b, k in enumerate(shape["new"]) for _ in range(k)], device="cuda")
        slot = s["table"].long()[row, torch.div(place, page, rounding_mode="floor")] * page + place % page
        pools = []
        for pool, x in ((s["K"], k), (s["V"], s["v"].double())):
            flat = pool.double().transpose(1, 2).reshape(-1, c["Hkv"], d)        # one row for each slot of the pool
            flat[slot] = x
            pools.append(flat.view(-1, page, c["Hkv"], d).transpose(1, 2))
        return q, pools[0], pools[1]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")

    def cached(pool, row, length):
        x = s[pool][row[: -(-length // page)].long()].permute(1, 0, 2, 3)
        return x.reshape(c["Hkv"], -1, d)[:, :length].double()

    for b in range(c["B"]):
        parts = [(s["table"][b], shape["own"][b])]
        for g in range(shape["groups"]):
            if shape["edges"][g] <= b < shape["edges"][g + 1]:
                parts.insert(0, (s["prefix_table"][g], shape["prefix"][g]))
        K, V = (torch.cat([cached(x, row, length) for row, length in parts], 1) for x in "KV")
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
