"""Plain 64-bit statements of the 4-bit cells, of attention over them and of a step's tables, with error bounds.

A rounding to type t is off by at most u(t) = finfo(t).eps / 2 relative to the value. The bounds are elementwise.
"""
import math

import torch

from paged_helpers import U, U32

LARGEST = 61440.0


def rounded(x):
    """x [..., d], any type -> (scale bytes [..., d / 16], codes [..., d], values [..., d] in float64), by the definition."""
    g = x.double().unflatten(-1, (-1, 16))
    a = g.abs().amax(-1)                              # NaN where there is one
    e = torch.floor(torch.log2(a.clamp(min=2.0 ** -14, max=LARGEST)))
    e = torch.where(torch.exp2(e) > a.clamp(min=2.0 ** -14), e - 1, e)       # log2 may round up
    unit = torch.exp2(e - 3)
    s = torch.ceil(a / unit) * unit
    fine = a <= LARGEST
    s = torch.where(fine, s, torch.full_like(s, math.nan))
    n = (torch.floor(torch.where(s[..., None] > 0, 8 * g / s[..., None], torch.zeros_like(g))) + 8).clamp(0, 15)
    v = (n - 7.5) * s[..., None] / 8
    byte = torch.where(fine, (s.to(torch.float16).view(torch.int16) >> 7).double(), torch.full_like(s, 255.0))
    return byte.to(torch.uint8), n.nan_to_num(0).to(torch.int64).flatten(-2), v.flatten(-2)


def code_bytes(n):
    """codes [..., d] -> bytes [..., d / 2]."""
    out = []
    for w in n.unflatten(-1, (-1, 8)).unbind(-2):
        for half in (0, 1):
            x = sum(w[..., half + 2 * i] << (4 * i) for i in range(4))
            x = ((x << 2) | (x >> 14)) & 0xffff
            out += [x & 255, x >> 8]
    return torch.stack(out, -1).to(torch.uint8)


def codes_of(raw):
    """bytes [..., d / 2] -> codes [..., d]."""
    b = raw.to(torch.int64)
    out = []
    for i in range(0, b.shape[-1], 4):
        halves = [b[..., i + 2 * h] | b[..., i + 2 * h + 1] << 8 for h in (0, 1)]
        halves = [(x >> 2) | ((x & 3) << 14) for x in halves]
        for k in range(4):
            out += [(halves[0] >> (4 * k)) & 15, (halves[1] >> (4 * k)) & 15]
    return torch.stack(out, -1)


def scales_of(raw):
    """scale bytes -> S in float64 (NaN for 255; the bytes from 248 on are no scales that a cache holds)."""
    r = raw.to(torch.int64)
    e, f = r >> 3, (r & 7).double()
    s = torch.where(e > 0, (1 + f / 8) * torch.exp2(e.double() - 15), f / 8 * 2.0 ** -14)
    return torch.where(r >= 248, torch.full_like(s, math.nan), s)


def views(pool, page, d):
    """[(codes [pages, Hkv, page, d / 2], scales [pages, Hkv, page, d / 16]) of keys, of values]: views where pages have one cell, else copies."""
    x = pool.unflatten(-1, (page // 16, 2, 16 * (d // 2 + d // 16)))
    out = []
    for i in range(2):
        c, s = x[..., i, : 8 * d], x[..., i, 8 * d:]
        out.append((c.unflatten(-1, (16, d // 2)).flatten(2, 3), s.unflatten(-1, (16, d // 16)).flatten(2, 3)))
    return out


def decoded(pool, page, d):
    """K, V [pages, Hkv, page, d] in float64."""
    return [(codes_of(c).double() - 7.5) * scales_of(s).repeat_interleave(16, -1) / 8 for c, s in views(pool, page, d)]


def put(pool, page, d, kv, where, row, byte, code):
    """Writes rows [..., Hkv, ...] at (page `where`, row `row`) of the pool: byte [n, Hkv, d / 16], code [n, Hkv, d]."""
    x = pool.unflatten(-1, (page // 16, 2, 16 * (d // 2 + d // 16)))[:, :, :, kv]
    x[..., : 8 * d].unflatten(-1, (16, d // 2))[where, :, row // 16, row % 16] = code_bytes(code)
    x[..., 8 * d:].unflatten(-1, (16, d // 16))[where, :, row // 16, row % 16] = byte


def attend(q, K, V, cu, lengths, table, scale, causal=True, cu_group=(), prefix_len=(), prefix_table=None, few=True):
    """(out, bound) in float64 over pools K, V in float64; rows behind cu[-1] are NaN in out. few: the kernel for few rows a sequence."""
    from paged_helpers import own_tokens
    n, H, d = q.shape
    Hkv = K.shape[1]
    G = H // Hkv
    out = torch.full((n, H, d), math.nan, dtype=torch.float64)
    bound = torch.zeros((n, H, d), dtype=torch.float64)
    u, wide = U[q.dtype], q.dtype == torch.float32
    for b in range(len(lengths)):
        t0, t1 = cu[b], cu[b + 1]
        if t0 == t1:
            continue
        k, v = own_tokens(K, table[b], lengths[b]), own_tokens(V, table[b], lengths[b])
        P = 0
        for g in range(len(prefix_len)):
            if cu_group[g] <= b < cu_group[g + 1]:
                P = prefix_len[g]
                k = torch.cat([own_tokens(K, prefix_table[g], P), k], 1)
                v = torch.cat([own_tokens(V, prefix_table[g], P), v], 1)
        L = k.shape[1]
        x = q[t0:t1].cpu().double().reshape(t1 - t0, Hkv, G, d)
        if L == 0:
            out[t0:t1] = 0
            continue
        s = torch.einsum("thgd,hld->thgl", x, k) * scale
        # scores: d products and sums, in the tensor cores' fp32 sums, which may cut off instead of rounding (2 u32 each); fp32
        # queries as two fp16 (2^-22); what is below 2^-39 of a row's largest coordinate is lost; the exponent's argument
        size = torch.einsum("thgd,hld->thgl", x.abs(), k.abs()) * scale
        floor = torch.einsum("thgd,hld->thgl", x.abs().amax(-1, keepdim=True).expand_as(x), k.abs()) * scale * 2.0 ** -39
        ds = (((2 * d + 4) * U32 + (2.0 ** -22 if wide else 0)) * size + floor).amax(-1, keepdim=True)
        i = torch.arange(t1 - t0)
        see = (P + lengths[b] - (t1 - t0) + 1 + i).clamp(min=P, max=L) if causal else torch.full((t1 - t0,), L)
        mask = torch.arange(L)[None] < see[:, None]
        s = s.masked_fill(~mask[:, None, None], -math.inf)
        m = s.amax(-1, keepdim=True).clamp(min=-1e300)
        p = torch.exp(s - m)
        l = p.sum(-1, keepdim=True)
        w = torch.where(l > 0, p / l, torch.zeros(()).double())
        y = torch.einsum("thgl,hld->thgd", w, v)
        a = torch.einsum("thgl,hld->thgd", w, v.abs())
        # weights: e^(2 ds) from the scores; exp2 and its argument (2^-20); L sums and as many joins, cut off again (2 u32); their own
        # rounding: fp16 (2^-11), as two fp16 (2^-22), or bf16 with the cubic that a part of them is made with; fp16 weights end
        # at 2^-25 where the largest is at least 2^6
        own = 2.0 ** -22 if wide else 2.0 ** -11 if few else 2.0 ** -8 + 2 * 7.5e-5
        rel = 2 * torch.expm1(ds) + 2.0 ** -20 + 4 * (L + 64) * U32 + own
        lost = 2.0 ** -31 * (v.abs().amax(1)[None, :, None] * see.double()[:, None, None, None]) if few else 0
        out[t0:t1] = y.reshape(t1 - t0, H, d)
        bound[t0:t1] = (rel * a + lost + u * (y.abs() + rel * a)).reshape(t1 - t0, H, d) + 1e-30
    return out, bound


class Setting4:
    """A pool of random bytes (scales that are NaN among them) with pages in random order, rounded tokens in the slots that sequences own, and a
    batch over it. Its other attributes are as paged_helpers.Setting's."""

    def __init__(self, new, own, H, Hkv, d, dtype, page=16, edges=(), prefix=(), seed=0, behind=0, spread=0.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.new, self.own, self.H, self.Hkv, self.d, self.dtype, self.page = list(new), list(own), H, Hkv, d, dtype, page
        self.edges, self.prefix = list(edges), list(prefix)
        counts = [-(-x // page) for x in self.own] + [-(-x // page) for x in self.prefix]
        pages = max(1, sum(counts)) + 3
        perm = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        self.pool = torch.randint(0, 256, (pages, Hkv, page * 2 * (d // 2 + d // 16)), generator=g, device="cuda").to(torch.uint8)
        B, wide = len(self.own), max([1] + counts[: len(self.own)])
        self.table = torch.full((B, wide), -1, dtype=torch.int32, device="cuda")
        self.ptable = torch.full((len(self.prefix), max([1] + counts[B:])), -1, dtype=torch.int32, device="cuda")
        at = 0
        for i, k in enumerate(counts):
            row, length = (self.table[i], self.own[i]) if i < B else (self.ptable[i - B], self.prefix[i - B])
            ids = perm[at:at + k]
            row[:k] = ids
            at += k
            if length:
                tok = torch.arange(length, device="cuda")
                for kv in range(2):
                    x = torch.randn(length, Hkv, d, generator=g, device="cuda")
                    if spread:
                        x = x * torch.exp(spread * torch.randn(length, Hkv, d // 16, 1, generator=g, device="cuda")).expand(-1, -1, -1, 16).reshape(x.shape)
                    byte, code, _ = rounded(x)
                    put(self.pool, page, d, kv, ids[tok // page].long(), tok % page, byte, code)
        self.cu = [0]
        for k in self.new:
            self.cu.append(self.cu[-1] + k)
        self.n = self.cu[-1] + behind
        ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        self.cu_q, self.lengths = ints(self.cu), ints(self.own)
        self.q = torch.randn(self.n, H, d, generator=g, device="cuda").to(dtype)
        self.k, self.v = (torch.randn(self.n, Hkv, d, generator=g, device="cuda").to(dtype) for _ in "kv")
        self.groups = dict(cu_group=ints(self.edges), prefix_len=ints(self.prefix), prefix_table=self.ptable) if self.prefix else {}

    def cache(self):
        from paper_2402_06082_b200 import binding
        return binding.PagedCache4(self.pool, self.page, self.d)

    def batch(self):
        from paper_2402_06082_b200 import binding
        return binding.PagedBatch(self.cu_q, self.lengths, self.table, **self.groups)

    def few(self):
        """Which kernel a call takes."""
        rows, groups, B = self.n * self.H // self.Hkv, len(self.prefix), len(self.own)
        return self.dtype == torch.float32 or rows <= 32 * (groups if 0 < groups < B else B)

    def want(self, scale, causal=True, few=None):
        K, V = decoded(self.pool, self.page, self.d)
        return attend(self.q, K, V, self.cu, self.own, self.table, scale, causal, self.edges, self.prefix, self.ptable, self.few() if few is None else few)


def step(lengths, table, free, count, added, page, n, ended=None, first=None):
    """subgen_page_step on host lists, one row after the other; table and free are changed in place. Rows and arguments are sound."""
    B, lengths, served = len(lengths), list(lengths), True
    for b in range(B):
        if ended and ended[b]:
            for k in range(-(-lengths[b] // page)):
                free[count] = table[b][k]
                count += 1
            lengths[b] = 0
    there, pages, tokens, cu, slots, positions = count, 0, 0, [0], [], []
    for b in range(B):
        held = -(-lengths[b] // page)
        want, k = -(-(lengths[b] + added[b]) // page) - held, added[b]
        pages, tokens = pages + want, tokens + k
        if (want and pages > there) or (k and tokens > n) or held + want > len(table[b]):
            served, k, want = False, 0, 0
        for i in range(want):
            count -= 1
            table[b][held + i] = free[count]
        for i in range(lengths[b], lengths[b] + k):
            slots.append(table[b][i // page] * page + i % page)
            positions.append(i + (first[b] if first else 0))
        lengths[b] += k
        cu.append(cu[-1] + k)
    pad = n - len(slots)
    return cu, lengths, count, slots + [-1] * pad, positions + [0] * pad, served
