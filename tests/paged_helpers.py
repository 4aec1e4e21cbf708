"""Plain 64-bit statements of the head norms with rotation, paged append and paged attention, with error bounds.

A rounding to type t is off by at most u(t) = finfo(t).eps / 2 relative to the value. The bounds are elementwise.
"""
import math

import torch

U32 = 2.0 ** -24
U = {torch.float32: U32, torch.bfloat16: 2.0 ** -8}


def freqs(rot, base=10000.0):
    return [base ** (-2.0 * i / rot) for i in range(rot // 2)]


def norm_rope(x, pos, w, f, rot, interleaved, eps):
    """x [n, heads, d] -> (y, bound) in float64 on the CPU; f: the frequencies or None."""
    dt = x.dtype
    x = x.detach().cpu().double()
    d = x.shape[-1]
    y = x
    if w is not None:
        y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.detach().cpu().double()
    size = y.abs()
    # the norm: a sum of d squares (d u32), mean, + eps, sqrt, reciprocal and two products (8 u32)
    rel = ((d / 2 + 8) if w is not None else 0) * U32
    if f is not None:
        a = torch.outer(pos.detach().cpu().double(), torch.tensor(f, dtype=torch.float64))
        cos, sin = a.cos()[:, None], a.sin()[:, None]
        y = y.clone()
        re, im = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
        p, q = y[..., re].clone(), y[..., im].clone()
        y[..., re], y[..., im] = p * cos - q * sin, q * cos + p * sin
        size = size.clone()
        size[..., re] = size[..., im] = p.abs() + q.abs()
        # the angle in half turns is rounded to 24 bits (pi u32); sine and cosine to 2 ulp (4 u32) from an angle that the
        # 64-bit reference itself has to |pos| * 2^-53; products and sum (3 u32)
        far = float(pos.abs().max()) if pos.numel() else 0.0
        rel += (math.pi + 4 + 3) * U32 + far * 2.0 ** -51
    bound = rel * size + (U[dt] * y.abs() if rel else 0) + 1e-37
    return y, bound


def own_tokens(pool, table_row, length):
    """[Hkv, length, d] of a sequence, on the CPU in float64."""
    page = pool.shape[2]
    ids = table_row[: -(-length // page)].long()
    x = pool[ids].permute(1, 0, 2, 3).reshape(pool.shape[1], -1, pool.shape[3])
    return x[:, :length].cpu().double()


def attend(q, K, V, cu, lengths, table, scale, causal=True, cu_group=(), prefix_len=(), prefix_table=None, base=None):
    """(out, bound) in float64 for host lists cu, lengths, cu_group, prefix_len; rows behind cu[-1] are NaN in out."""
    n, H, d = q.shape
    Hkv = K.shape[1]
    G = H // Hkv
    out = torch.full((n, H, d), math.nan, dtype=torch.float64)
    bound = torch.zeros((n, H, d), dtype=torch.float64)
    u = U[q.dtype]
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
        # scores: d products and sums in fp32, the scale and log2(e) in the exponent's argument, the largest taken off
        size = torch.einsum("thgd,hld->thgl", x.abs(), k.abs()) * scale
        ds = ((d + 4) * U32 * size).amax(-1, keepdim=True)
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
        # weights: e^(2 ds) from the scores, exp2 and its argument (|s| up to its range: 2^-21 with the fp32 rounding of an
        # argument of up to 64), L sums and as many joins; bf16: the weight itself, and 7.5e-5 of the cubic that some of the
        # weights are made with, which the sum of the weights has as well
        rel = 2 * torch.expm1(ds) + 2.0 ** -20 + 2 * (L + 64) * U32 + (u + 2 * 7.5e-5 if q.dtype == torch.bfloat16 else 0)
        out[t0:t1] = y.reshape(t1 - t0, H, d)
        bound[t0:t1] = (rel * a + u * (y.abs() + rel * a)).reshape(t1 - t0, H, d) + 1e-30
    return out, bound


def assert_within(got, want, bound, what=""):
    got = got.detach().cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what + ": NaN elsewhere"
    off = torch.where(torch.isnan(want), torch.zeros(()).double(), (got - want).abs() - bound)
    worst = float(off.max()) if off.numel() else 0.0
    assert worst <= 0, "%s: %.3g beyond the bound at %s" % (what, worst, tuple(int(x) for x in (off == off.max()).nonzero()[0]))


class Setting:
    """A pool with pages in random order, NaN in every slot that no sequence owns, and a batch over it."""

    def __init__(self, new, own, H, Hkv, d, dtype, page=16, edges=(), prefix=(), seed=0, behind=0, rows_first=False):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.new, self.own, self.H, self.Hkv, self.d, self.dtype, self.page = list(new), list(own), H, Hkv, d, dtype, page
        self.edges, self.prefix = list(edges), list(prefix)
        counts = [-(-x // page) for x in self.own] + [-(-x // page) for x in self.prefix]
        pages = max(1, sum(counts)) + 3
        perm = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        if rows_first:                                # [pages, page, Hkv, d] in memory
            self.K, self.V = (torch.randn(pages, page, Hkv, d, generator=g, device="cuda").to(dtype).transpose(1, 2) for _ in "KV")
        else:
            self.K, self.V = (torch.randn(pages, Hkv, page, d, generator=g, device="cuda").to(dtype) for _ in "KV")
        B, wide = len(self.own), max([1] + counts[: len(self.own)])
        self.table = torch.full((B, wide), -1, dtype=torch.int32, device="cuda")
        self.ptable = torch.full((len(self.prefix), max([1] + counts[B:])), -1, dtype=torch.int32, device="cuda")
        used, at = torch.zeros(pages, page, dtype=torch.bool, device="cuda"), 0
        for i, k in enumerate(counts):
            row, length = (self.table[i], self.own[i]) if i < B else (self.ptable[i - B], self.prefix[i - B])
            ids = perm[at:at + k]
            row[:k] = ids
            flat = torch.arange(k * page, device="cuda") < length
            used[ids.long()] = flat.view(k, page)
            at += k
        for x in (self.K, self.V):
            x.masked_fill_(~used[:, None, :, None], math.nan)
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
        return binding.PagedCache(self.K, self.V)

    def batch(self):
        from paper_2402_06082_b200 import binding
        return binding.PagedBatch(self.cu_q, self.lengths, self.table, **self.groups)

    def want(self, scale, causal=True):
        return attend(self.q, self.K, self.V, self.cu, self.own, self.table, scale, causal, self.edges, self.prefix, self.ptable)
