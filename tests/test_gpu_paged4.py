"""The 4-bit paged cache (append, load, attend) and the tables of a step against plain 64-bit statements."""
import math
import random

import pytest
import torch

import paged4_helpers as p4
from paged4_helpers import Setting4
from paged_helpers import assert_within, freqs, norm_rope

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _binding():
    from paper_2402_06082_b200 import binding
    return binding


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ---- append ----

def _odd_values(n, Hkv, d, dtype, seed):
    """Heads of all magnitudes: normal numbers, spread groups, zeros, borders between two codes, tiny ones, the largest."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(n, Hkv, d // 16, 16, generator=g, device="cuda") * torch.exp(4 * torch.randn(n, Hkv, d // 16, 1, generator=g, device="cuda"))
    kind = torch.randint(0, 8, (n, Hkv, d // 16, 1), generator=g, device="cuda")
    x = torch.where(kind == 1, torch.zeros_like(x), x)
    steps = torch.randint(-8, 9, x.shape, generator=g, device="cuda") * 0.125 * 2.0 ** torch.randint(-20, 12, kind.shape, generator=g, device="cuda")
    x = torch.where(kind == 2, steps, x)                                     # on the borders
    x = torch.where(kind == 3, x * 2.0 ** -20, x)
    x = torch.where(kind == 4, x * 2.0 ** -130, x)                           # denormal in fp32
    x = torch.where(kind == 5, torch.where(x > 0, -x * 2.0 ** -60, x), x)    # just below a border
    x = x.clamp(-61440.0, 61440.0).flatten(-2).to(dtype).float().clamp(-61440.0, 61440.0)
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d, Hkv, page", [(64, 1, 16), (64, 3, 32), (128, 2, 16), (128, 8, 128)])
def test_append_rounds_exactly(dtype, d, Hkv, page):
    """Without norm and rotation every byte is determined; slots of other tokens keep theirs."""
    s = Setting4([1, 7, 0, 40, 3], [1, 20, 5, 40, 130], Hkv, Hkv, d, dtype, page=page, seed=d + Hkv)
    k, v = _odd_values(s.n, Hkv, d, dtype, 5), _odd_values(s.n, Hkv, d, dtype, 6)
    want = s.pool.clone()
    seq = [b for b, m in enumerate(s.new) for _ in range(m)]
    at = torch.tensor([own - m + i for m, own in zip(s.new, s.own) for i in range(m)], device="cuda")
    where = s.table[torch.tensor(seq, device="cuda"), at // page].long()
    for kv, x in enumerate((k, v)):
        byte, code, _ = p4.rounded(x)
        p4.put(want, page, d, kv, where, at % page, byte, code)
    cache = s.cache()
    cache.append(s.batch(), k, v)
    assert torch.equal(s.pool, want) and cache.status() == 0
    K, V = cache.load(where * page + at % page, dtype)
    for got, x in ((K, k), (V, v)):
        assert torch.equal(got.double(), p4.rounded(x)[2])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d, rot, interleaved, norm", [(128, 128, False, True), (128, 128, True, False), (128, 48, False, True), (64, 16, False, False),
                                                       (64, 64, False, True), (64, 32, True, True), (128, 16, False, False), (64, 48, False, True)])
def test_append_with_rotation(dtype, d, rot, interleaved, norm):
    """Queries within their bound; a key's value off by half a step of its scale and the bound of what was rounded."""
    s = Setting4([1, 5, 33, 2], [40, 5, 100, 700], 8, 2, d, dtype, page=32, edges=[0, 2, 4], prefix=[50, 3], seed=3)
    b = _binding()
    g = torch.Generator(device="cuda").manual_seed(1)
    w = [(1 + 0.1 * torch.randn(d, generator=g, device="cuda")).to(dtype) if norm else None for _ in "qk"]
    cache = s.cache()
    q = cache.append(s.batch(), s.k, s.v, rope=b.Rope(d, rotary_dim=rot, interleaved=interleaved), q=s.q, wq=w[0], wk=w[1], eps=1e-5)
    at = [own - m + i for m, own in zip(s.new, s.own) for i in range(m)]
    seq = [x for x, m in enumerate(s.new) for _ in range(m)]
    pos = torch.tensor([a + s.prefix[0 if x < 2 else 1] for a, x in zip(at, seq)])
    assert_within(q, *norm_rope(s.q, pos, w[0], freqs(rot), rot, interleaved, 1e-5), "q")
    want, _ = norm_rope(s.k, pos, w[1], freqs(rot), rot, interleaved, 1e-5)
    _, off = norm_rope(s.k.float(), pos, None if w[1] is None else w[1].float(), freqs(rot), rot, interleaved, 1e-5)       # fp32 up to the rounding
    at, seq = torch.tensor(at, device="cuda"), torch.tensor(seq, device="cuda")
    K, V = cache.load(s.table[seq, at // 32].long() * 32 + at % 32, F32)
    # the scale may be the next one (an eighth more at most) where the largest magnitude moves by its bound
    scale = (want.abs() + off).unflatten(-1, (-1, 16)).amax(-1, keepdim=True).expand(-1, -1, -1, 16).flatten(-2) * 1.125
    assert ((K.double().cpu() - want).abs() <= scale / 16 + off).all()
    assert torch.equal(V.double(), p4.rounded(s.v)[2]) and cache.status() == 0


@pytest.mark.parametrize("dtype", [BF, F32])
def test_append_of_what_has_no_scale(dtype):
    b = _binding()
    s = Setting4([6], [6], 2, 2, 64, dtype, seed=1)
    k = s.k.clone()
    k[0, 0, 3], k[1, 1, 17], k[2, 0, 63], k[3, 0, 0] = math.nan, math.inf, -math.inf, 61696.0          # beyond 61440
    k[4, 1, 5] = 61440.0
    cache = s.cache()
    cache.append(s.batch(), k, s.v)
    K, _ = cache.load(s.table[0, 0].long() * 16 + torch.arange(6, device="cuda"), F32)
    want = p4.rounded(k)[2]
    assert torch.equal(K.isnan(), want.isnan()) and torch.equal(K.nan_to_num(), want.nan_to_num().float())
    assert int(want.isnan().sum()) == 4 * 16 and cache.status() == b.ST_RANGE


@pytest.mark.parametrize("fresh", [True, False])
def test_append_leaves_out(fresh):
    """Bad pages, tokens before their sequence, broken offsets: nothing is written for them, the status tells."""
    b = _binding()
    s = Setting4([3, 4, 2], [3, 2, 40], 4, 2, 64, BF, seed=2)      # two of sequence 1's tokens lie before it
    s.table[2, 2] = s.pool.shape[0]                                # and sequence 2's last page is none
    cache, before = s.cache(), s.pool.clone()
    out = None if fresh else torch.full_like(s.q, 7)
    q = cache.append(s.batch(), s.k, s.v, q=s.q, q_out=out)
    assert cache.status() == b.ST_PAGE and torch.equal(q, s.q)
    changed = {int(p) for p in (s.pool != before).flatten(1).any(1).nonzero()}
    assert changed == {int(s.table[0, 0]), int(s.table[1, 0])}
    before = s.pool.clone()
    for cu in ([0, 3, 2, 9], [-1, 3, 7, 9], [0, 3, 7, 10]):
        cache = s.cache()
        cache.append(b.PagedBatch(_ints(cu), s.lengths, s.table), s.k, s.v, q=s.q, q_out=None if fresh else torch.full_like(s.q, 7))
        assert cache.status() & b.ST_PAGE
    with pytest.raises(ValueError, match="rope"):
        cache.append(s.batch(), s.k, s.v, rope=b.Rope(128))
    with pytest.raises(ValueError, match="d = |shape"):
        cache.append(s.batch(), s.k[..., :32], s.v)
    with pytest.raises(ValueError):
        cache.append(s.batch(), s.k.half(), s.v.half())


# ---- load ----

@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_load(dtype, d):
    """All scales and codes, in slots of any order and more than once, padding, slots behind the pool, strided outputs."""
    b = _binding()
    Hkv, page, pages = 3, 32, 20
    g = torch.Generator(device="cuda").manual_seed(0)
    pool = torch.randint(0, 248, (pages, Hkv, b.PagedCache4.bytes(page, d)), generator=g, device="cuda").to(torch.uint8)
    cache = b.PagedCache4(pool, page, d)
    slots = torch.randint(0, pages * page, (1000,), generator=g, device="cuda")
    slots[5] = slots[6]
    slots[17] = -1
    slots[18] = -(2 ** 40)
    K, V = p4.decoded(pool, page, d)
    want = [x[slots.clamp(min=0) // page, :, slots.clamp(min=0) % page] * (slots >= 0)[:, None, None] for x in (K, V)]
    for got, w in zip(cache.load(slots, dtype), want):
        assert got.dtype is dtype and torch.equal(got.double(), w)
    assert cache.status() == 0
    wide = torch.full((1000, 2 * Hkv + 1, d), 7.0, device="cuda").to(dtype)
    again = cache.load(slots, dtype, K=wide[:, :Hkv], V=wide[:, Hkv + 1:])
    assert again[0].data_ptr() == wide.data_ptr() and torch.equal(wide[:, :Hkv].double(), want[0]) and torch.equal(wide[:, Hkv + 1:].double(), want[1])
    assert (wide[:, Hkv] == 7).all()
    heads = torch.empty(Hkv, 1000, d, dtype=dtype, device="cuda")            # as a prefill takes them
    cache.load(slots, dtype, K=heads.transpose(0, 1), V=torch.empty_like(heads).transpose(0, 1))
    assert torch.equal(heads.transpose(0, 1).double(), want[0])
    slots[3], slots[4] = pages * page, 2 ** 62
    K, V = cache.load(slots, dtype)
    assert K[3:5].isnan().all() and V[3:5].isnan().all() and not K[5:].isnan().any() and cache.status() == b.ST_PAGE
    assert cache.load(slots[:0], dtype)[0].shape == (0, Hkv, d)
    with pytest.raises(ValueError, match="slots"):
        cache.load(slots.int())


# ---- attend ----

LENGTHS = [(([1] * 9), [0 + 1, 2, 15, 16, 17, 127, 128, 129, 1000]), ([1, 2, 3, 1], [300, 33, 3, 2000]), ([1], [5000])]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d, H, Hkv", [(64, 8, 8), (64, 4, 2), (128, 8, 2), (128, 8, 1), (128, 4, 4)])
@pytest.mark.parametrize("new, own", LENGTHS)
def test_single_tokens(dtype, d, H, Hkv, new, own):
    s = Setting4(new, own, H, Hkv, d, dtype, page=16, seed=d + H, behind=2)
    cache = s.cache()
    out = torch.full((s.n, H, d), 5.0, device="cuda").to(dtype)
    got = cache.attend(s.batch(), s.q, scale=d ** -0.5, out=out)
    want, bound = s.want(d ** -0.5)
    assert_within(got[: s.cu[-1]], want[: s.cu[-1]], bound[: s.cu[-1]])
    assert (got[s.cu[-1]:] == 5).all() and cache.status() == 0
    assert torch.equal(cache.attend(s.batch(), s.q, scale=d ** -0.5)[: s.cu[-1]], got[: s.cu[-1]])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("new, own", [([4, 4, 3], [4, 130, 1000]), ([8, 1, 0, 5], [8, 900, 77, 6]), ([9, 30], [700, 31]), ([70, 3], [500, 300]), ([300], [300]),
                                      ([129, 64], [1025, 64])])
def test_drafts_and_prompts(dtype, page, causal, new, own):
    """From 4 rows a sequence to several hundred: all kernels."""
    s = Setting4(new, own, 8, 2, 128, dtype, page=page, seed=len(new))
    got = s.cache().attend(s.batch(), s.q, scale=0.1, causal=causal)
    assert_within(got, *s.want(0.1, causal))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d, H, Hkv", [(64, 8, 1), (128, 8, 2), (64, 4, 4)])
@pytest.mark.parametrize("new, own, edges, prefix", [
    ([1, 1, 1], [1, 30, 200], [0, 1, 3], [100, 1]), ([1] * 40, list(range(1, 41)), [0, 40], [1000]), ([2, 5, 1], [2, 9, 300], [0, 3], [0]),
    ([1, 3], [0, 3], [0, 1, 2], [17, 129]), ([60, 20, 90], [60, 100, 400], [0, 2, 3], [333, 128]), ([4] * 9, [4] * 9, [0, 3, 3, 9], [50, 60, 70])])
def test_shared_prefixes(dtype, d, H, Hkv, new, own, edges, prefix):
    s = Setting4(new, own, H, Hkv, d, dtype, page=16, edges=edges, prefix=prefix, seed=7)
    cache = s.cache()
    got = cache.attend(s.batch(), s.q, scale=d ** -0.5)
    assert_within(got, *s.want(d ** -0.5))
    assert cache.status() == 0


def test_rows_that_see_nothing():
    """More new tokens than the length says, empty sequences: 0, whatever the query is."""
    for new, own in (([3, 1, 2], [1, 0, 2]), ([40, 30], [10, 0]), ([1], [0])):
        for dtype in (BF, F32):
            s = Setting4(new, own, 8, 2, 64, dtype, seed=3)
            s.q[0] = math.nan
            got = s.cache().attend(s.batch(), s.q, scale=0.3)
            at = 0
            for m, o in zip(new, own):
                blind = max(0, m - o)
                assert (got[at:at + blind] == 0).all()
                if blind < m:
                    assert not got[at + blind:at + m].isnan().any()
                at += m


@pytest.mark.parametrize("new, own, edges, prefix", [([1, 2, 1], [300, 77, 5], [], []), ([4, 1], [500, 40], [], []), ([90, 4], [200, 100], [], []), ([1, 3], [9, 20], [0, 2], [150])])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_queries_that_are_not_finite(dtype, new, own, edges, prefix):
    """Their own rows are NaN and no other."""
    s = Setting4(new, own, 8, 2, 128, dtype, edges=edges, prefix=prefix, seed=11)
    clean = s.cache().attend(s.batch(), s.q, scale=0.1)
    s.q[0, 3, 5], s.q[1, 0, 0], s.q[1, 7, 127] = math.nan, math.inf, -math.inf
    got = s.cache().attend(s.batch(), s.q, scale=0.1)
    hit = torch.zeros(s.n, 8, dtype=torch.bool, device="cuda")
    hit[0, 3] = hit[1, 0] = hit[1, 7] = True
    assert got[hit].isnan().all() and torch.equal(got[~hit], clean[~hit])


@pytest.mark.parametrize("size", [2.0 ** -100, 2.0 ** -30, 2.0 ** 20, 2.0 ** 60])
@pytest.mark.parametrize("new, own", [([1, 3], [900, 40]), ([100], [300])])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_queries_of_any_size(dtype, new, own, size):
    """The scale undoes it: the same result to the bit, since every factor is a power of two."""
    s = Setting4(new, own, 4, 1, 128, dtype, seed=5)
    plain = s.cache().attend(s.batch(), s.q, scale=0.125)
    got = s.cache().attend(s.batch(), (s.q * size).to(dtype), scale=0.125 / size)
    assert torch.equal(plain, got)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("new, own", [([1, 1, 4], [2000, 64, 700]), ([60, 70], [300, 400])])
def test_spread_scales(dtype, new, own):
    """Groups of very different magnitudes; scores from -1000s to 1000s."""
    s = Setting4(new, own, 8, 2, 128, dtype, seed=6, spread=1.5)
    assert_within(s.cache().attend(s.batch(), s.q, scale=1.0), *s.want(1.0))


@pytest.mark.parametrize("new, own", [([1, 1], [400, 50]), ([12, 12], [400, 50]), ([100, 40], [400, 50])])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_bad_pages(dtype, new, own):
    b = _binding()
    s = Setting4(new, own, 4, 2, 64, dtype, page=16, seed=8)
    good = s.cache().attend(s.batch(), s.q, scale=0.2)
    for bad in (-1, s.pool.shape[0], 2 ** 31 - 1):
        was = int(s.table[0, 7])
        s.table[0, 7] = bad
        cache = s.cache()
        got = cache.attend(s.batch(), s.q, scale=0.2)
        assert cache.status() == b.ST_PAGE and got[new[0] - 1].isnan().all() and torch.equal(got[new[0]:], good[new[0]:])
        s.table[0, 7] = was
    for length in (-3, 26 * 16 + 1):
        cache = s.cache()
        got = cache.attend(b.PagedBatch(s.cu_q, _ints([length, own[1]]), s.table[:, :26].contiguous()), s.q, scale=0.2)
        assert cache.status() == b.ST_PAGE and got[: new[0]].isnan().all() and torch.equal(got[new[0]:], good[new[0]:])


@pytest.mark.parametrize("new", [[1, 2], [40, 60]])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_broken_offsets(dtype, new):
    b = _binding()
    s = Setting4(new, [70, 90], 4, 2, 64, dtype, seed=9)
    for cu in ([0, s.n + 1, s.n], [-1, 1, s.n], [0, 1, s.n + 1], [0, s.n, 1]):
        for out in (None, torch.full_like(s.q, 3)):
            cache = s.cache()
            got = cache.attend(b.PagedBatch(_ints(cu), s.lengths, s.table), s.q, scale=0.2, out=out)
            assert cache.status() == b.ST_PAGE and (got.isnan().all() if out is None else (got == 3).all())


def test_strides():
    """Queries that are slices of a projection, outputs with strides, a pool whose heads come before its pages."""
    for new, own in (([1, 2], [300, 40]), ([50, 20], [300, 40])):
        for dtype in (BF, F32):
            s = Setting4(new, own, 8, 2, 64, dtype, page=32, seed=10)
            want = s.cache().attend(s.batch(), s.q, scale=0.2)
            wide = torch.randn(s.n, 20, 64, device="cuda").to(dtype)
            wide[:, 4:12] = s.q
            out = torch.empty(8, s.n, 64, dtype=dtype, device="cuda")
            heads_first = torch.empty(2, s.pool.shape[0] + 1, s.pool.shape[2] + 48, dtype=torch.uint8, device="cuda")[:, 1:, 32:-16].transpose(0, 1)
            heads_first.copy_(s.pool)
            cache = _binding().PagedCache4(heads_first, 32, 64)
            got = cache.attend(s.batch(), wide[:, 4:12], scale=0.2, out=out.transpose(0, 1))
            assert got.data_ptr() == out.data_ptr() and torch.equal(got, want)


def test_more_than_4_gb():
    """Pages far out in a pool of more than 2^32 bytes."""
    b = _binding()
    pages, Hkv, page, d = 30000, 8, 128, 128
    pool = torch.empty(pages, Hkv, b.PagedCache4.bytes(page, d), dtype=torch.uint8, device="cuda")
    s = Setting4([1, 60], [500, 300], 32, Hkv, d, BF, page=page, seed=12)
    far = torch.arange(pages - 1, pages - 1 - s.pool.shape[0], -1, device="cuda")
    pool[far] = s.pool
    batch = b.PagedBatch(s.cu_q, s.lengths, torch.where(s.table >= 0, far[s.table.clamp(min=0).long()].int(), s.table))
    cache = b.PagedCache4(pool, page, d)
    assert torch.equal(cache.attend(batch, s.q, scale=0.1), s.cache().attend(s.batch(), s.q, scale=0.1))
    one = b.PagedBatch(s.cu_q[:2].contiguous(), s.lengths[:1].contiguous(), batch.tensors[2][:1].contiguous())
    here = b.PagedBatch(s.cu_q[:2].contiguous(), s.lengths[:1].contiguous(), s.table[:1].contiguous())
    assert torch.equal(cache.attend(one, s.q[:1], scale=0.1), s.cache().attend(here, s.q[:1], scale=0.1))
    k, v = s.k[:1].contiguous(), s.v[:1].contiguous()
    cache.append(one, k, v)
    at = batch.tensors[2][0, 499 // page].long() * page + 499 % page
    K, V = cache.load(at.view(1), F32)
    assert torch.equal(K.double(), p4.rounded(k)[2]) and torch.equal(V.double(), p4.rounded(v)[2]) and cache.status() == 0


def test_random_batches():
    r = random.Random(4)
    for i in range(60):
        d, dtype, page = r.choice([64, 128]), r.choice([BF, BF, F32]), r.choice([16, 32, 128])
        Hkv = r.choice([1, 2, 4])
        H = Hkv * r.choice([1, 2, 4, 8])
        B, most = r.randint(1, 12), r.choice([1, 3, 40])
        new = [r.randint(0, most) for _ in range(B)]
        own = [r.choice([0, 1, 16, r.randint(0, 700)]) for _ in range(B)]
        groups = r.choice([0, 0, 1, 3])
        edges = [0] + sorted(r.randint(0, B) for _ in range(groups - 1)) + [B] if groups else []
        prefix = [r.choice([0, 5, r.randint(0, 600)]) for _ in range(groups)]
        s = Setting4(new, own, H, Hkv, d, dtype, page=page, edges=edges, prefix=prefix, seed=i, behind=1)
        causal, scale = r.random() < 0.8, r.choice([0.05, d ** -0.5, 1.0])
        cache = s.cache()
        got = cache.attend(s.batch(), s.q, scale=scale, causal=causal)
        want, bound = s.want(scale, causal)
        assert_within(got[: s.cu[-1]], want[: s.cu[-1]], bound[: s.cu[-1]], "case %d" % i)
        assert cache.status() == 0


def test_many_sequences():
    r = random.Random(1)
    s = Setting4([1] * 1024, [r.randint(1, 90) for _ in range(1024)], 4, 1, 64, BF, seed=1)
    assert_within(s.cache().attend(s.batch(), s.q, scale=0.125), *s.want(0.125))


# ---- graphs, streams ----

@pytest.mark.parametrize("new", [[1, 1, 2], [30, 20, 25]])
def test_a_graph_with_lengths_that_change(new):
    s = Setting4(new, [900, 700, 300], 8, 2, 128, BF, seed=13)
    cache, batch = s.cache(), s.batch()
    cache.attend(batch, s.q, scale=0.1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = cache.attend(batch, s.q, scale=0.1)
    for own in ([900, 700, 300], [33, 640, 31], [130, 129, 128]):
        s.lengths.copy_(_ints(own))
        s.own = own
        out.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        assert_within(out, *s.want(0.1))


def test_two_streams_and_two_graphs():
    """Calls that overlap share nothing but the pool."""
    sets = [Setting4([1, 2], [3000, 700], 8, 2, 128, BF, seed=1), Setting4([60, 30], [500, 900], 8, 2, 128, BF, seed=2)]
    want = [s.cache().attend(s.batch(), s.q, scale=0.1) for s in sets]
    streams, graphs, outs = [torch.cuda.Stream() for _ in sets], [], []
    caches, batches = [s.cache() for s in sets], [s.batch() for s in sets]
    for s, c, b in zip(sets, caches, batches):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(c.attend(b, s.q, scale=0.1))
        graphs.append(g)
    torch.cuda.synchronize()
    for _ in range(20):
        eager = []
        for st, g, s, c, b in zip(streams, graphs, sets, caches, batches):
            with torch.cuda.stream(st):
                g.replay()
                eager.append(c.attend(b, s.q, scale=0.1))
    torch.cuda.synchronize()
    for o, e, w in zip(outs, eager, want):
        assert torch.equal(o, w) and torch.equal(e, w)


# ---- the tables of a step ----

def _tables(r, B, wide, pages, page, longest):
    lengths = [r.randint(0, min(longest, wide * page)) for _ in range(B)]
    ids = list(range(pages))
    r.shuffle(ids)
    table = [[-7] * wide for _ in range(B)]
    for b in range(B):
        for k in range(-(-lengths[b] // page)):
            table[b][k] = ids.pop()
    return lengths, table, ids


@pytest.mark.parametrize("seed", range(12))
def test_page_step(seed):
    """Random steps, some with too few pages, too few rows of tokens or too narrow tables, in place and not."""
    b = _binding()
    r = random.Random(seed)
    B, page, wide = r.choice([1, 2, 31, 64, 129, 1000, 1024]), r.choice([16, 64, 1024]), r.choice([3, 20])
    pages = B * wide // 2 + 5 if seed % 3 else B * wide + 9
    lengths, table, free = _tables(r, B, wide, pages, page, wide * page // 3)
    count = len(free)
    free += [99999] * (pages - count)
    for turn in range(4):
        most = r.choice([1, 5, page * 2])
        added = [r.choice([0, 1, r.randint(0, most)]) for _ in range(B)]
        ended = [int(r.random() < 0.2) for _ in range(B)]
        first = [r.randint(0, 1000) for _ in range(B)] if turn % 2 else None
        n = max(0, sum(added) + r.choice([-3, 0, 0, 7]))
        t = dict(lengths=_ints(lengths), table=_ints(table), free=_ints(free), count=_ints([count]))
        status = _ints([0])
        got = b.page_step(t["lengths"], t["table"], t["free"], t["count"], _ints(added), page, n, ended=_ints(ended), first=None if first is None else _ints(first),
                          in_place=turn < 2, status=status)
        was = lengths
        cu, lengths, count, slots, positions, served = p4.step(lengths, table, free, count, added, page, n, ended, first)
        assert got.cu_q.tolist() == cu and got.lengths.tolist() == lengths and got.free_count.tolist() == [count]
        assert got.slots.tolist() == slots and got.positions.tolist() == positions
        assert t["table"].tolist() == table and t["free"].tolist() == free
        assert int(status) == (0 if served else b.ST_CAPACITY)
        assert t["lengths"].tolist() == (lengths if turn < 2 else was)


def test_page_step_large():
    """Many tokens, many pages given back; a row that ends and begins again in one step."""
    b = _binding()
    r = random.Random(3)
    B, page, wide = 700, 16, 600
    pages = B * wide // 2 + 100
    lengths, table, free = _tables(r, B, wide, pages, page, 4000)
    count = len(free)
    free += [0] * (pages - count)
    added, ended = [r.randint(0, 400) for _ in range(B)], [int(r.random() < 0.5) for _ in range(B)]
    n = sum(added)
    t = [_ints(lengths), _ints(table), _ints(free), _ints([count])]
    got = b.page_step(*t, _ints(added), page, n, ended=_ints(ended))
    cu, lengths, count, slots, positions, served = p4.step(lengths, table, free, count, added, page, n, ended)
    assert served and got.slots.tolist() == slots and got.positions.tolist() == positions and got.cu_q.tolist() == cu
    assert t[0].tolist() == lengths and t[1].tolist() == table and t[2].tolist() == free and t[3].tolist() == [count]


def test_page_step_of_what_is_wrong():
    """Lengths, counts, tokens and entries that cannot be: the status tells, nothing outside is touched."""
    b = _binding()
    pages, page = 10, 16

    def go(lengths=(5, 20), added=(1, 1), table=((0, -1), (1, 2)), count=7, ended=None):
        status = _ints([0])
        guard = torch.full((3, pages), 55, dtype=torch.int32, device="cuda")
        guard[1] = _ints(list(range(3, 3 + pages)))
        x = b.page_step(_ints(lengths), _ints(table), guard[1], _ints([count]), _ints(added), page, 4, ended=None if ended is None else _ints(ended), status=status)
        assert (guard[0] == 55).all() and (guard[2] == 55).all()
        return x, int(status)

    x, st = go()
    assert st == 0 and x.slots.tolist() == [5, 2 * 16 + 4, -1, -1]
    x, st = go(lengths=(-1, 20))
    assert st == b.ST_PAGE and x.cu_q.tolist() == [0, 0, 1] and x.lengths.tolist() == [-1, 21]
    x, st = go(lengths=(5, 33), ended=(0, 1))
    assert st == b.ST_PAGE and x.lengths.tolist() == [6, 33] and x.free_count.tolist() == [7]
    x, st = go(added=(-4, 1))
    assert st == b.ST_PAGE and x.cu_q.tolist() == [0, 0, 1]
    for count in (-1, 11):
        x, st = go(count=count)
        assert st == b.ST_PAGE and x.cu_q.tolist() == [0, 1, 2] and x.free_count.tolist() == [0]
    x, st = go(table=((77, -1), (1, 2)))
    assert st == b.ST_PAGE and x.slots.tolist() == [-1, 2 * 16 + 4, -1, -1]
    x, st = go(count=10, ended=(1, 1), added=(0, 0))
    assert st == b.ST_PAGE and x.free_count.tolist() == [10] and x.lengths.tolist() == [0, 0]
    x, st = go(added=(2 ** 31 - 1, 1))
    assert st == b.ST_CAPACITY and x.cu_q.tolist() == [0, 0, 0]              # the tokens of both do not fit


# ---- all of them together ----

@pytest.mark.parametrize("dtype", [BF, F32])
def test_serving(dtype):
    """Requests that come, grow and end: tables, append, attention and the read-back of every step in one captured graph, against a plain
    cache that is kept token by token."""
    b = _binding()
    B, H, Hkv, d, page, n = 5, 8, 2, 64, 16, 48
    tables = b.PageTables(B, 12, 30, page, n)
    pool = torch.randint(0, 256, (30, Hkv, b.PagedCache4.bytes(page, d)), device="cuda").to(torch.uint8)
    cache = b.PagedCache4(pool, page, d)
    rope = b.Rope(d)
    q, k, v = (torch.empty(n, h, d, dtype=dtype, device="cuda") for h in (H, Hkv, Hkv))
    added, ended = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")

    def once():
        tables.step(added, ended)
        turned = cache.append(tables.batch, k, v, rope=rope, q=q)
        return turned, cache.attend(tables.batch, turned, scale=0.125), cache.load(tables.slots, F32)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):                                            # every kernel once before the capture
        once()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        turned, out, (K, V) = once()
    r = random.Random(0)
    kept = [([], []) for _ in range(B)]
    for turn in range(14):
        over = [int(r.random() < 0.15) for _ in range(B)]
        new = [r.choice([0, 1, 1, 2, r.randint(0, 20)]) for _ in range(B)]
        while sum(new) > n or any((0 if o else len(x[0])) + m > 12 * page for o, x, m in zip(over, kept, new)):
            new = [m // 2 for m in new]
        added.copy_(_ints(new))
        ended.copy_(_ints(over))
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        cu = tables.cu_q.tolist()
        got = [y - x for x, y in zip(cu, cu[1:])]
        assert got == new or tables.status() == b.ST_CAPACITY
        for i in range(B):
            if over[i]:
                kept[i] = ([], [])
            for t in range(cu[i], cu[i + 1]):
                assert int(tables.positions[t]) == len(kept[i][0])
                kept[i][0].append(K[t].cpu().double())
                kept[i][1].append(V[t].cpu().double())
        assert tables.lengths.tolist() == [len(x[0]) for x in kept]
        total = cu[-1]
        pos = tables.positions[:total].cpu()
        want, off = norm_rope(k[:total].float(), pos, None, freqs(d), d, False, 0.0)
        scale = (want.abs() + off).unflatten(-1, (-1, 16)).amax(-1, keepdim=True).expand(-1, -1, -1, 16).flatten(-2) * 1.125
        assert ((K[:total].cpu().double() - want).abs() <= scale / 16 + off).all()
        assert torch.equal(V[:total].double(), p4.rounded(v[:total])[2]) and (K[total:] == 0).all()
        longest = max([1] + [len(x[0]) for x in kept])
        pools = [torch.zeros(B, Hkv, longest, d, dtype=torch.float64) for _ in "KV"]
        for i, x in enumerate(kept):
            for p, y in zip(pools, x):
                if y:
                    p[i, :, : len(y)] = torch.stack(y, 1)
        table = torch.arange(B)[:, None]
        rows = n * H // Hkv
        want, bound = p4.attend(turned[:total], pools[0], pools[1], cu, [len(x[0]) for x in kept], table, 0.125, few=dtype == F32 or rows <= 32 * B)
        assert_within(out[:total], want, bound, "turn %d" % turn)
    assert cache.status() == 0


def test_prompt_into_subgen():
    """A prompt through the 4-bit cache into SubGen.prefill: the state is that of the values that the cache holds."""
    b = _binding()
    n, Hkv, d, page = 400, 2, 64, 32
    tables = b.PageTables(1, 16, 16, page, n)
    cache = b.PagedCache4(torch.empty(16, Hkv, b.PagedCache4.bytes(page, d), dtype=torch.uint8, device="cuda"), page, d)
    k, v = (torch.randn(n, Hkv, d, device="cuda").to(BF) for _ in "kv")
    x = tables.step(_ints([n]))
    cache.append(tables.batch, k, v)
    K, V = (torch.empty(1, Hkv, n, d, dtype=BF, device="cuda") for _ in "KV")
    cache.load(x.slots, BF, K=K[0].transpose(0, 1), V=V[0].transpose(0, 1))
    for got, y in ((K, k), (V, v)):
        assert torch.equal(got[0].transpose(0, 1).double(), p4.rounded(y)[2])
    states = []
    for a, c in ((K, V), (p4.rounded(k)[2].to(BF).transpose(0, 1)[None].contiguous(), p4.rounded(v)[2].to(BF).transpose(0, 1)[None].contiguous())):
        sg = b.SubGen(1, 4, d, 3.0, 4, 16, 8, seed=5, Hkv=Hkv, dtype=BF, m_max=256)
        sg.prefill(a, c)
        states.append([sg.export_state(0, h) for h in range(Hkv)])
    for s, t in zip(*states):
        assert s["m"] == t["m"] and s["mu"] == t["mu"] and (s["centre_tok"] == t["centre_tok"]).all() and (s["m_tok"] == t["m_tok"]).all()


def test_other_refusals():
    b = _binding()
    s = Setting4([1], [20], 4, 2, 64, BF, seed=1)
    cache, batch = s.cache(), s.batch()
    for call in (lambda: cache.attend(batch, s.q.cpu()), lambda: cache.attend(batch, s.q[..., :32]), lambda: cache.attend(batch, s.q.double()),
                 lambda: cache.attend(batch, s.q, out=s.q.float()), lambda: cache.load(torch.zeros(2, 2, dtype=torch.int64, device="cuda")),
                 lambda: b.PagedCache4(s.pool[..., :-16], 16, 64), lambda: b.PagedCache4(s.pool.int(), 16, 64),
                 lambda: b.page_step(_ints([1]), _ints([[1]]), _ints([1]), _ints([1]), _ints([1, 2]), 16, 4),
                 lambda: b.page_step(_ints([1]), _ints([1]), _ints([1]), _ints([1]), _ints([1]), 16, 4)):
        with pytest.raises(ValueError):
            call()
    for n in (-1, 2 ** 31, 2 ** 32 + 4, 2 ** 70, None):
        with pytest.raises(ValueError):
            b.page_step(_ints([1]), _ints([[1]]), _ints([1]), _ints([1]), _ints([1]), 16, n)
    with pytest.raises(b.SubgenError):
        cache.attend(batch, s.q, scale=0.0)
    with pytest.raises(b.SubgenError):
        cache.attend(batch, s.q, out=s.q)
    with pytest.raises(b.SubgenError, match="page"):
        b.page_step(_ints([1]), _ints([[1]]), _ints([1]), _ints([1]), _ints([1]), 24, 4)
