"""The 4-bit paged cache and the tables of a step where the calls of test_gpu_paged4.py do not go."""
import ctypes as C
import random
import sys

import pytest
import torch

import paged4_helpers as p4
from paged4_helpers import Setting4
from paged_helpers import assert_within

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _binding():
    from paper_2402_06082_b200 import binding
    return binding


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _stream():
    return torch.cuda.current_stream().cuda_stream


# ---- load ----

@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d, Hkv", [(64, 1), (64, 9), (128, 3)])
@pytest.mark.parametrize("side", [0, 1])
def test_load_of_one_side(dtype, d, Hkv, side):
    """The library's call with K or V alone: values, padding, and the status of a slot behind the pool."""
    b = _binding()
    page, pages, n = 32, 5, 70
    g = torch.Generator(device="cuda").manual_seed(d + Hkv)
    pool = torch.randint(0, 248, (pages, Hkv, b.PagedCache4.bytes(page, d)), generator=g, device="cuda").to(torch.uint8)
    slots = torch.randint(0, pages * page, (n,), generator=g, device="cuda")
    slots[2] = -1
    status = _ints([0])
    desc = b.Pages4Desc(pool.data_ptr(), pool.stride(0), pool.stride(1), pages, page, Hkv, d, status.data_ptr())
    want = p4.decoded(pool, page, d)[side][slots.clamp(min=0) // page, :, slots.clamp(min=0) % page]
    want[2] = 0
    for behind in (None, 0, n - 1):
        if behind is not None:
            slots[behind] = pages * page + 3
        out = torch.full((n, Hkv, d), 7.0, device="cuda").to(dtype)
        heads = [b.Heads(None, 0, 0), b.Heads(None, 0, 0)]
        heads[side] = b.Heads(out.data_ptr(), Hkv * d, d)
        assert b.load().subgen_paged4_load(desc, slots.data_ptr(), n, C.byref(heads[0]), C.byref(heads[1]), 0 if dtype is F32 else 1, _stream()) == 0
        kept = torch.ones(n, dtype=torch.bool, device="cuda")
        if behind is not None:
            kept[behind] = False
            if behind:
                kept[0] = False
            assert out[~kept].isnan().all()
        assert torch.equal(out[kept].double(), want[kept])
        assert int(status) == (0 if behind is None else b.ST_PAGE)
        status.zero_()


def test_load_refuses_outputs_without_keeping_them():
    b = _binding()
    cache = b.PagedCache4(torch.zeros(2, 2, b.PagedCache4.bytes(16, 64), dtype=torch.uint8, device="cuda"), 16, 64)
    slots = torch.zeros(3, dtype=torch.int64, device="cuda")
    good = torch.empty(3, 2, 64, dtype=BF, device="cuda")
    for bad in (torch.empty(3, 2, 128, dtype=BF, device="cuda"), torch.empty(3, 2, 64, device="cuda"), torch.empty(3, 2, 64, dtype=BF)):
        counts = [sys.getrefcount(x) for x in (good, bad)]
        for K, V in ((bad, None), (None, bad), (good, bad), (bad, good)):
            with pytest.raises(ValueError, match="must be a"):
                cache.load(slots, BF, K=K, V=V)
        with pytest.raises(b.SubgenError):                   # refused by the library
            cache.load(slots, BF, K=good, V=good)
        del K, V
        assert [sys.getrefcount(x) for x in (good, bad)] == counts


# ---- attend ----

def test_half_a_million_row_units():
    """fp32 rows by the million against a short memory: units of 8 rows, whose place in the division of the work is not walked to."""
    b = _binding()
    n, H, d, own = 1 << 19, 8, 64, 200
    s = Setting4([n], [own], H, 1, d, F32, page=64, seed=21)
    cache = s.cache()
    got = cache.attend(s.batch(), s.q, scale=0.125, causal=False)
    assert cache.status() == 0
    some = torch.cat([torch.arange(40), torch.randint(0, n, (200,), generator=torch.Generator().manual_seed(0)), torch.arange(n - 40, n)]).cuda()
    K, V = p4.decoded(s.pool, 64, d)
    want, bound = p4.attend(s.q[some], K, V, [0, len(some)], [own], s.table, 0.125, False)
    assert_within(got[some], want, bound)
    k, v = (x[s.table[0].long(), 0].flatten(0, 1)[:own].float() for x in (K, V))
    for i in range(0, n, 1 << 16):                           # every row: none is left out
        y = torch.softmax(s.q[i:i + (1 << 16)] @ k.T * 0.125, -1) @ v
        assert (got[i:i + (1 << 16)] - y).abs().max() < 1e-2


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("causal", [True, False])
def test_one_prompt_among_single_tokens(dtype, causal):
    """Hundreds of small row units of one sequence (fp32, and bf16 without a prefix), behind a prefix or not, some of them blind."""
    for new, own, edges, prefix in (([1] * 150 + [1000] + [1] * 150, [50] * 150 + [1030] + [9] * 150, [], []),
                                    ([1] * 140 + [999], [3] * 140 + [400], [0, 140, 141], [100, 130]), ([1] * 140 + [999], [3] * 140 + [400], [0, 141], [300])):
        s = Setting4(new, own, 4, 1, 64, dtype, seed=len(new), edges=edges, prefix=prefix)
        cache = s.cache()
        assert_within(cache.attend(s.batch(), s.q, scale=0.125, causal=causal), *s.want(0.125, causal))
        assert cache.status() == 0


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("new, own", [([1], [300]), ([5, 2], [5, 900]), ([80], [200])])
def test_scores_of_zero_whatever_the_scale(dtype, new, own):
    """Keys of zeros: every token weighs the same, also where queries times the scale leave fp32."""
    s = Setting4(new, own, 4, 1, 64, dtype, seed=31)
    for row, length in zip(s.table, own):
        tok = torch.arange(length, device="cuda")
        none = torch.zeros(length, 1, 64, device="cuda")
        p4.put(s.pool, 16, 64, 0, row[tok // 16].long(), tok % 16, *p4.rounded(none)[:2])
    cache = s.cache()
    plain = cache.attend(s.batch(), s.q, scale=1.0)
    assert not plain.isnan().any()
    s.q.fill_(2.0 ** 127)
    for scale in (1.0, 2.0 ** 14, 2.0 ** 100):
        assert torch.equal(cache.attend(s.batch(), s.q, scale=scale), plain)


@pytest.mark.parametrize("d, H, Hkv", [(64, 8, 1), (128, 8, 2), (128, 4, 4), (64, 2, 1)])
@pytest.mark.parametrize("new, own, edges, prefix, causal", [
    ([300], [300], [], [], True), ([129, 64], [1025, 200], [], [], True), ([70, 90], [500, 300], [], [], False), ([60, 70, 90], [60, 100, 400], [0, 2, 3], [333, 128], True),
    ([40] * 6, [40, 60, 80, 100, 500, 900], [0, 6], [1000], True), ([33, 40], [2000, 3000], [], [], True)])
def test_weights_of_units_of_256_rows(d, H, Hkv, new, own, edges, prefix, causal):
    """bf16 rows in units of 256: weights are off by fp16's rounding, an eighth of bf16's."""
    s = Setting4(new, own, H, Hkv, d, BF, page=32, seed=d + H, edges=edges, prefix=prefix)
    assert not s.few()
    got = s.cache().attend(s.batch(), s.q, scale=d ** -0.5, causal=causal)
    want, bound = s.want(d ** -0.5, causal, few=True)        # the bound of fp16 weights
    assert_within(got, want, bound)


@pytest.mark.parametrize("n", [1, 8, 100])
def test_weights_that_nearly_cancel(n):
    """Two tokens whose values cancel in some coordinate of some rows: there the weights' rounding shows, and bf16's would not do."""
    d, H = 64, 4
    s = Setting4([n], [2], H, 1, d, BF, seed=n)
    tok = torch.arange(2, device="cuda")
    steps = torch.zeros(2, 1, d, dtype=torch.int64, device="cuda")           # codes; scale 1: (code - 7.5) / 8
    steps[0] = 15
    steps[1, 0] = torch.arange(d, device="cuda") % 8                         # -0.9375 to -0.0625
    one = torch.full((2, 1, d // 16), 15 << 3, dtype=torch.uint8, device="cuda")
    p4.put(s.pool, 16, d, 1, s.table[0, tok // 16].long(), tok % 16, one, steps)
    steps[1] = 0
    one[1] = 0                                                               # a key of zeros
    p4.put(s.pool, 16, d, 0, s.table[0, tok // 16].long(), tok % 16, one, steps)
    score = torch.linspace(-2.8, 0.0, n * H, device="cuda").view(n, H, 1)
    s.q = (score / (0.9375 * d)).expand(n, H, d).to(BF).contiguous()
    want, bound = s.want(1.0, False, few=True)
    assert_within(s.cache().attend(s.batch(), s.q, scale=1.0, causal=False), want, bound)
    if n == 100:                                                             # what bf16 weights would give is beyond it
        x = s.q[..., :1].double().cpu() * 0.9375 * d
        V = p4.decoded(s.pool, 16, d)[1][s.table[0, 0].long(), 0, :2].cpu()
        w = torch.exp(x).to(BF).double()
        off = ((w * V[0] + V[1]) / (1 + torch.exp(x)) - want).abs() - bound
        assert float(off.max()) > 0


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("new, own, edges, prefix", [([1, 2], [200, 90], [], []), ([6, 1], [140, 30], [], []), ([300, 5], [300, 70], [], []), ([1, 3, 1], [5, 20, 9], [0, 2, 3], [50, 60])])
def test_groups_that_read_as_nan(dtype, new, own, edges, prefix):
    """A key's group makes the rows that see it NaN and no other; a value's group its 16 coordinates, in no row of another unit."""
    s = Setting4(new, own, 4, 1, 64, dtype, seed=17, edges=edges, prefix=prefix)
    clean = s.cache().attend(s.batch(), s.q, scale=0.125)
    assert not clean.isnan().any()
    for at in (own[0] - 1, max(0, own[0] - 3), 0):                           # own token `at` of sequence 0
        first = max(0, at - (own[0] - new[0]))                               # the first of its rows that sees it
        sees = torch.zeros(s.n, dtype=torch.bool, device="cuda")
        sees[first:new[0]] = True
        x = s.pool.unflatten(-1, (1, 2, 16 * (32 + 4)))
        page, row = int(s.table[0, at // 16]), at % 16
        for kv in range(2):
            was = x[page, 0, 0, kv, 16 * 32 + row * 4 + 2].clone()
            x[page, 0, 0, kv, 16 * 32 + row * 4 + 2] = 255                   # coordinates 32 to 47
            got = s.cache().attend(s.batch(), s.q, scale=0.125)
            x[page, 0, 0, kv, 16 * 32 + row * 4 + 2] = was
            if kv == 0:
                assert got[sees].isnan().all() and torch.equal(got[~sees], clean[~sees])
            else:
                assert got[sees][:, :, 32:48].isnan().all()
                rest = torch.cat((got[:, :, :32], got[:, :, 48:]), -1)
                assert torch.equal(rest, torch.cat((clean[:, :, :32], clean[:, :, 48:]), -1))
                assert torch.equal(got[new[0]:], clean[new[0]:])             # other sequences


# ---- the tables of a step ----

@pytest.mark.parametrize("n", [2 ** 31 - 1, 2 ** 31 - 4000])
def test_page_step_for_the_most_tokens(n):
    """Slots and positions of 2^31 - 1 tokens: all of them are written, the last row's too."""
    b = _binding()
    slots, positions = torch.full((n,), 5, dtype=torch.int64, device="cuda"), torch.full((n,), 5, dtype=torch.int32, device="cuda")
    wide = (2 ** 31 - 1024) // 1024 - 1
    added = [3, 0, wide * 1024]                              # the last row takes all but what is behind
    table = torch.zeros(3, wide, dtype=torch.int32, device="cuda")
    free = torch.arange(wide + 1, dtype=torch.int32, device="cuda")
    status = _ints([0])
    x = b.page_step(_ints([0, 0, 0]), table, free, _ints([wide + 1]), _ints(added), 1024, n, slots=slots, positions=positions, status=status)
    total = 3 + wide * 1024
    if total > n:
        assert int(status) == b.ST_CAPACITY and x.cu_q.tolist() == [0, 3, 3, 3]
        total = 3
    else:
        assert int(status) == 0 and x.cu_q.tolist() == [0, 3, 3, total]
        assert positions[:5].tolist() == [0, 1, 2, 0, 1] and slots[:5].tolist() == [wide * 1024, wide * 1024 + 1, wide * 1024 + 2, (wide - 1) * 1024, (wide - 1) * 1024 + 1]
        for at in (3 + 1024 * 1000, total - 1024):
            page = (at - 3) // 1024
            assert (slots[at:at + 1024] == (wide - 1 - page) * 1024 + torch.arange(1024, device="cuda")).all()
            assert (positions[at:at + 1024] == page * 1024 + torch.arange(1024, device="cuda")).all()
    step = 1 << 28
    for i in range(total, n, step):
        assert (slots[i:i + step] == -1).all() and (positions[i:i + step] == 0).all()
    for i in range(3, total, step):
        assert int(slots[i:min(i + step, total)].min()) >= 0


def _sources(cu, added, n):
    """By the definition: token i of a step is that row's token, counted from where `added` alone puts the row; below n, which no input passes."""
    out, at = [], 0
    for b, k in enumerate(added):
        out += [min(at + i, n - 1) for i in range(cu[b + 1] - cu[b])]
        at += max(k, 0)
    return out + [0] * (n - len(out))


@pytest.mark.parametrize("B, most, n", [(1, 5, 9), (40, 3, 70), (1024, 2, 900), (129, 60, 3000), (300, 60, 7000), (1000, 30, 14000)])
def test_sources(B, most, n):
    """Where a step's tokens lie in inputs that hold what was asked for, with rows that are not served; one kernel and two."""
    b = _binding()
    r = random.Random(B)
    for turn in range(3):
        added = [r.randint(0, most) for _ in range(B)]
        if turn == 2:
            added[B // 2] = 2 ** 31 - 1                      # nobody behind it is served
        lengths = [r.randint(0, 40) for _ in range(B)]
        if turn:
            lengths[B // 3] = -1                             # gets nothing, and its tokens are in the input
        pages = 5 * B + 200
        ids = list(range(pages))
        table = [[ids.pop() if k < -(-max(x, 0) // 16) else -1 for k in range(10)] for x in lengths]
        count = len(ids) if not turn else B // 2
        ids += [0] * (pages - len(ids))                      # the stack has room for all of the pool's pages
        sources, status = torch.full((n,), 9, dtype=torch.int32, device="cuda"), _ints([0])
        x = b.page_step(_ints(lengths), _ints(table), _ints(ids), _ints([count]), _ints(added), 16, n, sources=sources, status=status)
        cu = x.cu_q.tolist()
        if not turn:                                         # pages and places for all whose tokens come before the n-th
            total = 0
            for k, y, z in zip(added, cu, cu[1:]):
                total += k
                assert z - y == (k if total <= n else 0)
        assert sources.tolist() == _sources(cu, added, n)
        assert (x.slots[: cu[-1]] >= 0).all()


def test_page_tables_that_run_out():
    """Requests in a captured graph on a pool that is too small: tables, stack, lengths and inputs of every step as a host program has
    them, the values that are read back those of each request's own inputs."""
    b = _binding()
    B, Hkv, d, page, n, pages, wide = 6, 2, 64, 16, 64, 9, 5
    tables = b.PageTables(B, wide, pages, page, n)
    cache = b.PagedCache4(torch.zeros(pages, Hkv, b.PagedCache4.bytes(page, d), dtype=torch.uint8, device="cuda"), page, d)
    k, v = (torch.zeros(n, Hkv, d, device="cuda") for _ in "kv")
    added, ended = _ints([0] * B), _ints([0] * B)

    def once():
        tables.step(added, ended)
        i = tables.sources
        cache.append(tables.batch, k[i], v[i])
        return cache.load(tables.slots, F32)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        once()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        K, V = once()
    r = random.Random(5)
    lengths, table, free, count = [0] * B, [[0] * wide for _ in range(B)], list(range(pages - 1, -1, -1)), pages
    short = []
    for turn in range(25):
        over = [int(r.random() < 0.15) for _ in range(B)]
        new = [r.choice([0, 1, 5, 20]) for _ in range(B)]
        while sum(new) > n:
            new = [x // 2 for x in new]
        added.copy_(_ints(new))
        ended.copy_(_ints(over))
        for x in (k, v):
            x.copy_(torch.randn(x.shape, device="cuda"))
        tables._status.zero_()
        graph.replay()
        cu, lengths, count, slots, positions, served = p4.step(lengths, table, free, count, new, page, n, over)
        assert tables.status() == (0 if served else b.ST_CAPACITY)
        short.append(not served)
        assert tables.cu_q.tolist() == cu and tables.lengths.tolist() == lengths and tables.free_count.tolist() == [count]
        assert tables.table.tolist() == table and tables.free.tolist() == free
        assert tables.slots.tolist() == slots and tables.positions.tolist() == positions
        at, where = [sum(new[:i]) for i in range(B)], []
        for i in range(B):
            where += [at[i] + j for j in range(cu[i + 1] - cu[i])]
        for got, x in ((K, k), (V, v)):
            assert torch.equal(got[: cu[-1]].double(), p4.rounded(x[where])[2])
    assert any(short) and not all(short) and cache.status() == 0


def test_tables_made_in_a_capture_begin_anew():
    b = _binding()
    added = _ints([3, 20, 0])
    b.PageTables(3, 4, 10, 16, 32).step(added)               # the kernels, before the capture
    pool = torch.zeros(10, 1, b.PagedCache4.bytes(16, 64), dtype=torch.uint8, device="cuda")
    k = torch.full((32, 1, 64), 70000.0, device="cuda")      # beyond what has a scale
    b.PagedCache4(pool, 16, 64).append(b.PageTables(3, 4, 10, 16, 32).batch, k, k)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tables, cache = b.PageTables(3, 4, 10, 16, 32), b.PagedCache4(pool, 16, 64)
        tables.step(added)
        tables.step(added)
        cache.append(tables.batch, k, k)
    for _ in range(3):
        cache._status.fill_(b.ST_PAGE)
        graph.replay()
        assert tables.lengths.tolist() == [6, 40, 0] and tables.free_count.tolist() == [6] and tables.cu_q.tolist() == [0, 3, 23, 23]
        assert tables.table.tolist() == [[0, 0, 0, 0], [1, 2, 3, 0], [0, 0, 0, 0]] and tables.status() == 0
        assert cache.status() == b.ST_RANGE
