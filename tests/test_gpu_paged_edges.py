"""GPU tests of the paged operators at the edges of what a call may hold: values that are not finite, extreme values in masked
places, broken groups, far positions, outputs that nothing can be written to."""
import math
import os
import subprocess
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import paged_helpers as ph  # noqa: E402

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ---- attention ------------------------------------------------------------------------------------

SHAPES = {  # new, own, edges, prefix, H, Hkv
    "one token": ([1], [1], [], [], 4, 4),
    "four tokens": ([1, 4], [3, 4], [], [], 8, 2),
    "short prefix": ([1] * 3, [0] * 3, [0, 3], [3], 8, 4),
    "short and many": ([1, 2] * 40, [1, 3] * 40, [], [], 8, 2),
    "one tile": ([1], [20], [], [], 4, 4),
    "split over blocks": ([2], [9000], [], [], 8, 2),
    "a hundred rows": ([50], [700], [], [], 8, 4),
    "start of a prompt": ([300], [300], [], [], 4, 2),
    "two halves": ([300], [900], [], [], 4, 4),
    "behind a prefix": ([1, 3, 2], [30, 3, 200], [0, 3], [700], 8, 2),
    "many sequences": ([1] * 80, [10 + 9 * i for i in range(80)], [], [], 8, 2),
}


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("name", list(SHAPES))
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_queries_that_are_not_finite(dtype, d, name, value):
    """The softmax of scores that are NaN or infinite is NaN, also over one token; the other rows stay as they are."""
    new, own, edges, prefix, H, Hkv = SHAPES[name]
    s = ph.Setting(new, own, H, Hkv, d, dtype, 16, edges, prefix, seed=7)
    want, bound = s.want(0.1)
    bad = torch.zeros(s.n, H, dtype=torch.bool)
    for t in {0, 1, 2, s.n // 2, s.n - 1} & set(range(s.n)):
        for h in {0, H - 1}:
            s.q[t, h, (5 * t + h) % d] = value
            bad[t, h] = True
    want[bad] = math.nan
    ph.assert_within(s.cache().attend(s.batch(), s.q, scale=0.1), want, bound)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_rows_that_see_nothing_of_queries_that_are_not_finite(dtype):
    """More new tokens than the length says: the first ones see nothing and are 0 whatever they hold."""
    s = ph.Setting([5, 40], [2, 30], 4, 2, 64, dtype, 16, seed=2)
    want, bound = s.want(0.1)
    for t in (0, 1, 2, 5, 14):
        s.q[t] = math.nan
    ph.assert_within(s.cache().attend(s.batch(), s.q, scale=0.1), want, bound)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new, own, prefix, low", [
    (1, 256, 0, range(128)), (1, 256, 0, range(128, 256)), (1, 40, 0, range(39)), (2, 9000, 0, range(5000)), (60, 700, 0, range(500)),
    (300, 900, 0, range(128, 500)), (3, 200, 300, range(-300, 0)), (3, 200, 300, range(-300, 150)), (1, 129, 128, range(129)),
    (1, 40, 0, range(40)), (2, 9000, 0, range(9000)), (3, 200, 300, range(-300, 200)), (90, 300, 0, range(250))])
def test_scores_of_minus_infinity(dtype, d, new, own, prefix, low):
    """Keys whose products overflow have no weight, also where a block, a group of warps or a whole part of the row has no other;
    a row that sees none but those is NaN. Own tokens count from 0, the prefix's from -prefix."""
    s = ph.Setting([new], [own], 4, 2, d, dtype, 16, [0, 1] if prefix else [], [prefix] if prefix else [], seed=5)
    s.q.abs_().add_(1)
    scale, at = 0.25, []
    for j in low:
        row, i = (s.table[0], j) if j >= 0 else (s.ptable[0], prefix + j)
        at.append((int(row[i // 16]), i % 16))
    where = tuple(torch.tensor(x, device="cuda") for x in zip(*at))
    s.K[where[0], :, where[1]] = -8.0                  # d * 1 * 8 * scale = 128 below and more: no weight either
    want, bound = s.want(scale)
    s.K[where[0], :, where[1]] = torch.finfo(dtype).min
    for i in range(new):
        if all(j in low for j in range(-prefix, own - new + 1 + i)):
            want[i] = math.nan
    ph.assert_within(s.cache().attend(s.batch(), s.q, scale=scale), want, bound)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("name", list(SHAPES))
@pytest.mark.parametrize("scale", [3e4, 1e7, 1e9, 1e12, 1e30])
def test_scores_beyond_a_float_exponent(dtype, d, name, scale):
    """Finite scores of any size: where the largest is ahead by more than its rounding and 200, it has all the weight."""
    new, own, edges, prefix, H, Hkv = SHAPES[name]
    s = ph.Setting(new, own, H, Hkv, d, dtype, 16, edges, prefix, seed=8)
    got = s.cache().attend(s.batch(), s.q, scale=scale).cpu().double()
    clear = 0
    for b in range(len(new)):
        g = next((i for i in range(len(prefix)) if edges[i] <= b < edges[i + 1]), None)
        parts = ([(s.ptable[g], prefix[g])] if g is not None else []) + [(s.table[b], own[b])]
        k, v = (torch.cat([ph.own_tokens(pool, row, n) for row, n in parts], 1) for pool in (s.K, s.V))
        x = s.q[s.cu[b]:s.cu[b + 1]].cpu().double().view(new[b], Hkv, H // Hkv, d)
        sc = torch.einsum("thgd,hld->thgl", x, k) * scale
        size = torch.einsum("thgd,hld->thgl", x.abs(), k.abs()).amax(-1) * scale
        last = k.shape[1] - new[b] + torch.arange(new[b])
        sc.masked_fill_((torch.arange(k.shape[1]) > last[:, None])[:, None, None], -math.inf)
        two = torch.cat([sc, torch.full_like(sc[..., :1], -math.inf)], -1).topk(2, -1)
        ahead = (two.values[..., 0] - two.values[..., 1] > 200 + 4 * (d + 4) * ph.U32 * size).view(new[b], H)
        want = torch.stack([v[h][two.indices[:, h, :, 0].clamp(max=k.shape[1] - 1)] for h in range(Hkv)], 1).view(new[b], H, d)
        # its weight is any power of two up to 2^13, in the sum as it is, for the product rounded to bf16 (2^-8), perhaps by the
        # cubic in one and the same; 1 / sum, a product and the rounding of the output
        bound = (2 ** -7 + 2 ** -20 if dtype == BF16 else 2.0 ** -20) * want.abs()
        off = ((got[s.cu[b]:s.cu[b + 1]] - want).abs() > bound).any(-1)
        assert not (off & ahead).any() and torch.isfinite(got[s.cu[b]:s.cu[b + 1]]).all()
        clear += int(ahead.sum())
    assert clear > s.n * H // 2


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new, own, G", [(4, 5, 1), (8, 300, 1), (8, 8, 2), (20, 20, 4), (60, 61, 4), (200, 700, 1), (300, 300, 1)])
def test_extreme_values_that_a_row_does_not_see(dtype, d, new, own, G):
    """V of tokens behind a row's own is finite but the type's lowest: a weight that is not exactly 0 would show."""
    s = ph.Setting([new], [own], 2 * G, 2, d, dtype, 16, seed=3)
    want, bound = s.want(0.1)
    first = own - new + 1 if new < 64 else own - 20    # tokens from here on: rows up to the one before do not see them
    for j in range(first, own):
        s.V[int(s.table[0, j // 16]), :, j % 16] = torch.finfo(dtype).min
    rows = first - (own - new)
    out = s.cache().attend(s.batch(), s.q, scale=0.1)
    ph.assert_within(out[:rows], want[:rows], bound[:rows])


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new, own, G", [(4, 5, 1), (8, 300, 1), (20, 20, 4), (60, 61, 4), (200, 700, 1), (300, 300, 1)])
@pytest.mark.parametrize("value", ["lowest", "largest"])
def test_extreme_keys_that_a_row_does_not_see(dtype, d, new, own, G, value):
    """Keys behind a row's own whose products overflow, to either side or to NaN."""
    s = ph.Setting([new], [own], 2 * G, 2, d, dtype, 16, seed=4)
    want, bound = s.want(0.1)
    first = own - 2
    for j in range(first, own):
        s.K[int(s.table[0, j // 16]), :, j % 16] = torch.finfo(dtype).min if value == "lowest" else torch.finfo(dtype).max
    rows = first - (own - new)
    out = s.cache().attend(s.batch(), s.q, scale=0.1)
    ph.assert_within(out[:rows], want[:rows], bound[:rows])


def test_weights_of_the_cubic():
    """One token's weight against the largest's, from even to 2^-140 of it, by the place in the tile: within the bf16 bound."""
    n, d = 64, 64
    s = ph.Setting([1], [n], 1, 1, d, BF16, 64, seed=1)
    s.q.zero_()
    s.q[0, 0, 0] = 1
    K, V = s.K[int(s.table[0, 0]), 0], s.V[int(s.table[0, 0]), 0]
    for shift in (0.0, 0.37, 20.0):
        for last in (n - 1, n - 10):                   # the largest score by the cubic or not
            K.zero_()
            K[:, 0] = -torch.linspace(0, 97, n, device="cuda").to(BF16) - shift
            K[last, 0] = shift
            want, bound = s.want(1.0)
            ph.assert_within(s.cache().attend(s.batch(), s.q, scale=1.0), want, bound)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G, Hkv", [(8, 3), (8, 8), (4, 5), (1, 8)])
@pytest.mark.parametrize("seed", range(4))
def test_many_short_runs_of_two_halves(d, G, Hkv, seed):
    """Row units of more than 128 rows over a tile or two, between ones of one group alone: the groups' issuers get far apart."""
    g = torch.Generator().manual_seed(100 * seed + G)
    B = 150
    rows = torch.tensor([3, 40, 130, 180, 256, 300])[torch.randint(0, 6, (B,), generator=g)]
    new = ((rows + G - 1) // G).tolist()
    own = torch.tensor([1, 5, 60, 128, 129, 200, 300, 900])[torch.randint(0, 8, (B,), generator=g)].tolist()
    s = ph.Setting(new, own, G * Hkv, Hkv, d, BF16, 128, seed=seed)
    cache, batch = s.cache(), s.batch()
    want, bound = s.want(0.1)
    out = torch.full_like(s.q, 7.0)
    cache.attend(batch, s.q, scale=0.1, out=out)
    assert cache.status() == 0
    ph.assert_within(out, want, bound)
    for _ in range(20):
        again = torch.full_like(s.q, 7.0)
        cache.attend(batch, s.q, scale=0.1, out=again)
        assert torch.equal(again, out)
    assert cache.status() == 0


# ---- append ---------------------------------------------------------------------------------------

def _written(s, K0, tokens):
    """Exactly the slots of these tokens of s have changed."""
    where = [(b, s.own[b] - s.new[b] + i) for b in range(len(s.new)) for i in range(s.new[b])]
    changed = (torch.nan_to_num(s.K) != torch.nan_to_num(K0)).any(-1).any(1)
    want = torch.zeros_like(changed)
    for t in tokens:
        b, j = where[t]
        want[int(s.table[b, j // s.page]), j % s.page] = True
    assert torch.equal(changed, want)


BROKEN_GROUPS = {  # cu_group (of [0, 1, 3]), prefix_len (of [10, 20], tables of 32 tokens) -> tokens whose position is known, status
    "as it should be": ([0, 1, 3], [10, 20], [0, 1, 2, 3], 0),
    "whole tables": ([0, 1, 3], [32, 32], [0, 1, 2, 3], 0),
    "empty prefix": ([0, 0, 3], [10, 0], [0, 1, 2, 3], 0),
    "falls": ([0, 2, 1], [10, 20], [0, 1, 2], 8),
    "falls below 0": ([0, -1, 3], [10, 20], [0, 1, 2, 3], 8),
    "falls from the end": ([0, 3, 1], [10, 20], [0, 1, 2, 3], 8),
    "starts late": ([1, 2, 3], [10, 20], [1, 2, 3], 8),
    "ends early": ([0, 1, 2], [10, 20], [0, 1, 2], 8),
    "ends late": ([0, 1, 4], [10, 20], [0, 1, 2, 3], 8),
    "negative length": ([0, 1, 3], [10, -1], [0], 8),
    "beyond its table": ([0, 1, 3], [33, 20], [1, 2, 3], 8),
}


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("name", list(BROKEN_GROUPS))
def test_append_with_broken_groups(dtype, name):
    """A position that cannot be told is not made up: neither the key nor the query is written, and the status says so."""
    from paper_2402_06082_b200 import binding
    edges, lens, tokens, status = BROKEN_GROUPS[name]
    s = ph.Setting([1, 2, 1], [40, 30, 20], 4, 2, 64, dtype, 16, [0, 1, 3], [32, 32], seed=3)
    s.groups["cu_group"].copy_(_ints(edges))
    s.groups["prefix_len"].copy_(_ints(lens))
    rope = binding.Rope(64)
    cache, K0, q_out = s.cache(), s.K.clone(), torch.full_like(s.q, 7.0)
    cache.append(s.batch(), s.k, s.v, rope=rope, q=s.q, q_out=q_out)
    assert cache.status() == status
    _written(s, K0, tokens)
    seq = [0, 1, 1, 2]
    for t in range(4):
        if t not in tokens:
            assert bool((q_out[t] == 7).all())
            continue
        g = next(i for i in (0, 1) if edges[i] <= seq[t] < edges[i + 1])
        pos = torch.tensor([lens[g] + [39, 28, 29, 19][t]])
        ph.assert_within(q_out[t:t + 1], *ph.norm_rope(s.q[t:t + 1], pos, None, ph.freqs(64), 64, False, 0.0))


def test_append_where_two_groups_claim_a_sequence():
    from paper_2402_06082_b200 import binding
    s = ph.Setting([1, 2, 1], [40, 30, 20], 4, 2, 64, BF16, 16, [0, 1, 2, 3], [7, 7, 7], seed=3)
    s.groups["cu_group"].copy_(_ints([0, 3, 1, 3]))                # the first has all, the third the second and third sequence
    cache, K0 = s.cache(), s.K.clone()
    cache.append(s.batch(), s.k, s.v, rope=binding.Rope(64))
    assert cache.status() == 8
    _written(s, K0, [0])


def test_append_that_needs_no_prefix_length():
    """With positions, or without a rotation, groups are not looked at."""
    from paper_2402_06082_b200 import binding
    s = ph.Setting([1, 2, 1], [40, 30, 20], 4, 2, 64, BF16, 16, [0, 1, 3], [32, 32], seed=3)
    s.groups["prefix_len"].fill_(-1)
    cache, K0 = s.cache(), s.K.clone()
    cache.append(s.batch(), s.k, s.v)
    _written(s, K0, [0, 1, 2, 3])
    pos = _ints([3, 4, 5, 6])
    q = cache.append(s.batch(), s.k, s.v, rope=binding.Rope(64), positions=pos, q=s.q)
    ph.assert_within(q, *ph.norm_rope(s.q, pos, None, ph.freqs(64), 64, False, 0.0))
    assert cache.status() == 0


@pytest.mark.parametrize("G", [40, 100])
def test_append_positions_behind_many_groups(G):
    """More groups than a warp has lanes, some of them empty."""
    from paper_2402_06082_b200 import binding
    B = 120
    edges = sorted((i * i * B // (G * G)) for i in range(G + 1))
    prefix = [5 * i for i in range(G)]
    s = ph.Setting([1] * B, [1 + i % 30 for i in range(B)], 2, 1, 64, FP32, 16, edges, prefix, seed=1)
    cache = s.cache()
    q = cache.append(s.batch(), s.k, s.v, rope=binding.Rope(64), q=s.q)
    pos = torch.tensor([next(prefix[g] for g in range(G) if edges[g] <= b < edges[g + 1]) + b % 30 for b in range(B)])
    ph.assert_within(q, *ph.norm_rope(s.q, pos, None, ph.freqs(64), 64, False, 0.0))
    assert cache.status() == 0


def test_append_positions_beyond_31_bits():
    """The longest prefix and the longest sequence that tables can hold, all in one page."""
    from paper_2402_06082_b200 import binding
    page, most = 1024, 2 ** 21 - 2
    far = most * page
    K, V = (torch.zeros(1, 1, page, 64, device="cuda") for _ in "KV")
    cache, table = binding.PagedCache(K, V), torch.zeros(1, most, dtype=torch.int32, device="cuda")
    batch = binding.PagedBatch(_ints([0, 1]), _ints([far]), table, _ints([0, 1]), _ints([far]), table)
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k = (torch.randn(1, 1, 64, generator=g, device="cuda") for _ in "qk")
    out = cache.append(batch, k, k, rope=binding.Rope(64), q=q)
    assert cache.status() == 0
    pos = torch.tensor([2 * far - 1])
    ph.assert_within(out, *ph.norm_rope(q, pos, None, ph.freqs(64), 64, False, 0.0))
    want, bound = ph.norm_rope(k, pos, None, ph.freqs(64), 64, False, 0.0)
    ph.assert_within(K[0, :, page - 1], want[0], bound[0])
    assert torch.equal(V[0, :, page - 1], k[0])


@pytest.mark.parametrize("edges, tokens, status", [
    ([0, 1, 3, 4], [0, 1, 2, 3], 0), ([-1, 1, 3, 4], [1, 2, 3], 8), ([0, 1, 4, 6], [], 8), ([0, 1, 3, 2 ** 31 - 1], [0, 1, 2], 8),
    ([-2 ** 31, 1, 3, 4], [1, 2, 3], 8), ([-3, -2, -1, 4], [], 8)])
def test_append_edges_outside_the_rows(edges, tokens, status):
    """Edges below 0 or past n set the status also where no row of the call is theirs."""
    s = ph.Setting([1, 2, 1], [40, 30, 20], 4, 2, 64, FP32, 16)
    s.cu_q.copy_(_ints(edges))
    cache, K0, q_out = s.cache(), s.K.clone(), torch.full_like(s.q, 7.0)
    cache.append(s.batch(), s.k, s.v, q=s.q, q_out=q_out)
    assert cache.status() == status
    if edges[1:3] == [1, 3]:
        _written(s, K0, tokens)
        for t in range(4):
            assert bool((q_out[t] == 7).all()) == (t not in tokens)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_new_outputs_of_tokens_left_out(dtype):
    """Without q_out the tokens that are left out are NaN, the others as ever."""
    from paper_2402_06082_b200 import binding
    s = ph.Setting([1, 2, 1], [40, 30, 20], 40, 5, 64, dtype, 16, [0, 1, 3], [32, 32], seed=3)
    rope, cache = binding.Rope(64), s.cache()
    good = cache.append(s.batch(), s.k, s.v, rope=rope, q=s.q)
    assert torch.isfinite(good).all() and cache.status() == 0
    s.groups["prefix_len"][0] = 33
    q = cache.append(s.batch(), s.k, s.v, rope=rope, q=s.q)
    assert torch.isnan(q[0]).all() and torch.equal(q[1:], good[1:]) and cache.status() == 8
    s.groups["prefix_len"][0] = 32
    s.cu_q[3] = 9
    q = cache.append(s.batch(), s.k, s.v, rope=rope, q=s.q)
    assert torch.isnan(q[3]).all() and torch.equal(q[:3], good[:3])
    many = ph.Setting([3000], [3000], 8, 2, 64, dtype, 64, seed=1)  # a warp a token
    many.cu_q[1] = 3001
    assert torch.isnan(many.cache().append(many.batch(), many.k, many.v, q=many.q)).all()


# ---- attention that computes nothing --------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("new", [[1, 2, 1], [40, 300, 7]])
@pytest.mark.parametrize("d, H, Hkv", [(64, 4, 2), (128, 8, 8)])
def test_new_outputs_of_broken_offsets(dtype, new, d, H, Hkv):
    """All NaN, status 8; an output that was given stays as it is."""
    s = ph.Setting(new, [k + 20 for k in new], H, Hkv, d, dtype, 16, [0, 1, 3], [10, 20], seed=3, behind=2)
    cache, batch = s.cache(), s.batch()
    s.cu_q[1] = s.cu[2] + 1
    assert torch.isnan(cache.attend(batch, s.q)).all() and cache.status() == 8
    out = torch.full_like(s.q, 7.0)
    cache.attend(batch, s.q, out=out)
    assert bool((out == 7).all())
    s.cu_q[1] = s.cu[1]
    s.groups["cu_group"][2] = 2
    assert torch.isnan(cache.attend(batch, s.q)).all()


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_more_work_than_can_be_divided(dtype):
    """128 heads of a sequence that is as long as a table can hold (its pages are all the same one): refused on the device."""
    from paper_2402_06082_b200 import binding
    page, most, Hkv = 1024, 2 ** 21 - 2, 128
    K = torch.zeros(1, Hkv, page, 64, dtype=dtype, device="cuda")
    cache = binding.PagedCache(K, K)
    batch = binding.PagedBatch(_ints([0, 1]), _ints([most * page]), torch.zeros(1, most, dtype=torch.int32, device="cuda"))
    q = torch.zeros(1, Hkv, 64, dtype=dtype, device="cuda")
    out = torch.full_like(q, 7.0)
    cache.attend(batch, q, out=out)
    assert bool((out == 7).all()) and cache.status() == 16
    assert torch.isnan(cache.attend(batch, q)).all()
    batch.tensors[0][1] = 2                            # broken offsets as well: these are told
    cache = binding.PagedCache(K, K)
    cache.attend(batch, q, out=out)
    assert cache.status() == 8


# ---- captures and streams -------------------------------------------------------------------------

CAPTURE = """
import sys, torch
sys.path[:0] = [".", "tests"]
import paged_helpers as ph
from paper_2402_06082_b200 import binding
for dtype in (torch.bfloat16, torch.float32):
    for d, first, then in ((64, 1, 4000), (128, 4000, 1)):
        a, b = (ph.Setting([n], [n], 4, 4, d, dtype, 64, seed=n) for n in (first, then))
        rope = binding.Rope(d)
        for paged in (False, True):
            calls = []
            for s in (a, b):
                pos = torch.arange(s.n, dtype=torch.int32, device="cuda")
                cache, batch = s.cache(), s.batch()
                if paged: calls.append(lambda s=s, cache=cache, batch=batch: cache.append(batch, s.k, s.v, rope=rope, q=s.q))
                else: calls.append(lambda s=s, pos=pos: binding.qk_norm_rope(s.q, s.k, pos, rope)[0])
            calls[0]()
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                q = calls[1]()
            graph.replay()
            ph.assert_within(q, *ph.norm_rope(b.q, torch.arange(then), None, ph.freqs(d), d, False, 0.0))
print("captured")
"""


def test_capture_of_rotations_of_sizes_that_have_not_run():
    """One call of an operator, type and d loads what calls of other sizes need."""
    r = subprocess.run([sys.executable, "-c", CAPTURE], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured" in r.stdout, r.stderr[-2000:]


def test_causal_without_a_truth_value():
    s = ph.Setting([1], [5], 4, 2, 64, BF16)
    cache, batch = s.cache(), s.batch()
    with pytest.raises(ValueError, match="causal"):
        cache.attend(batch, s.q, causal=torch.ones(2))
    assert torch.equal(cache.attend(batch, s.q, causal=torch.ones(1)), cache.attend(batch, s.q, causal=1))


def test_status_of_a_cache_that_a_busy_stream_made():
    """A call on another stream right after the cache was made: the bit that it sets stays."""
    s = ph.Setting([1], [5], 4, 2, 64, BF16)
    s.table[0, 0] = -1
    batch = s.batch()
    s.cache().append(batch, s.k, s.v)
    torch.cuda.synchronize()
    busy, other = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(busy):
        torch.cuda._sleep(200_000_000)                 # a tenth of a second
        cache = s.cache()
    with torch.cuda.stream(other):
        cache.append(batch, s.k, s.v)
    assert cache.status() == 8


def test_a_cache_made_in_a_capture():
    s = ph.Setting([1, 2], [40, 30], 4, 2, 64, BF16)
    batch = s.batch()
    s.cache().attend(batch, s.q)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache = s.cache()
        out = cache.attend(batch, s.q, scale=0.2)
    graph.replay()
    ph.assert_within(out, *s.want(0.2))
    assert cache.status() == 0
