"""GPU tests of the head norms with rotation, the paged append and the paged attention, against 64-bit statements."""
import math
import os
import random
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import paged_helpers as ph  # noqa: E402

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32


def _randn(*shape, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


# ---- norms and rotation ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("d, rot, interleaved", [(128, 128, False), (128, 128, True), (128, 48, False), (64, 64, True), (64, 16, False), (64, 32, True)])
@pytest.mark.parametrize("n, H, Hkv", [(1, 32, 8), (3, 5, 2), (33, 1, 1), (700, 6, 6)])
def test_norm_rope(dtype, d, rot, interleaved, n, H, Hkv):
    from paper_2402_06082_b200 import binding
    qkv = _randn(n, (H + 2 * Hkv) * d, dtype=dtype, seed=n)
    q, k = qkv[:, : H * d].view(n, H, d), qkv[:, H * d: (H + Hkv) * d].view(n, Hkv, d)
    wq, wk = _randn(d, dtype=dtype, seed=1), _randn(d, dtype=dtype, seed=2)
    pos = torch.randint(0, 1 << 20, (n,), device="cuda", dtype=torch.int32, generator=torch.Generator(device="cuda").manual_seed(3))
    rope = binding.Rope(d, rotary_dim=rot, interleaved=interleaved)
    before = qkv.clone()
    for weights in ((wq, wk), (None, wk)):
        got = binding.qk_norm_rope(q, k, pos, rope, wq=weights[0], wk=weights[1], eps=1e-5)
        for x, w, y in zip((q, k), weights, got):
            want, bound = ph.norm_rope(x, pos, w, ph.freqs(rot), rot, interleaved, 1e-5)
            ph.assert_within(y, want, bound)
    assert torch.equal(qkv, before)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_norm_rope_forms(dtype):
    """One tensor alone, no rotation, no norm at all, far and negative positions, other frequencies, in place, other layouts."""
    from paper_2402_06082_b200 import binding
    n, H, d = 37, 3, 128
    x, w = _randn(n, H, d, dtype=dtype, seed=1), _randn(d, dtype=dtype, seed=2)
    x[5] = 0                                                       # a head of zeros: eps alone under the root
    y, none = binding.qk_norm_rope(x, None, wq=w)
    assert none is None
    ph.assert_within(y, *ph.norm_rope(x, None, w, None, 0, False, 1e-6))
    none, y = binding.qk_norm_rope(None, x)
    assert none is None and torch.equal(x, y)
    f = [0.37 ** i for i in range(64)]
    pos = torch.tensor([2 ** 31 - 1, -1, -2 ** 31] + list(range(n - 3)), dtype=torch.int32, device="cuda")
    rope = binding.Rope(d, inv_freq=f)
    want, bound = ph.norm_rope(x, pos, None, f, d, False, 0.0)
    _, y = binding.qk_norm_rope(None, x, pos, rope)
    ph.assert_within(y, want, bound)
    packed = torch.full((H, n, d), math.nan, dtype=dtype, device="cuda")          # the layout that the prefill calls take
    binding.qk_norm_rope(x, None, pos, rope, q_out=packed.transpose(0, 1))
    assert torch.equal(packed.transpose(0, 1), y)
    z = x.clone()
    binding.qk_norm_rope(z, None, pos, rope, q_out=z)
    assert torch.equal(z, y)
    e, _ = binding.qk_norm_rope(x[:0], None, pos[:0], rope)
    assert e.shape == (0, H, d)
    bad = x.clone()
    bad[0, 0, 0] = math.inf
    y, _ = binding.qk_norm_rope(bad, None, wq=w)
    assert torch.isnan(y[0, 0, 0]) and torch.isfinite(y[1:]).all() and torch.isfinite(y[0, 1:]).all()


# ---- append ---------------------------------------------------------------------------------------

APPENDS = [  # new, own, page, edges, prefix, behind
    ([1], [1], 16, [], [], 0),
    ([1, 1, 1], [16, 17, 1], 16, [], [], 0),
    ([0, 5, 40, 0, 1], [3, 5, 64, 0, 129], 32, [], [], 4),
    ([3, 1, 2], [10, 33, 2], 16, [0, 1, 3], [7, 48], 1),
    ([300, 7], [700, 7], 128, [0, 2], [1000], 0),
]


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("d, H, Hkv", [(128, 8, 2), (64, 3, 3)])
@pytest.mark.parametrize("case", APPENDS)
@pytest.mark.parametrize("norm", [False, True])
def test_append(dtype, d, H, Hkv, case, norm):
    from paper_2402_06082_b200 import binding
    new, own, page, edges, prefix, behind = case
    s = ph.Setting(new, own, H, Hkv, d, dtype, page, edges, prefix, seed=5, behind=behind, rows_first=norm)
    rope = binding.Rope(d)
    wq, wk = (_randn(d, dtype=dtype, seed=1), _randn(d, dtype=dtype, seed=2)) if norm else (None, None)
    K0, V0 = s.K.clone(), s.V.clone()
    q_out = torch.full_like(s.q, 7.0)
    cache = s.cache()
    got = cache.append(s.batch(), s.k, s.v, rope=rope, q=s.q, wq=wq, wk=wk, q_out=q_out)
    assert got is q_out and cache.status() == 0
    pos = []
    for b in range(len(new)):
        P = sum(p for i, p in enumerate(prefix) if edges[i] <= b < edges[i + 1])
        pos += [P + own[b] - new[b] + i for i in range(new[b])]
    m = s.cu[-1]
    pos = torch.tensor(pos, dtype=torch.int32)
    ph.assert_within(q_out[:m], *ph.norm_rope(s.q[:m], pos, wq, ph.freqs(d), d, False, 1e-6))
    assert bool((q_out[m:] == 7).all())                            # rows behind the last sequence
    want, bound = ph.norm_rope(s.k[:m], pos, wk, ph.freqs(d), d, False, 1e-6)
    touched = torch.zeros(K0.shape[0], page, dtype=torch.bool)
    for b in range(len(new)):
        for i in range(new[b]):
            j, t = own[b] - new[b] + i, s.cu[b] + i
            p, r = int(s.table[b, j // page]), j % page
            touched[p, r] = True
            ph.assert_within(s.K[p, :, r], want[t], bound[t])
            assert torch.equal(s.V[p, :, r], s.v[t])
    keep = ~touched.cuda()
    for x, x0 in ((s.K, K0), (s.V, V0)):                           # nothing else has changed
        a, b = x.transpose(1, 2)[keep], x0.transpose(1, 2)[keep]
        assert torch.equal(torch.nan_to_num(a, nan=9.0), torch.nan_to_num(b, nan=9.0))


def test_append_without_queries_given_positions():
    from paper_2402_06082_b200 import binding
    s = ph.Setting([2, 1], [5, 20], 4, 2, 64, BF16)
    pos = torch.tensor([100000, 3, 77], dtype=torch.int32, device="cuda")
    assert s.cache().append(s.batch(), s.k, s.v, rope=binding.Rope(64, rotary_dim=32, interleaved=True), positions=pos) is None
    want, bound = ph.norm_rope(s.k, pos, None, ph.freqs(32), 32, True, 0.0)
    ph.assert_within(s.K[int(s.table[1, 1]), :, 3], want[2], bound[2])
    s.cache().append(s.batch(), s.k, s.v)                          # neither norm nor rotation: bits as they are
    assert torch.equal(s.K[int(s.table[0, 0]), :, 3:5].transpose(0, 1), s.k[:2])


def test_append_leaves_bad_pages_alone():
    s = ph.Setting([1, 1, 1, 3], [5, 20, 17, 2], 4, 2, 64, FP32, behind=2)
    s.table[1, 1] = s.K.shape[0]                                   # outside the pool
    s.table[2, 1] = -1
    s.table[0, 0] = 0
    K0 = s.K.clone()
    cache = s.cache()
    cache.append(s.batch(), s.k, s.v)
    assert cache.status() == 8
    changed = (torch.nan_to_num(s.K) != torch.nan_to_num(K0)).any(-1).any(1)       # [pages, page]
    want = torch.zeros_like(changed)
    want[0, 4] = True
    want[int(s.table[3, 0]), :2] = True                            # the first of three tokens has no place in a length of 2
    assert torch.equal(changed, want)


@pytest.mark.parametrize("what", ["falls", "passes n", "starts late"])
def test_append_broken_offsets(what):
    """Rows that two sequences claim, or that there are not, are written for nobody; rows before cu_q[0] belong to nobody."""
    s = ph.Setting([1, 2, 1], [40, 30, 20], 4, 2, 64, FP32, 16)
    cache, K0 = s.cache(), s.K.clone()
    q_out = torch.full_like(s.q, 7.0)
    if what == "falls":
        s.cu_q.copy_(torch.tensor([0, 3, 1, 4], dtype=torch.int32))
        ours, tokens, status = [], [0, 3], 8          # rows 0 and 3 still have one sequence: [0, 3) and [1, 4) by the edges
    elif what == "passes n":
        s.cu_q[3] = 9
        ours, tokens, status = [(0, 39), (1, 28), (1, 29)], [0, 1, 2], 8
    else:
        s.cu_q.copy_(torch.tensor([1, 1, 3, 4], dtype=torch.int32))
        ours, tokens, status = [(1, 28), (1, 29), (2, 19)], [1, 2, 3], 0
    cache.append(s.batch(), s.k, s.v, q=s.q, q_out=q_out)
    assert cache.status() == status
    if what != "falls":
        changed = (torch.nan_to_num(s.K) != torch.nan_to_num(K0)).any(-1).any(1)
        want = torch.zeros_like(changed)
        for b, j in ours:
            want[int(s.table[b, j // 16]), j % 16] = True
        assert torch.equal(changed, want)
    for i in range(4):
        assert bool((q_out[i] == 7).all()) == (i not in tokens)


# ---- attention ------------------------------------------------------------------------------------

ATTENDS = {  # new, own, edges, prefix, behind
    "one of one": ([1], [1], [], [], 0),
    "steps": ([1] * 7, [1, 15, 16, 17, 128, 129, 700], [], [], 0),
    "empty ones": ([1, 0, 2, 1], [0, 40, 1, 64], [], [], 3),
    "shared": ([1] * 9, [1, 2, 30, 64, 65, 127, 200, 5, 1], [0, 9], [300], 0),
    "no own tokens": ([1, 1, 2], [0, 0, 0], [0, 3], [129], 1),
    "groups": ([1, 3, 1, 1, 2, 1, 40], [9, 3, 70, 1, 2, 300, 41], [0, 2, 2, 6, 7], [64, 50, 1000, 31], 2),
    "empty prefix": ([1, 2, 1], [5, 9, 0], [0, 2, 3], [0, 0], 0),
    "drafts": ([8, 1, 5, 7, 3], [8, 500, 77, 7, 130], [0, 5], [777], 0),
    "chunks": ([150, 257, 64], [150, 600, 64], [0, 3], [200], 5),
    "chunk alone": ([513], [1025], [], [], 0),
    "one long": ([1], [9001], [], [], 0),
    "many rows, one prefix": ([1] * 70, [1 + 3 * i for i in range(70)], [0, 70], [513], 0),
    "more new than own": ([5, 1], [2, 3], [0, 2], [40], 0),
}


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("d, H, Hkv, page", [(128, 8, 2, 16), (64, 4, 4, 64), (128, 8, 1, 128), (64, 2, 1, 1024)])
@pytest.mark.parametrize("name", list(ATTENDS))
def test_attend(dtype, d, H, Hkv, page, name):
    new, own, edges, prefix, behind = ATTENDS[name]
    s = ph.Setting(new, own, H, Hkv, d, dtype, page, edges, prefix, seed=len(name), behind=behind, rows_first=page == 64)
    cache, batch = s.cache(), s.batch()
    for causal in (True, False):
        out = torch.full_like(s.q, 7.0)
        assert cache.attend(batch, s.q, scale=1.5 * d ** -0.5, causal=causal, out=out) is out
        want, bound = s.want(1.5 * d ** -0.5, causal)
        m = s.cu[-1]
        ph.assert_within(out[:m], want[:m], bound[:m], "%s causal %s" % (name, causal))
        assert bool((out[m:] == 7).all())
        again = torch.full_like(s.q, 7.0)
        cache.attend(batch, s.q, scale=1.5 * d ** -0.5, causal=causal, out=again)
        assert torch.equal(out, again)
    assert cache.status() == 0


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_attend_large_scores(dtype):
    """Scores of some hundreds, rising and falling along the cache: the running maximum moves by more than any exponent holds."""
    s = ph.Setting([1, 3], [1500, 1400], 4, 2, 128, dtype, 16, [0, 2], [900], seed=3)
    ramp = torch.linspace(-6, 6, s.K.shape[0], device="cuda")[:, None, None, None]
    s.K.mul_(ramp.to(dtype))
    out = s.cache().attend(s.batch(), s.q, scale=2.0)
    want, bound = s.want(2.0)
    ph.assert_within(out, want, bound)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_attend_strided_queries(dtype):
    s = ph.Setting([1, 2, 1], [40, 300, 2], 8, 4, 64, dtype, 16, seed=3)
    wide = torch.full((s.n, 8 + 8, 64), math.nan, dtype=dtype, device="cuda")
    wide[:, :8] = s.q
    out = torch.full((8, s.n, 64), math.nan, dtype=dtype, device="cuda")
    s.cache().attend(s.batch(), wide[:, :8], scale=0.125, out=out.transpose(0, 1))
    want, bound = s.want(0.125)
    ph.assert_within(out.transpose(0, 1), want, bound)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("page", [16, 64])
def test_pools_that_are_halves_of_one_tensor(dtype, page):
    """K and V as [:, 0] and [:, 1] of [pages, 2, Hkv, page, d], and one head of several."""
    from paper_2402_06082_b200 import binding
    s = ph.Setting([1, 3], [200, 90], 4, 2, 128, dtype, page, [0, 2], [70], seed=6)
    both = torch.stack((s.K, s.V), 1)
    cache = binding.PagedCache(both[:, 0], both[:, 1])
    want, bound = s.want(0.1)
    ph.assert_within(cache.attend(s.batch(), s.q, scale=0.1), want, bound)
    one = binding.PagedCache(both[:, 0, 1:], both[:, 1, 1:])           # the second KV head and its two query heads
    ph.assert_within(one.attend(s.batch(), s.q[:, 2:], scale=0.1), want[:, 2:], bound[:, 2:])
    cache.append(s.batch(), s.k, s.v)
    assert torch.equal(both[int(s.table[0, 199 // page]), 0, :, 199 % page], s.k[0])
    assert torch.equal(both[int(s.table[1, 89 // page]), 1, :, 89 % page], s.v[3])


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_attend_bad_pages_and_lengths(dtype):
    """A page outside the pool or a length beyond its table: NaN for the rows that needed it, the others as ever."""
    s = ph.Setting([1, 1, 2, 1, 1, 1], [300, 20, 200, 5, 9, 40], 8, 2, 128, dtype, 16, [0, 5, 6], [100, 30], seed=3)
    want, bound = s.want(0.1)
    s.table[0, 3] = s.K.shape[0]
    s.table[2, 0] = -7
    s.lengths[3] = 10 ** 6
    s.lengths[4] = -1
    for b in (0, 2, 3, 4):
        want[s.cu[b]:s.cu[b + 1]] = math.nan
    cache = s.cache()
    ph.assert_within(cache.attend(s.batch(), s.q, scale=0.1), want, bound)
    assert cache.status() == 8
    s.ptable[1, 0] = 10 ** 9                                       # the second group's prefix
    want[s.cu[5]:] = math.nan
    ph.assert_within(cache.attend(s.batch(), s.q, scale=0.1), want, bound)
    s.ptable[0, 4] = -1                                            # the first one's, which is packed over its sequences
    want[:] = math.nan
    ph.assert_within(cache.attend(s.batch(), s.q, scale=0.1), want, bound)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H, Hkv, B, most_new, most_own", [
    (8, 2, 74, 1, 700), (8, 2, 80, 8, 1300), (32, 4, 37, 12, 600), (4, 4, 40, 40, 300), (16, 2, 150, 3, 140), (8, 8, 19, 2, 3000), (1, 1, 148, 33, 257), (8, 1, 150, 45, 400)])
def test_attend_wide_batches(dtype, d, H, Hkv, B, most_new, most_own):
    """Without prefixes and with at least as many sequences and KV heads as blocks; empty ones and more new than own among them."""
    g = torch.Generator().manual_seed(B + most_own)
    own = torch.randint(0, most_own + 1, (B,), generator=g).tolist()
    new = torch.randint(0, most_new + 1, (B,), generator=g).tolist()
    own[B // 3] = most_own
    new[B // 3] = most_new
    s = ph.Setting(new, own, H, Hkv, d, dtype, 64 if d == 64 else 16, seed=B, behind=2)
    cache, out = s.cache(), torch.full_like(s.q, 7.0)
    for causal in (True, False):
        cache.attend(s.batch(), s.q, scale=0.13, causal=causal, out=out)
        want, bound = s.want(0.13, causal)
        ph.assert_within(out[:s.cu[-1]], want[:s.cu[-1]], bound[:s.cu[-1]])
        assert bool((out[s.cu[-1]:] == 7).all())
    assert cache.status() == 0
    again = cache.attend(s.batch(), s.q, scale=0.13, causal=False)
    assert torch.equal(again[:s.cu[-1]], out[:s.cu[-1]])
    if s.cu[B // 3 + 1] > s.cu[B // 3]:
        s.table[B // 3, 0] = -3                        # its first page: all of its rows need it
        want[s.cu[B // 3]:s.cu[B // 3 + 1]] = math.nan
        ph.assert_within(cache.attend(s.batch(), s.q, scale=0.13, causal=False)[:s.cu[-1]], want[:s.cu[-1]], bound[:s.cu[-1]])
        assert cache.status() == 8


CAPTURE = """
import sys, torch
sys.path.insert(0, "tests")
import paged_helpers as ph
for dtype in (torch.bfloat16, torch.float32):
    one = ph.Setting([1], [40], 4, 2, 64, dtype)
    one.cache().attend(one.batch(), one.q)
    for new, own in (([1] * 80, [100] * 80), ([50, 60], [70, 80])):
        s = ph.Setting(new, own, 4, 2, 64, dtype)
        cache, batch, out = s.cache(), s.batch(), torch.zeros_like(s.q)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cache.attend(batch, s.q, scale=0.2, out=out)
        graph.replay()
        ph.assert_within(out, *s.want(0.2))
print("captured")
"""


def test_capture_of_sizes_that_have_not_run():
    """One call of a type and d loads what calls of other sizes need."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", CAPTURE], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured" in r.stdout, r.stderr[-2000:]


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("what", ["falls", "passes n", "negative", "groups end early", "groups fall"])
def test_attend_broken_offsets(dtype, what):
    s = ph.Setting([1, 2, 1], [40, 30, 20], 4, 2, 64, dtype, 16, [0, 1, 3], [10, 20], seed=3)
    if what == "falls":
        s.cu_q[1] = 4
    elif what == "passes n":
        s.cu_q[3] = 5
    elif what == "negative":
        s.cu_q[0] = -1
    elif what == "groups end early":
        s.groups["cu_group"][2] = 2
    else:
        s.groups["cu_group"][1] = 5
    out = torch.full_like(s.q, 7.0)
    cache = s.cache()
    cache.attend(s.batch(), s.q, out=out)
    assert cache.status() == 8 and bool((out == 7).all())


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("heads", [(4, 2), (8, 1)])
@pytest.mark.parametrize("edges", [[0, 1, 3, 2**31 - 1], [0, 2**31 - 1, 3, 4], [0, 1, -2**31, 4], [-2**31, 1, 3, 2**31 - 1], [0, 2**28, 2**29, 2**30]])
@pytest.mark.parametrize("groups", [[0, 3], [0, 1, 3]])
def test_attend_offsets_far_out(dtype, heads, edges, groups):
    """Offsets that would make rows by the billion of a group or a sequence: refused like any that pass n."""
    s = ph.Setting([1, 2, 1], [40, 30, 20], *heads, 64, dtype, 16, groups, [10] * (len(groups) - 1), seed=3)
    s.cu_q.copy_(torch.tensor(edges, dtype=torch.int32))
    out = torch.full_like(s.q, 7.0)
    cache = s.cache()
    cache.attend(s.batch(), s.q, out=out)
    assert cache.status() == 8 and bool((out == 7).all())


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_attend_in_a_graph_with_lengths_that_grow(dtype):
    from paper_2402_06082_b200 import binding
    s = ph.Setting([1, 1, 1], [200, 90, 130], 8, 2, 128, dtype, 16, [0, 3], [260], seed=3)
    full = list(s.own)
    rope = binding.Rope(128)
    cache, batch = s.cache(), s.batch()
    cache.append(batch, s.k, s.v, rope=rope, q=s.q)
    cache.attend(batch, s.q)                                       # loads the kernels before the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q = cache.append(batch, s.k, s.v, rope=rope, q=s.q)
        out = cache.attend(batch, q, scale=0.1)
    for step in range(3):
        s.own = [x - 40 + 20 * step for x in full]
        s.lengths.copy_(torch.tensor(s.own, dtype=torch.int32))
        s.k.copy_(_randn(*s.k.shape, dtype=dtype, seed=step))
        s.q.copy_(_randn(*s.q.shape, dtype=dtype, seed=9 + step))
        graph.replay()
        torch.cuda.synchronize()
        pos = torch.tensor([260 + x - 1 for x in s.own], dtype=torch.int32)
        ph.assert_within(q, *ph.norm_rope(s.q, pos, None, ph.freqs(128), 128, False, 0.0))
        s_q, s.q = s.q, q
        ph.assert_within(out, *s.want(0.1))
        s.q = s_q
    assert cache.status() == 0


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_attend_on_two_streams_at_once(dtype):
    a = ph.Setting([1] * 16, [3000] * 16, 8, 2, 128, dtype, 16, [0, 16], [5000], seed=1)
    b = ph.Setting([40, 9], [900, 2000], 8, 2, 128, dtype, 16, seed=2)
    alone = [x.cache().attend(x.batch(), x.q, scale=0.1) for x in (a, b)]
    torch.cuda.synchronize()
    streams, sets = [torch.cuda.Stream(), torch.cuda.Stream()], [(x.cache(), x.batch(), x.q) for x in (a, b)]
    outs = [[], []]
    for _ in range(20):
        for i, (cache, batch, q) in enumerate(sets):
            with torch.cuda.stream(streams[i]):
                outs[i].append(cache.attend(batch, q, scale=0.1))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, alone[i]) for x in outs[i])


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_attend_two_graphs_at_once(dtype):
    s = ph.Setting([1] * 12, [2000 + 31 * i for i in range(12)], 8, 2, 128, dtype, 16, [0, 12], [3000], seed=1)
    cache, batch = s.cache(), s.batch()
    alone = cache.attend(batch, s.q, scale=0.1)
    torch.cuda.synchronize()
    graphs, outs, streams = [], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(cache.attend(batch, s.q, scale=0.1))
        graphs.append(g)
    for _ in range(10):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, alone) for o in outs)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_as_many_sequences_as_there_may_be(dtype):
    """1000 sequences in 24 groups, some of them empty, and one more than there may be."""
    from paper_2402_06082_b200 import binding
    B, G = 1000, 24
    new = [i % 3 for i in range(B)]
    own = [new[i] + (7 * i) % 40 for i in range(B)]
    edges = sorted((i * i * B // (G * G)) for i in range(G + 1))
    s = ph.Setting(new, own, 2, 1, 64, dtype, 16, edges, [11 * i for i in range(G)], seed=1, behind=3)
    cache = s.cache()
    out = cache.attend(s.batch(), s.q, scale=0.2)
    want, bound = s.want(0.2)
    m = s.cu[-1]
    ph.assert_within(out[:m], want[:m], bound[:m])
    assert cache.status() == 0
    more = ph.Setting([1] * 1025, [1] * 1025, 2, 1, 64, dtype, 16)
    with pytest.raises(binding.SubgenError):
        more.cache().attend(more.batch(), more.q)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_sequences_that_read_the_same_pages(dtype):
    s = ph.Setting([2, 2, 1], [90, 90, 300], 4, 2, 128, dtype, 16, seed=5)
    s.table[1] = s.table[0]
    s.q[2:4] = s.q[0:2]
    out = s.cache().attend(s.batch(), s.q, scale=0.1)
    want, bound = s.want(0.1)
    ph.assert_within(out, want, bound)
    assert torch.equal(out[0:2], out[2:4])


def random_setting(seed):
    r = random.Random(seed)
    dtype, d, page = r.choice([BF16, BF16, FP32]), r.choice([64, 128]), r.choice([16, 32, 64, 128, 256, 1024])
    G, Hkv, B = r.choice([1, 2, 4, 8]), r.choice([1, 2, 3, 5]), r.randint(1, 20)
    top, long = r.choice([1, 1, 3, 9, 70, 300]), r.choice([1, 20, 130, 600, 3000])
    new = [r.choice([0, 1, r.randint(0, top)]) for _ in range(B)]
    new[r.randrange(B)] += 1
    own = [r.choice([k, k + r.randint(0, long), max(0, k - 1)]) for k in new]
    edges, prefix = [], []
    if r.random() < 0.7:
        g = r.randint(1, min(B, 4))
        edges = [0] + sorted(r.randint(0, B) for _ in range(g - 1)) + [B]
        prefix = [r.choice([0, r.randint(0, 40), r.randint(0, 2500)]) for _ in range(g)]
    return ph.Setting(new, own, G * Hkv, Hkv, d, dtype, page, edges, prefix, seed=seed, behind=r.choice([0, 0, 5]), rows_first=r.random() < 0.3), r


@pytest.mark.parametrize("seed", range(40))
def test_attend_random(seed):
    s, r = random_setting(seed)
    scale, causal, m = r.choice([0.05, s.d ** -0.5, 0.7]), r.random() < 0.8, s.cu[-1]
    cache = s.cache()
    out = cache.attend(s.batch(), s.q, scale=scale, causal=causal)
    want, bound = s.want(scale, causal)
    ph.assert_within(out[:m], want[:m], bound[:m], "seed %d" % seed)
    assert cache.status() == 0


def test_nothing_at_all():
    from paper_2402_06082_b200 import binding
    s = ph.Setting([1], [5], 4, 2, 64, BF16)
    none = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")  # noqa: E731
    empty = binding.PagedBatch(none(1), none(0), none(0, 4))
    cache = s.cache()
    assert cache.attend(empty, s.q).shape == s.q.shape and cache.append(empty, s.k, s.v) is None
    assert cache.attend(s.batch(), s.q[:0]).shape == (0, 4, 64) and cache.append(s.batch(), s.k[:0], s.v[:0], q=s.q[:0]).shape == (0, 4, 64)
    assert cache.status() == 0


def test_offsets_beyond_32_bits():
    """Pages that lie more than 2^32 bytes (and 2^31 elements) into the pool."""
    from paper_2402_06082_b200 import binding
    pages, Hkv, page, d = 70000, 4, 64, 128                        # 2.3e9 elements, 4.6 GB each
    K = torch.empty(pages, Hkv, page, d, dtype=BF16, device="cuda")
    V = torch.empty_like(K)
    s = ph.Setting([1, 3], [100, 70], 8, 4, d, BF16, page, seed=4)
    far = torch.tensor([69999, 3, 65537, 69998], dtype=torch.int32, device="cuda").view(2, 2)
    for i in range(2):
        for j in range(2):
            K[int(far[i, j])], V[int(far[i, j])] = s.K[int(s.table[i, j])], s.V[int(s.table[i, j])]
    want, bound = s.want(0.1)
    cache = binding.PagedCache(K, V)
    batch = binding.PagedBatch(s.cu_q, s.lengths, far)
    ph.assert_within(cache.attend(batch, s.q, scale=0.1), want, bound)
    cache.append(batch, s.k, s.v)
    assert torch.equal(K[69998, :, 70 - 64 - 3: 70 - 64].transpose(0, 1), s.k[1:4]) and torch.equal(V[3, :, 35], s.v[0])


# ---- a run of them together -----------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_a_prompt_and_steps_against_the_other_caches(dtype):
    """A shared prompt goes into the pool once, three sequences go on from it; the exact cache and SubGen (window over everything,
    so that its estimator is exact) get the same normed and rotated keys."""
    from paper_2402_06082_b200 import binding
    B, H, Hkv, d, P, steps, page = 3, 8, 2, 128, 150, 20, 16
    rope = binding.Rope(d, base=500000.0)
    wq, wk = (0.08 * (1 + _randn(d, dtype=dtype, seed=i).abs()) for i in (1, 2))
    ex = binding.ExactAttention(B, H, d, P + steps, Hkv=Hkv, dtype=dtype)
    sg = binding.SubGen(B, H, d, 0.5, 4, 16, P + steps, Hkv=Hkv, dtype=dtype, m_max=64)
    pages = 10 + B * 2
    K, V = (torch.full((pages, Hkv, page, d), math.nan, dtype=dtype, device="cuda") for _ in "KV")
    cache = binding.PagedCache(K, V)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    prefix = torch.arange(10, dtype=torch.int32, device="cuda").view(1, 10)
    qkv = _randn(P, (H + 2 * Hkv) * d, dtype=dtype, seed=3)
    cut = lambda x: (x[:, : H * d].unflatten(1, (H, d)), x[:, H * d: -Hkv * d].unflatten(1, (Hkv, d)), x[:, -Hkv * d:].unflatten(1, (Hkv, d)))  # noqa: E731
    q, k, v = cut(qkv)
    prompt = binding.PagedBatch(ints([0, P]), ints([P]), prefix)
    q1 = cache.append(prompt, k, v, rope=rope, wk=wk, q=q, wq=wq)
    assert torch.isfinite(cache.attend(prompt, q1)).all()
    q2, k2 = binding.qk_norm_rope(q, k, torch.arange(P, dtype=torch.int32, device="cuda"), rope, wq=wq, wk=wk)
    assert torch.equal(q1, q2)
    Kp, Vp = (x.transpose(0, 1)[None].expand(B, Hkv, P, d).contiguous() for x in (k2, v))
    ex.append(Kp, Vp)
    sg.prefill(Kp, Vp)
    lengths = ints([0] * B)
    table = (10 + torch.arange(B * 2, dtype=torch.int32, device="cuda")).view(B, 2)
    batch = binding.PagedBatch(ints(range(B + 1)), lengths, table, ints([0, B]), ints([P]), prefix)
    for i in range(steps):
        q, k, v = cut(_randn(B, (H + 2 * Hkv) * d, dtype=dtype, seed=100 + i))
        lengths += 1
        qr = cache.append(batch, k, v, rope=rope, wk=wk, q=q, wq=wq)
        out = cache.attend(batch, qr)
        _, kr = binding.qk_norm_rope(None, k, ints([P + i] * B), rope, wk=wk)
        vc = v.contiguous()
        tol = 1e-4 if dtype == FP32 else 2e-2                      # the other paths' own tolerance
        for other in (ex.step(qr, kr, vc), sg.step(qr, kr, vc)):
            assert float((out.double() - other.double()).norm(dim=-1).max() / other.double().norm(dim=-1).min()) <= 2 * tol
    assert cache.status() == 0 and sg.status() == 0


def test_other_device_and_type_are_refused():
    from paper_2402_06082_b200 import binding
    s = ph.Setting([1], [5], 4, 2, 64, BF16)
    cache, batch = s.cache(), s.batch()
    with pytest.raises(ValueError):
        cache.attend(batch, s.q.float())
    with pytest.raises(ValueError):
        cache.attend(batch, s.q.cpu())
    with pytest.raises(ValueError):
        cache.append(batch, s.k, s.v[:, :1])
    with pytest.raises(ValueError):
        cache.append(batch, s.k, s.v, rope=binding.Rope(128))
    with pytest.raises(ValueError):
        binding.PagedBatch(s.cu_q.long(), s.lengths, s.table)
    with pytest.raises(ValueError):
        binding.PagedBatch(s.cu_q, s.lengths, s.table, s.cu_q)
    with pytest.raises(binding.SubgenError):
        cache.attend(batch, s.q, scale=-1.0)
    with pytest.raises(binding.SubgenError):
        cache.attend(batch, s.q[:, :3])
    with pytest.raises(binding.SubgenError):
        cache.attend(batch, s.q, out=s.q)
