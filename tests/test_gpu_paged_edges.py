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
