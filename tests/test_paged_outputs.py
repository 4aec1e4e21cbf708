"""Outputs that the head norms, the paged append and the paged attention refuse, on the host: nothing is launched."""
import itertools

import pytest

from paper_2402_06082_b200 import binding

P = 1 << 20                                           # aligned addresses that nothing follows: the calls are refused first
D = 64


def _heads(p, ts, hs):
    return binding.Heads(p * P, ts, hs)


def _rotate(q, q_out, k=None, k_out=None, n=4, H=4, Hkv=2):
    none = binding.Heads(None, 0, 0)
    args = binding.QkArgs(q=q, q_out=q_out, k=k or none, k_out=k_out or none, n=n, H=H, Hkv=Hkv, d=D, dtype=0, eps=0.0)
    return binding.load().subgen_qk_norm_rope(args, None)


def _append(q, q_out, k=4, v=5, n=4, H=4):
    args = binding.QkArgs(q=q, q_out=q_out, k=_heads(k, 2 * D, D), v=_heads(v, 2 * D, D), n=n, H=H, eps=0.0)
    return binding.load().subgen_paged_append(_pages(), _batch(), args, None)


def _attend(q, out, n=4, H=4):
    return binding.load().subgen_paged_attend(_pages(), _batch(), binding.AttendArgs(q, out, 8 * P, 1 << 40, n, H, 1.0, 1), None)


def _pages():
    return binding.PagesDesc(K=6 * P, V=7 * P, page_stride=2 * 16 * D, head_stride=16 * D, row_stride=D, pages=10, page=16, Hkv=2, d=D, dtype=0)


def _batch():
    return binding.BatchDesc(B=2, cu_q=9 * P, lengths=9 * P, table=9 * P, table_stride=4, groups=0)


def _said():
    return binding.load().subgen_last_error().decode()


@pytest.mark.parametrize("call", [_rotate, _append, _attend])
@pytest.mark.parametrize("ts, hs", [(4 * D, D // 2), (D // 2, 4 * D), (D, D), (2 * D, D), (3 * D, D), (D, 3 * D), (2 * D, 3 * D), (4 * D - 4, D)])
def test_rows_that_overlap(call, ts, hs):
    assert call(_heads(1, 4 * D, D), _heads(2, ts, hs)) == -1 and "q_out" in _said() or "out" in _said()
    assert "rows overlap" in _said()


def _overlaps(ts, hs, n, H):
    at = sorted(t * ts + h * hs for t in range(n) for h in range(H))
    return any(b - a < D for a, b in zip(at, at[1:]))


def test_which_rows_overlap():
    """Against all rows' places. What is not refused for them is refused for another reason behind it: nothing is launched."""
    steps = [16, 48, 64, 68, 96, 128, 132, 192, 200, 256, 260, 320, 448, 640]
    for ts, hs, n, H in itertools.product(steps, steps, (1, 2, 3, 5), (1, 2, 3, 4)):
        rc = _rotate(_heads(1, 4 * D, D), _heads(2, ts, hs), k=_heads(3, 2 * D, D), k_out=_heads(1, 2 * D, D), n=n, H=H)
        real_ts, real_hs = (H * D if n == 1 else ts), (D if H == 1 else hs)
        assert rc == -1 and ("rows overlap" in _said()) == _overlaps(real_ts, real_hs, n, H), (ts, hs, n, H, _said())


@pytest.mark.parametrize("call", [_rotate, _append])
def test_an_input_in_another_layout(call):
    assert call(_heads(1, 4 * D, D), _heads(1, 8 * D, D)) == -1 and "strides" in _said()
    assert call(_heads(1, 4 * D, D), _heads(1, D, 4 * D)) == -1 and "strides" in _said()


def test_another_tensor_of_the_call():
    q, k = _heads(1, 4 * D, D), _heads(3, 2 * D, D)
    assert _rotate(q, _heads(3, 4 * D, D), k, _heads(5, 2 * D, D)) == -1 and "q_out must not be another" in _said()
    assert _rotate(q, _heads(5, 4 * D, D), k, _heads(5, 2 * D, D)) == -1 and "q_out must not be another" in _said()
    assert _rotate(q, _heads(5, 4 * D, D), k, _heads(1, 2 * D, D)) == -1 and "k_out must not be another" in _said()
    for p in (4, 5, 6, 7):
        assert _append(q, _heads(p, 4 * D, D)) == -1 and "another" in _said()
    for p in (6, 7):
        assert _attend(q, _heads(p, 4 * D, D)) == -1 and "another" in _said()


def test_more_heads_than_can_be_counted():
    """Sequences without new tokens count as well."""
    wide = 1 << 21
    pages = binding.PagesDesc(K=6 * P, V=7 * P, page_stride=wide * 16 * D, head_stride=16 * D, row_stride=D, pages=10, page=16, Hkv=wide, d=D, dtype=0)
    batch = _batch()
    batch.B = 1024
    args = binding.AttendArgs(_heads(1, wide * D, D), _heads(2, wide * D, D), 8 * P, 1 << 40, 1, wide, 1.0, 1)
    assert binding.load().subgen_paged_attend(pages, batch, args, None) == -1 and "too many rows" in _said()
