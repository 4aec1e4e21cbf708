"""Arguments that the head norms, the paged append and the paged attention refuse, on the host: nothing is launched."""
import ctypes as C

import pytest

from paper_2402_06082_b200 import binding

P = 1 << 20                                           # an aligned address that nothing follows: every call here is refused first


def _pages(**kw):
    f = dict(K=P, V=P, page_stride=8 * 16 * 128, head_stride=16 * 128, row_stride=128, pages=10, page=16, Hkv=8, d=128, dtype=1, status=None)
    f.update(kw)
    return binding.PagesDesc(**f)


def _batch(**kw):
    f = dict(B=2, cu_q=P, lengths=P, table=P, table_stride=4, groups=0)
    f.update(kw)
    return binding.BatchDesc(**f)


def _heads(**kw):
    f = dict(p=P, token_stride=1024, head_stride=128)
    f.update(kw)
    return binding.Heads(**f)


def _attend(pages=None, batch=None, q=None, out=None, n=2, H=32, scale=1.0, ws=P, size=1 << 40):
    pages, batch = pages or _pages(), batch or _batch()
    args = binding.AttendArgs(q or _heads(), out or _heads(p=2 * P), ws, size, n, H, scale, 1)
    return binding.load().subgen_paged_attend(pages, batch, args, None)             # (q and out differ unless a test says so)


def _qk(**kw):
    f = dict(q=_heads(p=None), k=_heads(), v=_heads(), n=2, H=32, Hkv=8, d=128, dtype=1, eps=1e-6)
    f.update(kw)
    return binding.QkArgs(**f)


def _append(pages=None, batch=None, **kw):
    pages, batch = pages or _pages(), batch or _batch()
    return binding.load().subgen_paged_append(pages, batch, _qk(**kw), None)


def _said():
    return binding.load().subgen_last_error().decode()


@pytest.mark.parametrize("call", [_attend, _append])
@pytest.mark.parametrize("kw, word", [
    (dict(page=24), "page"), (dict(page=8), "page"), (dict(page=2048), "page"), (dict(pages=0), "pages"), (dict(d=96), "d must be"),
    (dict(dtype=2), "dtype"), (dict(K=None), "K and V"), (dict(V=P + 8), "16 bytes"), (dict(row_stride=129), "16 bytes"),
    (dict(row_stride=64), "strides"), (dict(page_stride=0), "strides"), (dict(Hkv=0), "heads")])
def test_pools(call, kw, word):
    assert call(pages=_pages(**kw)) == -1 and word in _said()


@pytest.mark.parametrize("call", [_attend, _append])
@pytest.mark.parametrize("kw, word", [
    (dict(B=-1), "B and groups"), (dict(B=1024, groups=1), "at most 1024"), (dict(cu_q=None), "cu_q"), (dict(table_stride=0), "table_stride"),
    (dict(table_stride=1 << 27), "2^31"), (dict(groups=1), "cu_group"),
    (dict(groups=1, cu_group=P, prefix_len=P, prefix_table=P, prefix_stride=0), "prefix_stride")])
def test_batches(call, kw, word):
    assert call(batch=_batch(**kw)) == -1 and word in _said()


@pytest.mark.parametrize("call", [_attend, _append])
@pytest.mark.parametrize("page", [16, 128, 1024])
def test_longest_tables(call, page):
    """Lengths end far enough below 2^31 for an index that is rounded up to a tile to stay an int."""
    most = (2**31 - 1024) // page - 1
    for n, rc in ((most, 0), (most + 1, -1)):
        assert call(pages=_pages(page=page), batch=_batch(table_stride=n), n=0) == rc
        groups = dict(groups=1, cu_group=P, prefix_len=P, prefix_table=P, prefix_stride=n)
        assert call(pages=_pages(page=page), batch=_batch(**groups), n=0) == rc


def test_attend():
    assert _attend(H=12) == -1 and "H / Hkv" in _said()
    assert _attend(H=128) == -1 and "H / Hkv" in _said()
    for scale in (0.0, -1.0, float("nan"), float("inf"), 3e38):
        assert _attend(scale=scale) == -1 and "scale" in _said()
    assert _attend(n=-1) == -1 and "n must" in _said()
    assert _attend(n=1 << 30) == -1 and "rows" in _said()
    assert _attend(q=_heads(p=None)) == -1 and "q must not" in _said()
    assert _attend(out=_heads(p=P)) == -1 and "out must not be q" in _said()
    assert _attend(out=_heads(token_stride=1025)) == -1 and "out" in _said()
    assert _attend(ws=None) == -2 and "workspace" in _said()
    assert _attend(ws=P + 64) == -2 and "aligned" in _said()
    pages, bad, batch = _pages(), _pages(d=32), _batch()
    need = binding.load().subgen_paged_workspace_bytes(pages, batch, 2, 32)
    assert need > 0 and _attend(size=need - 1) == -2 and str(need) in _said()
    assert binding.load().subgen_paged_workspace_bytes(bad, batch, 2, 32) == 0
    assert _attend(q=_heads(token_stride=0)) == -1 and "positive" in _said()


def test_nothing_to_do():
    assert _attend(n=0) == 0 and _attend(batch=_batch(B=0)) == 0
    assert _append(n=0) == 0 and _append(batch=_batch(B=0)) == 0


def test_append():
    assert _append(k=_heads(p=None)) == -1 and "k must not" in _said()
    assert _append(v=_heads(head_stride=4)) == -1 and "v:" in _said()
    assert _append(q=_heads()) == -1 and "q_out" in _said()
    assert _append(rope=binding.RopeDesc(P, 24, 0)) == -1 and "rotary_dim" in _said()
    assert _append(rope=binding.RopeDesc(P, 256, 0)) == -1 and "rotary_dim" in _said()
    assert _append(wk=P + 2) == -1 and "aligned" in _said()
    assert _append(wk=P, eps=-1.0) == -1 and "eps" in _said()


def test_qk_norm_rope():
    def f(**kw):
        return binding.load().subgen_qk_norm_rope(_qk(**kw), None)
    h, none, r = _heads(), _heads(p=None), binding.RopeDesc(P, 128, 0)
    assert f(k=none) == -1 and "both" in _said()
    assert f(q=h, k=none) == -1 and "q_out" in _said()
    assert f(k_out=h, rope=r) == -1 and "positions" in _said()
    assert f(q=h, q_out=h, k_out=h, Hkv=0) == -1 and "heads" in _said()
    assert f(k_out=h, d=80) == -1 and "d must" in _said()
    assert f(k_out=h, positions=P, rope=r, wk=P, eps=float("nan")) == -1 and "eps" in _said()
    assert f(k_out=h, rope=r, n=0) == 0
    assert binding.load().subgen_qk_norm_rope(None, None) == -1 and "args" in _said()


def test_rope_words():
    L = binding.load()
    two_pi = 6.283185307179586476925286766559
    out = (C.c_uint64 * 4)()
    assert L.subgen_rope_words((C.c_double * 4)(two_pi / 4, two_pi, -two_pi / 8, 0.0), 4, out) == 0
    assert abs(out[0] - (1 << 62)) < 1 << 12 and min(out[1], (1 << 64) - out[1]) < 1 << 13 and out[3] == 0
    assert abs(out[2] - 7 * (1 << 61)) < 1 << 12
    assert L.subgen_rope_words((C.c_double * 1)(float("inf")), 1, out) == -1 and "finite" in _said()
    assert L.subgen_rope_words(None, 1, out) == -1
    # the fraction of a turn of a far position, from the word alone
    from decimal import Decimal, getcontext
    getcontext().prec = 60
    f = 10000.0 ** (-2.0 * 5 / 128)
    L.subgen_rope_words((C.c_double * 1)(f), 1, out)
    pi = Decimal("3.14159265358979323846264338327950288419716939937510582097494")
    for pos in (1, 131071, (1 << 31) - 1):
        want = (Decimal(f) / (2 * pi) * pos) % 1
        got = Decimal((out[0] * pos) % (1 << 64)) / (1 << 64)
        assert abs(got - want) < Decimal(2) ** -31


def test_python_refusals():
    import torch
    with pytest.raises(ValueError):
        binding.Rope(128, rotary_dim=20, device="cpu")
    with pytest.raises(ValueError):
        binding.Rope(64, rotary_dim=128, device="cpu")
    with pytest.raises(ValueError):
        binding.Rope(64, inv_freq=[1.0], device="cpu")
    with pytest.raises(ValueError, match="CUDA"):
        binding.PagedCache(torch.zeros(2, 1, 16, 64), torch.zeros(2, 1, 16, 64))
    with pytest.raises(ValueError, match="CUDA"):
        binding.qk_norm_rope(torch.zeros(1, 1, 64), None)
    with pytest.raises(ValueError):
        binding.qk_norm_rope(None, None)
    with pytest.raises(ValueError, match="CUDA"):
        binding.PagedBatch(torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(1, 1, dtype=torch.int32))
    with pytest.raises(ValueError):
        binding.qk_norm_rope(torch.zeros(1, 1, 64).half(), [1.0])
    with pytest.raises(TypeError):
        binding._calls.append(1, 2, 3)
