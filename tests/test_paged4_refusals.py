"""Arguments that the 4-bit cache and the tables of a step refuse, on the host: nothing is launched. And the plain format's own sense."""
import ctypes as C
import math
import os
import subprocess

import pytest
import torch

import paged4_helpers as p4
from paper_2402_06082_b200 import binding

P = 1 << 20                                           # an aligned address that nothing follows: every call here is refused first
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _said():
    return binding.load().subgen_last_error().decode()


def _pages(**kw):
    f = dict(pool=P, page_stride=8 * 2304, head_stride=2304, pages=10, page=16, Hkv=8, d=128, status=None)
    f.update(kw)
    return binding.Pages4Desc(**f)


def _batch(**kw):
    f = dict(B=2, cu_q=P, lengths=P, table=P, table_stride=4, groups=0)
    f.update(kw)
    return binding.BatchDesc(**f)


def _heads(**kw):
    f = dict(p=P, token_stride=1024, head_stride=128)
    f.update(kw)
    return binding.Heads(**f)


def _attend(pages=None, batch=None, q=None, out=None, n=2, H=32, scale=1.0, ws=P, size=1 << 40, dtype=1):
    args = binding.AttendArgs(q or _heads(token_stride=4096), out or _heads(p=2 * P, token_stride=4096), ws, size, n, H, scale, 1)
    return binding.load().subgen_paged4_attend(pages or _pages(), batch or _batch(), args, dtype, None)


def _append(pages=None, batch=None, **kw):
    f = dict(q=_heads(p=None), k=_heads(p=3 * P), v=_heads(p=4 * P), n=2, H=32, dtype=1, eps=1e-6)
    f.update(kw)
    return binding.load().subgen_paged4_append(pages or _pages(), batch or _batch(), binding.QkArgs(**f), None)


def _load(pages=None, slots=P, n=2, K=None, V=None, dtype=1):
    return binding.load().subgen_paged4_load(pages or _pages(), slots, n, K or _heads(p=2 * P), V or _heads(p=3 * P), dtype, None)


@pytest.mark.parametrize("call", [_attend, _append, _load])
@pytest.mark.parametrize("kw, word", [
    (dict(page=24), "page"), (dict(page=8), "page"), (dict(page=2048), "page"), (dict(pages=0), "pages"), (dict(d=96), "d must be"),
    (dict(pool=None), "pool"), (dict(pool=P + 8), "16 bytes"), (dict(head_stride=2312), "16 bytes"), (dict(head_stride=1152), "strides"),
    (dict(page_stride=0), "strides"), (dict(page=32), "strides"), (dict(Hkv=0), "heads")])
def test_pools(call, kw, word):
    assert call(pages=_pages(**kw)) == -1 and word in _said()


def test_an_axis_of_one():
    """Strides of one page and one head are not looked at: what is wrong here is n."""
    for kw in (dict(pages=1, page_stride=0), dict(Hkv=1, head_stride=7)):
        assert _attend(pages=_pages(**kw), n=-1) == -1 and "n must be" in _said()
        assert _append(pages=_pages(**kw), n=0) == 0 and _load(pages=_pages(**kw), n=0) == 0


@pytest.mark.parametrize("call", [_attend, _append])
@pytest.mark.parametrize("kw, word", [
    (dict(B=-1), "B and groups"), (dict(B=1024, groups=1), "at most 1024"), (dict(cu_q=None), "cu_q"), (dict(table_stride=0), "table_stride"),
    (dict(table_stride=1 << 27), "2^31"), (dict(groups=1), "cu_group")])
def test_batches(call, kw, word):
    assert call(batch=_batch(**kw)) == -1 and word in _said()


def test_attend():
    assert _attend(H=12) == -1 and "H / Hkv" in _said()
    assert _attend(H=128) == -1 and "H / Hkv" in _said()
    assert _attend(dtype=2) == -1 and "dtype" in _said()
    for scale in (0.0, -1.0, math.nan, math.inf, 3e38):
        assert _attend(scale=scale) == -1 and "scale" in _said()
    assert _attend(out=_heads(token_stride=4096)) == -1 and "out must not be q" in _said()
    assert _attend(pages=_pages(pool=2 * P)) == -1 and "another tensor" in _said()
    assert _attend(out=_heads(p=2 * P, token_stride=64)) == -1 and "16 bytes" in _said() or "rows overlap" in _said()
    assert _attend(size=1000) == -5 or "workspace" in _said()
    assert _attend(ws=P + 16) < 0 and "256-byte" in _said()
    assert _attend(q=_heads(p=None)) == -1 and "q must not be NULL" in _said()
    assert _attend(n=0) == 0 and _attend(batch=_batch(B=0)) == 0


def test_append():
    assert _append(dtype=7) == -1 and "dtype" in _said()
    assert _append(k=_heads(p=None)) == -1 and "k must not be NULL" in _said()
    assert _append(v=_heads(p=P + 2)) == -1 and "16 bytes" in _said()
    assert _append(q=_heads(p=5 * P, token_stride=4096), q_out=_heads(p=P, token_stride=4096)) == -1 and "another tensor" in _said()      # the pool
    assert _append(rope=binding.RopeDesc(P, 24, 0)) == -1 and "rotary_dim" in _said()
    assert _append(wk=P, eps=math.nan) == -1 and "eps" in _said()


def test_load():
    assert _load(slots=None) == -1 and "slots" in _said()
    assert _load(slots=P + 4) == -1 and "8-byte" in _said()
    assert _load(n=-1) == -1 and "n must be" in _said()
    assert _load(dtype=3) == -1 and "dtype" in _said()
    none = _heads(p=None)
    assert _load(K=none, V=none) == -1 and "both" in _said()
    assert _load(K=_heads(p=2 * P, head_stride=64)) == -1 and "rows overlap" in _said()
    assert _load(K=_heads(p=3 * P)) == -1 and "another tensor" in _said()
    assert _load(K=_heads(p=P)) == -1 and "another tensor" in _said()
    assert _load(V=_heads(p=2 * P + 4)) == -1 and "16 bytes" in _said()


def _step(**kw):
    f = dict(B=4, n=10, pages=100, page=16, table_stride=8, **{k: P for k in ("table", "free_pages", "free_count", "lengths", "added",
             "free_count_out", "lengths_out", "cu_q", "slots", "positions")})
    f.update(kw)
    return binding.load().subgen_page_step(binding.PageStepArgs(**f), None)


@pytest.mark.parametrize("kw, word", [
    (dict(B=0), "B must be"), (dict(B=1025), "B must be"), (dict(n=-1), "n >= 0"), (dict(pages=0), "pages"), (dict(page=12), "page"),
    (dict(page=2048), "page"), (dict(table_stride=0), "table_stride"), (dict(table_stride=1 << 27), "2^31"), (dict(slots=P + 4), "8-byte"), (dict(B=1024, table_stride=1 << 21), "2^31 - 1 pages")]
    + [({k: None}, "NULL") for k in ("table", "free_pages", "free_count", "lengths", "added", "free_count_out", "lengths_out", "cu_q", "slots", "positions")])
def test_step(kw, word):
    assert _step(**kw) == -1 and word in _said()


STRUCTS = {"subgen_pages4": binding.Pages4Desc, "subgen_page_step_args": binding.PageStepArgs}


def test_sizes_and_offsets(tmp_path):
    lines, want = ["#include <stddef.h>", "#include <stdio.h>", '#include "subgen.h"', "int main(void) {"], []
    for name, struct in STRUCTS.items():
        lines.append('printf("%%zu\\n", sizeof(%s));' % name)
        want.append(C.sizeof(struct))
        for field in struct._fields_:
            lines.append('printf("%%zu\\n", offsetof(%s, %s));' % (name, field[0]))
            want.append(getattr(struct, field[0]).offset)
    src = tmp_path / "sizes.c"
    src.write_text("\n".join(lines + ["return 0; }"]))
    exe = str(tmp_path / "sizes")
    subprocess.check_call(["gcc", "-I" + os.path.join(ROOT, "include"), "-o", exe, str(src)])
    assert [int(x) for x in subprocess.check_output([exe]).split()] == want


def test_the_plain_format():
    """Values are off by S / 16 at most and are exact in bf16 and fp16; bytes and codes come back."""
    g = torch.Generator().manual_seed(0)
    x = torch.randn(500, 64, generator=g) * torch.exp(4 * torch.randn(500, 4, 1, generator=g)).expand(-1, -1, 16).reshape(500, 64)
    x = x.clamp(-60000, 60000)
    byte, code, value = p4.rounded(x)
    s = p4.scales_of(byte).repeat_interleave(16, -1)
    assert ((value - x.double()).abs() <= s / 16).all()
    for dt in (torch.bfloat16, torch.float16):
        assert torch.equal(value.to(dt).double(), value)
    assert torch.equal(p4.codes_of(p4.code_bytes(code)), code)
    every = p4.scales_of(torch.arange(248, dtype=torch.uint8))
    all_values = ((torch.arange(16).double() - 7.5)[:, None] * every / 8)
    for dt in (torch.bfloat16, torch.float16):
        assert torch.equal(all_values.to(dt).double(), all_values)
    again, codes, values = p4.rounded(value)          # what it holds it holds again
    assert torch.equal(values, value) or (values - value).abs().max() <= (s / 16).max()


def test_wrapper_refusals():
    with pytest.raises(ValueError, match="CUDA tensor"):
        binding.PagedCache4(torch.zeros(2, 2, 2304, dtype=torch.uint8), 16, 128)
    with pytest.raises(ValueError):
        z = torch.zeros(4, dtype=torch.int32)
        binding.page_step(z, torch.zeros(4, 4, dtype=torch.int32), z, z[:1], z, 16, 4)
    assert binding.PagedCache4.bytes(16, 128) == 2304 and binding.PagedCache4.bytes(64, 64) == 4608
