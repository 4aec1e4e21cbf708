"""Refusals of the 4-bit cache's attention with code and text, and the plain format rounded twice, value by value."""
import torch

import paged4_helpers as p4
from test_paged4_refusals import P, _attend, _heads, _said

ENOMEM = -2                                           # SUBGEN_ENOMEM


def test_refused_outputs_and_workspaces():
    assert _attend(out=_heads(p=2 * P, token_stride=64)) == -1 and "rows overlap" in _said()
    assert _attend(out=_heads(p=2 * P, token_stride=4100)) == -1 and "16 bytes" in _said()
    assert _attend(size=1000) == ENOMEM and "workspace" in _said()
    assert _attend(ws=P + 16) == ENOMEM and "256-byte" in _said()
    assert _attend(ws=None) == ENOMEM and "workspace" in _said()


def test_values_rounded_again():
    """What the cells hold is off by S / 16 at most when it is rounded once more, S being its own group's new scale, no larger than the old."""
    g = torch.Generator().manual_seed(3)
    x = (torch.randn(500, 64, generator=g) * torch.exp(4 * torch.randn(500, 4, 1, generator=g)).expand(-1, -1, 16).reshape(500, 64)).clamp(-60000, 60000)
    byte, _, value = p4.rounded(x)
    again, _, values = p4.rounded(value)
    old, new = (p4.scales_of(b).repeat_interleave(16, -1) for b in (byte, again))
    assert (new <= old).all() and ((values - value).abs() <= new / 16).all()
