"""Frequencies that want a gradient are refused: rotary positions have none for them."""
from __future__ import annotations

import pytest
import torch

from paper_2412_19829_amd import binding as gb
from paper_2412_19829_amd.autograd import gformer_rotary_positions

gpu = pytest.mark.gpu


@pytest.mark.parametrize("learned", [lambda f: f.requires_grad_(True), torch.nn.Parameter, lambda f: f.requires_grad_(True) * 2.0])
@pytest.mark.parametrize("of_q", [False, True])
def test_refused_before_anything_is_called(learned, of_q, monkeypatch):
    monkeypatch.setattr(gb, "rotary_node", lambda *a: pytest.fail("called"))
    q = torch.zeros(3, 2, 64).requires_grad_(of_q)
    with pytest.raises(ValueError, match="freqs"):
        gformer_rotary_positions(q, None, learned(torch.ones(32)), positions=torch.zeros(3, dtype=torch.int32))


@gpu
@pytest.mark.parametrize("python", [False, True])
def test_both_makers_of_the_node(python, monkeypatch):
    if python:
        monkeypatch.setattr(gb, "rotary_node", lambda *a: None)
    gen = torch.Generator().manual_seed(1)
    q, freqs = torch.randn(3, 2, 64, generator=gen).cuda(), torch.rand(32, generator=gen).cuda()
    pos = torch.tensor([0, 5, 9], dtype=torch.int32, device="cuda")
    want, none = gformer_rotary_positions(q, None, freqs, positions=pos)
    assert none is None
    held = freqs.clone().requires_grad_(True)
    for x in (q, q.clone().requires_grad_(True)):
        with pytest.raises(ValueError, match="freqs"):
            gformer_rotary_positions(x, None, held, positions=pos)
        with torch.no_grad():                             # nothing is asked of them there
            got = gformer_rotary_positions(x, None, held, positions=pos)[0]
        assert torch.equal(got, want) and not got.requires_grad
    x = q.clone().requires_grad_(True)
    got = gformer_rotary_positions(x, None, held.detach(), positions=pos)[0]
    assert torch.equal(got, want) and torch.autograd.grad(got.sum(), x)[0] is not None
