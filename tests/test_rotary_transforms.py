"""Rotary positions under what the node has no rule for: an error, never a result without the derivative."""
from __future__ import annotations

import pytest
import torch
import torch.autograd.forward_ad as fwd

from paper_2412_19829_amd import binding as gb
from paper_2412_19829_amd.autograd import gformer_rotary_positions

gpu = pytest.mark.gpu


@pytest.fixture(params=["native", "python"])
def turn(request, monkeypatch):
    if request.param == "python":
        monkeypatch.setattr(gb, "rotary_node", lambda *a: None)
    freqs, pos = torch.rand(32).cuda(), torch.tensor([0, 5, 9], dtype=torch.int32, device="cuda")
    return lambda x, k=None: gformer_rotary_positions(x, k, freqs, positions=pos)


def rand(*shape):
    return torch.randn(*shape, device="cuda")


@gpu
@pytest.mark.parametrize("grad", [False, True])
def test_forward_mode(turn, grad):
    q, k = rand(3, 2, 64).requires_grad_(grad), rand(3, 1, 64)
    with fwd.dual_level():
        with pytest.raises((RuntimeError, NotImplementedError)):
            turn(fwd.make_dual(q, rand(3, 2, 64)))
        with pytest.raises((RuntimeError, NotImplementedError)):
            turn(q, fwd.make_dual(k, rand(3, 1, 64)))


@gpu
def test_functional_transforms(turn):
    q, many = rand(3, 2, 64), rand(4, 3, 2, 64)
    f = lambda x: turn(x)[0]
    for call in (lambda: torch.func.grad(lambda x: f(x).sum())(q), lambda: torch.func.vjp(f, q)[1](q), lambda: torch.func.jvp(f, (q,), (q,)),
                 lambda: torch.func.vmap(f)(many), lambda: torch.func.functionalize(f)(q)):
        with pytest.raises((RuntimeError, ValueError, NotImplementedError)):
            call()


@gpu
def test_many_gradients_at_once(turn):
    q = rand(3, 2, 64).requires_grad_(True)
    out = turn(q)[0]
    with pytest.raises((RuntimeError, ValueError, NotImplementedError)):
        torch.autograd.grad(out, q, rand(4, 3, 2, 64), is_grads_batched=True, retain_graph=True)
    g = rand(3, 2, 64)                                    # and the graph is whole
    assert torch.autograd.grad(out, q, g)[0].shape == g.shape
