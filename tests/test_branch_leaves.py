"""Gradients of the residual branch's autograd forms at leaves: each leaf has a gradient of its own, that a second pass adds to."""
from __future__ import annotations

import pytest
import torch

from paper_2102_08124_b200 import binding_branch, branch


def _plain(monkeypatch):
    """The binding's two functions as torch formulas, with its way of returning one tensor as dh and dx where p is 0."""
    def forward(x, weight=None, eps=1e-5, residual=None, p=0.0, seed=0, offset=0, offset_dev=None, y=None, sum_out=None):
        h = x if residual is None else x + residual
        rstd = ((h * h).mean(1) + eps).rsqrt()
        y.copy_(h * rstd[:, None] * (1 if weight is None else weight))
        if sum_out is not None:
            sum_out.copy_(h)
        return y, sum_out, rstd

    def backward(dy, h, rstd, weight=None, dsum=None, p=0.0, seed=0, offset=0, offset_dev=None, want_dh=True, want_weight=True):
        g, xh = dy * (1 if weight is None else weight), h * rstd[:, None]
        dh = rstd[:, None] * (g - xh * (g * xh).mean(1, keepdim=True)) + (0 if dsum is None else dsum)
        return dh, dh, (dy * xh).sum(0) if want_weight else None

    monkeypatch.setattr(binding_branch, "tm_rms_norm", forward)
    monkeypatch.setattr(binding_branch, "tm_rms_norm_backward", backward)


def _passes(device, p, shape=(3, 5, 24)):
    g = torch.Generator().manual_seed(2)
    leaf = lambda *s: torch.randn(*s, generator=g).to(device).requires_grad_()
    x, r, w = leaf(*shape), leaf(*shape), leaf(shape[-1])
    c, e = (torch.randn(*shape, generator=g).to(device) for _ in range(2))

    def once():
        y, h = branch.rms_norm(x, w, residual=r, p=p, seed=3, offset=4)
        ((y * c).sum() + (h * e).sum()).backward()

    once()
    first = [t.grad.clone() for t in (x, r, w)]
    once()
    assert len({t.grad.untyped_storage().data_ptr() for t in (x, r, w)}) == 3
    for t, f in zip((x, r, w), first):
        assert torch.equal(t.grad, 2 * f)                  # the same numbers twice: their sum is exact
    x.grad.zero_()
    assert torch.equal(r.grad, 2 * first[1])


def test_two_passes_with_plain_formulas(monkeypatch):
    _plain(monkeypatch)
    _passes("cpu", 0.0)


@pytest.mark.gpu
@pytest.mark.parametrize("p", [0.0, 0.3])
def test_two_passes(p):
    _passes("cuda", p)


@pytest.mark.gpu
@pytest.mark.parametrize("p", [0.0, 0.3])
def test_a_leaf_that_is_input_and_residual_at_once(p):
    """Its gradient is the sum of both."""
    x = torch.randn(6, 40, device="cuda", requires_grad=True)
    a, b = (x.detach().clone().requires_grad_() for _ in range(2))
    c = torch.randn(6, 40, device="cuda")
    for f in (lambda u, v: branch.rms_norm(u, residual=v, p=p, seed=3)[0], lambda u, v: branch.dropout(u, p, 3, residual=v)):
        x.grad = a.grad = b.grad = None
        (f(x, x) * c).sum().backward()
        (f(a, b) * c).sum().backward()
        assert torch.equal(x.grad, a.grad + b.grad)


@pytest.mark.gpu
def test_two_passes_of_dropout():
    x, r = (torch.randn(6, 40, device="cuda", requires_grad=True) for _ in range(2))
    c = torch.randn(6, 40, device="cuda")
    kept = c.clone()
    branch.dropout(x, 0.3, 5, residual=r).backward(c)
    first = [x.grad.clone(), r.grad.clone()]
    branch.dropout(x, 0.3, 5, residual=r).backward(c)
    assert torch.equal(x.grad, 2 * first[0]) and torch.equal(r.grad, 2 * first[1]) and torch.equal(c, kept)
