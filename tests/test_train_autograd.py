"""The autograd forms of the training operators: second derivatives, gradients in both types, shapes."""
from __future__ import annotations

import pytest
import torch

from paper_2102_08124_b200.distill import distill_backward, distill_loss, layer_norm, teacher_lists
from tests import train_ref as ref

pytestmark = pytest.mark.gpu


def test_a_second_differentiation_is_refused():
    """A gradient penalty through these operators would lose terms: it raises instead."""
    x, r, w = (torch.randn(*s, device="cuda", requires_grad=True) for s in ((5, 16), (5, 16), (16,)))
    y, h = layer_norm(x, w, residual=r)
    (g,) = torch.autograd.grad((y.square() + h).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        g.square().sum().backward()
    z = torch.randn(4, 50, device="cuda", requires_grad=True)
    lists = teacher_lists(torch.randn(4, 50, device="cuda"), 5)
    (g,) = torch.autograd.grad(distill_loss(z, lists).sum(), z, create_graph=True)
    with pytest.raises(RuntimeError):
        g.square().sum().backward()


def test_one_differentiation_with_a_graph_kept():
    x = torch.randn(5, 16, device="cuda", requires_grad=True)
    y, _ = layer_norm(x)
    c = torch.randn_like(y)
    first = torch.autograd.grad((y * c).sum(), x, create_graph=True)[0]
    second = torch.autograd.grad((y * c).sum(), x)[0]
    assert torch.equal(first, second)


def test_a_residual_of_another_shape_is_refused():
    """(2, 3, n) and (3, 2, n) have as many rows, but not the same ones."""
    from paper_2102_08124_b200 import TmError
    x = torch.randn(2, 3, 16, device="cuda")
    for other in (x.transpose(0, 1), x.reshape(6, 16), x[:1], x[..., :8]):
        with pytest.raises(TmError):
            layer_norm(x, residual=other)


def test_a_gradient_that_the_loss_does_not_have_is_refused():
    from paper_2102_08124_b200 import TmError
    z = torch.randn(4, 50, device="cuda", requires_grad=True)
    lists = teacher_lists(torch.randn(4, 50, device="cuda"), 5)
    weight = torch.ones(4, device="cuda", requires_grad=True)
    with pytest.raises(TmError):
        distill_loss(z, lists, weight)
    with pytest.raises(TmError):
        distill_loss(z, lists._replace(values=lists.values.clone().requires_grad_()))
    with pytest.raises(TmError):
        distill_loss(z, lists._replace(lse=lists.lse.clone().requires_grad_()))
    distill_loss(z, lists, weight.detach()).sum().backward()
    with torch.no_grad():
        distill_loss(z, lists, weight)


def test_ids_that_were_left_out_are_seen():
    import paper_2102_08124_b200 as tm
    z = torch.randn(4, 50, device="cuda", requires_grad=True)
    lists = teacher_lists(torch.randn(4, 50, device="cuda"), 5)
    bad = lists._replace(ids=lists.ids.clone())
    bad.ids[2, 1] = 50
    for call in (lambda l, s: distill_loss(z, l, status=s), lambda l, s: distill_backward(z * 1, l, status=s)):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        call(lists, status)
        assert int(status) == 0
        call(bad, status)
        assert int(status) == tm.TM_DEV_BADID
