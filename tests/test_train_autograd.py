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


def _norm64(x, r, w, b):
    h = x + r
    m = h.mean(-1, keepdim=True)
    return (h - m) / ((h - m).square().mean(-1, keepdim=True) + 1e-5).sqrt() * w + b, h


@pytest.mark.parametrize("shape", [(3, 11, 200), (40, 1024), (2, 9000)])
def test_layer_norm_gradients_in_bf16(shape):
    """Against 64-bit autograd: the stored sum, y's gradient and the result are rounded to bf16 once each (2^-9 of an entry, or of the largest
    one where it enters all of a row); the sums over n rows add theirs like n^(1/2)."""
    torch.manual_seed(6)
    n = shape[-1]
    leaf = lambda *s: torch.randn(*s, device="cuda").bfloat16().requires_grad_()
    x, r, w, b = leaf(*shape), leaf(*shape), leaf(n), leaf(n)
    c, e = (torch.randn(*shape, device="cuda").bfloat16() for _ in range(2))
    y, h = layer_norm(x, w, b, residual=r)
    torch.autograd.backward([y, h], [c, e])
    X, R, W, B = (t.detach().double().requires_grad_() for t in (x, r, w, b))
    Y, H = _norm64(X, R, W, B)
    torch.autograd.backward([Y, H], [c.double(), e.double()])
    close = lambda got, want, unit: float((got.double() - want).abs().max()) <= unit * float(want.abs().max())
    assert close(y.detach(), Y.detach(), 2.0 ** -8) and close(h.detach(), H.detach(), 2.0 ** -8)
    assert close(x.grad, X.grad, 2.0 ** -6) and close(r.grad, R.grad, 2.0 ** -6)
    assert close(w.grad, W.grad, 2.0 ** -6) and close(b.grad, B.grad, 2.0 ** -7)


@pytest.mark.parametrize("tail", [False, True])
def test_distill_gradients_in_bf16(tail):
    """Against 64-bit autograd: every entry of the gradient is rounded to bf16 once, beside fp32 exponentials."""
    torch.manual_seed(7)
    rows, vocab, t, scale = 9, 3001, 1.5, 2.0
    teacher, z = (3 * torch.randn(3, 3, vocab, device="cuda") for _ in range(2))
    z = z.bfloat16().requires_grad_()
    lists = teacher_lists(teacher.reshape(rows, vocab), 20, t)
    lists = lists if tail else lists._replace(lse=None)
    up, weight = torch.rand(rows, device="cuda") + 0.5, torch.rand(rows, device="cuda")
    loss = distill_loss(z, lists, weight, scale)
    (loss * up).sum().backward()
    Z = z.detach().double().reshape(rows, vocab).requires_grad_()
    logq, at = (Z / t).log_softmax(1), lists.ids.long()
    v = lists.values.double() / t
    logp = v - lists.lse.double()[:, None] if tail else v.log_softmax(1)
    want = (logp.exp() * (logp - logq.gather(1, at))).sum(1)
    if tail:
        out = torch.ones_like(logq, dtype=torch.bool).scatter_(1, at, False)
        rest = 1 - logp.exp().sum(1)
        want = want + rest * (rest.log() - logq.masked_fill(~out, -torch.inf).logsumexp(1))
    want = want * scale * weight.double()
    (want * up).sum().backward()
    reach = float((z.detach().float() / t).abs().max())
    unit = 4 * ref.sum_unit(vocab, reach)
    assert bool(((loss - want).abs() <= unit * (2 + reach) * scale).all())
    size = Z.grad.abs() + (scale / t * up * weight).double()[:, None] * (logq.detach().exp() + torch.zeros_like(logq).scatter_(1, at, logp.exp()))
    assert bool(((z.grad.reshape(rows, vocab).double() - Z.grad).abs() <= 2.0 ** -8 * Z.grad.abs() + 2 * unit * size).all())


@pytest.mark.parametrize("shape", [(4, 16), (2, 3, 16)])
def test_outputs_can_be_written_to_in_place(shape):
    """y is not needed for the gradient, so it may change; the sum is, so a change is noticed."""
    x, r = (torch.randn(*shape, device="cuda", requires_grad=True) for _ in range(2))
    c = torch.randn(*shape, device="cuda")
    y, h = layer_norm(x, residual=r)
    want = torch.autograd.grad((2 * y * c).sum() + h.sum(), (x, r))
    y, h = layer_norm(x, residual=r)
    y.mul_(2.0)
    got = torch.autograd.grad((y * c).sum() + h.sum(), (x, r))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    y, h = layer_norm(x, residual=r)
    h.add_(1.0)
    with pytest.raises(RuntimeError, match="inplace"):
        (y * c).sum().backward()
    with torch.no_grad():
        y, h = layer_norm(x, residual=r)
        h.add_(y)


@pytest.mark.parametrize("rows", [0, 1, 5])
def test_slices_and_no_rows(rows):
    """Inputs whose rows are apart, gradients that are expanded, no rows at all."""
    x, r = (torch.randn(rows, 48, device="cuda", requires_grad=True) for _ in range(2))
    w = torch.randn(16, device="cuda", requires_grad=True)
    y, h = layer_norm(x[:, 8:24], w, residual=r.reshape(rows, 3, 16)[:, 1])
    (y.sum() + 2 * h.sum()).backward()
    X, R, W = (t.detach().double().requires_grad_() for t in (x, r, w))
    Y, H = _norm64(X[:, 8:24], R[:, 16:32], W, 0.0)
    (Y.sum() + 2 * H.sum()).backward()
    for got, want in ((x, X), (r, R), (w, W)):
        assert got.grad.shape == want.grad.shape and torch.allclose(got.grad.double(), want.grad, rtol=0, atol=2e-4)
    z = torch.randn(rows, 80, device="cuda", requires_grad=True)
    lists = teacher_lists(torch.randn(rows, 50, device="cuda"), 5)
    loss = distill_loss(z[:, 10:60], lists)
    loss.sum().backward()
    b = z.detach()[:, 10:60].clone().requires_grad_()
    one = distill_backward(b * 1, lists)
    assert torch.allclose(loss, one, rtol=1e-5, atol=1e-6) and torch.allclose(z.grad[:, 10:60], b.grad, rtol=0, atol=1e-6)
    assert not z.grad[:, :10].any() and not z.grad[:, 60:].any()
