"""The operators of the training step together: their autograd forms against 64-bit autograd, and the example that distils a dense
network into its 2:4 pruning."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_import_needs_no_device():
    code = "import paper_2102_08124_b200.distill as d, sys; assert 'torch' not in sys.modules; d.TeacherLists"
    subprocess.run([sys.executable, "-c", code], cwd=ROOT, check=True)


def norm64(x, w, b, eps):
    m = x.mean(-1, keepdim=True)
    return (x - m) / ((x - m).square().mean(-1, keepdim=True) + eps).sqrt() * w + b


# fp32 against fp64: a gradient is a sum of n terms of which each takes a few roundings, an error of some n^(1/2) 2^-24 against terms
# of their sum's size; 1e-4 of the largest entry leaves a factor of about 30 at n = 400.
TOL = 1e-4


def close(got, want):
    assert float((got.double() - want).abs().max()) <= TOL * float(want.abs().max())


@pytest.mark.gpu
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("use_sum", [False, True])
def test_layer_norm_gradients(residual, use_sum):
    import torch
    from paper_2102_08124_b200.distill import layer_norm
    torch.manual_seed(3)
    leaf = lambda *s: torch.randn(*s, device="cuda").requires_grad_()
    x, r, w, b = leaf(2, 7, 100), leaf(2, 7, 100), leaf(100), leaf(100)
    c, e = torch.randn(2, 7, 100, device="cuda"), torch.randn(2, 7, 100, device="cuda")
    y, h = layer_norm(x, w, b, 1e-5, residual=r if residual else None)
    ((y * c).sum() + ((h * e).sum() if use_sum else 0)).backward()
    X, R, W, B = (t.detach().double().requires_grad_() for t in (x, r, w, b))
    H = X + R if residual else X * 1
    Y = norm64(H, W, B, 1e-5)
    ((Y * c).sum() + ((H * e).sum() if use_sum else 0)).backward()
    close(y.detach(), Y.detach())
    for got, want in ((x, X), (w, W), (b, B)) + (((r, R),) if residual else ()):
        close(got.grad, want.grad)
    assert residual or r.grad is None


@pytest.mark.gpu
def test_sum_alone_has_its_gradient():
    import torch
    from paper_2102_08124_b200.distill import layer_norm
    x, r = torch.randn(3, 8, device="cuda", requires_grad=True), torch.randn(3, 8, device="cuda", requires_grad=True)
    _, h = layer_norm(x, residual=r)
    h.sum().backward()
    assert torch.equal(x.grad, torch.ones_like(x)) and torch.equal(r.grad, torch.ones_like(r))


@pytest.mark.gpu
def test_distill_loss_gradients_and_the_one_pass_form():
    import torch
    from paper_2102_08124_b200.distill import distill_backward, distill_loss, teacher_lists
    torch.manual_seed(4)
    T, k, rows, vocab = 1.5, 5, 6, 301
    teacher, z = 3 * torch.randn(rows, vocab, device="cuda"), 3 * torch.randn(rows, vocab, device="cuda")
    lists = teacher_lists(teacher, k, T)
    grad, weight = torch.rand(rows, device="cuda") + 0.5, torch.rand(rows, device="cuda")
    a = z.clone().requires_grad_()
    loss = distill_loss(a, lists, weight, scale=2.0)
    (loss * grad).sum().backward()
    A, P = z.double().requires_grad_(), (teacher.double() / T).log_softmax(1)
    Q, at = (A / T).log_softmax(1), lists.ids.long()
    p, q = P.gather(1, at).exp(), Q.gather(1, at)
    rest_p = 1 - p.sum(1)
    rest_q = 1 - q.exp().sum(1)
    want = 2.0 * weight.double() * ((p * (p.log() - q)).sum(1) + rest_p * (rest_p.log() - rest_q.log()))
    (want * grad).sum().backward()
    close(loss.detach(), want.detach())
    close(a.grad, A.grad)
    b, c = z.clone().requires_grad_(), z.clone().requires_grad_()
    one = distill_backward(b * 1, lists, weight, scale=2.0)
    distill_loss(c * 1, lists, weight, scale=2.0).sum().backward()
    close(one, want.detach())
    close(b.grad, c.grad.double())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_example_recovers_what_pruning_lost(dtype):
    import torch
    from paper_2102_08124_b200.distill import train
    losses = train(steps=40, rows=256, vocab=1031, width=64, blocks=2, k=16, dtype=getattr(torch, dtype))
    assert all(l == l and l >= 0 for l in losses)
    assert losses[-1] < 0.8 * losses[0]
