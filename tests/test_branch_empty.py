"""The autograd forms on tensors without rows or without columns, and on a single row without a leading dimension."""
from __future__ import annotations

import pytest
import torch

from paper_2102_08124_b200.branch import _rows

SHAPES = [(0,), (7,), (3, 0), (0, 5), (2, 0, 5), (2, 3, 0), (0, 0), (4, 1)]


@pytest.mark.parametrize("shape", SHAPES)
def test_rows(shape):
    t = torch.arange(1.0 * torch.Size(shape).numel()).view(shape)
    m = _rows(t)
    assert m.shape == (torch.Size(shape[:-1]).numel(), shape[-1]) and torch.equal(m.flatten(), t.flatten())


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("p", [0.0, 0.5])
def test_gradients(shape, p):
    from paper_2102_08124_b200.branch import dropout, rms_norm
    from paper_2102_08124_b200.distill import layer_norm
    leaf = lambda *s: torch.randn(*s, device="cuda").requires_grad_()
    for residual in (False, True):
        for f in (lambda x, r, w: rms_norm(x, w, residual=r, p=p, seed=1)[0], lambda x, r, w: dropout(x, p, 1, residual=r),
                  lambda x, r, w: layer_norm(x, w, w, residual=r)[0]):
            x, r, w = leaf(*shape), leaf(*shape) if residual else None, leaf(shape[-1])
            y = f(x, r, w)
            assert y.shape == shape
            (y.sum() + 0 * w.sum()).backward()
            assert x.grad.shape == shape and (r is None or r.grad.shape == shape) and w.grad.shape == w.shape
            if torch.Size(shape).numel() == 0:
                assert bool((w.grad == 0).all())
