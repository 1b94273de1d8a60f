"""Zeros keep their sign in dropout where nothing is added, as x / (1 - p) and x itself have it."""
from __future__ import annotations

import pytest
import torch

import paper_2102_08124_b200 as tm
from tests import branch_ref as ref

pytestmark = pytest.mark.gpu
BITS = {torch.float32: torch.int32, torch.bfloat16: torch.int16}


def _zeros(rows, cols, kind):
    """Zeros of both signs, and other numbers."""
    g = torch.Generator().manual_seed(cols)
    x = torch.randn(rows, cols, generator=g)
    x[:, ::3] = -0.0
    x[:, 1::3] = 0.0
    return x.to(kind).cuda()


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (5, 8), (40, 264), (7, 1001), (33, 1024)])
def test_signs_of_zeros(rows, cols, kind):
    x, bits = _zeros(rows, cols, kind), BITS[kind]
    assert torch.equal(tm.tm_dropout(x, 0.0, 1).view(bits), x.view(bits))
    y = tm.tm_dropout(x, 0.4, 7)
    stay = torch.from_numpy(ref.kept(rows, cols, 0.4, 7, 0)[0]).cuda()
    assert torch.equal(torch.signbit(y), torch.signbit(x) & stay)
    # a sum of a zero of either sign and its negative, or of two positive ones, is +0; of two negative ones -0
    z = tm.tm_dropout(x, 0.0, 1, residual=torch.full_like(x, -0.0))
    assert torch.equal(z.view(bits), x.view(bits))
    assert not bool(torch.signbit(tm.tm_dropout(x, 0.0, 1, residual=torch.zeros_like(x))[x == 0]).any())
