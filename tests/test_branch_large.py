"""Matrices whose offsets pass 32 bits: the last rows against the same rows alone, or against the formula where the row's number counts."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2102_08124_b200 as tm
from tests import branch_ref as ref

pytestmark = pytest.mark.gpu
SEED, OFFSET = 123456789, 42


@pytest.fixture(scope="module")
def matrix():
    """[134000, 16385] in bf16, 2^31 elements passed at row 131072 or so; rows off every boundary; its last rows are random, the others zeros."""
    x = torch.zeros(134000, 16385, device="cuda", dtype=torch.bfloat16)
    x[-3:] = torch.randn(3, 16385, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    return x


@pytest.mark.parametrize("cols", [16000, 16377, 16385])
def test_norm(matrix, cols):
    x = matrix[:, :cols]
    y, _, rstd = tm.tm_rms_norm(x, y=torch.empty_like(matrix)[:, :cols])
    last = x[-3:].clone()
    y3, _, r3 = tm.tm_rms_norm(last)
    assert torch.allclose(y[-3:].float(), y3.float(), rtol=2.0 ** -7, atol=1e-6) and torch.allclose(rstd[-3:], r3, rtol=2.0 ** -18)
    assert bool((y[:-3].view(torch.int16) == 0).all())
    dh, _, dw = tm.tm_rms_norm_backward(x, x, rstd, dh=y)
    dh3, _, dw3 = tm.tm_rms_norm_backward(last, last, r3)
    assert torch.allclose(dh[-3:].float(), dh3.float(), rtol=2.0 ** -7, atol=1e-3) and torch.allclose(dw.float(), dw3.float(), rtol=2.0 ** -7, atol=1e-5)
    assert bool((dh[:-3].view(torch.int16) & 0x7FFF == 0).all())


def test_dropout(matrix):
    p, rows = 0.3, matrix.shape[0]
    for cols in (16384, 16385):
        y = tm.tm_dropout(matrix[:, :cols], p, SEED, OFFSET, y=torch.empty_like(matrix)[:, :cols])
        words = ref.philox(np.arange((cols + 7) // 8, dtype=np.uint64)[None, :], np.arange(rows - 3, rows, dtype=np.uint64)[:, None], OFFSET, SEED)
        stay = np.stack([words & 0xFFFF, words >> 16], -1).reshape(3, -1)[:, :cols] >= round(65536 * p)
        assert np.array_equal((y[-3:] != 0).cpu().numpy(), stay & (matrix[-3:, :cols] != 0).cpu().numpy())
        assert bool((y[:-3].view(torch.int16) & 0x7FFF == 0).all())


def test_verification():
    """One draw a row of [17000, 131072]: the last rows have one likely token each, at different places."""
    z = torch.full((17000, 131072), -50.0, device="cuda", dtype=torch.bfloat16)
    at = torch.tensor([5, 70001, 131071], device="cuda")
    z[-3:].scatter_(1, at[:, None], 0.0)
    z[:-3, 9] = 0.0
    tokens, _, logp = tm.tm_verify_draft(z, None, torch.empty(17000, 0, dtype=torch.int32, device="cuda"), SEED)
    assert tokens[-3:, 0].tolist() == at.tolist() and bool((tokens[:-3] == 9).all()) and float(logp.abs().max()) < 1e-6
