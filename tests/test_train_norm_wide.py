"""Forward layer norm of wide bf16 rows on both sides of the number of rows that decides how many threads share one."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2102_08124_b200 as tm
from tests import train_ref as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("rows,cols", [(7, 8200), (500, 8200), (1200, 8200), (450, 16384), (700, 16384), (300, 12001), (800, 12001), (700, 16383)])
def test_few_and_many_wide_rows(rows, cols, residual):
    g = torch.Generator("cuda").manual_seed(rows)
    x, r = (torch.randn(rows, cols, device="cuda", generator=g).bfloat16() for _ in range(2))
    w, b = torch.rand(cols, device="cuda", generator=g) + 0.5, torch.randn(cols, device="cuda", generator=g)
    y, s, mean, rstd = tm.tm_layer_norm(x, w, b, residual=r if residual else None)
    pick = np.r_[0, np.arange(1, rows, 37), rows - 1]
    f = lambda t: t[pick].double().cpu().numpy()
    wd, bd = w.double().cpu().numpy(), b.double().cpu().numpy()
    yd, hd, md, sd = ref.norm(f(x), f(r) if residual else None, wd, bd, 1e-5)
    top = np.abs(hd).max(1)
    assert np.all(np.abs(f(y) - yd) <= ref.norm_bounds(hd, sd, wd, bd, yd, "bf16"))
    assert np.all(np.abs(f(mean) - md) <= 64 * ref.U32 * top) and np.all(np.abs(f(rstd) - sd) <= 64 * ref.U32 * sd * (1 + top * sd))
    assert s is None if not residual else np.all(np.abs(f(s) - hd) <= (ref.U16 + ref.U32) * np.abs(hd))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_without_columns(dtype):
    """The mean and deviation of nothing are NaN, not what the memory held."""
    x = torch.empty((5, 0), dtype=dtype, device="cuda")
    mean, rstd = torch.zeros(5, device="cuda"), torch.zeros(5, device="cuda")
    y, s, _, _ = tm.tm_layer_norm(x, residual=x, mean_out=mean, rstd_out=rstd)
    assert y.shape == s.shape == (5, 0) and torch.isnan(mean).all() and torch.isnan(rstd).all()
    dx, dw, db = tm.tm_layer_norm_backward(x, x, mean, rstd)
    assert dx.shape == (5, 0) and dw.shape == db.shape == (0,)
    assert tm.tm_layer_norm(x, want_stats=False)[0].shape == (5, 0)
