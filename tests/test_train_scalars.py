"""Scalars of the training operators at the ends of their ranges.  No GPU needed for what is refused."""
from __future__ import annotations

import numpy as np
import pytest

import paper_2102_08124_b200 as tm
from tests.test_train_refusals import _distill, _top, lib  # noqa: F401  (lib: a fixture)


@pytest.mark.parametrize("t", [1e-39, 2.0 ** -149, -0.0])
def test_temperatures_below_the_normal_range_are_refused(lib, t):  # noqa: F811
    assert _top(lib, t=t) == tm.TM_ERR_RANGE
    assert all(_distill(lib, which, t=t) == tm.TM_ERR_RANGE for which in ("loss", "grad", "both"))


@pytest.mark.gpu
@pytest.mark.parametrize("k", [-1, 0, 257, 10 ** 12, 2 ** 32 + 1])
def test_list_lengths_are_refused_before_anything_is_created(k):
    import torch
    z = torch.zeros(4, 300, device="cuda")
    with pytest.raises(tm.TmError) as e:
        tm.tm_top_logits(z, k)
    assert e.value.code == tm.TM_ERR_RANGE


def _rounded(x):
    """As fp32 has it: infinite past its range."""
    with np.errstate(over="ignore"):
        return float(np.float32(x))


@pytest.mark.gpu
@pytest.mark.parametrize("t", [2.0 ** -126, 2.0 ** -60, 2.0 ** 60, 2.0 ** 126])
def test_extreme_temperatures(t):
    """At one end only the largest logit counts, at the other all count alike."""
    import torch
    z = torch.from_numpy((np.random.Generator(np.random.PCG64(1)).permutation(3000)[None] / 8).astype(np.float32)).cuda()
    values, ids, lse = tm.tm_top_logits(z, 4, t)
    n = 3000 if t > 1 else 1
    want = float(z.max()) / t + np.log(n)
    near = lambda got, want, unit: got == _rounded(want) or abs(got - want) <= unit * abs(want)
    assert near(float(lse), want, 2.0 ** -20)
    own = torch.zeros_like(values)
    loss, stats = tm.tm_distill_loss(z, own, ids, temperature=t, scale=t)
    loss2, d = tm.tm_distill_loss_grad(z, own, ids, temperature=t, scale=t)
    d2 = tm.tm_distill_grad(z, own, ids, stats, temperature=t, scale=t)
    q = torch.zeros_like(z)
    q[0, ids[0, 0]] = 1.0
    q = q if t < 1 else torch.full_like(q, 1 / 3000)
    q[0, ids[0].long()] -= 0.25
    gap = 4 * float(values[0, 0]) - float(values.sum())                    # sum of the listed logits' distances from the largest
    want = 0.25 * gap + t * np.log(0.25) if t < 1 else t * np.log(0.25 * 3000)
    assert near(float(loss), want, 2.0 ** -18) and torch.equal(loss, loss2)
    assert float((d - q).abs().max()) <= 2.0 ** -20 and float((d2 - q).abs().max()) <= 2.0 ** -20
