"""Logits that a mask has set to a large negative value, and rows whose logits share a large offset: lists, loss and gradient."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2102_08124_b200 as tm
from tests import train_ref as ref
from tests.test_train_distill_tail import _run

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
LEVELS = [-1e4, -1e6, -1e8, -1e9, -1e10, -1e12, -1e20, -1e30, -1e37]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("t", [1.0, 0.5, 3.0])
@pytest.mark.parametrize("vocab", [40, 3001, 70000])
def test_lists_beside_masks_and_of_masked_rows(vocab, t, dtype):
    rng = np.random.Generator(np.random.PCG64(vocab))
    levels = LEVELS + [-x for x in LEVELS]
    z = np.empty((2 * len(levels), vocab))
    for i, level in enumerate(levels):
        z[2 * i] = np.where(rng.random(vocab) < 0.5, -abs(level), rng.standard_normal(vocab))
        z[2 * i + 1] = level
    host = torch.from_numpy(z.astype(np.float32)).to(DT[dtype])
    zd = host.double().numpy()
    k = 16
    values, ids, lse = (x.double().cpu().numpy() for x in tm.tm_top_logits(host.cuda(), k, t))
    for r in range(len(z)):
        v, i = ref.top(zd[r], k)
        assert np.array_equal(ids[r], i) and np.array_equal(values[r], v), r
        want = zd[r].max() / t + ref.log_sum_exp((zd[r] - zd[r].max()) / t)               # no digit lost to an offset
        ordinary = np.abs(zd[r][np.abs(zd[r]) < 100] / t).max(initial=0.0)
        assert abs(lse[r] - want) <= ref.sum_unit(vocab, ordinary) + 2 * ref.U32 * abs(want), (r, lse[r], want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("t", [1.0, 0.5, 3.0])
@pytest.mark.parametrize("vocab", [40, 4001, 70000])
@pytest.mark.parametrize("tail", [False, True])
def test_masked_logits_outside_the_list_are_no_mass(tail, vocab, t, dtype):
    """Unlisted logits of a mask's size give the same bits as -Inf, and leave the rest's term out."""
    rng = np.random.Generator(np.random.PCG64(3))
    k, rows = 20, 3
    ids = np.stack([rng.permutation(vocab)[:k] for _ in range(rows)]).astype(np.int32)
    v = rng.standard_normal((rows, k)).astype(np.float32)
    lse = np.array([ref.log_sum_exp(x.astype(np.float64) / t) + 0.2 for x in v], np.float32) if tail else None
    listed = rng.standard_normal((rows, k))
    results = []
    for mask in [-np.inf, float(torch.finfo(DT[dtype]).min)] + LEVELS[2:]:
        z = np.full((rows, vocab), mask)
        np.put_along_axis(z, ids.astype(np.int64), listed, 1)
        results.append(_run(torch.from_numpy(z.astype(np.float32)).to(DT[dtype]).cuda(), v, ids, lse, t, 1.0))
    assert np.isfinite(results[0][0]).all() and np.isfinite(results[0][3]).all() and np.isfinite(results[0][4]).all()
    for other in results[1:]:
        assert all(np.array_equal(a, b) for a, b in zip(results[0], other))
