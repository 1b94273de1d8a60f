"""Lists as long as they may be, over many short rows."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2102_08124_b200 as tm
from tests import train_ref as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("k", [128, 129, 200, 256])
@pytest.mark.parametrize("rows,vocab", [(1000, 130), (700, 1030), (600, 2311), (500, 4000), (400, 8000)])
def test_long_lists_of_many_short_rows(rows, vocab, k, dtype):
    rng = np.random.Generator(np.random.PCG64(k + vocab))
    z = torch.from_numpy(np.round(rng.standard_normal((rows, vocab)) * 64).astype(np.float32) / 16).to(dtype)      # many equal ones
    values, ids, lse = (t.double().cpu().numpy() for t in tm.tm_top_logits(z.cuda(), k, 1.5))
    exact = z.double().numpy()
    for r in range(0, rows, 7):
        v, i = ref.top(exact[r], k)
        assert np.array_equal(ids[r], i) and np.array_equal(values[r], v), r
    want = np.array([ref.log_sum_exp(x / 1.5) for x in exact])
    assert np.all(np.abs(lse - want) <= ref.sum_unit(vocab, np.abs(exact).max() / 1.5) + 2 * ref.U32 * np.abs(want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_largest_vocabulary(dtype):
    from tests.test_train_distill import _check_distill, _check_top, _matrix
    rng = np.random.Generator(np.random.PCG64(1))
    vocab, k, t = 1 << 22, 100, 1.5
    z, zd = _matrix(rng.standard_normal((2, vocab), dtype=np.float32) * 2, dtype)
    _check_top(z, zd, 200, t)
    ids = np.stack([rng.permutation(vocab)[:k] for _ in range(2)]).astype(np.int32)
    values = np.sort(rng.standard_normal((2, k)).astype(np.float32) + 9)[:, ::-1].copy()
    lse = np.array([ref.log_sum_exp(x.astype(np.float64) / t) + 0.2 for x in values], np.float32)
    for teacher_lse in (lse, None):
        _check_distill(z, zd, values, ids, teacher_lse, None, t, 1.0, dtype, inplace=teacher_lse is None)
