"""Lists of rows with more logits at the bound than the buffer of a thread block holds: equal logits, masked rows, many rows a block."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2102_08124_b200 as tm
from tests import train_ref as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab,rows", [(4000, 1300), (32001, 700), (131072, 400)])
def test_equal_logits_in_many_rows(vocab, rows, dtype):
    """Every block goes from rows that overflow its buffer to rows that do not, and back; the same bits every time."""
    kinds = np.zeros((5, vocab), np.float32)
    kinds[0] = 1.5                                                         # constant
    kinds[1] = -np.inf                                                     # masked
    kinds[2, vocab // 2:] = 1.0                                            # two levels
    kinds[3] = np.random.Generator(np.random.PCG64(vocab)).standard_normal(vocab)
    kinds[4] = np.finfo(np.float32).min
    kinds = torch.from_numpy(kinds).to(dtype)
    order = torch.arange(rows) * 7 % 5
    z = kinds.cuda()[order.cuda()]
    k = 100
    first = tm.tm_top_logits(z, k, 2.0)
    for _ in range(5):
        again = tm.tm_top_logits(z, k, 2.0)
        assert all(torch.equal(a, b) for a, b in zip(first, again))
    exact = kinds.double().numpy()
    values, ids, lse = (t.cpu() for t in first)
    for kind in range(5):
        v, i = ref.top(exact[kind], k)
        mine = order == kind
        assert torch.equal(ids[mine], torch.from_numpy(i.astype(np.int32)).expand(int(mine.sum()), k))
        assert torch.equal(values[mine].double(), torch.from_numpy(v).expand(int(mine.sum()), k))
        want = ref.log_sum_exp(exact[kind] / 2.0)
        finite = np.abs(exact[kind][np.isfinite(exact[kind])] / 2.0)
        bound = ref.sum_unit(vocab, finite.max() if finite.size else 0.0) + 2 * ref.U32 * abs(want) if np.isfinite(want) else 0.0
        got = lse[mine].double()
        assert torch.all((got == want) | ((got - want).abs() <= bound))
