"""A refused draft whose rows are equal leaves nothing of p - q, whatever the rows' sums were rounded to: the token is the one that the target's row alone gives."""
from __future__ import annotations

import pytest
import torch

import paper_2102_08124_b200 as tm

pytestmark = pytest.mark.gpu
SEED, OFFSET = 31, 1 << 40


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("temperature", [1.0, 0.3])
@pytest.mark.parametrize("batch,vocab", [(3, 200003), (40, 131072), (300, 70001), (310, 1500)])
def test_equal_rows(batch, vocab, kind, temperature):
    g = torch.Generator("cuda").manual_seed(vocab)
    rows = torch.randn(batch, vocab + 3, device="cuda", generator=g)[:, :vocab].to(kind)
    rows[:, 7] = float("-inf")                             # drafted, and impossible: refused
    target = rows.repeat_interleave(2, 0)                  # the second position is not reached
    draft = torch.empty(batch, vocab + 5, device="cuda", dtype=kind)[:, 3:vocab + 3]      # on other boundaries, so that its sums are cut otherwise
    draft.copy_(rows)
    ids = torch.full((batch, 1), 7, device="cuda", dtype=torch.int32)
    tokens, accepted, _ = tm.tm_verify_draft(target, draft, ids, SEED, OFFSET, temperature=temperature)
    alone, _, _ = tm.tm_verify_draft(rows, None, ids[:, :0], SEED, OFFSET, temperature=temperature)
    assert bool((accepted == 0).all()) and torch.equal(tokens[:, 0], alone[:, 0])
