"""Verification by clusters that go through several rounds, of two positions or of eight: drafts refused in the first, a middle and the last round,
sequences that end early, against the 64-bit form."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import tests.test_branch_verify as verify

# Blocks of a sequence (on 148 multiprocessors) and positions of a round: 2 and 2; 4 and 2; 8 and 8; 8 and 2; 1 and 8; 1 and 2
CASES = [(100, 3, 70001), (40, 5, 70001), (20, 5, 131072), (5, 7, 200003), (60, 20, 3000), (310, 6, 1500)]


def _inputs(batch, drafted, vocab, dtype):
    """Drafters from good to bad over the batch; every fifth sequence has fewer drafts."""
    target, draft, ids = verify._inputs(batch, drafted, vocab, dtype, 100 + batch, noise=0.0)
    g = torch.Generator().manual_seed(vocab)
    noise = torch.tensor([0.02, 0.4, 1.2])[torch.arange(batch) % 3][:, None, None]
    draft = (draft.float() + noise * torch.randn(draft.shape, generator=g)).to(draft.dtype)
    u = torch.rand(batch, drafted, vocab, generator=g).clamp(1e-7, 1 - 1e-7)
    ids = (draft.float() - torch.log(-torch.log(u))).argmax(-1).int()
    lengths = torch.where(torch.arange(batch) % 5 == 4, torch.arange(batch) % drafted, drafted)
    ids[torch.arange(drafted) >= lengths[:, None]] = -1
    return target, draft, ids, lengths.numpy()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("batch,drafted,vocab", CASES)
@pytest.mark.parametrize("certain", [False, True])
def test_rounds(batch, drafted, vocab, dtype, certain):
    target, draft, ids, lengths = _inputs(batch, drafted, vocab, dtype)
    if certain:                                            # likely tokens, so that some stay
        ids = torch.where(ids >= 0, target[:, :drafted].float().argmax(-1).int(), ids)
        target = target * 2
    tokens, accepted, _ = verify._check(target, None if certain else draft, ids, least=0.95)
    refused = accepted < lengths
    assert refused.any()
    if not certain:
        assert (accepted == lengths).any()
        assert batch < 20 or ((accepted[refused] == 0).any() and (accepted[refused] >= drafted // 2).any())
