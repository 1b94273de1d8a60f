"""Rounds of drafting whose networks give rows that nothing can be drawn from: the sequences end, and no negative token is looked up."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2102_08124_b200 import TM_DEV_NONFINITE, binding_branch, draft
from tests import branch_ref as ref

VOCAB, BATCH, DRAFTS = 11, 40, 3


def _plain(monkeypatch):
    def verify(logits, draft_logits, ids, seed, offset=0, temperature=1.0, want_logp=True, status=None):
        batch, drafted = ids.shape
        z = logits.double().numpy().reshape(batch, drafted + 1, -1)
        q = None if draft_logits is None else draft_logits.double().numpy().reshape(batch, drafted, -1)
        tokens, accepted, logp, _ = ref.verify(z, q, ids.numpy(), seed, offset, temperature, temperature)
        if status is not None and np.isnan(logp).any():
            status |= TM_DEV_NONFINITE
        return torch.from_numpy(tokens).int(), torch.from_numpy(accepted).int(), None

    monkeypatch.setattr(binding_branch, "tm_verify_draft", verify)


def _networks(device, bad_target=None, bad_drafter=None):
    """Tables of logits; the rows of the given tokens are NaN."""
    g = torch.Generator().manual_seed(1)
    z = 0.7 * torch.randn(VOCAB, VOCAB, generator=g)
    q = z + 0.3 * torch.randn(VOCAB, VOCAB, generator=g)
    if bad_target is not None:
        z[bad_target] = float("nan")
    if bad_drafter is not None:
        q[bad_drafter] = float("nan")

    def network(table):
        table = table.to(device)

        def logits(tokens):
            assert bool((tokens >= 0).all()) and bool((tokens < VOCAB).all())
            return table[tokens.long()]

        return logits

    return network(z), network(q)


def _rounds(device):
    last = (torch.arange(BATCH) % VOCAB).to(device)
    status = torch.zeros(1, dtype=torch.int32, device=device)
    fine, accepted = draft.speculate(*_networks(device), last, DRAFTS, 5, status=status)
    assert int(status) == 0 and bool((fine.gather(1, accepted.long()[:, None]) >= 0).all())

    # the drafter has nothing behind token 4: the drafts end there, and the target goes on
    out, accepted = draft.speculate(*_networks(device, bad_drafter=4), last, DRAFTS, 5, status=status)
    assert int(status) == TM_DEV_NONFINITE
    assert bool((out.gather(1, accepted.long()[:, None]) >= 0).all()) and bool((accepted[last == 4] == 0).all())
    given = torch.cat([last[:, None].to(out.dtype), out[:, :-1]], 1)
    stays = torch.arange(DRAFTS, device=device) < accepted[:, None]
    assert not bool((stays & (given[:, :DRAFTS] == 4)).any())

    # the target has nothing behind token 4: those sequences end, the others are as before
    target, drafter = _networks(device, bad_target=4)
    status.zero_()
    out, accepted = draft.speculate(target, drafter, last, DRAFTS, 5, status=status)
    new = out.gather(1, accepted.long()[:, None])[:, 0]
    assert int(status) == TM_DEV_NONFINITE
    assert bool((out[last == 4] == -1).all()) and bool((accepted[last == 4] == 0).all())
    same = (new >= 0)
    assert 0 < int((~same).sum()) < BATCH and torch.equal(out[same], fine[same])

    # and stay ended, whatever the next round draws
    again, accepted = draft.speculate(target, drafter, new, DRAFTS, 5, DRAFTS + 1, status=status)
    assert bool((again[new < 0] == -1).all()) and bool((accepted[new < 0] == 0).all()) and bool((again[new >= 0] >= -1).all())
    none, accepted = draft.speculate(target, drafter, new, 0, 5, status=status)
    assert none.shape == (BATCH, 1) and bool((none[new < 0] == -1).all())

    assert 0 <= draft.share_that_stays(*_networks(device), last, DRAFTS, 2, 5) <= 1
    for bad in (dict(bad_target=4), dict(bad_drafter=4)):
        with pytest.raises(FloatingPointError):
            draft.share_that_stays(*_networks(device, **bad), last, DRAFTS, 2, 5)


def test_rounds_with_the_plain_form(monkeypatch):
    _plain(monkeypatch)
    _rounds("cpu")


@pytest.mark.gpu
def test_rounds():
    _rounds("cuda")
