"""Verification of drafted tokens against a 64-bit form, token for token, and the distribution of what comes out."""
from __future__ import annotations

import numpy as np
import pytest

from tests import branch_ref as ref

pytestmark = pytest.mark.gpu
SEED, OFFSET = 0xA5A5_1234_0F0F_9876, (2 << 32) + 9


def _inputs(batch, drafted, vocab, dtype, seed, noise=0.5, spread=2.0):
    import torch
    kind = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    g = torch.Generator().manual_seed(seed)
    target = (spread * torch.randn(batch, drafted + 1, vocab, generator=g)).to(kind)
    draft = (target[:, :drafted].float() + noise * torch.randn(batch, drafted, vocab, generator=g)).to(kind)
    u = torch.rand(batch, drafted, vocab, generator=g).clamp(1e-7, 1 - 1e-7)
    ids = (draft.float() - torch.log(-torch.log(u))).argmax(-1).int() if drafted else torch.empty(batch, 0, dtype=torch.int32)
    return target, draft, ids


def _check(target, draft, ids, t=1.0, td=None, least=0.9, seed=SEED, status=None, **kw):
    """Runs the kernel on [batch, positions, vocab] tensors and compares; returns what it gave."""
    import torch
    import paper_2102_08124_b200 as tm
    vocab = target.shape[2]
    td = t if td is None else td
    two = lambda a: a.reshape(-1, vocab).cuda()
    tokens, accepted, logp = tm.tm_verify_draft(two(target), None if draft is None else two(draft), ids.cuda(), seed, OFFSET, temperature=t, draft_temperature=td,
                                                status=status, **kw)
    tokens, accepted, logp = tokens.cpu().numpy(), accepted.cpu().numpy(), logp.double().cpu().numpy()
    f64 = lambda a: None if a is None else a.double().numpy()
    want, count, want_logp, sure = ref.verify(f64(target), f64(draft), ids.numpy(), seed, OFFSET, float(np.float32(t)), float(np.float32(td)))
    assert sure.mean() >= least
    assert np.array_equal(tokens[sure], want[sure]) and np.array_equal(accepted[sure], count[sure])
    # a log-sum-exp of fp32 exponentials, their exponents rounded twice: 2^-22 (1 + |x|) relative, |x| below 64 where there is mass
    assert np.allclose(logp[sure], want_logp[sure], rtol=4 * ref.U32, atol=2e-5, equal_nan=True)
    return tokens, accepted, logp


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("batch,drafted,vocab", [(1, 0, 1), (3, 2, 1), (5, 3, 2), (40, 4, 3), (33, 1, 5), (64, 8, 8), (20, 5, 31), (17, 3, 33), (50, 4, 1000), (7, 6, 1023),
                                                 (300, 2, 1024), (3, 5, 4099), (9, 3, 32001), (2, 4, 32768), (160, 1, 8000), (1, 3, 131072), (2, 2, 200003)])
def test_tokens(batch, drafted, vocab, dtype):
    target, draft, ids = _inputs(batch, drafted, vocab, dtype, batch + vocab)
    _check(target, draft, ids, least=0.9 if batch > 9 else 0.0)


@pytest.mark.parametrize("t,td", [(0.5, 0.5), (1.7, 1.0), (0.05, 0.2), (30.0, 30.0)])
def test_temperatures(t, td):
    target, draft, ids = _inputs(60, 3, 500, "f32", 3)
    _check(target, draft, ids, t, td)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_lengths(dtype):
    """Sequences end anywhere; what stands behind a negative id is not looked at."""
    import torch
    target, draft, ids = _inputs(40, 6, 700, dtype, 8, noise=0.1)
    n = torch.arange(40) % 7
    ids[torch.arange(6) >= n[:, None]] = -1
    ids[5, 5] = 3                                              # n = 5: behind it, nothing
    ids[12, 0] = -7
    tokens, accepted, _ = _check(target, draft, ids)
    assert (accepted <= np.minimum(n.numpy(), 6)).all() and accepted[12] == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masks(dtype):
    """Tokens at -Inf or the type's lowest value have no probability, in the target, the drafter, or both; offsets change nothing."""
    import torch
    target, draft, ids = _inputs(64, 3, 900, dtype, 4)
    low = torch.finfo(target.dtype).min
    target[:16, :, 100:] = float("-inf")
    draft[8:24, :, :450] = float("-inf")
    target[32:40, :, ::2] = low
    draft[32:40, :, 1::2] = low
    target[40:48] += 300.0
    target[48:56, 1:] = low                                   # a row of one value alone: all equal
    ids[3, 0] = 500                                           # p = 0: refused, whatever u is
    ids[20, 0] = 10                                           # q = 0 at a drafted token: stays, should p be positive
    tokens, accepted, _ = _check(target, draft, ids)
    assert (tokens[:16] < 100).all() and accepted[3] == 0 and accepted[20] >= 1


def test_one_token_left():
    import torch
    target, draft, ids = _inputs(8, 2, 50, "f32", 5)
    target[:4] = float("-inf")
    target[:4, :, 7] = -1e30
    tokens, accepted, logp = _check(target, draft, ids)
    assert all(tokens[b, accepted[b]] == 7 for b in range(4)) and np.abs(logp[:4]).max() == 0


def test_equal_rows_are_never_refused():
    target, _, ids = _inputs(200, 5, 300, "bf16", 6)
    tokens, accepted, _ = _check(target, target[:, :5].clone(), ids)
    assert (accepted == 5).all()


def test_refused_with_nothing_left_draws_from_the_target():
    """p = q, the draft has no probability in either."""
    target, _, ids = _inputs(100, 1, 64, "f32", 7)
    target[:, 0, 9] = float("-inf")
    ids[:] = 9
    tokens, accepted, _ = _check(target, target[:, :1].clone(), ids)
    assert (accepted == 0).all() and (tokens[:, 0] != 9).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_certain_drafter(dtype):
    """Without the drafter's logits a draft stays with the target's probability, and is not drawn after it was refused."""
    target, _, _ = _inputs(200, 3, 40, dtype, 9)
    ids = target[:, :3].float().argmax(-1).int()
    ids[::3] = 5
    tokens, accepted, _ = _check(target, None, ids)
    for b in range(200):
        if accepted[b] < 3:
            assert tokens[b, accepted[b]] != ids[b, accepted[b]]


def test_bad_rows_and_ids_are_shown():
    import torch
    import paper_2102_08124_b200 as tm
    cases = []
    for k, (where, value) in enumerate([("t", float("nan")), ("t", float("inf")), ("d", float("nan")), ("d", float("inf")), ("t", None), ("d", None)]):
        target, draft, ids = _inputs(6, 3, 200, "f32", 20 + k, noise=0.0)
        rows = target if where == "t" else draft
        if value is None:
            rows[2, 1] = float("-inf")
        else:
            rows[2, 1, 199] = value
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        tokens, accepted, logp = _check(target, draft, ids, status=status)
        assert int(status) == tm.TM_DEV_NONFINITE and accepted[2] == 1 and tokens[2].tolist()[1:] == [-1] * 3 and np.isnan(logp[2, 1])
    # behind the last row that is reached nothing is looked at
    target, draft, ids = _inputs(4, 2, 100, "f32", 30)
    target[:, 0, 3] = float("-inf")
    ids[:, 0] = 3
    target[:, 1:] = float("nan")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    _, accepted, _ = _check(target, draft, ids, status=status)
    assert int(status) == 0 and (accepted == 0).all()
    target, draft, ids = _inputs(4, 2, 100, "f32", 31, noise=0.0)
    ids[1, 1], ids[2, 0] = 100, 2 ** 31 - 1
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    _, accepted, _ = _check(target, draft, ids, status=status)
    assert int(status) == tm.TM_DEV_BADID and accepted.tolist() == [2, 1, 0, 2]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [0, 1, 3])
def test_rows_that_start_anywhere(dtype, shift):
    import torch
    import paper_2102_08124_b200 as tm
    batch, drafted, vocab = 6, 2, 3001
    target, draft, ids = _inputs(batch, drafted, vocab, dtype, 11)
    plain = tm.tm_verify_draft(target.reshape(-1, vocab).cuda(), draft.reshape(-1, vocab).cuda(), ids.cuda(), SEED, OFFSET)

    def strided(a, pitch, at):
        t = torch.full((a.shape[0] * a.shape[1], pitch), float("nan"), dtype=a.dtype, device="cuda")[:, at:at + vocab]
        t.copy_(a.reshape(-1, vocab))
        return t

    got = tm.tm_verify_draft(strided(target, 3008, shift), strided(draft, 3010, 2 * shift), ids.cuda(), SEED, OFFSET)
    assert torch.equal(got[0], plain[0]) and torch.equal(got[1], plain[1])
    assert torch.allclose(got[2], plain[2], rtol=0, atol=2e-5)


def test_same_input_same_answer_and_outputs_that_are_passed_in():
    import torch
    import paper_2102_08124_b200 as tm
    target, draft, ids = _inputs(30, 3, 5000, "bf16", 12)
    a = (target.reshape(-1, 5000).cuda(), draft.reshape(-1, 5000).cuda(), ids.cuda(), SEED)
    first = tm.tm_verify_draft(*a)
    out = (torch.full((30, 4), 77, dtype=torch.int32, device="cuda"), torch.full((30,), 77, dtype=torch.int32, device="cuda"), torch.full((30, 4), 7.0, device="cuda"))
    again = tm.tm_verify_draft(*a, tokens_out=out[0], accepted_out=out[1], logp_out=out[2])
    assert all(x is y for x, y in zip(out, again)) and all(torch.equal(x, y) for x, y in zip(first, again))
    assert tm.tm_verify_draft(*a, want_logp=False)[2] is None
    step = torch.tensor([5], dtype=torch.int64, device="cuda")
    other = tm.tm_verify_draft(*a, 5)
    assert not torch.equal(other[0], first[0]) and torch.equal(other[0], tm.tm_verify_draft(*a, offset_dev=step)[0])
    empty = tm.tm_verify_draft(a[0][:0], a[1][:0], ids[:0].cuda(), 1)
    assert empty[0].shape == (0, 4) and empty[1].shape == (0,)


@pytest.mark.parametrize("certain", [False, True])
def test_what_comes_out_is_distributed_as_the_target(certain):
    """Drafts drawn from q, 100000 sequences of one pair of rows: every token's count of the first place within six deviations of p."""
    import torch
    import paper_2102_08124_b200 as tm
    n, vocab = 100_000, 13
    g = torch.Generator().manual_seed(1)
    z, y = 1.5 * torch.randn(vocab, generator=g), 1.5 * torch.randn(vocab, generator=g)
    p, q = torch.softmax(z.double(), 0), torch.softmax(y.double(), 0)
    ids = torch.full((n, 1), 4, dtype=torch.int32) if certain else torch.multinomial(q, n, True, generator=g).int()[:, None]
    tokens, accepted, _ = tm.tm_verify_draft(z.repeat(2 * n, 1).cuda(), None if certain else y.repeat(n, 1).cuda(), ids.cuda(), 99)
    count = torch.bincount(tokens[:, 0].cpu().long(), minlength=vocab).double()
    assert bool(((count - n * p).abs() <= 6 * (n * p * (1 - p)).sqrt()).all())
    stay = float(p[4]) if certain else float(torch.minimum(p, q).sum())
    assert abs(float(accepted.double().mean()) - stay) <= 6 * (stay * (1 - stay) / n) ** 0.5
    # the bonus token, where the draft stayed, is the target's too
    bonus = tokens[:, 1][accepted == 1].cpu().long()
    m = bonus.numel()
    assert bool(((torch.bincount(bonus, minlength=vocab).double() - m * p).abs() <= 6 * (m * p * (1 - p)).sqrt()).all())


@pytest.mark.parametrize("kind", ["drafter", "certain", "none"])
def test_near_keys_are_told_apart(kind):
    """Enough sequences that a few dozen have two keys, or the two sides of a test, within 2^-11 of each other."""
    target, draft, ids = _inputs(30000, 0 if kind == "none" else 1, 24, "f32", 40)
    _check(target, draft if kind == "drafter" else None, ids, least=0.97)
