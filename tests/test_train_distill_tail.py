"""The distillation loss and its gradient where the student's mass outside the list is far below the fp32 range: finite gaps of any size
between listed and unlisted logits."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2102_08124_b200 as tm
from tests import train_ref as ref

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _formula(z, v, ids, lse_t, t, scale):
    """train_ref.distill for a teacher with a remaining mass, the gradient's q / q_rest taken in logarithms."""
    j = ids[ids >= 0]
    out = np.ones(z.size, bool)
    out[j] = False
    lse = ref.log_sum_exp(z / t)
    logq = z / t - lse
    logp = v[ids >= 0].astype(np.float64) / t - lse_t
    p, log_rest = np.exp(logp), ref.log_sum_exp(logq[out])
    rest = 1.0 - p.sum()
    loss = (p * (logp - logq[j])).sum() + rest * (np.log(rest) - log_rest)
    share = np.where(out, np.exp(np.where(out, logq - log_rest, 0.0)), 0.0)              # q_j / q_rest
    grad = np.exp(logq) - rest * share
    grad[j] -= p
    # as in train_ref: units of fp32 exponentials whose exponents reach the largest |z| / T, |v| / T and logs
    reach = max(np.abs(z / t).max(), np.abs(v / t).max(), abs(lse), abs(lse_t))
    unit = 2 * ref.sum_unit(z.size, reach)
    b_loss = abs(scale) * unit * (3 + reach + abs(np.log(rest)) + abs(log_rest)) + ref.U32 * abs(scale * loss)
    b_grad = abs(scale) / t * (unit * np.exp(logq) + share * unit * (1 + 2 * rest))
    b_grad[j] += abs(scale) / t * unit * p
    return scale * loss, scale / t * grad, lse, log_rest, b_loss, b_grad, unit


def _run(z, v, ids, lse, t, scale):
    dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()
    kw = dict(teacher_lse=dev(lse), temperature=t, scale=scale)
    loss, stats = tm.tm_distill_loss(z, dev(v), dev(ids), **kw)
    grad = tm.tm_distill_grad(z, dev(v), dev(ids), stats, **kw)
    loss2, grad2 = tm.tm_distill_loss_grad(z, dev(v), dev(ids), **kw)
    return [x.double().cpu().numpy() for x in (loss, loss2, stats, grad, grad2)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("t", [1.0, 0.5, 3.0])
@pytest.mark.parametrize("vocab", [301, 9000, 32001, 200003])
@pytest.mark.parametrize("gap", [20, 60, 86, 88, 100, 1000])                             # of z / T
def test_finite_gaps(gap, vocab, t, dtype):
    rng = np.random.Generator(np.random.PCG64(gap + vocab))
    rows, k, scale = 6, 64, 2.0
    ids = np.stack([rng.permutation(vocab)[:k] for _ in range(rows)]).astype(np.int32)
    z = np.zeros((rows, vocab))
    for r in range(rows):
        level = -gap * t
        z[r] = level                                                                     # all alike
        if r % 3 == 1:
            z[r] = level * 2                                                             # one, the others far below it
            z[r, (ids[r].max() + 1) % vocab] = level
        if r % 3 == 2:
            z[r] = level + rng.standard_normal(vocab) * t
        if r >= 3:
            ids[r, 16:] = -1
        z[r, ids[r][ids[r] >= 0]] = 0.0 if r % 2 else rng.standard_normal((ids[r] >= 0).sum()) * t
    v = np.sort(rng.standard_normal((rows, k)) + 3, axis=1)[:, ::-1].astype(np.float32)
    rest = rng.uniform(0.1, 0.4, rows)
    lse = np.array([ref.log_sum_exp(v[r][ids[r] >= 0].astype(np.float64) / t) for r in range(rows)]) - np.log1p(-rest)
    lse = lse.astype(np.float32)
    host = torch.from_numpy(z.astype(np.float32)).to(DT[dtype])
    zd = host.double().numpy()
    loss, loss2, stats, grad, grad2 = _run(host.cuda(), v, ids, lse, t, scale)
    for r in range(rows):
        want, dz, l, log_rest, bl, bg, unit = _formula(zd[r], v[r], ids[r], float(lse[r]), t, scale)
        assert abs(loss[r] - want) <= bl and abs(loss2[r] - want) <= bl, (r, loss[r], loss2[r], want, bl)
        assert abs(stats[r, 0] - l) <= 2 * unit and abs(stats[r, 1] - log_rest) <= 2 * unit + 2 * ref.U32 * abs(log_rest), (r, stats[r], l, log_rest)
        bound = 2 * bg + (ref.out_unit(dtype) + 4 * ref.U32) * np.abs(dz) + 2.0 ** -126 * (1 + scale)
        for name, g in (("both", grad2), ("grad", grad)):
            wrong = ~(np.abs(g[r] - dz) <= bound)
            assert not wrong.any(), (r, name, wrong.sum(), np.flatnonzero(wrong)[:4], g[r][wrong][:4], dz[wrong][:4])
