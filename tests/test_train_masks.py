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


def _offset_rows(rng, vocab, k, offset, dtype, spread):
    """Rows whose logits are small multiples of 1/16 plus an offset that keeps them exact; the rows without it."""
    z = np.round(rng.standard_normal((3, vocab)) * spread * 16) / 16
    ids = np.stack([rng.permutation(vocab)[:k] for _ in range(3)]).astype(np.int32)
    host = torch.from_numpy((z + offset).astype(np.float32)).to(DT[dtype])
    assert np.array_equal(host.double().numpy() - offset, z)
    return host.cuda(), z, ids, rng.standard_normal((3, k)).astype(np.float32) + 2


def _shared_offset(offset, spread, vocab, t, tail, dtype):
    """An offset that all logits share changes neither loss nor gradient: the bounds are those of the rows without it."""
    rng = np.random.Generator(np.random.PCG64(abs(int(min(offset, 1e6))) + vocab))
    k, scale = 24, 1.5
    z, zd, ids, v = _offset_rows(rng, vocab, k, offset, dtype, spread)
    lse_t = np.array([ref.log_sum_exp(x.astype(np.float64) / t) + 0.25 for x in v], np.float32) if tail else None
    loss, loss2, stats, grad, grad2 = _run(z, v, ids, lse_t, t, scale)
    for r in range(3):
        want, dz, lse, _, (bl, bg) = ref.distill(zd[r], v[r].astype(np.float64), ids[r], float(lse_t[r]) if tail else None, 1.0, t, scale)
        assert abs(loss[r] - want) <= bl and abs(loss2[r] - want) <= bl, (r, loss[r], loss2[r], want, bl)
        shifted = lse + offset / t
        with np.errstate(over="ignore"):
            rounded = np.float32(shifted)
        assert stats[r, 0] == rounded or abs(stats[r, 0] - shifted) <= 4 * ref.sum_unit(vocab, abs(lse)) + 2 * ref.U32 * abs(shifted)   # (it may be past fp32's range)
        bound = 2 * bg + (ref.out_unit(dtype) + 4 * ref.U32) * np.abs(dz) + 2.0 ** -126 * (1 + scale / t)      # exponentials below the normal range are zero
        # the gradient from the statistics: a log-sum-exp inside +-1024 is rounded to fp32, an error of all q and q / q_rest (bg holds them times unit)
        reach = max(np.abs(zd[r] / t).max(), np.abs(v[r] / t).max(), abs(lse), abs(lse_t[r]) if tail else 0.0)
        stored = ref.U32 * abs(shifted) * bg / (2 * ref.sum_unit(vocab, reach)) if abs(shifted) < 1024 else 0.0
        for name, g, bound in (("both", grad2, bound), ("grad", grad, bound + stored)):
            wrong = ~(np.abs(g[r] - dz) <= bound)
            assert not wrong.any(), (r, name, wrong.sum(), np.flatnonzero(wrong)[:4], g[r][wrong][:4], dz[wrong][:4])


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("t", [1.0, 0.0625, 3.0])                                        # 0.0625: scaled differences do not reach the larger offsets
@pytest.mark.parametrize("vocab", [40, 4001, 70000])
@pytest.mark.parametrize("offset", [0.0, 600.0, -4096.0, 2.0 ** 18, -2.0 ** 19])
def test_an_offset_that_all_logits_share(offset, vocab, t, tail):
    _shared_offset(offset, 1.5, vocab, t, tail, "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("t", [1.0, 0.5, 3.0])
@pytest.mark.parametrize("vocab", [40, 4001, 70000])
@pytest.mark.parametrize("offset", [-2.0 ** 33, 2.0 ** 40, -2.0 ** 100, -2.0 ** 127])
def test_rows_of_one_level(offset, vocab, t, tail, dtype):
    """A row that is masked from end to end is a uniform one."""
    _shared_offset(offset, 0.0, vocab, t, tail, dtype)


@pytest.mark.parametrize("rows,vocab", [(2, 200003), (700, 5000)])
def test_gradients_on_the_logits_of_rows_with_an_offset(rows, vocab):
    """The second reading of such a row comes before anything is written, by any block that shares it."""
    rng = np.random.Generator(np.random.PCG64(rows))
    z = torch.from_numpy((np.round(rng.standard_normal((rows, vocab)) * 32) / 16 + 8192.0 * (np.arange(rows) % 2 * 2 - 1)[:, None]).astype(np.float32)).cuda()
    z[::5] -= 8192.0 * (torch.arange(rows, device="cuda")[::5, None] % 2 * 2 - 1)       # some rows without
    values, ids, lse = tm.tm_top_logits(z, 30, 1.0)
    z += torch.round(torch.randn(z.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(1)) * 4) / 16
    stats = tm.tm_distill_loss(z, values, ids)[1]
    want = tm.tm_distill_grad(z, values, ids, stats)
    both = tm.tm_distill_loss_grad(z, values, ids)[1]
    assert float((want - both).abs().max()) <= 2 * ref.sum_unit(vocab, 40.0) + 2.0 ** -14  # q at most 1; the statistics' rounding inside +-1024
    again = z.clone()
    assert torch.equal(tm.tm_distill_grad(again, values, ids, stats, dlogits=again), want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("t", [1.0, 0.25])
@pytest.mark.parametrize("vocab", [301, 5000, 70000])
@pytest.mark.parametrize("gap", [2048.0, 32768.0, 524288.0])                             # of z / T
def test_masks_that_still_count(gap, vocab, t, dtype):
    """Unlisted logits of one level, far below the listed ones: each gets an equal share of the teacher's remaining mass, by any of the entries."""
    rng = np.random.Generator(np.random.PCG64(vocab))
    rows, k = 3, 30
    ids = np.stack([rng.permutation(vocab)[:k] for _ in range(rows)]).astype(np.int32)
    v = (rng.standard_normal((rows, k)) + 3).astype(np.float32)
    rest = np.array([0.05, 0.2, 0.5])
    lse = (np.array([ref.log_sum_exp(x.astype(np.float64) / t) for x in v]) - np.log1p(-rest)).astype(np.float32)
    z = np.full((rows, vocab), -gap * t)
    np.put_along_axis(z, ids.astype(np.int64), rng.standard_normal((rows, k)), 1)
    loss, loss2, stats, grad, grad2 = _run(torch.from_numpy(z.astype(np.float32)).to(DT[dtype]).cuda(), v, ids, lse, t, 1.0)
    for r in range(rows):
        p_rest = 1.0 - np.exp(v[r].astype(np.float64) / t - float(lse[r])).sum()
        unit = ref.sum_unit(vocab, max(np.abs(v[r] / t).max(), abs(lse[r])))             # of p_rest, and of a sum of equal exponentials
        out = np.setdiff1d(np.arange(vocab), ids[r])
        want = -p_rest / t / (vocab - k)
        for g in (grad[r, out], grad2[r, out]):
            assert np.all(np.abs(g - want) <= (ref.out_unit(dtype) + 4 * ref.U32) * abs(want) + 4 * unit / t / (vocab - k)), (r, g[:3], want)
