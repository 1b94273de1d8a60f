"""A teacher's largest logits and the distillation loss with its gradient on the GPU against the formulas in 64 bits: types,
vocabularies from one to past every form's limit, odd pitches, ties, masked and non-finite logits, lists of every length, padding,
repeated and foreign ids, idle rows, in-place gradients."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2102_08124_b200 as tm
from tests import train_ref as ref

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
VOCABS = [1, 2, 7, 8, 31, 64, 255, 256, 1000, 1001, 4096, 5003, 16384, 32001, 50000, 131072, 200003]


def _matrix(values, dtype, pad=0, shift=0):
    """A CUDA matrix with `pad` unused columns between rows, `shift` elements past an aligned start; and its exact values."""
    host = torch.from_numpy(np.asarray(values, dtype=np.float32)).to(DT[dtype])
    rows, cols = host.shape
    store = torch.full((rows * (cols + pad) + shift + 8,), float("nan"), dtype=DT[dtype], device="cuda")
    view = store[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(host)
    return view, host.double().numpy()


def _check_top(z, zd, k, t, status=None):
    values, ids, lse = tm.tm_top_logits(z, k, t, status=status)
    values, ids, lse = values.double().cpu().numpy(), ids.cpu().numpy(), lse.double().cpu().numpy()
    for r in range(zd.shape[0]):
        v, i = ref.top(zd[r], k)
        assert np.array_equal(ids[r], i), (r, np.flatnonzero(ids[r] != i)[:5])
        assert np.array_equal(values[r], v, equal_nan=True), r
        want = np.nan if np.isnan(zd[r]).any() else ref.log_sum_exp(zd[r] / t)
        finite = np.abs(zd[r][np.isfinite(zd[r])] / t)
        bound = ref.sum_unit(zd.shape[1], finite.max() if finite.size else 0.0) + 2 * ref.U32 * abs(want)
        assert (np.isnan(want) and np.isnan(lse[r])) or lse[r] == want or abs(lse[r] - want) <= bound, (r, lse[r], want, bound)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", VOCABS)
def test_top_logits(vocab, dtype):
    rng = np.random.Generator(np.random.PCG64(vocab))
    for rows, pad, shift, k, t in [(1, 0, 0, 1, 1.0), (3, 0, 0, 64, 2.0), (9, 8, 0, 7, 0.7), (4, 3, 1, 256, 1.0), (160 if vocab < 20000 else 2, 1, 3, 20, 3.0)]:
        z, zd = _matrix(rng.standard_normal((rows, vocab)) * 3, dtype, pad, shift)
        _check_top(z, zd, k, t)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [9, 1001, 32000, 131073])
def test_top_logits_ties_and_orders(vocab, dtype):
    """Equal logits go by the lower id, whatever the order of the row; the largest ones crowd in few places."""
    rng = np.random.Generator(np.random.PCG64(vocab + 1))
    ramp = np.arange(vocab) / 64.0
    crowd = np.where(np.arange(vocab) % 512 < 8, 5.0 + rng.standard_normal(vocab), -5.0 + rng.standard_normal(vocab))
    few = rng.integers(-3, 3, vocab).astype(np.float64)
    masked = np.where(rng.random(vocab) < 0.9, -np.inf, rng.standard_normal(vocab))
    half = np.where(np.arange(vocab) < vocab // 2, 1.0, 0.0)
    zeros = np.where(rng.random(vocab) < 0.5, 0.0, -0.0)
    rows = [ramp, -ramp, crowd, few, masked, half, half[::-1], zeros, np.full(vocab, 1.5), np.full(vocab, -np.inf), np.full(vocab, np.finfo(np.float32).min)]
    z, zd = _matrix(np.stack(rows), dtype)
    for k in (1, 13, 256):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        _check_top(z, zd, k, 1.0, status)
        assert int(status.item()) == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_top_logits_non_finite(dtype):
    rng = np.random.Generator(np.random.PCG64(5))
    a = rng.standard_normal((4, 3001))
    a[1, 77], a[1, 2000] = np.inf, np.inf
    a[2, 5], a[2, 4], a[2, 9] = np.nan, -np.nan, np.inf
    a[3, :50] = -np.inf
    z, zd = _matrix(a, dtype)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    _check_top(z, zd, 8, 1.0, status)
    assert int(status.item()) == tm.TM_DEV_NONFINITE


def _lists(rng, rows, vocab, k, dtype_scale=3.0):
    """k different ids a row with teacher logits; some lists short, some empty."""
    ids = np.stack([rng.permutation(vocab)[:k] if vocab >= k else np.append(rng.permutation(vocab), np.full(k - vocab, -1)) for _ in range(rows)]).astype(np.int32)
    values = np.sort(rng.standard_normal((rows, k)) * 2 + 4, axis=1)[:, ::-1].astype(np.float32)
    return values.copy(), ids


def _check_distill(z, zd, values, ids, lse_t, weight, t, scale, dtype, status_bits=0, inplace=False):
    dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()
    kw = dict(teacher_lse=dev(lse_t), row_weight=dev(weight), temperature=t, scale=scale)
    v, i = dev(values), dev(ids)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    loss, stats = tm.tm_distill_loss(z, v, i, status=status, **kw)
    up = np.random.Generator(np.random.PCG64(9)).uniform(0.5, 1.5, zd.shape[0]).astype(np.float32)
    part = tm.tm_distill_grad(z, v, i, stats, grad_loss=dev(up), status=status, **kw)
    if inplace:
        buffer = z.clone()
        loss2, both = tm.tm_distill_loss_grad(buffer, v, i, dlogits=buffer, status=status, **kw)
        again = z.clone()
        assert torch.equal(tm.tm_distill_grad(again, v, i, stats, grad_loss=dev(up), dlogits=again, **kw), part)
    else:
        loss2, both = tm.tm_distill_loss_grad(z, v, i, status=status, **kw)
    assert int(status.item()) == status_bits
    loss, loss2, stats, part, both = (x.double().cpu().numpy() for x in (loss, loss2, stats, part, both))
    u_out = ref.out_unit(dtype)
    for r in range(zd.shape[0]):
        want, grad, lse, rest, (bl, bg) = ref.distill(zd[r], values[r].astype(np.float64), ids[r], None if lse_t is None else float(lse_t[r]),
                                                      1.0 if weight is None else float(weight[r]), t, scale)
        if not np.isfinite(want):
            assert loss[r] == want and loss2[r] == want, (r, loss[r], want)
        else:
            assert abs(loss[r] - want) <= bl and abs(loss2[r] - want) <= bl, (r, loss[r], loss2[r], want, bl)
        assert abs(stats[r, 0] - lse) <= 4 * ref.sum_unit(zd.shape[1], abs(lse)) + 2 * ref.U32 * abs(lse), r
        assert stats[r, 1] == rest or abs(stats[r, 1] - rest) <= 8 * ref.sum_unit(zd.shape[1], max(abs(lse), np.abs(zd[r][np.isfinite(zd[r])]).max(initial=0) / t)) + 2 * ref.U32 * abs(rest), r
        tiny = 2.0 ** -126 * (1 + abs(scale))                             # exponentials below the normal range are zero
        for got, f in ((both[r], 1.0), (part[r], float(up[r]))):
            bound = (2 * bg + 4 * ref.U32 * np.abs(grad)) * f + u_out * np.abs(grad * f) + tiny
            wrong = ~(np.abs(got - grad * f) <= bound)
            assert not wrong.any(), (r, f, wrong.sum(), np.flatnonzero(wrong)[:4], np.abs(got - grad * f)[wrong].max(), bound[wrong].min())


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", VOCABS)
def test_distill(vocab, dtype, tail):
    rng = np.random.Generator(np.random.PCG64(vocab + 7))
    for n, (rows, pad, shift, k, t, scale) in enumerate([(1, 0, 0, 1, 1.0, 1.0), (5, 0, 0, 64, 2.0, 0.25), (7, 8, 0, 5, 0.7, 3.0), (3, 3, 1, 256, 1.0, 1.0),
                                                         (160 if vocab < 20000 else 2, 1, 3, 17, 4.0, 16.0)]):
        values, ids = _lists(rng, rows, vocab, k)
        a = rng.standard_normal((rows, vocab)) * 2
        for r in range(rows):
            kept = ids[r] >= 0
            a[r, ids[r][kept]] += 0.5 * values[r][kept]
        if rows > 2:
            ids[1, (k + 1) // 2:] = -1                                     # a short list, and one without entries
            ids[2] = -1
        z, zd = _matrix(a, dtype, pad, shift)
        lse = None
        if tail:                                                           # 10 % to 40 % of the teacher's mass elsewhere
            lse = np.array([ref.log_sum_exp(values[r][ids[r] >= 0].astype(np.float64) / t) if (ids[r] >= 0).any() else 1.0 for r in range(rows)])
            lse = (lse - np.log1p(-rng.uniform(0.1, 0.4, rows))).astype(np.float32)
        weight = None
        if n % 2:
            weight = rng.uniform(0.5, 2.0, rows).astype(np.float32)
            weight[rows // 2] = 0.0
        _check_distill(z, zd, values, ids, lse, weight, t, scale, dtype, inplace=n % 2 == 0)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("rows,vocab,k,dtype", [(5000, 301, 9, "f32"), (4100, 1000, 40, "bf16"), (1501, 4099, 20, "bf16"), (900, 16384, 64, "f32"), (620, 40001, 33, "bf16")])
def test_more_rows_than_the_device_holds(rows, vocab, k, dtype, tail):
    """Every thread block has many rows, idle ones among them."""
    rng = np.random.Generator(np.random.PCG64(rows))
    values, ids = _lists(rng, rows, vocab, k)
    ids[rng.random(rows) < 0.1, k // 2:] = -1
    ids[rng.random(rows) < 0.05] = -1
    weight = np.where(rng.random(rows) < 0.2, 0.0, rng.uniform(0.5, 1.5, rows)).astype(np.float32)
    z, zd = _matrix(rng.standard_normal((rows, vocab), dtype=np.float32) * 2, dtype)
    lse = np.array([ref.log_sum_exp(v.astype(np.float64) / 1.5) + 0.2 for v in values], np.float32) if tail else None
    _check_distill(z, zd, values, ids, lse, weight, 1.5, 1.0, dtype, inplace=tail)
    if tail:
        _check_top(z, zd, k, 1.5)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("vocab", [40, 3001, 40000])
def test_bad_and_repeated_ids(vocab, tail):
    rng = np.random.Generator(np.random.PCG64(21))
    values, ids = _lists(rng, 6, vocab, 20)
    z, zd = _matrix(rng.standard_normal((6, vocab)), "f32")
    ids[0, 5], ids[0, 19] = ids[0, 2], ids[0, 2]                           # the first of equal ids counts
    ids[1, 0] = vocab
    ids[2, 7] = 2 ** 31 - 1
    ids[3] = ids[3, 0]
    ids[4, 3] = -2 ** 31
    lse = np.full(6, 9.0, np.float32) if tail else None
    _check_distill(z, zd, values, ids, lse, None, 1.0, 1.0, "f32", status_bits=tm.TM_DEV_BADID)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tail", [False, True])
def test_whole_vocabulary_listed_and_masked_logits(tail, dtype):
    """Nothing left outside the list (no mass for the rest), logits of -Inf outside and inside it, a teacher entry of -Inf."""
    rng = np.random.Generator(np.random.PCG64(31))
    vocab = 48
    values, ids = _lists(rng, 5, vocab, vocab)
    a = rng.standard_normal((5, vocab))
    ids[1, 30:] = -1
    a[1, np.setdiff1d(np.arange(vocab), ids[1])] = -np.inf                 # the student has no mass outside
    a[2, ids[2, 40:]] = -np.inf
    values[2, 40:] = -np.inf                                               # neither has the teacher there
    a[3, ids[3, 3]] = -np.inf                                              # the loss is infinite, the gradient is not
    z, zd = _matrix(a, dtype)
    lse = np.array([ref.log_sum_exp(v.astype(np.float64)) + 0.1 for v in values], np.float32) if tail else None
    _check_distill(z, zd, values, ids, lse, None, 1.0, 1.0, dtype)


def test_idle_rows_do_not_read_their_logits():
    z = torch.full((6, 5000), float("nan"), device="cuda")
    z[1] = 0.0
    ids = torch.arange(8, dtype=torch.int32, device="cuda").repeat(6, 1)
    ids[4:] = -1
    values = torch.zeros(6, 8, device="cuda")
    weight = torch.zeros(6, device="cuda")
    weight[1] = 1.0
    weight[4:] = 1.0
    for lse in (None, torch.full((6,), 4.0, device="cuda")):
        loss, stats = tm.tm_distill_loss(z, values, ids, teacher_lse=lse, row_weight=weight)
        loss2, dz = tm.tm_distill_loss_grad(z, values, ids, teacher_lse=lse, row_weight=weight)
        dz2 = tm.tm_distill_grad(z, values, ids, stats, teacher_lse=lse, row_weight=weight)
        idle = torch.tensor([0, 2, 3, 4, 5], device="cuda")
        assert torch.all(loss[idle] == 0) and torch.all(stats[idle] == 0) and torch.all(dz[idle] == 0) and torch.all(dz2[idle] == 0)
        assert loss[1] > 0 and torch.equal(loss, loss2) and torch.isfinite(dz).all()
    empty = torch.zeros((6, 0), dtype=torch.int32, device="cuda")
    loss, dz = tm.tm_distill_loss_grad(z, torch.zeros((6, 0), device="cuda"), empty)
    assert torch.all(loss == 0) and torch.all(dz == 0)


def test_non_finite_logits_stay_in_their_row():
    rng = np.random.Generator(np.random.PCG64(41))
    values, ids = _lists(rng, 4, 2000, 9)
    z, zd = _matrix(rng.standard_normal((4, 2000)), "f32")
    clean = tm.tm_distill_loss_grad(z, torch.from_numpy(values).cuda(), torch.from_numpy(ids).cuda())
    z2 = z.clone()
    z2[1, 1500], z2[2, 3] = float("nan"), float("inf")
    loss, dz = tm.tm_distill_loss_grad(z2, torch.from_numpy(values).cuda(), torch.from_numpy(ids).cuda())
    for r in (0, 3):
        assert torch.equal(loss[r], clean[0][r]) and torch.equal(dz[r], clean[1][r])
    assert torch.isnan(loss[1]) and torch.isnan(loss[2]) and torch.isnan(dz[1]).all()


@pytest.mark.parametrize("tail", [False, True])
def test_gradient_against_differences(tail):
    """dlogits . v equals the central difference of the loss, on the 64-bit formula."""
    rng = np.random.Generator(np.random.PCG64(51))
    values, ids = _lists(rng, 3, 60, 6)
    z, zd = _matrix(rng.standard_normal((3, 60)), "f32")
    lse = np.array([ref.log_sum_exp(v.astype(np.float64) / 1.5) + 0.3 for v in values], np.float32) if tail else None
    _, dz = tm.tm_distill_loss_grad(z, torch.from_numpy(values).cuda(), torch.from_numpy(ids).cuda(), teacher_lse=None if lse is None else torch.from_numpy(lse).cuda(),
                                    temperature=1.5, scale=2.0)
    dz = dz.double().cpu().numpy()
    for r in range(3):
        v = rng.standard_normal(60)
        f = lambda a: ref.distill(a, values[r].astype(np.float64), ids[r], None if lse is None else float(lse[r]), 1.0, 1.5, 2.0)[0]
        e = 1e-5
        assert abs((f(zd[r] + e * v) - f(zd[r] - e * v)) / (2 * e) - (dz[r] * v).sum()) <= 1e-4 * np.abs(dz[r] * v).sum()


def test_lists_of_a_teacher_feed_the_loss():
    """tm_top_logits -> tm_distill: a student equal to its teacher has loss 0 (its list, and the rest as one class) and gradient 0."""
    torch.manual_seed(0)
    teacher = torch.randn(33, 5001, device="cuda") * 3
    values, ids, lse = tm.tm_top_logits(teacher, 40, 2.0)
    loss, dz = tm.tm_distill_loss_grad(teacher, values, ids, teacher_lse=lse, temperature=2.0)
    assert loss.abs().max() < 1e-5 and dz.abs().max() < 1e-6
    first = tm.tm_distill_loss_grad(teacher + 0.1 * torch.randn_like(teacher), values, ids, teacher_lse=lse, temperature=2.0)
    assert first[0].min() > 0


def test_same_bits_on_another_stream_and_in_a_graph():
    rng = np.random.Generator(np.random.PCG64(61))
    values, ids = _lists(rng, 40, 9000, 24)
    z, _ = _matrix(rng.standard_normal((40, 9000)), "bf16")
    v, i = torch.from_numpy(values).cuda(), torch.from_numpy(ids).cuda()
    want = tm.tm_distill_loss_grad(z, v, i) + tm.tm_top_logits(z, 24)
    out = [torch.empty_like(t) for t in want]
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        tm.tm_distill_loss_grad(z, v, i, loss_out=out[0], dlogits=out[1], stream=side)
        tm.tm_top_logits(z, 24, values_out=out[2], ids_out=out[3], lse_out=out[4], stream=side)
    for _ in range(2):
        for t in out:
            t.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_offsets_past_32_bits():
    """Rows that start more than 2^31 elements into the matrix."""
    cols, stride = 1000, 1 << 27
    store = torch.zeros(17 * stride + cols, dtype=torch.bfloat16, device="cuda")
    z = torch.as_strided(store, (18, cols), (stride, 1))
    z.copy_(torch.randn(18, cols, generator=torch.Generator("cuda").manual_seed(1), device="cuda"))
    tight = z.contiguous()
    got, want = tm.tm_top_logits(z, 8), tm.tm_top_logits(tight, 8)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    loss, _ = tm.tm_distill_loss(z, want[0], want[1], teacher_lse=want[2])
    loss2, dz2 = tm.tm_distill_loss_grad(tight, want[0], want[1], teacher_lse=want[2])
    assert torch.equal(loss, loss2)
    y, _, mean, rstd = tm.tm_layer_norm(z)
    assert torch.equal(y, tm.tm_layer_norm(tight)[0])
    dz = tm.tm_distill_loss_grad(z, want[0], want[1], teacher_lse=want[2], dlogits=z)[1]
    assert torch.equal(dz.contiguous(), dz2)


def test_binding_refuses_mismatched_tensors():
    z = torch.zeros(4, 8, device="cuda")
    v, i = torch.zeros(4, 2, device="cuda"), torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    for call in (lambda: tm.tm_distill_loss(z, v[:3], i), lambda: tm.tm_distill_loss(z, v, i.long()), lambda: tm.tm_distill_loss(z, v.double(), i),
                 lambda: tm.tm_distill_loss(z, v, i, teacher_lse=torch.zeros(3, device="cuda")), lambda: tm.tm_distill_loss(z, v, i, row_weight=torch.zeros(4)),
                 lambda: tm.tm_distill_loss_grad(z, v, i, dlogits=torch.zeros(4, 9, device="cuda")), lambda: tm.tm_distill_grad(z, v, i, torch.zeros(4, device="cuda")),
                 lambda: tm.tm_distill_loss(z.half(), v, i), lambda: tm.tm_top_logits(z, 0), lambda: tm.tm_top_logits(z, 257), lambda: tm.tm_top_logits(z.t(), 2),
                 lambda: tm.tm_top_logits(z, 2, temperature=0.0)):
        with pytest.raises(tm.TmError):
            call()
