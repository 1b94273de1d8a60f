"""Layer norm on the GPU, forward and backward, against the formulas in 64 bits: types, widths on both sides of every form's limit,
odd pitches, residual and extra gradient, in-place outputs, degenerate rows, few and many rows."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2102_08124_b200 as tm
from tests import train_ref as ref

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _matrix(rng, rows, cols, dtype, pad=0, shift=0, scale=1.0, offset=0.0):
    """A CUDA matrix with `pad` unused columns between rows, `shift` elements past an aligned start; and its exact values."""
    host = torch.from_numpy((rng.standard_normal((rows, cols)) * scale + offset).astype(np.float32)).to(DT[dtype])
    store = torch.full((rows * (cols + pad) + shift + 8,), float("nan"), dtype=DT[dtype], device="cuda")
    view = store[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(host)
    return view, host.double().numpy()


def _vector(rng, n, dtype, scale, offset):
    host = torch.from_numpy((rng.standard_normal(n) * scale + offset).astype(np.float32)).to(DT[dtype])
    return host.cuda(), host.double().numpy()


def _near(got, want, bound, what):
    got = got.double().cpu().numpy()
    wrong = ~(np.abs(got - want) <= bound)
    assert not wrong.any(), "%s: %d of %d off, worst by %g where %g is allowed" % (
        what, wrong.sum(), wrong.size, np.abs(got - want)[wrong].max(), np.asarray(bound)[wrong].min() if np.ndim(bound) else bound)


WIDTHS = [1, 2, 7, 8, 63, 64, 65, 136, 255, 256, 257, 1000, 1001, 1024, 1026, 2048, 2049, 4096, 4104, 8191, 8192, 8200, 12288, 16384, 16385, 20002]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", WIDTHS)
def test_forward_and_backward(cols, dtype):
    rng = np.random.Generator(np.random.PCG64(cols))
    for n, (rows, pad, shift, res, wdtype) in enumerate([(1, 0, 0, True, "f32"), (33, 0, 0, False, dtype), (5, 8, 0, True, dtype), (6, 3, 1, True, "f32"), (3, 2, 2, False, "f32")]):
        x, xd = _matrix(rng, rows, cols, dtype, pad, shift, 1.5, 0.5)
        r, rd = _matrix(rng, rows, cols, dtype, pad, shift) if res else (None, None)
        w, wd = _vector(rng, cols, wdtype, 0.3, 1.0)
        b, bd = _vector(rng, cols, wdtype, 0.1, 0.0)
        y, s, mean, rstd = tm.tm_layer_norm(x, w, b, 1e-5, residual=r)
        yd, hd, md, sd = ref.norm(xd, rd, wd, bd, 1e-5)
        _near(y, yd, ref.norm_bounds(hd, sd, wd, bd, yd, dtype), (n, "y"))
        top = np.abs(hd).max(1)
        _near(mean, md, 64 * ref.U32 * top, (n, "mean"))
        _near(rstd, sd, 64 * ref.U32 * sd * (1 + top * sd), (n, "rstd"))
        assert (s is None) == (not res)
        if res:
            _near(s, hd, ref.out_unit(dtype) * np.abs(hd) + ref.U32 * np.abs(hd), (n, "sum"))
        # backward of the stored matrix with the statistics in hand
        h, hd = (s, s.double().cpu().numpy()) if res else (x, xd)
        dy, dyd = _matrix(rng, rows, cols, dtype, pad, shift, 0.1)
        ds, dsd = _matrix(rng, rows, cols, dtype, 0, 0, 0.1) if n % 2 == 0 else (None, None)
        dx, dw, db = tm.tm_layer_norm_backward(dy, h, mean, rstd, w, dsum=ds)
        m64, r64 = mean.double().cpu().numpy(), rstd.double().cpu().numpy()
        dxd, dwd, dbd, xh, g = ref.norm_backward(dyd, hd, m64, r64, wd, dsd)
        bx, bw, bb = ref.norm_backward_bounds(dyd, hd, m64, r64, wd, dxd, dwd, dbd, xh, g, dtype, wdtype)
        _near(dx, dxd, bx + (0 if dsd is None else 2 * ref.U32 * np.abs(dsd)), (n, "dx"))
        _near(dw, dwd, bw, (n, "dweight"))
        _near(db, dbd, bb, (n, "dbias"))


@pytest.mark.parametrize("rows,cols,dtype", [(3000, 40, "bf16"), (2500, 256, "f32"), (4001, 1024, "bf16"), (1500, 1032, "f32"), (700, 4096, "bf16"), (640, 8192, "f32"), (300, 9001, "bf16")])
def test_more_rows_than_the_device_holds(rows, cols, dtype):
    rng = np.random.Generator(np.random.PCG64(rows))
    x, xd = _matrix(rng, rows, cols, dtype, offset=1.0)
    w, wd = _vector(rng, cols, "f32", 0.3, 1.0)
    y, _, mean, rstd = tm.tm_layer_norm(x, w, None)
    yd, hd, md, sd = ref.norm(xd, None, wd, 0.0, 1e-5)
    _near(y, yd, ref.norm_bounds(hd, sd, wd, np.zeros(1), yd, dtype), "y")
    dy, dyd = _matrix(rng, rows, cols, dtype, scale=0.1)
    dx, dw, db = tm.tm_layer_norm_backward(dy, x, mean, rstd, w)
    m64, r64 = mean.double().cpu().numpy(), rstd.double().cpu().numpy()
    dxd, dwd, dbd, xh, g = ref.norm_backward(dyd, xd, m64, r64, wd, None)
    bx, bw, bb = ref.norm_backward_bounds(dyd, xd, m64, r64, wd, dxd, dwd, dbd, xh, g, dtype, "f32")
    _near(dx, dxd, bx, "dx")
    _near(dw, dwd, bw, "dweight")
    _near(db, dbd, bb, "dbias")
    # the same bits again, and without the parameters' gradients
    dx2, dw2, db2 = tm.tm_layer_norm_backward(dy, x, mean, rstd, w)
    dx3, none_w, none_b = tm.tm_layer_norm_backward(dy, x, mean, rstd, w, want_params=False)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2) and torch.equal(db, db2) and torch.equal(dx, dx3) and none_w is None and none_b is None


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [40, 1001, 4096, 20001])
def test_outputs_on_inputs_and_without_parameters(cols, dtype):
    rng = np.random.Generator(np.random.PCG64(7))
    rows = 37
    x, _ = _matrix(rng, rows, cols, dtype)
    r, _ = _matrix(rng, rows, cols, dtype)
    y, s, mean, rstd = tm.tm_layer_norm(x, residual=r)
    one, zero = torch.ones(cols, device="cuda"), torch.zeros(cols, device="cuda")
    y1 = tm.tm_layer_norm(x, one, zero, residual=r)[0]
    assert torch.equal(y, y1)                                             # NULL parameters are ones and zeros
    x2, r2 = x.clone(), r.clone()
    tm.tm_layer_norm(x2, residual=r2, y=x2, sum_out=r2)
    assert torch.equal(x2, y) and torch.equal(r2, s)
    dy, _ = _matrix(rng, rows, cols, dtype)
    ds, _ = _matrix(rng, rows, cols, dtype)
    dx, dw, db = tm.tm_layer_norm_backward(dy, s, mean, rstd, dsum=ds)
    for name in ("dy", "h", "dsum"):
        t = {"dy": dy.clone(), "h": s.clone(), "dsum": ds.clone()}
        dx2, dw2, db2 = tm.tm_layer_norm_backward(t["dy"], t["h"], mean, rstd, dsum=t["dsum"], dx=t[name])
        assert torch.equal(dx2, dx) and torch.equal(dw2, dw) and torch.equal(db2, db), name


@pytest.mark.parametrize("rows,cols,dtype", [(20000, 24, "f32"), (9000, 300, "bf16"), (5000, 1024, "bf16"), (5000, 1001, "f32"), (2500, 4095, "bf16"), (900, 8192, "f32"), (700, 9000, "bf16")])
def test_outputs_on_inputs_with_many_rows(rows, cols, dtype):
    """Rows are read ahead of their turn while others are written: the same bits as with outputs of their own."""
    rng = np.random.Generator(np.random.PCG64(8))
    x, _ = _matrix(rng, rows, cols, dtype)
    r, _ = _matrix(rng, rows, cols, dtype)
    y, s, mean, rstd = tm.tm_layer_norm(x, residual=r)
    dx, dw, db = tm.tm_layer_norm_backward(x, s, mean, rstd, dsum=r)
    for name in ("dy", "h", "dsum"):
        t = {"dy": x.clone(), "h": s.clone(), "dsum": r.clone()}
        dx2, dw2, db2 = tm.tm_layer_norm_backward(t["dy"], t["h"], mean, rstd, dsum=t["dsum"], dx=t[name])
        assert torch.equal(dx2, dx) and torch.equal(dw2, dw) and torch.equal(db2, db), name
    x2, r2 = x.clone(), r.clone()
    tm.tm_layer_norm(x2, residual=r2, y=r2, sum_out=x2)
    assert torch.equal(r2, y) and torch.equal(x2, s)


def test_degenerate_rows():
    """Constant rows (no variance), rows of one column, no rows, a large offset."""
    for cols in (1, 8, 1000, 4096, 17000):
        x = torch.full((3, cols), 2.5, device="cuda")
        y, _, mean, rstd = tm.tm_layer_norm(x)
        assert torch.all(mean == 2.5) and torch.allclose(rstd, torch.full_like(rstd, 1e-5 ** -0.5), rtol=1e-6) and torch.all(y == 0)
        dx, dw, db = tm.tm_layer_norm_backward(torch.ones_like(x), x, mean, rstd)
        assert torch.all(dx == 0) and torch.all(dw == 0) and torch.all(db == 3)
    x = torch.empty((0, 24), device="cuda")
    y, _, mean, rstd = tm.tm_layer_norm(x)
    dx, dw, db = tm.tm_layer_norm_backward(x, x, mean, rstd)
    assert y.shape == (0, 24) and torch.all(dw == 0) and torch.all(db == 0) and dw.shape == (24,)
    rng = np.random.Generator(np.random.PCG64(3))
    x = torch.from_numpy((rng.standard_normal((4, 1024)) * 0.01 + 100.0).astype(np.float32)).cuda()     # the mean is 10^4 deviations away
    y = tm.tm_layer_norm(x)[0].double().cpu().numpy()
    yd, hd, _, sd = ref.norm(x.double().cpu().numpy(), None, 1.0, 0.0, 1e-5)
    assert np.all(np.abs(y - yd) <= ref.norm_bounds(hd, sd, np.ones(1), np.zeros(1), yd, "f32"))
    bad = torch.ones((3, 1024), device="cuda")
    bad[1, 5] = float("nan")
    y = tm.tm_layer_norm(bad)[0]
    assert torch.isnan(y[1]).all() and torch.isfinite(y[0]).all() and torch.isfinite(y[2]).all()         # a bad row stays by itself


@pytest.mark.parametrize("cols", [9, 130])
def test_gradient_against_differences(cols):
    """dx . v and dweight . u equal the central differences of sum(dy * y), taken on the 64-bit formula."""
    rng = np.random.Generator(np.random.PCG64(cols))
    h, hd = _matrix(rng, 4, cols, "f32")
    w, wd = _vector(rng, cols, "f32", 0.3, 1.0)
    dy, dyd = _matrix(rng, 4, cols, "f32")
    _, _, mean, rstd = tm.tm_layer_norm(h, w)
    dx, dw, db = (t.double().cpu().numpy() for t in tm.tm_layer_norm_backward(dy, h, mean, rstd, w))
    v, u = rng.standard_normal(hd.shape), rng.standard_normal(cols)
    f = lambda hh, ww: (dyd * ref.norm(hh, None, ww, 0.0, 1e-5)[0]).sum()
    e = 1e-5
    # the difference's own error is of order e^2; the gradient's that of fp32
    assert abs((f(hd + e * v, wd) - f(hd - e * v, wd)) / (2 * e) - (dx * v).sum()) <= 1e-4 * np.abs(dx * v).sum()
    assert abs((f(hd, wd + e * u) - f(hd, wd - e * u)) / (2 * e) - (dw * u).sum()) <= 1e-4 * np.abs(dw * u).sum()
    assert np.allclose(db, dyd.sum(0), rtol=0, atol=1e-5)


def test_streams_and_capture():
    rng = np.random.Generator(np.random.PCG64(11))
    x, _ = _matrix(rng, 64, 1024, "bf16")
    dy, _ = _matrix(rng, 64, 1024, "bf16")
    w = torch.ones(1024, device="cuda")
    y, _, mean, rstd = tm.tm_layer_norm(x, w)
    want = tm.tm_layer_norm_backward(dy, x, mean, rstd, w)
    ws = torch.empty(tm.tm_layer_norm_workspace_bytes(64, 1024), dtype=torch.uint8, device="cuda")
    out = [torch.empty_like(t) for t in want]
    y2 = torch.empty_like(y)
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        tm.tm_layer_norm(x, w, y=y2, mean_out=mean, rstd_out=rstd, stream=side)
        tm.tm_layer_norm_backward(dy, x, mean, rstd, w, dx=out[0], dweight_out=out[1], dbias_out=out[2], workspace=ws, stream=side)
    for _ in range(2):
        for t in out + [y2]:
            t.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y2, y) and all(torch.equal(a, b) for a, b in zip(out, want))


def test_binding_refuses_mismatched_tensors():
    x = torch.zeros(4, 8, device="cuda")
    for call in (lambda: tm.tm_layer_norm(x, torch.ones(7, device="cuda")), lambda: tm.tm_layer_norm(x, torch.ones(8, device="cuda"), torch.ones(8, device="cuda").bfloat16()),
                 lambda: tm.tm_layer_norm(x, residual=torch.zeros(4, 9, device="cuda")), lambda: tm.tm_layer_norm(x, residual=x.bfloat16()),
                 lambda: tm.tm_layer_norm(x.t()), lambda: tm.tm_layer_norm(torch.zeros(1, 8, device="cuda").expand(4, 8)),
                 lambda: tm.tm_layer_norm(x, y=torch.zeros(3, 8, device="cuda")), lambda: tm.tm_layer_norm(x, mean_out=torch.zeros(3, device="cuda")),
                 lambda: tm.tm_layer_norm_backward(x, x, torch.zeros(4, device="cuda"), torch.zeros(3, device="cuda")),
                 lambda: tm.tm_layer_norm_backward(x, x, torch.zeros(4, device="cuda"), torch.zeros(4, device="cuda"), workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(tm.TmError):
            call()
