"""Root-mean-square norm of dropout and residual, forward and backward, against 64-bit formulas."""
from __future__ import annotations

import numpy as np
import pytest

from tests import branch_ref as ref
from tests.test_branch_dropout import _matrix

pytestmark = pytest.mark.gpu
SEED, OFFSET, EPS = 0x0123456789ABCDEF, (3 << 32) + 17, 1e-5
SIZES = [(1, 1, "plain"), (2, 7, "plain"), (1, 8, "plain"), (9, 31, "off"), (5, 64, "plain"), (150, 72, "padded"), (40, 255, "plain"), (333, 256, "plain"), (17, 257, "off"),
         (21, 512, "plain"), (70, 520, "plain"), (1200, 1000, "padded"), (601, 1001, "plain"), (16, 1024, "plain"), (1500, 1024, "off"), (9, 2000, "plain"), (10, 2047, "plain"),
         (1, 4096, "plain"), (640, 4096, "plain"), (5, 4100, "padded"), (3, 8191, "plain"), (310, 8192, "plain"), (301, 8200, "off"), (2, 12000, "plain"), (400, 16384, "plain"),
         (6, 16380, "padded"), (3, 16385, "plain"), (2, 20000, "plain"), (2, 40001, "off")]


def _weight(cols, wdtype, seed=7):
    import torch
    g = torch.Generator().manual_seed(seed)
    w = (1 + 0.3 * torch.randn(cols, generator=g)).to({"f32": torch.float32, "bf16": torch.bfloat16}[wdtype]).cuda()
    return w, w.double().cpu().numpy()


def _host(t):
    return None if t is None else t.double().cpu().numpy()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,layout", SIZES)
@pytest.mark.parametrize("residual,p", [(False, 0.0), (True, 0.0), (True, 0.1), (False, 0.4)])
def test_forward(rows, cols, layout, dtype, residual, p):
    import paper_2102_08124_b200 as tm
    x, x64 = _matrix(rows, cols, dtype, layout, 3)
    r, r64 = _matrix(rows, cols, dtype, layout, 4) if residual else (None, None)
    w, w64 = _weight(cols, "f32" if (rows + cols) % 2 else dtype)
    y, s, rstd = tm.tm_rms_norm(x, w, EPS, residual=r, p=p, seed=SEED, offset=OFFSET)
    h, dh = ref.total(x64, r64, p, SEED, OFFSET)
    want, want_r = ref.rms(h, w64, EPS)
    by, br = ref.rms_bounds(h, dh, w64, want_r, want)
    u = ref.out_unit(dtype)
    assert (np.abs(_host(y) - want) <= by + u * (np.abs(want) + by)).all()
    assert (np.abs(_host(rstd) - want_r) <= br).all()
    assert (s is None) == (not residual and p == 0)
    if s is not None:
        assert (np.abs(_host(s) - h) <= dh + u * (np.abs(h) + dh)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,layout", SIZES)
@pytest.mark.parametrize("dsum,p", [(False, 0.0), (True, 0.0), (True, 0.1), (False, 0.4)])
def test_backward(rows, cols, layout, dtype, dsum, p):
    import paper_2102_08124_b200 as tm
    h, h64 = _matrix(rows, cols, dtype, layout, 5)
    dy, dy64 = _matrix(rows, cols, dtype, layout, 6)
    e, e64 = _matrix(rows, cols, dtype, layout, 8) if dsum else (None, None)
    wdtype = "f32" if (rows + cols) % 2 else dtype
    w, w64 = _weight(cols, wdtype)
    _, _, rstd = tm.tm_rms_norm(h, w, EPS)
    dh, dx, dw = tm.tm_rms_norm_backward(dy, h, rstd, w, dsum=e, p=p, seed=SEED, offset=OFFSET)
    r64 = _host(rstd)
    want, want_w, xh, g = ref.rms_backward(dy64, h64, r64, w64, e64)
    bx, bw = ref.rms_backward_bounds(dy64, r64, e64, want, want_w, xh, g)
    u = ref.out_unit(dtype)
    assert (np.abs(_host(dh) - want) <= bx + u * (np.abs(want) + bx)).all()
    assert (np.abs(_host(dw) - want_w) <= bw + ref.out_unit(wdtype) * (np.abs(want_w) + bw)).all()
    if p == 0:
        assert dx is dh
    else:
        stay, f = ref.kept(rows, cols, p, SEED, OFFSET)
        want_x, b = np.where(stay, want * f, 0), bx * f + 2 * ref.U32 * np.abs(want) * f
        assert (np.abs(_host(dx) - want_x) <= b + u * (np.abs(want_x) + b)).all()
        assert (_host(dx)[~stay] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("group", [0, 32, 64, 128])
@pytest.mark.parametrize("rows,cols,layout", [s for s in SIZES if s[0] * s[1] < 2_000_000])
def test_eight_bits(rows, cols, layout, dtype, group):
    import paper_2102_08124_b200 as tm
    residual = cols % 3 != 0
    x, x64 = _matrix(rows, cols, dtype, layout, 3)
    r, r64 = _matrix(rows, cols, dtype, layout, 4) if residual else (None, None)
    w, w64 = _weight(cols, "f32" if (rows + cols) % 2 else dtype)
    y8, scales, s = tm.tm_rms_norm_e4m3(x, w, EPS, residual=r, group=group)
    h, dh = ref.total(x64, r64, 0.0, 0, 0)
    y, rstd = ref.rms(h, w64, EPS)
    by, _ = ref.rms_bounds(h, dh, w64, rstd, y)
    at = np.arange(cols) // (group or cols)
    most = np.stack([np.abs(y[:, at == k]).max(1) for k in range(at[-1] + 1)], 1)
    near = np.stack([by[:, at == k].max(1) for k in range(at[-1] + 1)], 1)
    want = np.maximum(most / 448, 2.0 ** -126)
    bs = near / 448 + 3 * ref.U32 * want                       # the quotient by 448 is a product with a rounded 1 / 448
    assert scales.shape == want.shape and (np.abs(_host(scales) - want) <= bs).all()
    sc = _host(scales)[:, at]
    t = y / sc                                                  # what is rounded, within the bound of y and three units: inverse, product, scale
    bt = by / sc + 4 * ref.U32 * np.abs(t)
    got = _host(y8.float())
    assert (np.abs(got - np.clip(t, -448, 448)) <= bt + ref.e4m3_step(np.abs(t) + bt) / 2).all()
    if residual:
        assert (np.abs(_host(s) - h) <= dh + ref.out_unit(dtype) * (np.abs(h) + dh)).all()
    else:
        assert s is None


def test_rows_of_zeros_infinities_and_nan():
    import torch
    import paper_2102_08124_b200 as tm
    x = torch.randn(6, 300, device="cuda")
    x[1] = 0
    x[2, 7] = float("inf")
    x[3, 299] = float("nan")
    x[4] = 1e-30
    w = torch.ones(300, device="cuda")
    y, _, rstd = tm.tm_rms_norm(x, w, 0.0)
    assert bool(torch.isfinite(y[0]).all()) and bool(torch.isnan(y[1]).all()) and float(rstd[1]) == float("inf")       # 0 / 0, as written
    y, _, _ = tm.tm_rms_norm(x, w, 1e-5)
    assert bool((y[1] == 0).all()) and bool(torch.isnan(y[3]).all())
    assert bool(torch.isnan(y[2, 7])) and bool((torch.cat([y[2, :7], y[2, 8:]]) == 0).all())
    assert bool(torch.isfinite(y[4:]).all())
    for group in (0, 32, 64, 128):
        y8, scales, _ = tm.tm_rms_norm_e4m3(x, w, 1e-5, group=group)
        v = y8.float()
        assert bool(torch.isfinite(scales).all()) and bool((scales > 0).all())
        assert torch.equal(torch.isnan(v), torch.isnan(y)) and bool((v[1] == 0).all()) and bool((scales[1] == 2.0 ** -126).all())
        assert bool((torch.cat([v[2, :7], v[2, 8:]]) == 0).all())


def test_outputs_may_lie_on_inputs():
    import torch
    import paper_2102_08124_b200 as tm
    for rows, cols in ((64, 1024), (33, 1001), (5, 20000)):
        x, r, w = torch.randn(rows, cols, device="cuda"), torch.randn(rows, cols, device="cuda"), torch.rand(cols, device="cuda")
        y, s, _ = tm.tm_rms_norm(x, w, residual=r, p=0.2, seed=4)
        a, b = x.clone(), r.clone()
        tm.tm_rms_norm(a, w, residual=b, p=0.2, seed=4, y=a, sum_out=b)
        assert torch.equal(a, y) and torch.equal(b, s)
        a, b = x.clone(), r.clone()
        tm.tm_rms_norm(a, w, residual=b, p=0.2, seed=4, y=b, sum_out=a)
        assert torch.equal(b, y) and torch.equal(a, s)
        q, scales, _ = tm.tm_rms_norm_e4m3(x, w, residual=r, group=64)
        a, b = x.clone(), r.clone()
        q2, scales2, s2 = tm.tm_rms_norm_e4m3(a, w, residual=b, group=64, sum_out=b)
        assert torch.equal(q.view(torch.uint8), q2.view(torch.uint8)) and torch.equal(scales, scales2) and torch.equal(a, x)
        _, _, rstd = tm.tm_rms_norm(s, w)
        dy, e = torch.randn_like(x), torch.randn_like(x)
        dh, dx, dw = tm.tm_rms_norm_backward(dy, s, rstd, w, dsum=e, p=0.2, seed=4)
        for first, second in ((0, 1), (1, 2), (2, 0)):
            t = [dy.clone(), s.clone(), e.clone()]
            _, _, dw2 = tm.tm_rms_norm_backward(t[0], t[1], rstd, w, dsum=t[2], p=0.2, seed=4, dh=t[first], dx=t[second])
            assert torch.equal(t[first], dh) and torch.equal(t[second], dx) and torch.equal(dw2, dw)


def test_what_is_not_wanted_and_no_rows():
    import torch
    import paper_2102_08124_b200 as tm
    x, w = torch.randn(8, 100, device="cuda"), torch.rand(100, device="cuda")
    y, s, rstd = tm.tm_rms_norm(x, w, p=0.5, seed=1, want_sum=False, want_stats=False)
    assert s is None and rstd is None and torch.equal(y, tm.tm_rms_norm(x, w, p=0.5, seed=1)[0])
    rstd = tm.tm_rms_norm(x, w)[2]
    dh, dx, dw = tm.tm_rms_norm_backward(x, x, rstd, w, p=0.5, seed=1, want_dh=False, want_weight=False)
    assert dh is None and dw is None and torch.equal(dx, tm.tm_rms_norm_backward(x, x, rstd, w, p=0.5, seed=1)[1])
    assert torch.equal(tm.tm_rms_norm(x)[0], tm.tm_rms_norm(x, torch.ones(100, device="cuda"))[0])
    none = x[:0]
    y, s, rstd = tm.tm_rms_norm(none, w, residual=none)
    assert y.shape == (0, 100) and rstd.shape == (0,)
    dh, _, dw = tm.tm_rms_norm_backward(none, none, rstd, w)
    assert dh.shape == (0, 100) and bool((dw == 0).all())
    assert bool(torch.isnan(tm.tm_rms_norm(x[:, :0])[2]).all())
    y8, scales, _ = tm.tm_rms_norm_e4m3(none, w)
    assert y8.shape == (0, 100) and scales.shape == (0, 1)


def test_same_input_same_bits():
    import torch
    import paper_2102_08124_b200 as tm
    h, dy, w = torch.randn(3000, 1000, device="cuda"), torch.randn(3000, 1000, device="cuda"), torch.rand(1000, device="cuda")
    rstd = tm.tm_rms_norm(h, w)[2]
    first = tm.tm_rms_norm_backward(dy, h, rstd, w, p=0.1, seed=2)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, tm.tm_rms_norm_backward(dy, h, rstd, w, p=0.1, seed=2)))


def test_gradient_against_differences():
    """Central differences of the forward pass in fp64 arithmetic of the formula, at the kernel's own dropout."""
    import torch
    import paper_2102_08124_b200 as tm
    rows, cols, p = 3, 40, 0.3
    x, r, w = (torch.randn(rows, cols, device="cuda"), torch.randn(rows, cols, device="cuda"), 1 + 0.2 * torch.randn(cols, device="cuda"))
    _, s, rstd = tm.tm_rms_norm(x, w, EPS, residual=r, p=p, seed=SEED)
    dy = torch.randn(rows, cols, device="cuda")
    dh, dx, dw = tm.tm_rms_norm_backward(dy, s, rstd, w, p=p, seed=SEED)
    x64, r64, w64, dy64 = (_host(t) for t in (x, r, w, dy))

    def loss(x_, r_, w_):
        return (ref.rms(ref.total(x_, r_, p, SEED, 0)[0], w_, EPS)[0] * dy64).sum()

    step = 1e-4                                               # differences: step^2 / 6 of a third derivative of order 1, beside fp32's 1e-6
    for got, k in ((dx, 0), (dh, 1), (dw, 2)):
        args = [x64, r64, w64]
        flat = _host(got).reshape(-1)
        for i in range(0, flat.size, 7):
            up, down = args[k].copy().reshape(-1), args[k].copy().reshape(-1)
            up[i] += step
            down[i] -= step
            a, b = list(args), list(args)
            a[k], b[k] = up.reshape(args[k].shape), down.reshape(args[k].shape)
            assert abs((loss(*a) - loss(*b)) / (2 * step) - flat[i]) < 1e-4


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("cols", [9, 17, 255, 505, 1001, 2041, 3001, 5001, 9001, 16377, 16383])
def test_rows_do_not_see_their_neighbours(cols, dtype):
    """Every other row is NaN and Inf; the rows between, and what lies before and behind the matrix, stay as they are."""
    import torch
    import paper_2102_08124_b200 as tm
    kind, rows = getattr(torch, dtype), 37
    g = torch.Generator("cuda").manual_seed(cols)
    flat = lambda: torch.randn(rows * cols + 32, device="cuda", generator=g).to(kind)
    for shift in (0, 3):
        stores = {k: flat() for k in ("x", "r", "dy", "e")}
        part = {k: t[16 + shift:16 + shift + rows * cols].view(rows, cols) for k, t in stores.items()}
        for k, t in part.items():
            t[1::2] = float("nan")
            t[1::2, ::2] = float("inf")
        w = torch.rand(cols, device="cuda", generator=g)
        out = {k: torch.full((rows * cols + 32,), 7.0, device="cuda", dtype=kind) for k in ("y", "s", "dh", "dx")}
        o = {k: t[16 + shift:16 + shift + rows * cols].view(rows, cols) for k, t in out.items()}
        _, _, rstd = tm.tm_rms_norm(part["x"], w, residual=part["r"], p=0.3, seed=1, y=o["y"], sum_out=o["s"])
        tm.tm_rms_norm_backward(part["dy"], o["s"], rstd, w, dsum=part["e"], p=0.3, seed=1, dh=o["dh"], dx=o["dx"])
        alone = {k: t.clone().nan_to_num(0.0, 0.0, 0.0) for k, t in part.items()}
        y, s, r2 = tm.tm_rms_norm(alone["x"], w, residual=alone["r"], p=0.3, seed=1)
        dh, dx, _ = tm.tm_rms_norm_backward(alone["dy"], s, r2, w, dsum=alone["e"], p=0.3, seed=1)
        for got, want in ((o["y"], y), (o["s"], s), (o["dh"], dh), (o["dx"], dx)):
            # the same kernel or one that adds a row's terms in another order, of which the row's factor holds 2^-18
            assert torch.allclose(got[::2].float(), want[::2].float(), rtol=2.0 ** -7 if dtype == "bfloat16" else 2.0 ** -16, atol=1e-5)
        for t in out.values():
            assert bool((t[:16 + shift] == 7).all()) and bool((t[16 + shift + rows * cols:] == 7).all())
