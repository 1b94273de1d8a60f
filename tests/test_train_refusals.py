"""The operators of the training step refuse bad arguments before anything is launched.  No GPU needed."""
from __future__ import annotations

import pytest

import paper_2102_08124_b200 as tm
from paper_2102_08124_b200 import binding_train

A = 0x10000  # a fake, well-aligned, never dereferenced device address


@pytest.fixture(scope="module")
def lib():
    from paper_2102_08124_b200 import build
    build.build()
    return binding_train._lib()


def _norm(lib, **kw):
    a = dict(x=A, ld_x=8, res=None, ld_res=8, dtype=0, rows=4, cols=8, w=A, b=A, wdtype=0, eps=1e-5, s=None, ld_s=8, y=A, ld_y=8, mean=A, rstd=A)
    a.update(kw)
    return lib.tm_layer_norm(a["x"], a["ld_x"], a["res"], a["ld_res"], a["dtype"], a["rows"], a["cols"], a["w"], a["b"], a["wdtype"], a["eps"], a["s"],
                             a["ld_s"], a["y"], a["ld_y"], a["mean"], a["rstd"], None)


@pytest.mark.parametrize("args,code", [
    (dict(dtype=2), 5), (dict(wdtype=-1), 5), (dict(rows=-1), 2), (dict(cols=-8), 2), (dict(ld_x=7), 2), (dict(ld_y=7), 2), (dict(res=A, ld_res=7), 2),
    (dict(s=A, ld_s=0), 2), (dict(rows=1 << 40, ld_x=1 << 40), 2), (dict(eps=-1.0), 11), (dict(eps=float("nan")), 11), (dict(eps=float("inf")), 11),
    (dict(x=None), 1), (dict(y=None), 1), (dict(x=A + 2), 6), (dict(y=A + 1), 6), (dict(res=A + 2), 6), (dict(s=A + 2), 6), (dict(w=A + 2), 6),
    (dict(b=A + 1), 6), (dict(mean=A + 2), 6), (dict(rstd=A + 2), 6), (dict(dtype=1, x=A + 1), 6), (dict(rows=0, x=None, y=None), 0), (dict(cols=0, ld_x=0, ld_y=0), 0),
])
def test_layer_norm(lib, args, code):
    assert _norm(lib, **args) == code


def _back(lib, **kw):
    a = dict(dy=A, ld_dy=8, h=A, ld_h=8, dtype=0, rows=4, cols=8, w=A, wdtype=0, mean=A, rstd=A, ds=None, ld_ds=8, dx=A, ld_dx=8, dw=A, db=A, ws=A, n=1 << 30)
    a.update(kw)
    return lib.tm_layer_norm_backward(a["dy"], a["ld_dy"], a["h"], a["ld_h"], a["dtype"], a["rows"], a["cols"], a["w"], a["wdtype"], a["mean"], a["rstd"],
                                      a["ds"], a["ld_ds"], a["dx"], a["ld_dx"], a["dw"], a["db"], a["ws"], a["n"], None)


@pytest.mark.parametrize("args,code", [
    (dict(dtype=3), 5), (dict(wdtype=2), 5), (dict(rows=-1), 2), (dict(ld_dy=7), 2), (dict(ld_h=0), 2), (dict(ld_dx=7), 2), (dict(ds=A, ld_ds=7), 2),
    (dict(dy=None), 1), (dict(h=None), 1), (dict(mean=None), 1), (dict(rstd=None), 1), (dict(dx=None), 1), (dict(dy=A + 2), 6), (dict(h=A + 2), 6),
    (dict(dx=A + 2), 6), (dict(ds=A + 2), 6), (dict(w=A + 2), 6), (dict(dw=A + 2), 6), (dict(db=A + 2), 6), (dict(mean=A + 1), 6), (dict(rstd=A + 2), 6),
    (dict(ws=None), 8), (dict(ws=A + 128), 8), (dict(n=255), 8), (dict(cols=0), 0), (dict(rows=0, dw=None, db=None, ws=None), 0),
])
def test_layer_norm_backward(lib, args, code):
    assert _back(lib, **args) == code


def test_workspace_sizes(lib):
    f = tm.tm_layer_norm_workspace_bytes
    assert f(0, 8) > 0 and f(8, 0) > 0 and f(1, 1) % 256 == 0
    assert f(1, 1024) >= 2 * 1024 * 4 and f(16384, 1024) >= f(64, 1024) and f(1 << 20, 1024) == f(1 << 21, 1024)


def _top(lib, **kw):
    a = dict(z=A, dtype=0, rows=4, vocab=8, ld=8, k=3, t=1.0, v=A, i=A, lse=A, st=A)
    a.update(kw)
    return lib.tm_top_logits(a["z"], a["dtype"], a["rows"], a["vocab"], a["ld"], a["k"], a["t"], a["v"], a["i"], a["lse"], a["st"], None)


@pytest.mark.parametrize("args,code", [
    (dict(dtype=2), 5), (dict(rows=-1), 2), (dict(vocab=-1), 2), (dict(ld=7), 2), (dict(vocab=1 << 31, ld=1 << 31), 2), (dict(k=0), 11), (dict(k=257), 11),
    (dict(t=0.0), 11), (dict(t=-1.0), 11), (dict(t=float("inf")), 11), (dict(t=float("nan")), 11), (dict(z=None), 1), (dict(v=None), 1), (dict(i=None), 1),
    (dict(z=A + 2), 6), (dict(v=A + 2), 6), (dict(i=A + 2), 6), (dict(lse=A + 2), 6), (dict(st=A + 2), 6), (dict(rows=0, z=None), 0),
])
def test_top_logits(lib, args, code):
    assert _top(lib, **args) == code


def _distill(lib, which, **kw):
    a = dict(z=A, dtype=0, rows=4, vocab=8, ld=8, v=A, i=A, k=3, lse=None, w=None, t=1.0, scale=1.0, loss=A, stats=A, g=None, dz=A, ld_d=8, st=None)
    a.update(kw)
    head = (a["z"], a["dtype"], a["rows"], a["vocab"], a["ld"], a["v"], a["i"], a["k"], a["lse"], a["w"], a["t"], a["scale"])
    if which == "loss":
        return lib.tm_distill_loss(*head, a["loss"], a["stats"], a["st"], None)
    if which == "grad":
        return lib.tm_distill_grad(*head, a["stats"], a["g"], a["dz"], a["ld_d"], a["st"], None)
    return lib.tm_distill_loss_grad(*head, a["loss"], a["dz"], a["ld_d"], a["st"], None)


@pytest.mark.parametrize("which", ["loss", "grad", "both"])
@pytest.mark.parametrize("args,code", [
    (dict(dtype=2), 5), (dict(rows=-1), 2), (dict(vocab=-1), 2), (dict(ld=7), 2), (dict(vocab=1 << 31, ld=1 << 31), 2), (dict(k=-1), 11), (dict(k=257), 11),
    (dict(t=0.0), 11), (dict(t=float("nan")), 11), (dict(scale=float("inf")), 11), (dict(z=None), 1), (dict(v=None), 1), (dict(i=None), 1),
    (dict(z=A + 2), 6), (dict(v=A + 2), 6), (dict(i=A + 2), 6), (dict(lse=A + 2), 6), (dict(w=A + 2), 6), (dict(st=A + 2), 6), (dict(rows=0, z=None), 0),
])
def test_distill(lib, which, args, code):
    assert _distill(lib, which, **args) == code


@pytest.mark.parametrize("which,args,code", [
    ("loss", dict(loss=None), 1), ("loss", dict(loss=A + 2), 6), ("loss", dict(stats=A + 2), 6), ("grad", dict(stats=None), 1), ("grad", dict(stats=A + 2), 6),
    ("grad", dict(g=A + 2), 6), ("grad", dict(dz=None), 1), ("grad", dict(dz=A + 2), 6), ("grad", dict(ld_d=7), 2), ("both", dict(loss=None), 1),
    ("both", dict(dz=None), 1), ("both", dict(loss=A + 2), 6), ("both", dict(dz=A + 1), 6), ("both", dict(ld_d=7), 2),
])
def test_distill_outputs(lib, which, args, code):
    assert _distill(lib, which, **args) == code


def test_status_string(lib):
    assert "out of range" in tm.tm_status_string(tm.TM_ERR_RANGE)


def test_binding_refuses_host_tensors():
    import torch
    x = torch.zeros(4, 8)
    one, ids = torch.zeros(4), torch.zeros(4, 2, dtype=torch.int32)
    for call in (lambda: tm.tm_layer_norm(x), lambda: tm.tm_layer_norm_backward(x, x, one, one), lambda: tm.tm_top_logits(x, 2),
                 lambda: tm.tm_distill_loss(x, torch.zeros(4, 2), ids), lambda: tm.tm_distill_loss_grad(x, torch.zeros(4, 2), ids),
                 lambda: tm.tm_distill_grad(x, torch.zeros(4, 2), ids, torch.zeros(4, 2))):
        with pytest.raises(tm.TmError):
            call()
    with pytest.raises(tm.TmError):
        tm.tm_layer_norm(x.half())
