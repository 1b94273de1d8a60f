"""The residual branch's operators and draft verification refuse bad arguments before anything is launched.  No GPU needed."""
from __future__ import annotations

import pytest

import paper_2102_08124_b200 as tm
from paper_2102_08124_b200 import binding_branch

A = 0x10000  # a fake, well-aligned, never dereferenced device address


@pytest.fixture(scope="module")
def lib():
    from paper_2102_08124_b200 import build
    build.build()
    return binding_branch._lib()


def _drop(lib, **kw):
    a = dict(x=A, ld_x=8, res=None, ld_res=8, dtype=0, rows=4, cols=8, p=0.5, off=None, y=A, ld_y=8)
    a.update(kw)
    return lib.tm_dropout(a["x"], a["ld_x"], a["res"], a["ld_res"], a["dtype"], a["rows"], a["cols"], a["p"], 1, 2, a["off"], a["y"], a["ld_y"], None)


COMMON = [(dict(dtype=2), 5), (dict(rows=-1), 2), (dict(cols=-8), 2), (dict(ld_x=7), 2), (dict(ld_y=7), 2), (dict(res=A, ld_res=7), 2), (dict(rows=1 << 40, ld_x=1 << 40), 2),
          (dict(x=None), 1), (dict(y=None), 1), (dict(x=A + 2), 6), (dict(res=A + 2), 6), (dict(dtype=1, x=A + 1), 6), (dict(rows=0, x=None, y=None), 0),
          (dict(cols=0, ld_x=0, ld_y=0), 0)]
RANDOM = [(dict(p=-0.1), 11), (dict(p=1.0), 11), (dict(p=float("nan")), 11), (dict(off=A + 4), 6), (dict(rows=1 << 32), 2)]


@pytest.mark.parametrize("args,code", COMMON + RANDOM + [(dict(y=A + 2), 6)])
def test_dropout(lib, args, code):
    assert _drop(lib, **args) == code


def _norm(lib, **kw):
    a = dict(x=A, ld_x=8, res=None, ld_res=8, dtype=0, rows=4, cols=8, w=A, wdtype=0, eps=1e-5, p=0.5, off=None, s=None, ld_s=8, y=A, ld_y=8, rstd=A)
    a.update(kw)
    return lib.tm_rms_norm(a["x"], a["ld_x"], a["res"], a["ld_res"], a["dtype"], a["rows"], a["cols"], a["w"], a["wdtype"], a["eps"], a["p"], 1, 2, a["off"], a["s"], a["ld_s"],
                           a["y"], a["ld_y"], a["rstd"], None)


NORM = [(dict(wdtype=-1), 5), (dict(s=A, ld_s=0), 2), (dict(eps=-1.0), 11), (dict(eps=float("nan")), 11), (dict(eps=float("inf")), 11), (dict(s=A + 2), 6), (dict(w=A + 2), 6),
        (dict(rstd=A + 2), 6)]


@pytest.mark.parametrize("args,code", COMMON + RANDOM + NORM + [(dict(y=A + 1), 6)])
def test_rms_norm(lib, args, code):
    assert _norm(lib, **args) == code


def _norm8(lib, **kw):
    a = dict(x=A, ld_x=8, res=None, ld_res=8, dtype=0, rows=4, cols=8, w=A, wdtype=0, eps=1e-5, group=32, s=None, ld_s=8, y=A, ld_y=8, scales=A, rstd=None)
    a.update(kw)
    return lib.tm_rms_norm_e4m3(a["x"], a["ld_x"], a["res"], a["ld_res"], a["dtype"], a["rows"], a["cols"], a["w"], a["wdtype"], a["eps"], a["group"], a["s"], a["ld_s"], a["y"],
                                a["ld_y"], a["scales"], a["rstd"], None)


@pytest.mark.parametrize("args,code", COMMON + NORM + [(dict(group=g), 11) for g in (-1, 1, 16, 33, 96, 256)] + [(dict(scales=None), 1), (dict(scales=A + 2), 6)])
def test_rms_norm_e4m3(lib, args, code):
    assert _norm8(lib, **args) == code


def _back(lib, **kw):
    a = dict(dy=A, ld_dy=8, h=A, ld_h=8, dtype=0, rows=4, cols=8, w=A, wdtype=0, rstd=A, ds=None, ld_ds=8, p=0.5, off=None, dh=A, ld_dh=8, dx=A, ld_dx=8, dw=A, ws=A, n=1 << 30)
    a.update(kw)
    return lib.tm_rms_norm_backward(a["dy"], a["ld_dy"], a["h"], a["ld_h"], a["dtype"], a["rows"], a["cols"], a["w"], a["wdtype"], a["rstd"], a["ds"], a["ld_ds"], a["p"], 1, 2,
                                    a["off"], a["dh"], a["ld_dh"], a["dx"], a["ld_dx"], a["dw"], a["ws"], a["n"], None)


@pytest.mark.parametrize("args,code", RANDOM + [
    (dict(dtype=3), 5), (dict(wdtype=2), 5), (dict(rows=-1), 2), (dict(ld_dy=7), 2), (dict(ld_h=0), 2), (dict(ld_dh=7), 2), (dict(ld_dx=7), 2), (dict(ds=A, ld_ds=7), 2),
    (dict(dy=None), 1), (dict(h=None), 1), (dict(rstd=None), 1), (dict(dh=None, dx=None), 1), (dict(dy=A + 2), 6), (dict(h=A + 2), 6), (dict(dh=A + 2), 6), (dict(dx=A + 2), 6),
    (dict(ds=A + 2), 6), (dict(w=A + 2), 6), (dict(dw=A + 2), 6), (dict(rstd=A + 2), 6), (dict(ws=None), 8), (dict(ws=A + 128), 8), (dict(n=127), 8), (dict(cols=0), 0),
    (dict(rows=0, dw=None, ws=None), 0),
])
def test_rms_norm_backward(lib, args, code):
    assert _back(lib, **args) == code


def test_workspace_sizes(lib):
    f = tm.tm_rms_norm_workspace_bytes
    assert f(0, 8) > 0 and f(8, 0) > 0 and f(1, 1) % 256 == 0
    assert f(1, 1024) >= 1024 * 4 and f(16384, 1024) >= f(64, 1024) and f(1 << 20, 1024) == f(1 << 21, 1024)


def _verify(lib, **kw):
    a = dict(z=A, dtype=0, batch=4, drafted=2, vocab=8, ld=8, d=A, ld_d=8, ids=A, t=1.0, td=1.0, off=None, tok=A, acc=A, lp=A, st=A)
    a.update(kw)
    return lib.tm_verify_draft(a["z"], a["dtype"], a["batch"], a["drafted"], a["vocab"], a["ld"], a["d"], a["ld_d"], a["ids"], a["t"], a["td"], 1, 2, a["off"], a["tok"], a["acc"],
                               a["lp"], a["st"], None)


@pytest.mark.parametrize("args,code", [
    (dict(dtype=2), 5), (dict(batch=-1), 2), (dict(batch=1 << 31), 2), (dict(drafted=-1), 2), (dict(drafted=1025), 2), (dict(vocab=0), 2), (dict(vocab=(1 << 22) + 1, ld=1 << 23, ld_d=1 << 23), 2),
    (dict(ld=7), 2), (dict(ld_d=7), 2), (dict(ld=1 << 60), 2), (dict(t=0.0), 11), (dict(td=0.0), 11), (dict(t=float("nan")), 11), (dict(td=float("inf")), 11), (dict(t=-1.0), 11),
    (dict(z=None), 1), (dict(ids=None), 1), (dict(tok=None), 1), (dict(acc=None), 1), (dict(z=A + 2), 6), (dict(d=A + 2), 6), (dict(ids=A + 2), 6), (dict(tok=A + 1), 6),
    (dict(acc=A + 2), 6), (dict(lp=A + 2), 6), (dict(st=A + 2), 6), (dict(off=A + 4), 6), (dict(batch=0, z=None), 0),
])
def test_verify_draft(lib, args, code):
    assert _verify(lib, **args) == code


def test_binding_refuses_host_tensors_and_bad_numbers():
    import torch
    x, one, ids = torch.zeros(4, 8), torch.zeros(4), torch.zeros(2, 1, dtype=torch.int32)
    for call in (lambda: tm.tm_dropout(x, 0.5, 1), lambda: tm.tm_rms_norm(x), lambda: tm.tm_rms_norm_e4m3(x), lambda: tm.tm_rms_norm_backward(x, x, one),
                 lambda: tm.tm_verify_draft(x, None, ids, 1)):
        with pytest.raises(tm.TmError):
            call()
    for seed, offset in ((-1, 0), (1 << 64, 0), (0, -1), (0, 1 << 64)):
        with pytest.raises(tm.TmError) as e:
            binding_branch._whole(seed, offset)
        assert e.value.code == tm.TM_ERR_RANGE
