"""Rows that all start off a 16-byte boundary, more of them than a grid takes in one turn: the norm, its 8-bit output and its backward pass against the
64-bit formulas, and rows between rows of NaN."""
from __future__ import annotations

import pytest
import torch

import paper_2102_08124_b200 as tm
import tests.test_branch_rms as rms

pytestmark = pytest.mark.gpu


# Rows side by side: each repeats the lead of the one `period` rows above it.  Widths for every number of threads that share a row.
@pytest.mark.parametrize("residual,p", [(False, 0.0), (True, 0.0), (True, 0.1), (False, 0.4)])
@pytest.mark.parametrize("rows,cols,dtype", [(5000, 3001, "f32"), (1500, 2050, "f32"), (1200, 4093, "f32"), (9000, 99, "bf16"), (9000, 300, "bf16"), (5000, 999, "bf16"),
                                             (3000, 1001, "bf16"), (3000, 3001, "bf16"), (1001, 5002, "bf16"), (700, 8180, "bf16"), (500, 9001, "bf16")])
def test_forward(rows, cols, dtype, residual, p):
    rms.test_forward(rows, cols, "plain", dtype, residual, p)


@pytest.mark.parametrize("dsum,p", [(False, 0.0), (True, 0.0), (True, 0.1), (False, 0.4)])
@pytest.mark.parametrize("rows,cols,dtype", [(2000, 3001, "f32"), (9000, 99, "bf16"), (9000, 300, "bf16"), (5000, 999, "bf16"), (3000, 1001, "bf16"), (3000, 3001, "bf16"),
                                             (1001, 5002, "bf16"), (700, 8180, "bf16"), (500, 9001, "bf16")])
def test_backward(rows, cols, dtype, dsum, p):
    rms.test_backward(rows, cols, "plain", dtype, dsum, p)


@pytest.mark.parametrize("group", [0, 64])
@pytest.mark.parametrize("rows,cols,dtype", [(5000, 3001, "f32"), (1200, 4093, "f32"), (5000, 999, "bf16"), (3000, 1001, "bf16"), (2000, 3001, "bf16"), (501, 9001, "bf16")])
def test_eight_bits(rows, cols, dtype, group):
    rms.test_eight_bits(rows, cols, "plain", dtype, group)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,cols", [(37, 9), (37, 255), (37, 1001), (4001, 1001), (37, 2500), (37, 3001), (2001, 3001), (37, 4091), (37, 5001), (37, 9001), (37, 16377)])
def test_rows_do_not_see_their_neighbours(rows, cols, dtype):
    """Without dropout: every other row is NaN and Inf; the rows between, and what lies before and behind the matrices, stay as they are."""
    kind, guard = getattr(torch, dtype), 32
    g = torch.Generator("cuda").manual_seed(cols)
    for shift in (0, 3):
        def inside(store):
            return store[16 + shift:16 + shift + rows * cols].view(rows, cols)

        part = {k: inside(torch.randn(rows * cols + guard, device="cuda", generator=g).to(kind)) for k in ("x", "r", "dy", "e")}
        for t in part.values():
            t[1::2] = float("nan")
            t[1::2, ::2] = float("inf")
        w = torch.rand(cols, device="cuda", generator=g)
        out = {k: torch.full((rows * cols + guard,), 7.0, device="cuda", dtype=kind) for k in ("y", "s", "dh", "s8")}
        out["y8"] = torch.full((rows * cols + guard,), 7.0, device="cuda").to(torch.float8_e4m3fn)
        o = {k: inside(t) for k, t in out.items()}
        _, _, rstd = tm.tm_rms_norm(part["x"], w, residual=part["r"], y=o["y"], sum_out=o["s"])
        tm.tm_rms_norm_backward(part["dy"], o["s"], rstd, w, dsum=part["e"], dh=o["dh"])
        _, scales, _ = tm.tm_rms_norm_e4m3(part["x"], w, residual=part["r"], y8=o["y8"], sum_out=o["s8"])
        alone = {k: t.clone().nan_to_num(0.0, 0.0, 0.0) for k, t in part.items()}
        y, s, r2 = tm.tm_rms_norm(alone["x"], w, residual=alone["r"])
        dh, _, _ = tm.tm_rms_norm_backward(alone["dy"], s, r2, w, dsum=alone["e"])
        _, scales2, _ = tm.tm_rms_norm_e4m3(alone["x"], w, residual=alone["r"])
        for got, want in ((o["y"], y), (o["dh"], dh)):
            # the same kernel or one that adds a row's terms in another order, of which the row's factor holds 2^-18
            assert torch.allclose(got[::2].float(), want[::2].float(), rtol=2.0 ** -7 if dtype == "bfloat16" else 2.0 ** -16, atol=1e-5)
        assert torch.equal(o["s"][::2], s[::2]) and torch.equal(o["s8"][::2], s[::2])      # one addition and one rounding
        assert torch.allclose(scales[::2], scales2[::2], rtol=2.0 ** -18)
        # y from its 8 bits: half a step of 2^-3, or of the smallest numbers' 2^-9, times the scale
        assert bool(((o["y8"].float() * scales)[::2] - y[::2].float()).abs().le(y[::2].float().abs() * (2.0 ** -4 + 2.0 ** -7) + scales[::2] * 2.0 ** -9).all())
        for t in out.values():
            v = t.float()
            assert bool((v[:16 + shift] == 7).all()) and bool((v[16 + shift + rows * cols:] == 7).all())
