"""Dropout from the counter-based generator against a 64-bit form: which elements stay is exact."""
from __future__ import annotations

import numpy as np
import pytest

from tests import branch_ref as ref

SEED, OFFSET = 0xFEDCBA9876543210, (7 << 32) + 5


def test_generator_gives_the_published_words():
    words = lambda c, k: ref.philox(c[0], c[1], c[2] | c[3] << 32, k[0] | k[1] << 32).tolist()
    ones = 0xFFFFFFFF
    assert words((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert words((ones,) * 4, (ones,) * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert words((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0)) == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def _matrix(rows, cols, dtype, layout, seed):
    """A device matrix and its values: side by side, padded rows on 16-byte boundaries, or rows that start anywhere."""
    import torch
    kind = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    g = torch.Generator().manual_seed(seed)
    wide = {"plain": cols, "padded": (cols + 15) // 8 * 8, "off": cols + 3}[layout]
    t = torch.randn(rows, wide, generator=g).to(kind).cuda()
    t = t[:, 1:cols + 1] if layout == "off" else t[:, :cols]
    return t, t.double().cpu().numpy()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,layout", [(1, 1, "plain"), (3, 7, "plain"), (2, 8, "plain"), (5, 9, "off"), (64, 1024, "plain"), (33, 1001, "plain"),
                                              (7, 1001, "padded"), (1, 70001, "plain"), (300, 264, "off"), (4097, 40, "padded")])
@pytest.mark.parametrize("p,residual", [(0.1, False), (0.5, True), (0.0, True), (0.99999, False)])
def test_dropout(rows, cols, layout, dtype, p, residual):
    import paper_2102_08124_b200 as tm
    x, x64 = _matrix(rows, cols, dtype, layout, 1)
    r, r64 = _matrix(rows, cols, dtype, layout, 2) if residual else (None, None)
    y = tm.tm_dropout(x, p, SEED, OFFSET, residual=r).double().cpu().numpy()
    want, bound = ref.total(x64, r64, p, SEED, OFFSET)
    assert (np.abs(y - want) <= bound + ref.out_unit(dtype) * (np.abs(want) + bound)).all()
    if not residual and p > 0:
        stay, _ = ref.kept(rows, cols, p, SEED, OFFSET)
        assert np.array_equal(y != 0, stay & (x64 != 0))


@pytest.mark.gpu
def test_share_that_stays():
    import torch
    import paper_2102_08124_b200 as tm
    for p in (0.1, 0.25, 0.9):
        y = tm.tm_dropout(torch.ones(1024, 1024, device="cuda"), p, 11)
        n, q = 1 << 20, 1 - round(65536 * p) / 65536
        assert abs(float((y != 0).sum()) - n * q) < 6 * (n * q * (1 - q)) ** 0.5
        assert abs(float(y.double().mean()) - 1) < 6 * ((1 - q) / q / n) ** 0.5


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_what_is_dropped_is_gone(dtype):
    """Inf and NaN do not reach the output from a dropped place; with a residual its value stands there."""
    import torch
    import paper_2102_08124_b200 as tm
    kind = getattr(torch, dtype)
    x = torch.full((16, 100), float("nan"), device="cuda", dtype=kind)
    x[8:] = float("inf")
    r = torch.randn(16, 100, device="cuda").to(kind)
    stay = torch.from_numpy(ref.kept(16, 100, 0.5, 3, 0)[0]).cuda()
    y, z = tm.tm_dropout(x, 0.5, 3), tm.tm_dropout(x, 0.5, 3, residual=r)
    assert bool((y[~stay] == 0).all()) and torch.equal(z[~stay], r[~stay])
    assert bool(torch.isnan(y[:8][stay[:8]]).all()) and bool((y[8:][stay[8:]] == float("inf")).all())


@pytest.mark.gpu
def test_seeds_offsets_and_the_device_offset():
    import torch
    import paper_2102_08124_b200 as tm
    x = torch.ones(64, 512, device="cuda")
    base = tm.tm_dropout(x, 0.3, 5, 100)
    assert torch.equal(base, tm.tm_dropout(x, 0.3, 5, 100))
    for seed, offset in ((6, 100), (5, 101), (5 + (1 << 32), 100), (5, 100 + (1 << 32))):
        assert not torch.equal(base, tm.tm_dropout(x, 0.3, seed, offset))
    step = torch.tensor([60], dtype=torch.int64, device="cuda")
    assert torch.equal(base, tm.tm_dropout(x, 0.3, 5, 40, offset_dev=step))
    assert torch.equal(tm.tm_dropout(x, 0.3, 5, (1 << 64) - 10, offset_dev=step), tm.tm_dropout(x, 0.3, 5, 50))      # modulo 2^64


@pytest.mark.gpu
def test_in_place_and_the_gradient_is_the_same_call():
    import torch
    import paper_2102_08124_b200 as tm
    x, r = torch.randn(37, 333, device="cuda"), torch.randn(37, 333, device="cuda")
    want = tm.tm_dropout(x, 0.2, 9, residual=r)
    a, b = x.clone(), r.clone()
    assert tm.tm_dropout(a, 0.2, 9, residual=r, y=a) is a and torch.equal(a, want)
    assert tm.tm_dropout(x, 0.2, 9, residual=b, y=b) is b and torch.equal(b, want)
    dy = torch.randn(37, 333, device="cuda")
    stay, factor = ref.kept(37, 333, 0.2, 9, 0)
    back = tm.tm_dropout(dy, 0.2, 9).double().cpu().numpy()
    assert np.allclose(back, dy.double().cpu().numpy() * stay * factor, rtol=3 * ref.U32, atol=0)


@pytest.mark.gpu
def test_nothing_to_do():
    import torch
    import paper_2102_08124_b200 as tm
    for shape in ((0, 8), (8, 0), (0, 0)):
        assert tm.tm_dropout(torch.empty(shape, device="cuda"), 0.5, 1).shape == shape
