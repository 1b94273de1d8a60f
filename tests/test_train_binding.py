"""What the binding of the training operators refuses, and what it does with buffers of the caller's."""
from __future__ import annotations

import pytest
import torch

import paper_2102_08124_b200 as tm

pytestmark = pytest.mark.gpu


def test_a_workspace_that_the_gpu_cannot_use_is_refused():
    x, stat = torch.zeros(4, 8, device="cuda"), torch.zeros(4, device="cuda")
    n = tm.tm_layer_norm_workspace_bytes(4, 8)
    for workspace in (torch.empty(n, dtype=torch.uint8), torch.empty(n, dtype=torch.uint8).pin_memory(), torch.empty(2 * n, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(tm.TmError):
            tm.tm_layer_norm_backward(x, x, stat, stat, workspace=workspace)
    tm.tm_layer_norm_backward(x, x, stat, stat, workspace=torch.empty(n, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [40, 1001, 9000, 20000])
def test_a_sum_that_was_passed_in_is_written_without_a_residual(cols, dtype):
    x = torch.randn(7, cols, device="cuda").to(dtype)
    out = torch.full_like(x, float("nan"))
    y, s, _, _ = tm.tm_layer_norm(x, sum_out=out)
    assert s is out and torch.equal(out, x) and torch.equal(y, tm.tm_layer_norm(x)[0]) and tm.tm_layer_norm(x)[1] is None
