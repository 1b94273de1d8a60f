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
