"""The example's network with dropout, forward and backward pass, in a captured graph: every replay drops other elements, those of an eager step at its
offset."""
from __future__ import annotations

import pytest
import torch

from paper_2102_08124_b200.distill import Blocks

pytestmark = pytest.mark.gpu
VOCAB, WIDTH, BLOCKS, ROWS, P, SEED, FIRST = 97, 48, 2, 40, 0.25, 11, (1 << 33) + 3


@pytest.mark.parametrize("norm", ["layer", "rms"])
def test_replays(norm):
    dense = Blocks(VOCAB, WIDTH, BLOCKS, torch.float32, "cuda", seed=3, norm=norm)
    g = torch.Generator("cuda").manual_seed(4)
    tokens, c = torch.randint(VOCAB, (ROWS,), device="cuda", generator=g), torch.randn(ROWS, VOCAB, device="cuda", generator=g)
    masked = [p.detach() * (torch.arange(p.shape[1], device="cuda") % 4 < 2) for p in dense.linear]
    step = torch.zeros(1, dtype=torch.int64, device="cuda")

    def once(offset, offset_dev):
        net = dense.copy()                                 # leaves of this pass alone
        out = net.logits(tokens, masked, P, SEED, offset, offset_dev)
        return [out.detach()] + list(torch.autograd.grad((out * c).sum(), list(net.parameters())))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        once(FIRST, step)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = once(FIRST, step)
        step += BLOCKS + 1
    step.zero_()
    before = None
    for i in range(3):
        graph.replay()
        # the same kernels on the same numbers, but for library products, which may split a sum otherwise: 400 additions of fp32 at most in each of a
        # dozen layers one after the other
        want = once(FIRST + i * (BLOCKS + 1), None)
        for a, b in zip(got, want):
            assert float((a - b).abs().max()) <= 1e-4 * float(b.abs().max())
        if before is not None:
            assert not torch.allclose(got[0], before, rtol=1e-2, atol=1e-2)
        before = got[0].clone()
