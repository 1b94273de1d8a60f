"""Calls on a stream that is not torch's current one, without outputs or workspaces of the caller's: what they create belongs to that stream."""
from __future__ import annotations

import pytest
import torch

import paper_2102_08124_b200 as tm

pytestmark = pytest.mark.gpu
DELAY = 50_000_000                                                         # clocks, some 25 ms: far longer than the kernels of a call


def _calls():
    g = torch.Generator("cuda").manual_seed(5)
    x, dy = (torch.randn(512, 1024, device="cuda", generator=g) for _ in range(2))
    w = torch.rand(1024, device="cuda", generator=g)
    _, _, mean, rstd = tm.tm_layer_norm(x, w)
    z = torch.randn(96, 5000, device="cuda", generator=g)
    values, ids, lse = tm.tm_top_logits(z, 12)
    student = z + torch.randn(96, 5000, device="cuda", generator=g)
    _, stats = tm.tm_distill_loss(student, values, ids, lse)
    mask = tm.tm_find_mask_batched([x], 2, 4, tm.TM_APPROX)[0][0]
    other = tm.tm_nm_mask_1d(x, 2, 4)[0]
    first = lambda out: [t for t in out if t is not None]
    return {
        "layer_norm": lambda s: first(tm.tm_layer_norm(x, w, residual=dy, stream=s)),
        "layer_norm_backward": lambda s: first(tm.tm_layer_norm_backward(dy, x, mean, rstd, w, stream=s)),
        "top_logits": lambda s: first(tm.tm_top_logits(z, 12, stream=s)),
        "distill_loss": lambda s: first(tm.tm_distill_loss(student, values, ids, lse, stream=s)),
        "distill_grad": lambda s: [tm.tm_distill_grad(student, values, ids, stats, teacher_lse=lse, stream=s)],
        "distill_loss_grad": lambda s: first(tm.tm_distill_loss_grad(student, values, ids, lse, stream=s)),
        "find_mask_batched": lambda s: [o for part in tm.tm_find_mask_batched([x], 2, 4, tm.TM_APPROX, stream=s)[:2] for o in part],
        "nm_mask_1d": lambda s: first(tm.tm_nm_mask_1d(x, 2, 4, stream=s)),
        "mask_violations": lambda s: [tm.tm_mask_violations(x, mask, stream=s)],
        "mask_hamming": lambda s: [tm.tm_mask_hamming(mask, other, stream=s)],
        "compress_2_4": lambda s: first(tm.tm_compress_2_4(x, mask, stream=s)),
    }


NAMES = ["layer_norm", "layer_norm_backward", "top_logits", "distill_loss", "distill_grad", "distill_loss_grad", "find_mask_batched", "nm_mask_1d",
         "mask_violations", "mask_hamming", "compress_2_4"]


@pytest.mark.parametrize("name", NAMES)
def test_outputs_do_not_wait_for_the_current_stream(name):
    """The current stream is busy, and writes to memory that it has given back: neither reaches the call's outputs."""
    call = _calls()[name]
    want = [t.clone() for t in call(None)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(DELAY)
    for t in [torch.empty_like(o) for o in want] + [torch.empty(1 << 22, dtype=torch.uint8, device="cuda") for _ in range(4)]:
        t.fill_(77)                                                        # written after the delay, given back before the call
    del t
    got = call(side)
    side.synchronize()
    kept = [t.clone() for t in got]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) and torch.equal(c, b) for a, b, c in zip(got, want, kept))


@pytest.mark.parametrize("name", NAMES)
def test_hidden_workspaces_are_not_given_away(name):
    """A busy side stream still has the call before it when the current stream takes memory and fills it."""
    call = _calls()[name]
    want = [t.clone() for t in call(None)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(DELAY)
    got = call(side)
    mine = [torch.full((n,), 77, dtype=torch.uint8, device="cuda") for n in (256, 4096, 65536, 1 << 20, 1 << 21, 1 << 22, 1 << 23) for _ in range(4)]
    torch.cuda.synchronize()
    assert all(bool((t == 77).all()) for t in mine)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_stream_of_another_device_is_refused():
    class Elsewhere:
        device, cuda_stream = torch.device("cuda", 7), 0
    with pytest.raises(tm.TmError):
        tm.tm_layer_norm(torch.zeros(2, 8, device="cuda"), stream=Elsewhere())
