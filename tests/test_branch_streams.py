"""The residual branch's operators and draft verification on other streams than torch's current one, two at once, and in captured graphs."""
from __future__ import annotations

import pytest
import torch

import paper_2102_08124_b200 as tm

pytestmark = pytest.mark.gpu
DELAY = 50_000_000                                                         # clocks, some 25 ms: far longer than the kernels of a call


def _calls():
    g = torch.Generator("cuda").manual_seed(5)
    x, r, dy = (torch.randn(512, 1024, device="cuda", generator=g) for _ in range(3))
    w = torch.rand(1024, device="cuda", generator=g)
    _, h, rstd = tm.tm_rms_norm(x, w, residual=r)
    z = torch.randn(64, 5000, device="cuda", generator=g)
    d = z.view(16, 4, 5000)[:, :3].reshape(48, 5000) + 0.5 * torch.randn(48, 5000, device="cuda", generator=g)
    ids = torch.randint(5000, (16, 3), device="cuda", generator=g, dtype=torch.int32)
    first = lambda out: [t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t for t in out if t is not None]
    return {
        "dropout": lambda s: [tm.tm_dropout(x, 0.3, 1, residual=r, stream=s)],
        "rms_norm": lambda s: first(tm.tm_rms_norm(x, w, residual=r, p=0.2, seed=3, stream=s)),
        "rms_norm_e4m3": lambda s: first(tm.tm_rms_norm_e4m3(x, w, residual=r, group=64, stream=s)),
        "rms_norm_backward": lambda s: first(tm.tm_rms_norm_backward(dy, h, rstd, w, p=0.2, seed=3, stream=s)),
        "verify_draft": lambda s: first(tm.tm_verify_draft(z, d, ids, 7, stream=s)),
        "verify_none": lambda s: first(tm.tm_verify_draft(z, None, ids[:0].new_empty(64, 0), 7, stream=s)),
    }


NAMES = ["dropout", "rms_norm", "rms_norm_e4m3", "rms_norm_backward", "verify_draft", "verify_none"]


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


@pytest.mark.parametrize("name", NAMES)
def test_two_streams_at_once_and_two_captured_graphs(name):
    """Calls that overlap, eager and replayed, share nothing."""
    call = _calls()[name]
    want = [t.clone() for t in call(None)]
    sides, got = [torch.cuda.Stream() for _ in range(2)], []
    for s in sides:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        got += [call(s) for s in sides]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(call(None))
        graphs.append(g)
    for _ in range(3):
        for o in outs:
            for t in o:
                t.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, sides):
            with torch.cuda.stream(s):
                for _ in range(4):
                    g.replay()
        torch.cuda.synchronize()
        got += [[t.clone() for t in o] for o in outs]
    assert all(torch.equal(a, b) for o in got for a, b in zip(o, want))


def test_a_stream_of_another_device_is_refused():
    class Elsewhere:
        device, cuda_stream = torch.device("cuda", 7), 0
    x = torch.zeros(2, 8, device="cuda")
    for call in (lambda s: tm.tm_dropout(x, 0.5, 1, stream=s), lambda s: tm.tm_rms_norm(x, stream=s), lambda s: tm.tm_rms_norm_e4m3(x, stream=s),
                 lambda s: tm.tm_verify_draft(x, None, torch.zeros(2, 0, device="cuda", dtype=torch.int32), 1, stream=s)):
        with pytest.raises(tm.TmError):
            call(Elsewhere())


def test_device_offset_in_a_graph():
    x, step = torch.ones(8, 256, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    z = torch.randn(8, 500, device="cuda")
    none = torch.zeros(8, 0, device="cuda", dtype=torch.int32)
    calls = lambda offset, dev: (tm.tm_dropout(x, 0.5, 3, offset, offset_dev=dev), tm.tm_rms_norm(x, p=0.5, seed=3, offset=offset, offset_dev=dev)[0],
                                 tm.tm_rms_norm_backward(x, x, x[:, 0].contiguous(), p=0.5, seed=3, offset=offset, offset_dev=dev)[1],
                                 tm.tm_verify_draft(z, None, none, 3, offset, offset_dev=dev)[0])
    calls(0, step)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        outs = calls(10, step)
        step += 1
    step.zero_()
    for i in range(3):
        g.replay()
        assert all(torch.equal(a, b) for a, b in zip(outs, calls(10 + i, None)))
