"""The autograd forms of dropout and the root-mean-square norm against 64-bit autograd, and the operators together: a student that trains with
them, drafts for its teacher, and is checked."""
from __future__ import annotations

import os
import subprocess
import sys

import pytest

from tests import branch_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SEED, OFFSET = 77, 5


def test_import_needs_no_device():
    code = "import paper_2102_08124_b200.branch, paper_2102_08124_b200.draft, sys; assert 'torch' not in sys.modules"
    subprocess.run([sys.executable, "-c", code], cwd=ROOT, check=True)


# fp32 against fp64: a gradient is a sum of n terms of which each takes a few roundings, an error of some n^(1/2) 2^-24 against terms
# of their sum's size; 1e-4 of the largest entry leaves a factor of about 30 at n = 400.
TOL = 1e-4


def close(got, want, tol=TOL):
    assert float((got.double() - want).abs().max()) <= tol * float(want.abs().max())


def drop64(x, p, seed, offset):
    import torch
    if p == 0:
        return x
    stay, factor = ref.kept(x.numel() // x.shape[-1], x.shape[-1], p, seed, offset)
    return torch.where(torch.from_numpy(stay).cuda().view(x.shape), x * factor, 0.0)


@pytest.mark.gpu
@pytest.mark.parametrize("p", [0.0, 0.3])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("use", ["y", "sum", "both"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_rms_norm_gradients(p, residual, use, dtype):
    import torch
    from paper_2102_08124_b200.branch import rms_norm
    torch.manual_seed(3)
    kind = getattr(torch, dtype)
    leaf = lambda *s: torch.randn(*s, device="cuda").to(kind).requires_grad_()
    x, r, w = leaf(2, 7, 100), leaf(2, 7, 100), leaf(100)
    c, e = (torch.randn(2, 7, 100, device="cuda").to(kind) for _ in range(2))
    y, h = rms_norm(x, w, 1e-5, residual=r if residual else None, p=p, seed=SEED, offset=OFFSET)
    X, R, W = (t.detach().double().requires_grad_() for t in (x, r, w))
    H = drop64(X, p, SEED, OFFSET) + (R if residual else 0)
    Y = H / (H.square().mean(-1, keepdim=True) + 1e-5).sqrt() * W
    pick = lambda a, b, u, v: (a * u).sum() * (use != "sum") + (b * v).sum() * (use != "y")
    pick(y, h, c, e).backward()
    pick(Y, H, c.double(), e.double()).backward()
    # bf16: y, the sum (which the backward pass takes) and the gradients are rounded, 2^-8 each, and gradients add where the sum is x itself
    tol = TOL if dtype == "float32" else 4 * 2.0 ** -8
    close(y.detach(), Y.detach(), tol)
    pairs = [(x, X)] + ([(r, R)] if residual else []) + ([(w, W)] if use != "sum" else [])
    for got, want in pairs:
        close(got.grad, want.grad, tol)
    assert residual or r.grad is None


@pytest.mark.gpu
@pytest.mark.parametrize("residual", [False, True])
def test_dropout_gradients_of_first_and_second_order(residual):
    import torch
    from paper_2102_08124_b200.branch import dropout
    x, r = (torch.randn(3, 5, 60, device="cuda", requires_grad=True) for _ in range(2))
    y = dropout(x, 0.4, SEED, OFFSET, residual=r if residual else None)
    X, R = (t.detach().double().requires_grad_() for t in (x, r))
    Y = drop64(X, 0.4, SEED, OFFSET) + (R if residual else 0)
    close(y.detach(), Y.detach())
    y.pow(3).sum().backward(retain_graph=True)
    Y.pow(3).sum().backward(retain_graph=True)
    close(x.grad, X.grad)
    if residual:
        close(r.grad, R.grad)
    g, G = (torch.autograd.grad(b.pow(3).sum(), a, create_graph=True)[0] for a, b in ((x, y), (X, Y)))
    close(torch.autograd.grad(g.square().sum(), x)[0], torch.autograd.grad(G.square().sum(), X)[0])


@pytest.mark.gpu
def test_refusals_and_second_derivatives():
    import torch
    from paper_2102_08124_b200 import TmError
    from paper_2102_08124_b200.branch import dropout, rms_norm
    x = torch.randn(2, 3, 16, device="cuda", requires_grad=True)
    for other in (x.transpose(0, 1), x.reshape(6, 16), x[:1], x[..., :8]):
        for f in (lambda: rms_norm(x, residual=other), lambda: dropout(x, 0.5, 1, residual=other)):
            with pytest.raises(TmError):
                f()
    y, _ = rms_norm(x, p=0.5, seed=1)
    (g,) = torch.autograd.grad(y.square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        g.square().sum().backward()


@pytest.mark.gpu
def test_a_raised_device_offset_is_seen_before_the_backward_pass():
    """The backward pass would drop other elements than the forward pass did: autograd refuses."""
    import torch
    from paper_2102_08124_b200.branch import dropout, rms_norm
    x, step = torch.randn(4, 32, device="cuda", requires_grad=True), torch.zeros(1, dtype=torch.int64, device="cuda")
    for f in (lambda: dropout(x, 0.5, 1, offset_dev=step), lambda: rms_norm(x, p=0.5, seed=1, offset_dev=step)[0]):
        y = f()
        step += 1
        with pytest.raises(RuntimeError):
            y.sum().backward()


@pytest.mark.gpu
@pytest.mark.parametrize("norm", ["layer", "rms"])
def test_a_captured_step_draws_new_numbers_at_every_replay(norm):
    """Forward and backward pass of the example's network in a graph, against eager steps at the same offsets."""
    import torch
    from paper_2102_08124_b200.branch import dropout, rms_norm
    x, dy, w = torch.randn(32, 96, device="cuda"), torch.randn(32, 96, device="cuda"), torch.rand(96, device="cuda")
    step = torch.zeros(1, dtype=torch.int64, device="cuda")

    def once(offset, offset_dev, leaf):
        h = rms_norm(leaf, w, p=0.25, seed=9, offset=offset, offset_dev=offset_dev)[0] if norm == "rms" else leaf * 1
        y = dropout(h, 0.25, 9, offset + 1000, residual=x, offset_dev=offset_dev)
        return y.detach(), torch.autograd.grad(y, leaf, dy)[0]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        once(0, step, x.clone().requires_grad_())
    torch.cuda.current_stream().wait_stream(side)
    leaf = x.clone().requires_grad_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, g = once(0, step, leaf)
        step += 1
    step.zero_()
    for i in range(3):
        graph.replay()
        want = once(i, None, x.clone().requires_grad_())
        assert torch.equal(y, want[0]) and torch.equal(g, want[1])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_the_network_with_dropout_and_rms_norm(dtype):
    """Logits and gradients of the whole student (masked layers, norms, dropout) against the same network in 64 bits."""
    import torch
    from paper_2102_08124_b200.distill import Blocks
    torch.manual_seed(0)
    net = Blocks(97, 48, 2, getattr(torch, dtype), "cuda", norm="rms").copy()
    masked = [p.detach() * (torch.arange(p.shape[1], device="cuda") % 4 < 2) for p in net.linear]
    tokens = torch.randint(97, (40,), device="cuda")
    out = net.logits(tokens, masked, 0.2, SEED, OFFSET)
    c = torch.randn(40, 97, device="cuda")
    (out.float() * c).sum().backward()
    to64 = lambda t: t.detach().double()
    weights, masks = [to64(p).requires_grad_() for p in net.linear], [to64(p) for p in masked]
    norms, embedding, head = [to64(p).requires_grad_() for p in net.norm_weight], to64(net.embedding), to64(net.head)

    class Through(torch.autograd.Function):                # the dense copy's gradient is that of the masked weight
        @staticmethod
        def forward(ctx, dense, kept):
            return kept.clone()

        @staticmethod
        def backward(ctx, g):
            return g, None

    h, update = embedding[tokens], None
    for i in range(3):
        h = h if update is None else h + drop64(update, 0.2, SEED, OFFSET + i)
        y = h / (h.square().mean(-1, keepdim=True) + 1e-5).sqrt() * norms[i]
        if i < 2:
            a, b = (Through.apply(weights[2 * i + k], masks[2 * i + k]) for k in (0, 1))
            update = torch.nn.functional.gelu(y @ a.t()) @ b.t()
    want = y @ head.t()
    (want * c).sum().backward()
    # bf16: every layer's tensors are rounded to 2^-8 of themselves, some 30 roundings one after the other, which add up like a random walk
    tol = 2e-4 if dtype == "float32" else 12 * 2.0 ** -8
    close(out.detach(), want.detach(), tol)
    for got, w64 in list(zip(net.linear, weights)) + list(zip(net.norm_weight, norms)):
        close(got.grad, w64.grad, tol)


@pytest.mark.gpu
@pytest.mark.parametrize("norm,dropout", [("rms", 0.1), ("rms", 0.0), ("layer", 0.1)])
def test_example_trains(norm, dropout):
    from paper_2102_08124_b200.distill import train
    losses = train(steps=3, rows=64, vocab=515, width=64, blocks=1, k=8, evaluate=1, norm=norm, dropout=dropout)
    assert len(losses) == 4 and all(l == l and l >= 0 for l in losses)


@pytest.mark.gpu
def test_example_drafts():
    """Tokens of a round: the drafts that stayed, one more from the vocabulary, -1 behind; a drafter that is the target keeps all its drafts."""
    import torch
    from paper_2102_08124_b200 import draft
    from paper_2102_08124_b200.distill import Blocks
    target, other = (Blocks(515, 64, 1, torch.float32, "cuda", seed=k, norm="rms") for k in (0, 1))
    last = torch.randint(515, (50,), device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    with torch.no_grad():
        out, accepted = draft.speculate(target.logits, other.logits, last, 3, 1, status=status)
        for b in range(50):
            n = int(accepted[b])
            assert all(0 <= t < 515 for t in out[b, :n + 1].tolist()) and all(t == -1 for t in out[b, n + 1:].tolist())
        out, accepted = draft.speculate(target.logits, target.logits, last, 3, 1)
        assert bool((accepted == 3).all())
        out, accepted = draft.speculate(target.logits, other.logits, last, 0, 1)
        assert out.shape == (50, 1) and bool((accepted == 0).all())
    assert int(status) == 0
    shares = draft.run(steps=2, rows=64, vocab=515, width=64, blocks=1, drafts=2, rounds=2, batch=16)
    assert len(shares) == 3 and all(0 <= s <= 1 for s in shares)


@pytest.mark.gpu
def test_a_product_in_eight_bits():
    """The norm's 8-bit output times 8-bit weights against the product in 64 bits of what they stand for."""
    import torch
    import paper_2102_08124_b200 as tm
    from paper_2102_08124_b200.draft import Rows8
    x, w = torch.randn(48, 256, device="cuda", dtype=torch.bfloat16), torch.randn(96, 256, device="cuda")
    y8, scales, _ = tm.tm_rms_norm_e4m3(x)
    rows = Rows8(w)
    got = rows.product(y8, scales).double()
    want = (y8.double() * scales.double()) @ (rows.values.double() * rows.scale.double()).t()
    size = (y8.double() * scales.double()).abs() @ (rows.values.double() * rows.scale.double()).abs().t()
    # products of e4m3 numbers are exact in fp32; 256 additions of at least 14 bits, and the rounding to bf16
    assert bool(((got - want).abs() <= 256 * 2.0 ** -14 * size + 2.0 ** -8 * want.abs()).all())
