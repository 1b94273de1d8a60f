"""A pruned network trained against the dense one that it came from: autograd forms of the layer norm with residual sum and of the
distillation loss, the teacher's side of it, and a small example that runs them with the masked layers.

    python -m paper_2102_08124_b200.distill --steps 60

The teacher keeps, for every token, its k largest logits and the log-sum-exp of all of them (k 8-byte entries instead of the whole
vocabulary); the student's loss is the divergence from that, with the unlisted logits as one more class."""
from __future__ import annotations

import argparse
from typing import NamedTuple, Optional

from . import binding as tm
from . import binding_train as tt
from .branch import _rows, dropout, rms_norm
from .refresh import MaskRefresher, masked_linear

_functions = None


class TeacherLists(NamedTuple):
    """What the loss needs of a teacher's logits [rows, vocab], at one temperature."""
    values: object              # float32 [rows, k], largest first
    ids: object                 # int32 [rows, k]
    lse: object                 # float32 [rows]
    temperature: float


def teacher_lists(logits, k: int, temperature: float = 1.0, status=None) -> TeacherLists:
    values, ids, lse = tt.tm_top_logits(logits.detach(), k, temperature, status=status)
    return TeacherLists(values, ids, lse, temperature)


def _make():
    import torch
    from torch.autograd.function import once_differentiable              # second derivatives are refused, not left out

    class Norm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, residual, weight, bias, eps):
            if residual is not None and residual.shape != x.shape:       # rows of other shapes could still be as many
                raise tm.TmError(2, "residual must have the shape of x")
            x2 = _rows(x)
            # outputs of x's shape, of which the kernel gets views: a view itself could not be written to in place
            y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
            h = None if residual is None else torch.empty_like(y)
            _, _, mean, rstd = tt.tm_layer_norm(x2, weight, bias, eps, residual=None if residual is None else _rows(residual), y=y.view(x2.shape),
                                                sum_out=None if h is None else h.view(x2.shape))
            ctx.save_for_backward(x2 if h is None else h, mean, rstd, weight)
            ctx.shape, ctx.params = x.shape, (weight is not None or bias is not None, bias.dtype if bias is not None else None)
            ctx.set_materialize_grads(False)
            # without a residual the sum is x itself, whose other uses reach x by their own way
            return y, h

        @staticmethod
        @once_differentiable
        def backward(ctx, dy, dsum):
            h, mean, rstd, weight = ctx.saved_tensors
            h = _rows(h)
            want = ctx.params[0] and any(ctx.needs_input_grad[2:4])
            dsum = None if dsum is None else _rows(dsum)
            if dy is None:                                  # only the sum was used
                dy = torch.zeros_like(h)
            dx, dw, db = tt.tm_layer_norm_backward(_rows(dy), h, mean, rstd, weight, dsum=dsum, want_params=want, params_dtype=ctx.params[1])
            dx = dx.view(ctx.shape)
            need = ctx.needs_input_grad
            return dx if need[0] else None, dx if need[1] else None, dw if need[2] else None, db if need[3] else None, None

    class Loss(torch.autograd.Function):
        @staticmethod
        def forward(ctx, logits, values, ids, lse, row_weight, temperature, scale, status):
            z = _rows(logits)
            loss, stats = tt.tm_distill_loss(z, values, ids, lse, row_weight, temperature, scale, want_stats=ctx.needs_input_grad[0], status=status)
            ctx.save_for_backward(z, values, ids, lse, row_weight, stats)
            ctx.scalars = (temperature, scale, logits.shape)
            return loss

        @staticmethod
        @once_differentiable
        def backward(ctx, grad):
            z, values, ids, lse, row_weight, stats = ctx.saved_tensors
            temperature, scale, shape = ctx.scalars
            d = tt.tm_distill_grad(z, values, ids, stats, grad.contiguous(), lse, row_weight, temperature, scale)
            return (d.view(shape),) + (None,) * 7

    return Norm, Loss


def _get():
    global _functions
    if _functions is None:
        _functions = _make()
    return _functions


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, residual=None):
    """Differentiable layer norm over the last dimension of x (+ residual).  Returns (y, the sum), the sum being x without a residual."""
    y, h = _get()[0].apply(x, residual, weight, bias, eps)
    return y, x if residual is None else h


def distill_loss(logits, teacher: TeacherLists, row_weight=None, scale: float = 1.0, status=None):
    """Differentiable loss of every row of logits [..., vocab] (float32 [rows]).  status (int32[1] or None): TM_DEV_BADID for ids that were left out."""
    import torch
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (teacher.values, teacher.lse, row_weight)):
        raise tm.TmError(2, "the loss has a gradient for its logits alone: detach the teacher's lists and the row weights")
    return _get()[1].apply(logits, teacher.values, teacher.ids, teacher.lse, row_weight, teacher.temperature, scale, status)


def distill_backward(logits, teacher: TeacherLists, row_weight=None, scale: float = 1.0, status=None):
    """Adds the gradient of the summed loss to everything that logits [..., vocab] came from, and returns the loss of every row: loss and
    gradient in one pass over the logits, for a step that has no other use of the loss."""
    loss, d = tt.tm_distill_loss_grad(_rows(logits.detach()), teacher.values, teacher.ids, teacher.lse, row_weight, teacher.temperature, scale, status=status)
    logits.backward(d.view(logits.shape))
    return loss


class Blocks:
    """A small pre-norm network over token ids: embedding, blocks of norm, wide linear, gelu, linear, and a norm before the output layer.
    norm: "layer", or "rms" (without the biases)."""

    def __init__(self, vocab: int, width: int, blocks: int, dtype, device, seed: int = 0, norm: str = "layer"):
        import torch
        if norm not in ("layer", "rms"):
            raise ValueError("norm must be layer or rms")
        self.norm = norm
        g = torch.Generator(device="cpu").manual_seed(seed)

        def weight(rows, cols, scale):
            return (torch.randn(rows, cols, generator=g) * scale).to(device=device, dtype=dtype)

        self.embedding = weight(vocab, width, 1.0)
        self.linear = []                                    # in, out, in, out, ...
        for _ in range(blocks):
            self.linear += [weight(4 * width, width, width ** -0.5), weight(width, 4 * width, (4 * width) ** -0.5)]
        self.norm_weight = [torch.ones(width, dtype=dtype, device=device) for _ in range(blocks + 1)]
        self.norm_bias = [torch.zeros(width, dtype=dtype, device=device) for _ in range(blocks + 1)] if norm == "layer" else []
        self.head = weight(vocab, width, 2.0 * width ** -0.5)

    def parameters(self):
        return self.linear + self.norm_weight + self.norm_bias

    def copy(self) -> "Blocks":
        other = object.__new__(Blocks)
        other.norm = self.norm
        other.embedding, other.head = self.embedding, self.head          # shared, not trained
        for name in ("linear", "norm_weight", "norm_bias"):
            setattr(other, name, [p.detach().clone().requires_grad_() for p in getattr(self, name)])
        return other

    def _norm(self, i, update, h, p, seed, offset, offset_dev):
        """Norm i of h + dropout(update): (y, the sum)."""
        if self.norm == "rms":
            return rms_norm(h if update is None else update, self.norm_weight[i], residual=None if update is None else h, p=0.0 if update is None else p,
                            seed=seed, offset=offset + i, offset_dev=offset_dev)
        if update is not None and p > 0:
            h, update = dropout(update, p, seed, offset + i, residual=h, offset_dev=offset_dev), None
        return layer_norm(h if update is None else update, self.norm_weight[i], self.norm_bias[i], residual=None if update is None else h)

    def logits(self, tokens, masked: Optional[list] = None, p: float = 0.0, seed: int = 0, offset: int = 0, offset_dev=None):
        """masked: the linear layers' masked weights; None runs the dense ones.  p: dropout of the blocks' outputs, from seed and as many offsets as
        there are norms.  offset_dev (int64[1] on the device, or None) is added to them when the kernels run: for a captured step, which raises it by
        that many behind its backward pass."""
        import torch
        h, update = self.embedding[tokens], None
        for i in range(len(self.linear) // 2):
            y, h = self._norm(i, update, h, p, seed, offset, offset_dev)
            a, b = self.linear[2 * i], self.linear[2 * i + 1]
            if masked is None:
                update = torch.nn.functional.gelu(y @ a.t()) @ b.t()
            else:
                update = masked_linear(torch.nn.functional.gelu(masked_linear(y, a, masked[2 * i])), b, masked[2 * i + 1])
        y, _ = self._norm(len(self.linear) // 2, update, h, p, seed, offset, offset_dev)
        return y @ self.head.t()


def train(steps: int = 60, rows: int = 512, vocab: int = 4099, width: int = 256, blocks: int = 2, k: int = 32, temperature: float = 2.0,
          lr: float = 1e-3, period: int = 1, dtype=None, device: str = "cuda", seed: int = 0, evaluate: int = 20, report=None, norm: str = "layer",
          dropout: float = 0.0, networks: Optional[list] = None):
    """Distils a dense network into its 2:4 transposable pruning; returns the mean losses on held-out tokens, before, during and after.
    dropout: of the student's blocks while it trains.  networks: a list that receives the teacher, the student and the student's masked weights."""
    import torch
    dtype = dtype or torch.float32
    teacher = Blocks(vocab, width, blocks, dtype, device, seed, norm)
    student = teacher.copy()
    refresher = MaskRefresher([p.detach() for p in student.linear], N=2, M=4, period=period, method=tm.TM_EXACT, use_graph=False)
    optimizer = torch.optim.Adam(student.parameters(), lr=lr)
    g = torch.Generator(device="cpu").manual_seed(seed + 1)

    def batch():
        return torch.randint(vocab, (rows,), generator=g).to(device)

    def held_out(tokens, lists):
        with torch.no_grad():
            return float(distill_loss(student.logits(tokens, refresher.masked_weights), lists).mean())

    test = batch()
    with torch.no_grad():
        test_lists = teacher_lists(teacher.logits(test), k, temperature)
    losses = [held_out(test, test_lists)]
    for i in range(1, steps + 1):
        tokens = batch()
        with torch.no_grad():
            lists = teacher_lists(teacher.logits(tokens), k, temperature)
        optimizer.zero_grad(set_to_none=True)
        distill_backward(student.logits(tokens, refresher.masked_weights, dropout, seed, i * (blocks + 1)), lists, scale=temperature ** 2 / rows)
        optimizer.step()
        refresher.step(i)
        if i % evaluate == 0 or i == steps:
            losses.append(held_out(test, test_lists))
            if report:
                report("step %d: loss %.5f (dense weights pruned without training %.5f), %d mask bits changed" % (i, losses[-1], losses[0], refresher.changed_bits[-1]))
    if networks is not None:
        networks[:] = [teacher, student, refresher.masked_weights]
    return losses


def main(argv=None):
    p = argparse.ArgumentParser(description="Distil a small dense network into its 2:4 transposable pruning.")
    p.add_argument("--steps", type=int, default=60)
    p.add_argument("--rows", type=int, default=512)
    p.add_argument("--vocab", type=int, default=4099)
    p.add_argument("--width", type=int, default=256)
    p.add_argument("--blocks", type=int, default=2)
    p.add_argument("--k", type=int, default=32)
    p.add_argument("--temperature", type=float, default=2.0)
    p.add_argument("--dtype", choices=["float32", "bfloat16"], default="float32")
    p.add_argument("--norm", choices=["layer", "rms"], default="layer")
    p.add_argument("--dropout", type=float, default=0.0)
    a = vars(p.parse_args(argv))
    import torch
    a["dtype"] = getattr(torch, a["dtype"])
    losses = train(report=print, **a)
    print("loss %.5f -> %.5f" % (losses[0], losses[-1]))
    return losses


if __name__ == "__main__":
    main()
