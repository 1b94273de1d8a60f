"""A pruned student as the drafter of the teacher that it was distilled from: the student proposes tokens, the teacher checks them in one pass, and
what comes out is distributed as the teacher's own tokens.  The share of drafts that stay says how near the student is.

    python -m paper_2102_08124_b200.draft --steps 60
"""
from __future__ import annotations

import argparse

from . import binding_branch as bb
from .distill import train


def draw(logits, seed: int, offset: int = 0, temperature: float = 1.0, status=None):
    """One token from softmax(logits / temperature) of every row (int32 [rows]); -1 where a row holds NaN, +Inf or nothing but -Inf, which `status`
    (int32[1] or None) shows too."""
    import torch
    none = torch.empty((logits.shape[0], 0), dtype=torch.int32, device=logits.device)
    return bb.tm_verify_draft(logits, None, none, seed, offset, temperature=temperature, want_logp=False, status=status)[0][:, 0]


def speculate(target, drafter, last, drafts: int, seed: int, offset: int = 0, temperature: float = 1.0, status=None):
    """One round for sequences whose last tokens are `last` [batch]: `drafts` tokens from the drafter, one after the other, then the target's
    check of all of them.  target and drafter map tokens [n] to the next token's logits [n, vocab].  Takes drafts + 1 offsets.
    Returns (tokens [batch, drafts + 1], accepted [batch]): the drafts that stayed, one more token, and -1 behind it.
    A sequence has ended where its last token is negative, as it is behind a row of the target's that nothing can be drawn from: it stays
    at -1.  A row of the drafter's of that kind ends the sequence's drafts of the round.  Negative tokens reach neither network (token 0 does, and
    its logits are not used).  status: shows such rows, the drafter's too."""
    import torch
    tokens, rows = [last], []
    for i in range(drafts):
        rows.append(drafter(tokens[-1].clamp_min(0)))
        tokens.append(torch.where(tokens[-1] < 0, -1, draw(rows[-1], seed, offset + i, temperature, status)))
    given = torch.stack(tokens, 1)                                       # [batch, drafts + 1]
    logits = target(given.clamp_min(0).reshape(-1))
    draft_logits = torch.stack(rows, 1).reshape(-1, logits.shape[1]) if drafts else None
    out, accepted, _ = bb.tm_verify_draft(logits, draft_logits, given[:, 1:].contiguous().int(), seed, offset + drafts, temperature=temperature,
                                          want_logp=False, status=status)
    return torch.where(last[:, None] < 0, -1, out), accepted


def share_that_stays(target, drafter, last, drafts: int, rounds: int, seed: int, temperature: float = 1.0) -> float:
    """Share of the tested drafts that stayed, over `rounds` rounds."""
    import torch
    kept = tested = 0
    status = torch.zeros(1, dtype=torch.int32, device=last.device)
    for i in range(rounds):
        out, accepted = speculate(target, drafter, last, drafts, seed, i * (drafts + 1), temperature, status)
        last = out.gather(1, accepted.long()[:, None])[:, 0]
        kept += int(accepted.sum())
        tested += int((accepted + (accepted < drafts)).sum())
    if int(status):
        raise FloatingPointError("a row of logits holds NaN, +Inf or nothing but -Inf")
    return kept / max(tested, 1)


class Rows8:
    """A weight [out, in] in 8 bits with a scale a row, for products with tm_rms_norm_e4m3's output (group 0).  Both dimensions are multiples of 16."""

    def __init__(self, weight):
        import torch
        w = weight.detach().float()
        self.scale = (w.abs().amax(1, keepdim=True) / 448.0).clamp_min(2.0 ** -126)
        self.values = (w / self.scale).to(torch.float8_e4m3fn)

    def product(self, y8, scales):
        import torch
        return torch._scaled_mm(y8, self.values.t(), scale_a=scales, scale_b=self.scale.t(), out_dtype=torch.bfloat16)


def eight_bit_logits(blocks, masked):
    """The forward pass of a trained "rms" network in bfloat16 whose blocks' first products run in 8 bits: tokens [n] to logits."""
    import torch
    first = [Rows8(masked[2 * i]) for i in range(len(masked) // 2)]

    def logits(tokens):
        h, update = blocks.embedding[tokens], None
        for i, w in enumerate(first):
            y8, scales, total = bb.tm_rms_norm_e4m3(h if update is None else update, blocks.norm_weight[i], residual=None if update is None else h)
            h = h if total is None else total
            update = torch.nn.functional.gelu(w.product(y8, scales)) @ masked[2 * i + 1].t()
        y, _, _ = bb.tm_rms_norm(update, blocks.norm_weight[-1], residual=h, want_sum=False, want_stats=False)
        return y @ blocks.head.t()

    return logits


def run(steps: int = 60, rows: int = 512, vocab: int = 4099, width: int = 256, blocks: int = 2, drafts: int = 4, rounds: int = 8, batch: int = 64,
        dropout: float = 0.05, seed: int = 0, report=None):
    """Shares of drafts that stay: the pruned network without training, the distilled one, and that one with products in 8 bits."""
    import torch
    found = []
    for n in (0, steps):
        networks = []
        train(steps=n, rows=rows, vocab=vocab, width=width, blocks=blocks, dtype=torch.bfloat16, seed=seed, norm="rms", dropout=dropout, networks=networks)
        teacher, student, masked = networks
        last = torch.randint(vocab, (batch,), generator=torch.Generator().manual_seed(seed + 2)).to(teacher.embedding.device)
        with torch.no_grad():
            drafters = [lambda t: student.logits(t, masked)] + ([eight_bit_logits(student, masked)] if n else [])
            for d in drafters:
                found.append(share_that_stays(teacher.logits, d, last, drafts, rounds, seed + 3))
    if report:
        report("drafts that stay: %.3f pruned, %.3f distilled, %.3f with products in 8 bits" % tuple(found))
    return found


def main(argv=None):
    p = argparse.ArgumentParser(description="Distil a pruned network and let it draft for its teacher.")
    for name, default in (("steps", 60), ("rows", 512), ("vocab", 4099), ("width", 256), ("blocks", 2), ("drafts", 4), ("rounds", 8), ("batch", 64)):
        p.add_argument("--" + name, type=int, default=default)
    p.add_argument("--dropout", type=float, default=0.05)
    return run(report=print, **vars(p.parse_args(argv)))


if __name__ == "__main__":
    main()
