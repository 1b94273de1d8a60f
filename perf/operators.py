"""Cases, plain forms and 64-bit values of the operators that train a pruned network from its dense teacher.

Layer normalisation with a residual sum (forward, backward), the largest logits of a teacher with the log of its softmax
sum, and the distillation loss against such a list with its gradient.  `run` computes them from elementary torch operations
in 32 bits, or, where `own` is set, through this package's entry points.
"""
from __future__ import annotations

import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_ELEM = {"f32": 4, "bf16": 2}
_LARGEST = 4096 * 131072 * 2       # bytes of the largest logits


def listed():
    return [
        # one position of a network that answers: the norm after a residual branch, no statistics kept; latency is all there is
        _norm("norm_token", 1, 1024, "bf16", "bf16", residual=True, stats=False),
        # hidden size 1024 (the BERT-large-shaped layers of the benchmark), 32 sequences of 512 tokens, one training step's forward
        _norm("norm_train", 16384, 1024, "bf16", "f32", residual=True, stats=True),
        # a width that no vector divides, in 32 bits, nothing to add
        _norm("norm_odd", 4097, 1001, "f32", "f32", residual=False, stats=True),
        # the backward pass of a small micro-batch: the reduction over rows has few rows to share out
        _norm_back("norm_back_small", 64, 1024, "f32", "f32", dsum=False),
        # the backward pass of norm_train, with the gradient that arrives past the branch
        _norm_back("norm_back_train", 16384, 1024, "bf16", "f32", dsum=True),
        # wide rows that start on no vector boundary
        _norm_back("norm_back_wide", 2047, 8191, "bf16", "bf16", dsum=False),
        # the teacher's list for one position
        _top("top_one", 1, 32768, "f32", 20, 1.0),
        # the teacher's lists for a batch, large vocabulary
        _top("top_batch", 4096, 131072, "bf16", 64, 2.0),
        # evaluation: the loss alone, odd vocabulary, lists of several lengths, no tail
        _distill("distill_eval", "distill_loss", 2048, 32001, "f32", 32, 1.0, tail=False, short=True),
        # the backward pass after it, from the statistics that the forward pass left
        _distill("distill_back", "distill_grad", 2048, 32001, "bf16", 32, 2.0, tail=True, short=False),
        # loss and gradient in one call for a handful of positions
        _distill("distill_step_small", "distill_step", 8, 32768, "f32", 16, 1.0, tail=True, short=False),
        # loss and gradient in one call for a training batch, large vocabulary, the teacher's remaining mass as one more class
        _distill("distill_step_batch", "distill_step", 4096, 131072, "bf16", 64, 2.0, tail=True, short=True),
    ]


def _norm(name, rows, cols, dtype, wdtype, residual, stats):
    return {"name": name, "op": "norm", "rows": rows, "cols": cols, "dtype": dtype, "wdtype": wdtype, "residual": residual, "stats": stats}


def _norm_back(name, rows, cols, dtype, wdtype, dsum):
    return {"name": name, "op": "norm_back", "rows": rows, "cols": cols, "dtype": dtype, "wdtype": wdtype, "dsum": dsum}


def _top(name, rows, vocab, dtype, k, temperature):
    return {"name": name, "op": "top", "rows": rows, "vocab": vocab, "dtype": dtype, "k": k, "temperature": temperature}


def _distill(name, op, rows, vocab, dtype, k, temperature, tail, short):
    return {"name": name, "op": op, "rows": rows, "vocab": vocab, "dtype": dtype, "k": k, "temperature": temperature, "tail": tail, "short": short}


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["norm", "norm_back", "top", "distill_loss", "distill_grad", "distill_step"])
    dtype = rng.choice(["f32", "bf16"])
    if op in ("norm", "norm_back"):
        cols = spread(64, 16384)
        rows = spread(1, min(32768, (1 << 25) // cols))
        wdtype = rng.choice(["f32", dtype])
        case = (_norm("", rows, cols, dtype, wdtype, rng.random() < 0.5, rng.random() < 0.8) if op == "norm"
                else _norm_back("", rows, cols, dtype, wdtype, rng.random() < 0.5))
    else:
        vocab = spread(1000, 131072)
        rows = spread(1, min(4096, _LARGEST // (vocab * _ELEM[dtype])))
        k = spread(1, 128)
        temperature = round(rng.uniform(0.5, 4.0), 2)
        case = (_top("", rows, vocab, dtype, k, temperature) if op == "top"
                else _distill("", op, rows, vocab, dtype, k, temperature, rng.random() < 0.5, rng.random() < 0.5))
    del case["name"]
    return case


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, dtype = case["op"], _TYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    s = dict(case)
    rows = case["rows"]
    if op in ("norm", "norm_back"):
        cols, wdtype = case["cols"], _TYPES[case["wdtype"]]
        spread, shift = torch.exp(0.5 * normal(cols)), 0.5 * normal(cols)          # channels differ in scale and offset
        s["weight"] = (1.0 + 0.2 * normal(cols)).to(wdtype)
        s["bias"] = (0.1 * normal(cols)).to(wdtype)
        s["x"] = (normal(rows, cols) * spread + shift).to(dtype)
        if op == "norm":
            s["residual_in"] = normal(rows, cols).to(dtype) if case["residual"] else None
        else:
            h = s["x"].float()
            s["mean"] = h.mean(1)
            s["rstd"] = torch.rsqrt((h - s["mean"][:, None]).square().mean(1) + 1e-5)
            s["dy"] = (0.02 * normal(rows, cols)).to(dtype)
            s["dsum_in"] = (0.02 * normal(rows, cols)).to(dtype) if case["dsum"] else None
        return s
    vocab, k, t = case["vocab"], case["k"], case["temperature"]
    z = normal(rows, vocab).mul_(2.0)
    if op == "top":
        s["logits"] = z.to(dtype)
        return s
    # a list of k different ids a row, their teacher logits in falling order, and a student that half follows the teacher
    step = torch.randint(1, vocab // k + 1, (rows, 1), generator=g, device="cuda")
    start = torch.randint(0, vocab, (rows, 1), generator=g, device="cuda")
    ids = (start + step * torch.arange(k, device="cuda")) % vocab
    values = (6.0 + 2.0 * normal(rows, k)).sort(dim=1, descending=True).values
    z.scatter_add_(1, ids, 0.6 * values)
    s["logits"] = z.to(dtype)
    lengths = torch.randint(1, k + 1, (rows, 1), generator=g, device="cuda") if case["short"] else torch.full((rows, 1), k, device="cuda")
    kept = torch.arange(k, device="cuda") < lengths
    s["ids"] = torch.where(kept, ids, -1).to(torch.int32)
    s["values"] = values
    s["teacher_lse"] = None
    if case["tail"]:                                                               # 2 % to 30 % of the teacher's mass outside the list
        outside = 0.02 + 0.28 * torch.rand(rows, generator=g, device="cuda")
        s["teacher_lse"] = torch.logsumexp((values / t).masked_fill(~kept, -math.inf), 1) - torch.log1p(-outside)
    weight = torch.ones(rows, device="cuda")
    weight[torch.randperm(rows, generator=g, device="cuda")[:_idle(case)]] = 0.0   # padding positions
    s["row_weight"] = weight
    s["scale"] = t * t / rows
    if op == "distill_grad":
        s["grad_loss"] = 0.5 + torch.rand(rows, generator=g, device="cuda")
        zt = s["logits"].float() / t
        lse = torch.logsumexp(zt, 1)
        tail = torch.zeros_like(lse)
        if case["tail"]:
            spare = torch.where(kept, ids, vocab)
            listed_ = torch.zeros(rows, vocab + 1, dtype=torch.bool, device="cuda").scatter_(1, spare, True)[:, :vocab]
            tail = torch.logsumexp(zt.masked_fill_(listed_, -math.inf), 1) - lse
        s["stats"] = torch.stack([lse, tail], 1) * (weight != 0)[:, None]
    return s


def _idle(case):
    return case["rows"] // 8


def run(s):
    return (_own if own else _plain)[s["op"]](s)


# ---- the package's entry points ------------------------------------------------------------------------------------

def _own_norm(s):
    import paper_2102_08124_b200 as tm
    y, total, mean, rstd = tm.tm_layer_norm(s["x"], s["weight"], s["bias"], 1e-5, residual=s["residual_in"], want_stats=s["stats"])
    return {"y": y, "sum": total, "mean": mean, "rstd": rstd}


def _own_norm_back(s):
    import paper_2102_08124_b200 as tm
    dx, dweight, dbias = tm.tm_layer_norm_backward(s["dy"], s["x"], s["mean"], s["rstd"], s["weight"], dsum=s["dsum_in"])
    return {"dx": dx, "dweight": dweight, "dbias": dbias}


def _own_top(s):
    import paper_2102_08124_b200 as tm
    values, ids, lse = tm.tm_top_logits(s["logits"], s["k"], s["temperature"])
    return {"values": values, "ids": ids, "lse": lse}


def _own_distill_loss(s):
    import paper_2102_08124_b200 as tm
    loss, stats = tm.tm_distill_loss(s["logits"], s["values"], s["ids"], teacher_lse=s["teacher_lse"], row_weight=s["row_weight"],
                                     temperature=s["temperature"], scale=s["scale"])
    return {"loss": loss, "stats": stats}


def _own_distill_grad(s):
    import paper_2102_08124_b200 as tm
    return {"dlogits": tm.tm_distill_grad(s["logits"], s["values"], s["ids"], s["stats"], grad_loss=s["grad_loss"], teacher_lse=s["teacher_lse"],
                                          row_weight=s["row_weight"], temperature=s["temperature"], scale=s["scale"])}


def _own_distill_step(s):
    import paper_2102_08124_b200 as tm
    loss, dlogits = tm.tm_distill_loss_grad(s["logits"], s["values"], s["ids"], teacher_lse=s["teacher_lse"], row_weight=s["row_weight"],
                                            temperature=s["temperature"], scale=s["scale"])
    return {"loss": loss, "dlogits": dlogits}


# ---- plain forms ---------------------------------------------------------------------------------------------------

def _plain_norm(s):
    h = s["x"].float()
    if s["residual_in"] is not None:
        h = h + s["residual_in"].float()
    mean = h.mean(1, keepdim=True)
    centred = h - mean
    rstd = torch.rsqrt((centred * centred).mean(1, keepdim=True) + 1e-5)
    y = centred * rstd * s["weight"].float() + s["bias"].float()
    kind = s["x"].dtype
    return {"y": y.to(kind), "sum": h.to(kind) if s["residual_in"] is not None else None,
            "mean": mean[:, 0] if s["stats"] else None, "rstd": rstd[:, 0] if s["stats"] else None}


def _plain_norm_back(s):
    dy, rstd = s["dy"].float(), s["rstd"][:, None]
    xhat = (s["x"].float() - s["mean"][:, None]) * rstd
    gy = dy * s["weight"].float()
    dx = (gy - gy.mean(1, keepdim=True) - xhat * (gy * xhat).mean(1, keepdim=True)) * rstd
    if s["dsum_in"] is not None:
        dx = dx + s["dsum_in"].float()
    return {"dx": dx.to(s["x"].dtype), "dweight": (dy * xhat).sum(0).to(s["weight"].dtype), "dbias": dy.sum(0).to(s["weight"].dtype)}


def _plain_top(s):
    z = s["logits"].float()
    # one whole number per logit that orders by (value, lower index first): the pattern of the value, then the index from above
    bits = z.view(torch.int32)
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
    index = torch.arange(z.shape[1], device=z.device)
    best = ((order << 32) + (0x7FFFFFFF - index)).topk(s["k"], dim=1).values
    ids = 0x7FFFFFFF - (best & 0xFFFFFFFF)
    zt = z / s["temperature"]
    top = zt.amax(1, keepdim=True)
    lse = top[:, 0] + torch.log(torch.exp(zt - top).sum(1))
    return {"values": z.gather(1, ids), "ids": ids.int(), "lse": lse}


def _teacher(s):
    """The list's probabilities and their logs (0 where the entry is padding), the mass outside it, and which entries count."""
    kept = s["ids"] >= 0
    v = (s["values"] / s["temperature"]).masked_fill(~kept, -math.inf)
    if s["teacher_lse"] is not None:
        logp = v - s["teacher_lse"][:, None]
    else:
        top = v.amax(1, keepdim=True)
        logp = v - top - torch.log(torch.exp(v - top).sum(1, keepdim=True))
    p = torch.exp(logp)
    rest = (1.0 - p.sum(1)).clamp_min(0.0) if s["teacher_lse"] is not None else torch.zeros_like(p[:, 0])
    return p, torch.where(kept, logp, 0.0), rest, kept


def _outside(s, kept):
    """1 for the logits that the row's list leaves out, 0 for the listed ones."""
    rows, vocab = s["logits"].shape
    at = s["ids"].clamp_min(0).long()
    return 1.0 - torch.zeros(rows, vocab, device=at.device).scatter_add_(1, at, kept.float()), at


def _gradient(s, zt, lse, log_rest, p, rest, at, outside, upstream):
    q = torch.exp(zt - lse[:, None])
    d = q - outside * q * (rest * torch.exp(-log_rest))[:, None] if s["teacher_lse"] is not None else q
    d = d.scatter_add(1, at, -p)
    return (d * upstream[:, None]).to(s["logits"].dtype)


def _loss(s, want_gradient):
    p, logp, rest, kept = _teacher(s)
    zt = s["logits"].float() / s["temperature"]
    top = zt.amax(1, keepdim=True)
    e = torch.exp(zt - top)
    total = e.sum(1)
    lse = top[:, 0] + torch.log(total)
    at = s["ids"].clamp_min(0).long()
    loss = (p * (logp - (zt.gather(1, at) - lse[:, None]))).sum(1)
    log_rest, outside = torch.zeros_like(lse), None
    if s["teacher_lse"] is not None:
        outside, at = _outside(s, kept)
        log_rest = torch.log((e * outside).sum(1)) - torch.log(total)
        loss = loss + torch.where(rest > 0, rest * (torch.log(rest) - log_rest), 0.0)
    weight = s["row_weight"] * s["scale"]
    on = (s["row_weight"] != 0).float()
    if not want_gradient:
        return {"loss": loss * weight, "stats": torch.stack([lse, log_rest], 1) * on[:, None]}
    return {"loss": loss * weight, "dlogits": _gradient(s, zt, lse, log_rest, p, rest, at, outside, weight / s["temperature"])}


def _plain_distill_grad(s):
    p, _, rest, kept = _teacher(s)
    outside, at = _outside(s, kept) if s["teacher_lse"] is not None else (None, s["ids"].clamp_min(0).long())
    zt = s["logits"].float() / s["temperature"]
    upstream = s["row_weight"] * s["grad_loss"] * (s["scale"] / s["temperature"])
    return {"dlogits": _gradient(s, zt, s["stats"][:, 0], s["stats"][:, 1], p, rest, at, outside, upstream)}


_own = {"norm": _own_norm, "norm_back": _own_norm_back, "top": _own_top, "distill_loss": _own_distill_loss, "distill_grad": _own_distill_grad,
        "distill_step": _own_distill_step}
_plain = {"norm": _plain_norm, "norm_back": _plain_norm_back, "top": _plain_top, "distill_loss": lambda s: _loss(s, False),
          "distill_grad": _plain_distill_grad, "distill_step": lambda s: _loss(s, True)}


# ---- what a pass cannot do without ---------------------------------------------------------------------------------

def work(case):
    op, rows, e = case["op"], case["rows"], _ELEM[case["dtype"]]
    if op in ("norm", "norm_back"):
        cols, w = case["cols"], _ELEM[case["wdtype"]]
        n = rows * cols
        if op == "norm":
            return {"bytes": n * e * (4 if case["residual"] else 2) + 2 * cols * w + (8 * rows if case["stats"] else 0), "flops": 8 * n}
        return {"bytes": n * e * (4 if case["dsum"] else 3) + 3 * cols * w + 8 * rows, "flops": 14 * n}
    vocab, k = case["vocab"], case["k"]
    n = rows * vocab
    if op == "top":
        return {"bytes": n * e + rows * (8 * k + 4), "flops": 4 * n}
    on = rows - _idle(case)                                  # a padding position's logits need not be read; its gradient is written
    lists = on * k * 8 + rows * 4 + (on * 4 if case["tail"] else 0)
    if op == "distill_loss":
        return {"bytes": on * vocab * e + lists + rows * 12, "flops": 4 * on * vocab}
    extra = on * 12 if op == "distill_grad" else rows * 4
    return {"bytes": on * vocab * e + n * e + lists + extra, "flops": (6 if op == "distill_grad" else 9) * on * vocab}


# ---- the same from the definitions, in 64 bits ---------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    op, rows = case["op"], case["rows"]
    if op == "norm":
        h = s["x"].double()
        if s["residual_in"] is not None:
            h += s["residual_in"].double()
        var, mean = torch.var_mean(h, dim=1, correction=0)
        rstd = 1.0 / (var + 1e-5).sqrt()
        y = torch.addcmul(s["bias"].double(), (h - mean.unsqueeze(1)) / (var + 1e-5).sqrt().unsqueeze(1), s["weight"].double())
        return {"y": y, "sum": h if case["residual"] else None, "mean": mean if case["stats"] else None, "rstd": rstd if case["stats"] else None}
    if op == "norm_back":
        n = case["cols"]
        dy, c, r = s["dy"].double(), s["x"].double() - s["mean"].double().unsqueeze(1), s["rstd"].double().unsqueeze(1)
        u = dy * s["weight"].double()
        dx = r / n * (n * u - u.sum(1, keepdim=True) - c * r.square() * (u * c).sum(1, keepdim=True))
        if s["dsum_in"] is not None:
            dx += s["dsum_in"].double()
        return {"dx": dx, "dweight": torch.einsum("ij,ij,i->j", dy, c, r[:, 0]), "dbias": dy.sum(0)}
    t, chunk = case["temperature"], max(1, (1 << 27) // case["vocab"])
    parts = [_exact_rows(s, case, t, slice(a, min(rows, a + chunk))) for a in range(0, rows, chunk)]
    return {name: torch.cat([p[name] for p in parts]) for name in parts[0]}


def _exact_rows(s, case, t, at):
    z = s["logits"][at].double()
    logq = torch.log_softmax(z / t, 1)
    if case["op"] == "top":
        order = torch.sort(z, dim=1, descending=True, stable=True)
        return {"values": order.values[:, :case["k"]].clone(), "ids": order.indices[:, :case["k"]].int(), "lse": torch.logsumexp(z / t, 1)}
    ids, v, w = s["ids"][at].long(), s["values"][at].double() / t, s["row_weight"][at].double()
    valid = ids >= 0
    column = torch.where(valid, ids, case["vocab"])           # padding goes to a column of its own
    if case["tail"]:
        p = torch.where(valid, torch.exp(v - s["teacher_lse"][at].double()[:, None]), 0.0)
        rest = (1.0 - p.sum(1)).clamp_min(0.0)
    else:
        p = torch.softmax(torch.where(valid, v, -math.inf), 1)
        rest = torch.zeros(len(w), dtype=torch.float64, device=w.device)
    target = torch.zeros(z.shape[0], case["vocab"] + 1, dtype=torch.float64, device=z.device).scatter_(1, column, p)[:, :-1]
    unlisted = torch.ones(z.shape[0], case["vocab"] + 1, dtype=torch.bool, device=z.device).scatter_(1, column, False)[:, :-1]
    if case["op"] == "distill_grad":
        stats = s["stats"][at].double()
        lse, log_rest = stats[:, 0], stats[:, 1]
        q = torch.exp(z / t - lse[:, None])
    else:
        lse, q = torch.logsumexp(z / t, 1), logq.exp()
        log_rest = torch.logsumexp(logq.masked_fill(~unlisted, -math.inf), 1) if case["tail"] else torch.zeros_like(lse)
    scale = w * s["scale"] / t
    if case["op"] == "distill_grad":
        scale = scale * s["grad_loss"][at].double()
    if case["op"] != "distill_loss":
        if case["tail"]:
            target = torch.where(unlisted, q * (rest / log_rest.exp())[:, None], target)
        gradient = (q - target) * scale[:, None]
        if case["op"] == "distill_grad":
            return {"dlogits": gradient}
    picked = logq.gather(1, ids.clamp_min(0))
    loss = torch.where(p > 0, torch.xlogy(p, p) - p * picked, 0.0).sum(1)
    if case["tail"]:
        loss = loss + torch.where(rest > 0, torch.xlogy(rest, rest) - rest * log_rest, 0.0)
    loss = loss * w * s["scale"]
    if case["op"] == "distill_step":
        return {"loss": loss, "dlogits": gradient}
    return {"loss": loss, "stats": torch.stack([lse, log_rest], 1) * (w != 0)[:, None]}
