"""Cases, plain forms and 64-bit values of the operators of a pruned network's residual branch, and of its use as a drafter of its teacher.

Dropout from a counter-based generator, root-mean-square norm of a residual sum with that dropout (forward, with an output in 8 bits,
backward), and verification of drafted tokens against the target's probabilities.  `run` computes them from elementary torch
operations in 32 bits (the verification in 64: a whole number hangs on every comparison), or, where `own` is set, through this
package's entry points.

Random numbers are Philox4x32 with ten rounds, key = the two halves of the seed, counter = (block, row, the two halves of the offset).  Dropout: a
block is eight columns of a row, sixteen bits each, low half of the first word first; an element stays where its bits are not below round(65536 p),
and is divided by the share that stays.  Verification: a block is four tokens, a word w each, and u = (w + 1/2) / 2^32; the
acceptance of draft i of a row takes word i of the blocks from 2^31 on.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_ELEM = {"f32": 4, "bf16": 2}
_LARGEST = 256 * 11 * 131072 * 2      # bytes of the largest logits, the target's and the drafter's
_EPS = 1e-5
_STAYS = 0.8                          # drafts that are accepted, about: the drafter's logits are the target's with noise


def listed():
    return [
        # the backward pass of dropout for a small micro-batch
        _drop("drop_small", 64, 1024, "f32", 0.1, residual=False),
        # hidden size 1024 (the BERT-large-shaped layers of the benchmark), 32 sequences of 512 tokens: dropout and the residual's addition
        _drop("drop_train", 16384, 1024, "bf16", 0.1, residual=True),
        # one position of a network that answers; latency is all there is
        _rms("rms_token", 1, 1024, "bf16", "bf16", 0.0, residual=True, stats=False),
        # one training step's forward: dropout, residual, norm
        _rms("rms_train", 16384, 1024, "bf16", "f32", 0.1, residual=True, stats=True),
        # a width that no vector divides, in 32 bits, nothing to add
        _rms("rms_odd", 4097, 1001, "f32", "f32", 0.0, residual=False, stats=True),
        # one position, for a product in 8 bits with a scale a row
        _rms8("rms8_token", 1, 4096, "bf16", "bf16", 0, residual=True),
        # a prompt of 8192 positions, a scale for every 128 columns
        _rms8("rms8_prompt", 8192, 4096, "bf16", "bf16", 128, residual=True),
        # the backward pass of a small micro-batch: the sum over rows has few rows to share out
        _back("back_small", 64, 1024, "f32", "f32", 0.1, dsum=False),
        # the backward pass of rms_train, with the gradient that arrives past the branch
        _back("back_train", 16384, 1024, "bf16", "f32", 0.1, dsum=True),
        # wide rows that start on no vector boundary
        _back("back_wide", 2047, 8191, "bf16", "bf16", 0.0, dsum=False),
        # four drafts of one conversation
        _verify("verify_one", 1, 4, 32768, "f32", 1.0, ragged=False),
        # five drafts, or fewer, for each sequence of a large batch, large vocabulary
        _verify("verify_batch", 256, 5, 131072, "bf16", 0.8, ragged=True),
    ]


def _drop(name, rows, cols, dtype, p, residual):
    return {"name": name, "op": "drop", "rows": rows, "cols": cols, "dtype": dtype, "p": p, "residual": residual}


def _rms(name, rows, cols, dtype, wdtype, p, residual, stats):
    return {"name": name, "op": "rms", "rows": rows, "cols": cols, "dtype": dtype, "wdtype": wdtype, "p": p, "residual": residual, "stats": stats}


def _rms8(name, rows, cols, dtype, wdtype, group, residual):
    return {"name": name, "op": "rms8", "rows": rows, "cols": cols, "dtype": dtype, "wdtype": wdtype, "group": group, "residual": residual}


def _back(name, rows, cols, dtype, wdtype, p, dsum):
    return {"name": name, "op": "back", "rows": rows, "cols": cols, "dtype": dtype, "wdtype": wdtype, "p": p, "dsum": dsum}


def _verify(name, rows, drafts, vocab, dtype, temperature, ragged):
    return {"name": name, "op": "verify", "rows": rows, "drafts": drafts, "vocab": vocab, "dtype": dtype, "temperature": temperature, "ragged": ragged}


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["drop", "rms", "rms8", "back", "verify", "verify"])
    dtype = rng.choice(["f32", "bf16"])
    if op == "verify":
        vocab, drafts = spread(1000, 131072), rng.randint(0, 8)
        rows = spread(1, min(256, _LARGEST // ((2 * drafts + 1) * vocab * _ELEM[dtype])))
        case = _verify("", rows, drafts, vocab, dtype, round(rng.uniform(0.5, 1.5), 2), rng.random() < 0.5)
    else:
        cols = spread(64, 16384)
        rows = spread(1, min(32768, (1 << 25) // cols))
        wdtype, p, flag = rng.choice(["f32", dtype]), rng.choice([0.0, 0.1, round(rng.uniform(0.01, 0.6), 3)]), rng.random() < 0.5
        if op == "drop":
            case = _drop("", rows, cols, dtype, max(p, 0.05), flag)
        elif op == "rms":
            case = _rms("", rows, cols, dtype, wdtype, p, flag, rng.random() < 0.8)
        elif op == "rms8":
            case = _rms8("", rows, cols, dtype, wdtype, rng.choice([0, 32, 64, 128]), flag)
        else:
            case = _back("", rows, cols, dtype, wdtype, p, flag)
    del case["name"]
    return case


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, dtype, rows = case["op"], _TYPES[case["dtype"]], case["rows"]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    s = dict(case)
    s["seed"], s["offset"] = 0x9E3779B97F4A7C15 * (seed + 1) % (1 << 64), seed % 1000 + (1 << 33)
    if op == "verify":
        _prepare_verify(s, g, normal, dtype)
        return s
    cols = case["cols"]
    spread = torch.exp(0.5 * normal(cols))                                         # channels differ in scale
    if op != "drop":
        s["weight"] = (1.0 + 0.2 * normal(cols)).to(_TYPES[case["wdtype"]])
    if op == "back":
        s["h"] = (normal(rows, cols) * spread).to(dtype)
        s["rstd"] = torch.rsqrt(s["h"].float().square().mean(1) + _EPS)
        s["dy"] = (0.02 * normal(rows, cols)).to(dtype)
        s["dsum_in"] = (0.02 * normal(rows, cols)).to(dtype) if case["dsum"] else None
    else:
        s["x"] = (normal(rows, cols) * spread).to(dtype)
        s["residual_in"] = normal(rows, cols).to(dtype) if case["residual"] else None
    return s


def _prepare_verify(s, g, normal, dtype):
    """Logits with a head of 32 likely tokens a row, a drafter that follows them with some noise, and drafts drawn from its softmax."""
    rows, drafts, vocab = s["rows"], s["drafts"], s["vocab"]
    target = torch.empty(rows, drafts + 1, vocab, dtype=dtype, device="cuda")
    draft = torch.empty(rows, drafts, vocab, dtype=dtype, device="cuda")
    ids = torch.empty(rows, drafts, dtype=torch.int32, device="cuda")
    for i in range(drafts + 1):
        z = normal(rows, vocab).mul_(2.0)
        z.scatter_add_(1, torch.randint(0, vocab, (rows, 32), generator=g, device="cuda"), 7.0 + 2.0 * normal(rows, 32))
        target[:, i] = z
        if i < drafts:
            z += 0.5 * normal(rows, vocab)
            draft[:, i] = z
            u = torch.rand(rows, vocab, generator=g, device="cuda").clamp_(1e-7, 1 - 1e-7)
            ids[:, i] = (draft[:, i].float() / s["temperature"] - torch.log(-torch.log(u))).argmax(1)
    if s["ragged"]:
        lengths = torch.randint(0, drafts + 1, (rows, 1), generator=g, device="cuda")
        ids[torch.arange(drafts, device="cuda") >= lengths] = -1
    s["logits"], s["draft_logits"], s["draft_ids"] = target.view(-1, vocab), draft.view(-1, vocab), ids


def run(s):
    return (_own if own else _plain)[s["op"]](s)


# ---- the package's entry points ------------------------------------------------------------------------------------

def _own_drop(s):
    import paper_2102_08124_b200 as tm
    return {"y": tm.tm_dropout(s["x"], s["p"], s["seed"], s["offset"], residual=s["residual_in"])}


def _own_rms(s):
    import paper_2102_08124_b200 as tm
    y, total, rstd = tm.tm_rms_norm(s["x"], s["weight"], _EPS, residual=s["residual_in"], p=s["p"], seed=s["seed"], offset=s["offset"], want_stats=s["stats"])
    return {"y": y, "sum": total, "rstd": rstd}


def _own_rms8(s):
    import paper_2102_08124_b200 as tm
    y8, scales, total = tm.tm_rms_norm_e4m3(s["x"], s["weight"], _EPS, residual=s["residual_in"], group=s["group"])
    return {"y8": y8, "scales": scales, "sum": total}


def _own_back(s):
    import paper_2102_08124_b200 as tm
    dh, dx, dweight = tm.tm_rms_norm_backward(s["dy"], s["h"], s["rstd"], s["weight"], dsum=s["dsum_in"], p=s["p"], seed=s["seed"], offset=s["offset"])
    return {"dh": dh, "dx": dx, "dweight": dweight}


def _own_verify(s):
    import paper_2102_08124_b200 as tm
    tokens, accepted, logp = tm.tm_verify_draft(s["logits"], s["draft_logits"], s["draft_ids"], s["seed"], s["offset"], temperature=s["temperature"])
    return {"tokens": tokens, "accepted": accepted, "logp": logp}


# ---- plain forms ---------------------------------------------------------------------------------------------------

def _philox(c0, c1, offset, seed):
    """Words 0 to 3 for counters (c0, c1, offset), whole numbers below 2^32 held in int64."""
    low = 0xFFFFFFFF
    c2, c3 = torch.full_like(c0, offset & low), torch.full_like(c0, offset >> 32)
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack([c0, c1, c2, c3], -1)


def _grid(rows, blocks):
    c0 = torch.arange(blocks, device="cuda").expand(rows, blocks)
    return c0, torch.arange(rows, device="cuda")[:, None].expand(rows, blocks)


def _dropped(v, s):
    """v (float32) with its dropped elements at zero and the others divided by the share that stays."""
    limit = int(round(65536 * s["p"]))
    if limit == 0:
        return v
    rows, cols = v.shape
    w = _philox(*_grid(rows, (cols + 7) // 8), s["offset"], s["seed"])
    bits = torch.stack([w & 0xFFFF, w >> 16], -1).reshape(rows, -1)[:, :cols]
    return torch.where(bits >= limit, v * (65536 / (65536 - limit)), 0.0)


def _sum(s):
    h = _dropped(s["x"].float(), s) if "p" in s else s["x"].float()
    return h if s["residual_in"] is None else h + s["residual_in"].float()


def _plain_drop(s):
    return {"y": _sum(s).to(s["x"].dtype)}


def _plain_rms(s):
    h, kind = _sum(s), s["x"].dtype
    rstd = torch.rsqrt((h * h).mean(1, keepdim=True) + _EPS)
    more = s["residual_in"] is not None or s["p"] > 0
    return {"y": (h * rstd * s["weight"].float()).to(kind), "sum": h.to(kind) if more else None, "rstd": rstd[:, 0] if s["stats"] else None}


def _plain_rms8(s):
    h, kind = _sum(s), s["x"].dtype
    rows, cols = h.shape
    y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + _EPS) * s["weight"].float()
    width = s["group"] or cols
    groups = (cols + width - 1) // width
    padded = torch.nn.functional.pad(y, (0, groups * width - cols)).view(rows, groups, width)
    scales = (padded.abs().amax(2) / 448.0).clamp_min(2.0 ** -126)
    q = (padded / scales[:, :, None]).clamp(-448.0, 448.0).view(rows, -1)[:, :cols]
    return {"y8": q.to(torch.float8_e4m3fn), "scales": scales, "sum": h.to(kind) if s["residual_in"] is not None else None}


def _plain_back(s):
    dy, rstd = s["dy"].float(), s["rstd"][:, None]
    xh, g = s["h"].float() * rstd, dy * s["weight"].float()
    dh = (g - xh * (g * xh).mean(1, keepdim=True)) * rstd
    if s["dsum_in"] is not None:
        dh = dh + s["dsum_in"].float()
    kind = s["h"].dtype
    return {"dh": dh.to(kind), "dx": _dropped(dh, s).to(kind), "dweight": (dy * xh).sum(0).to(s["weight"].dtype)}


def _uniform(words):
    return (words.double() + 0.5) * 2.0 ** -32


def _plain_verify(s):
    rows, drafts, vocab, t = s["rows"], s["drafts"], s["vocab"], s["temperature"]
    target, draft, ids = s["logits"].view(rows, -1, vocab), s["draft_logits"].view(rows, -1, vocab), s["draft_ids"].long()
    if drafts:
        def at(z, i):                                                              # log softmax at the given tokens
            z = z.double() / t
            top = z.amax(-1, keepdim=True)
            return (z.gather(-1, i[..., None]) - top)[..., 0] - torch.log(torch.exp(z - top).sum(-1))

        safe = ids.clamp_min(0)
        logp, logq = at(target[:, :drafts], safe), at(draft, safe)
        c0 = (torch.arange((drafts + 3) // 4, device="cuda") + (1 << 31)).expand(rows, -1)
        u = _uniform(_philox(c0, torch.arange(rows, device="cuda")[:, None].expand_as(c0), s["offset"], s["seed"]).reshape(rows, -1)[:, :drafts])
        good = (ids >= 0) & (u * torch.exp(logq) < torch.exp(logp))
        accepted = good.long().cumprod(1).sum(1)
    else:
        accepted = torch.zeros(rows, dtype=torch.long, device="cuda")
    row = torch.arange(rows, device="cuda")

    def softmax(z):
        z = z.double() / t
        e = torch.exp(z - z.amax(1, keepdim=True))
        return e / e.sum(1, keepdim=True)

    p = softmax(target[row, accepted])
    r = p
    if drafts:
        last = accepted.clamp_max(drafts - 1)
        refused = (accepted < drafts) & (ids[row, last] >= 0)
        r = torch.where(refused[:, None], (p - softmax(draft[row, last])).clamp_min(0.0), p)
        r = torch.where((r > 0).any(1, keepdim=True), r, p)
    u = _uniform(_philox(*_grid(rows, (vocab + 3) // 4), s["offset"], s["seed"]).reshape(rows, -1)[:, :vocab])
    token = (r / -torch.log1p(-u)).argmax(1)
    place = torch.arange(drafts + 1, device="cuda")
    tokens = torch.where(place < accepted[:, None], torch.nn.functional.pad(ids, (0, 1)), -1).scatter(1, accepted[:, None], token[:, None])
    chosen = torch.where(place == accepted[:, None], torch.log(p.gather(1, token[:, None])), 0.0)
    if drafts:
        chosen = torch.where(place < accepted[:, None], torch.nn.functional.pad(logp, (0, 1)), chosen)
    return {"tokens": tokens.int(), "accepted": accepted.int(), "logp": chosen.float()}


_own = {"drop": _own_drop, "rms": _own_rms, "rms8": _own_rms8, "back": _own_back, "verify": _own_verify}
_plain = {"drop": _plain_drop, "rms": _plain_rms, "rms8": _plain_rms8, "back": _plain_back, "verify": _plain_verify}


# ---- what a pass cannot do without ---------------------------------------------------------------------------------

def work(case):
    op, rows, e = case["op"], case["rows"], _ELEM[case["dtype"]]
    if op == "verify":
        # a row of the target's is read for every position that is reached, one of the drafter's where a draft stands there
        drafts, vocab = case["drafts"], case["vocab"]
        lengths = range(drafts + 1) if case["ragged"] else [drafts]
        reached = [sum(_STAYS ** i for i in range(n)) for n in lengths]
        both, alone = sum(reached) / len(reached), sum(_STAYS ** n for n in lengths) / len(lengths)
        read = rows * (2 * both + alone) * vocab
        return {"bytes": read * e + rows * (drafts * 4 + (drafts + 1) * 8 + 4), "flops": 4 * read + 30 * rows * vocab}
    cols = case["cols"]
    n, w = rows * cols, _ELEM[case.get("wdtype", case["dtype"])]
    random = 9 * n if case.get("p", 0.0) > 0 else 0
    if op == "drop":
        return {"bytes": n * e * (3 if case["residual"] else 2), "flops": 2 * n + random}
    if op == "rms":
        more = case["residual"] or case["p"] > 0
        return {"bytes": n * e * (2 + case["residual"] + more) + cols * w + (4 * rows if case["stats"] else 0), "flops": 5 * n + random}
    if op == "rms8":
        groups = -(-cols // case["group"]) if case["group"] else 1
        return {"bytes": n * (e * (3 if case["residual"] else 1) + 1) + cols * w + 4 * rows * groups, "flops": 8 * n}
    return {"bytes": n * e * (3 + case["dsum"] + (case["p"] > 0)) + 2 * cols * w + 4 * rows, "flops": 10 * n + random}


# ---- the same from the definitions, in 64 bits ---------------------------------------------------------------------

def _words(block, row, offset, seed):
    """The generator's words in numpy, for arrays of block and row numbers of one shape: shape + (4,), uint32."""
    m, s32 = np.uint64(0xFFFFFFFF), np.uint64(32)
    x = [np.asarray(block, np.uint64), np.asarray(row, np.uint64), np.uint64(offset & 0xFFFFFFFF), np.uint64(offset >> 32)]
    key = [seed % (1 << 32), seed // (1 << 32)]
    for _ in range(10):
        first, third = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(third >> s32) ^ x[1] ^ np.uint64(key[0]), third & m, (first >> s32) ^ x[3] ^ np.uint64(key[1]), first & m]
        key = [(key[0] + 0x9E3779B9) % (1 << 32), (key[1] + 0xBB67AE85) % (1 << 32)]
    return np.stack(np.broadcast_arrays(*x), -1).astype(np.uint32)


def _kept(case, s):
    """Which elements stay, and what they are multiplied by."""
    rows, cols, limit = case["rows"], case["cols"], int(round(65536 * case["p"]))
    w = _words(np.arange((cols + 7) // 8)[None, :], np.arange(rows)[:, None], s["offset"], s["seed"])
    bits = w.view(np.uint16).reshape(rows, -1)[:, :cols]                            # little end first
    return torch.from_numpy(bits >= limit).cuda(), 1.0 / (1.0 - limit / 65536.0)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "verify":
        return _exact_verify(case, s)
    if op == "back":
        r, dy, h, w = s["rstd"].double()[:, None], s["dy"].double(), s["h"].double(), s["weight"].double()
        dot = torch.einsum("ij,ij,j->i", dy, h, w)[:, None]
        dh = r * dy * w - h * r.pow(3) * dot / case["cols"]
        if s["dsum_in"] is not None:
            dh += s["dsum_in"].double()
        dx = dh
        if case["p"] > 0:
            kept, factor = _kept(case, s)
            dx = (dh * factor).masked_fill(~kept, 0.0)
        return {"dh": dh, "dx": dx, "dweight": torch.einsum("ij,ij,i->j", dy, h, r[:, 0])}
    h = s["x"].double()
    if case.get("p", 0.0) > 0:
        kept, factor = _kept(case, s)
        h = (h * factor).masked_fill(~kept, 0.0)
    if s["residual_in"] is not None:
        h = h + s["residual_in"].double()
    if op == "drop":
        return {"y": h}
    norm = (h.square().sum(1) / case["cols"] + _EPS).sqrt()
    y = h / norm[:, None] * s["weight"].double()
    more = s["residual_in"] is not None or case.get("p", 0.0) > 0
    if op == "rms":
        return {"y": y, "sum": h if more else None, "rstd": 1.0 / norm if case["stats"] else None}
    parts = y.split(case["group"] or case["cols"], dim=1)
    scales = torch.stack([p.abs().amax(1) for p in parts], 1) / 448.0
    q = torch.cat([p / scales[:, k:k + 1] for k, p in enumerate(parts)], 1)         # before they are rounded to 8 bits
    return {"y8": q, "scales": scales, "sum": h if more else None}


def _exact_verify(case, s):
    rows, drafts, vocab, t = case["rows"], case["drafts"], case["vocab"], case["temperature"]
    ids = s["draft_ids"].cpu().numpy()
    tokens, accepted, chosen = np.full((rows, drafts + 1), -1, np.int32), np.zeros(rows, np.int32), np.zeros((rows, drafts + 1))
    tests = (_words(np.arange(1 << 31, (1 << 31) + (drafts + 3) // 4)[None, :], np.arange(rows)[:, None], s["offset"], s["seed"]).reshape(rows, -1)
             .astype(np.float64) + 0.5) / 2.0 ** 32
    row = lambda z, k: torch.log_softmax(z[k].double() / t, 0)
    for b in range(rows):
        n, out = 0, None
        while n < drafts and ids[b, n] >= 0:
            logp, logq, x = row(s["logits"], b * (drafts + 1) + n), row(s["draft_logits"], b * drafts + n), int(ids[b, n])
            if tests[b, n] >= float(torch.exp(logp[x] - logq[x])):
                out = (logp.exp() - logq.exp()).clamp_min(0.0)
                break
            tokens[b, n], chosen[b, n] = x, float(logp[x])
            n += 1
        logp = row(s["logits"], b * (drafts + 1) + n)
        if out is None or not bool((out > 0).any()):
            out = logp.exp()
        w = torch.from_numpy(_words(np.arange((vocab + 3) // 4), b, s["offset"], s["seed"]).reshape(-1)[:vocab].astype(np.float64)).cuda()
        race = torch.log(out) - torch.log(-torch.log1p(-(w + 0.5) / 2.0 ** 32))
        x = int(race.argmax())
        tokens[b, n], chosen[b, n], accepted[b] = x, float(logp[x]), n
    return {"tokens": tokens, "accepted": accepted, "logp": chosen}
