"""Plain 64-bit implementations (numpy) of the residual branch's operators and of draft verification, and bounds on what 32-bit arithmetic
may differ by."""
from __future__ import annotations

import numpy as np

U32, U16 = 2.0 ** -24, 2.0 ** -8          # unit roundoff of fp32 and of bf16


def out_unit(dtype: str) -> float:
    return U16 if dtype == "bf16" else U32


def philox(block, row, offset, seed):
    """Philox4x32 with ten rounds: the four words of every (block, row), uint32 [..., 4]."""
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    c = [np.array(v, np.uint64) for v in np.broadcast_arrays(block, row, offset & 0xFFFFFFFF, offset >> 32)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> half) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> half) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, -1).astype(np.uint32)


# ---- dropout and norm ------------------------------------------------------------------------------------------------

def kept(rows, cols, p, seed, offset):
    """(which elements stay, the factor of those that do)."""
    limit = min(65535, int(round(65536 * p)))
    w = philox(np.arange((cols + 7) // 8, dtype=np.uint64)[None, :], np.arange(rows, dtype=np.uint64)[:, None], offset, seed)
    bits = np.stack([w & 0xFFFF, w >> 16], -1).reshape(rows, -1)[:, :cols]
    return bits >= limit, 65536.0 / (65536 - limit)


def dropped(x, p, seed, offset):
    if p == 0:
        return x
    stay, factor = kept(*x.shape, p, seed, offset)
    return np.where(stay, x * factor, 0.0)


def total(x, res, p, seed, offset):
    """(h, bound on its fp32 error): the factor and the product round, then the sum."""
    d = dropped(x, p, seed, offset)
    h = d if res is None else d + res
    return h, U32 * (2 * np.abs(d) * (p > 0) + np.abs(h) * (res is not None))


def rms(h, w, eps):
    rstd = 1.0 / np.sqrt((h * h).mean(1) + eps)
    return h * rstd[:, None] * w, rstd


def rms_bounds(h, dh, w, rstd, y):
    """Bounds in fp32, before y is rounded to its type.  A sum of squares has at most 64 additions in a row a thread, a tree, and its terms' roundings,
    all of one sign: 80 units of itself, so 40 of rstd, and a root, a quotient and the mean's two more; dh is the error of h."""
    lift = 2 * np.sqrt((dh * dh).mean(1)) * rstd                                   # what dh does to the root of the mean square, relative
    br = rstd * (44 * U32 + lift)
    return (46 * U32 + lift[:, None]) * np.abs(y) + dh * np.abs(w) * rstd[:, None], br


def rms_backward(dy, h, rstd, w, dsum):
    xh = h * rstd[:, None]
    g = dy * w
    dh = rstd[:, None] * (g - xh * (g * xh).mean(1, keepdims=True))
    return dh + (0 if dsum is None else dsum), (dy * xh).sum(0), xh, g


def rms_backward_bounds(dy, rstd, dsum, dh, dweight, xh, g):
    """The row's sum has its terms' roundings and at most 64 + 16 additions in a row: 84 units of the sum of magnitudes."""
    r = rstd[:, None]
    size = np.abs(g) + np.abs(xh) * np.abs(g * xh).mean(1, keepdims=True)
    bx = 88 * U32 * r * size + U32 * (np.abs(dh) + (0 if dsum is None else np.abs(dsum)))
    n = dy.shape[0] + 64                                                           # additions of a column's sum, in any order
    return bx, n * U32 * np.abs(dy * xh).sum(0)


def e4m3_step(t):
    """Distance of neighbours in e4m3 around t."""
    e = np.floor(np.log2(np.maximum(np.abs(t), 2.0 ** -6)))
    return 2.0 ** (e - 3)


# ---- verification ----------------------------------------------------------------------------------------------------

def log_softmax(z):
    m = z.max()
    return z - m - np.log(np.exp(z - m).sum())


def verify(target, draft, ids, seed, offset, t, td):
    """target float64 [batch, drafted + 1, vocab], draft [batch, drafted, vocab] or None.  Returns (tokens, accepted, logp, sure): sure[b] is
    false where a comparison of sequence b was closer than fp32 sums can tell (2^-18 relative)."""
    batch, more, vocab = target.shape
    drafted, close = more - 1, 2.0 ** -18
    tokens, accepted = np.full((batch, more), -1, np.int64), np.zeros(batch, np.int64)
    logps, sure = np.zeros((batch, more)), np.ones(batch, bool)
    tests = philox((1 << 31) + np.arange((drafted + 3) // 4, dtype=np.uint64)[None, :], np.arange(batch, dtype=np.uint64)[:, None], offset, seed)
    tests = (tests.reshape(batch, -1) + 0.5) * 2.0 ** -32
    words = philox(np.arange((vocab + 3) // 4, dtype=np.uint64)[None, :], np.arange(batch, dtype=np.uint64)[:, None], offset, seed)
    noise = -np.log1p(-(words.reshape(batch, -1)[:, :vocab] + 0.5) * 2.0 ** -32)
    for b in range(batch):
        r = None
        for n in range(more):
            z = target[b, n] / t
            x = ids[b, n] if n < drafted else -1
            fine = not np.isnan(z).any() and not np.isposinf(z).any() and not np.isneginf(z).all()
            if fine and 0 <= x < vocab and draft is not None:
                y = draft[b, n] / td
                fine = not np.isnan(y).any() and not np.isposinf(y).any() and not np.isneginf(y).all()
            if not fine:
                logps[b, n] = np.nan
                break
            logp = log_softmax(z)
            p = np.exp(logp)
            if 0 <= x < vocab:
                q = np.exp(log_softmax(y)) if draft is not None else (np.arange(vocab) == x) * 1.0
                lhs = tests[b, n] * q[x]
                sure[b] &= abs(lhs - p[x]) > close * p[x] or p[x] == 0
                if lhs < p[x]:
                    tokens[b, n], logps[b, n] = x, logp[x]
                    continue
                r = np.maximum(p - q, 0.0)
                sure[b] &= r.sum() == 0 or r.sum() > 2.0 ** -10          # a difference of sums that each hold 2^-22
            if r is None or not (r > 0).any():
                r = p
            key = r / noise[b]
            x = int(key.argmax())
            best = key[x]
            key[x] = 0.0
            sure[b] &= key.max() < best * (1 - (close if r is p else 2.0 ** -8))
            tokens[b, n], logps[b, n] = x, logp[x]
            break
        accepted[b] = n
    return tokens, accepted, logps, sure
