"""Plain 64-bit implementations (numpy) of the operators of the training step, and bounds on what 32-bit arithmetic may differ by."""
from __future__ import annotations

import numpy as np

U32, U16 = 2.0 ** -24, 2.0 ** -8          # unit roundoff of fp32 and of bf16


def out_unit(dtype: str) -> float:
    return U16 if dtype == "bf16" else U32


# ---- layer norm ------------------------------------------------------------------------------------------------------

def norm(x, res, w, b, eps):
    h = x if res is None else x + res
    mean = h.mean(1)
    rstd = 1.0 / np.sqrt(((h - mean[:, None]) ** 2).mean(1) + eps)
    xh = (h - mean[:, None]) * rstd[:, None]
    return xh * w + b, h, mean, rstd


def norm_bounds(h, rstd, w, b, y, dtype):
    """A row's mean and rstd are sums of at most 64 sequential fp32 additions a thread, then a tree: 64 units of the row's largest
    magnitude cover them and the few roundings after; y is rounded once more to its type."""
    top = np.abs(h).max(1, keepdims=True)
    return out_unit(dtype) * np.abs(y) + 64 * U32 * (top * rstd[:, None] * (1 + np.abs(y)) * np.maximum(np.abs(w), 1) + np.abs(b))


def norm_backward(dy, h, mean, rstd, w, dsum):
    xh = (h - mean[:, None]) * rstd[:, None]
    g = dy * w
    dx = rstd[:, None] * (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True))
    return dx + (0 if dsum is None else dsum), (dy * xh).sum(0), dy.sum(0), xh, g


def norm_backward_bounds(dy, h, mean, rstd, w, dx, dweight, dbias, xh, g, dtype, wdtype):
    r = rstd[:, None]
    off = U32 * (np.abs(h) + np.abs(mean[:, None])) * r * 4                        # of xh: a difference of two fp32 numbers
    size = np.abs(g) + np.abs(g).mean(1, keepdims=True) + np.abs(xh) * np.abs(g * xh).mean(1, keepdims=True)
    wrong = off * np.abs(g * xh).mean(1, keepdims=True) + np.abs(xh) * (np.abs(g) * off).mean(1, keepdims=True)
    bx = out_unit(dtype) * np.abs(dx) + 64 * U32 * r * size + r * wrong
    n = dy.shape[0] + 64                                                           # additions of a column's sum, in any order
    bw = out_unit(wdtype) * np.abs(dweight) + n * U32 * np.abs(dy * xh).sum(0) + (np.abs(dy) * off).sum(0)
    bb = out_unit(wdtype) * np.abs(dbias) + n * U32 * np.abs(dy).sum(0)
    return bx, bw, bb


# ---- lists and distillation ------------------------------------------------------------------------------------------

def log_sum_exp(a):
    if a.size == 0:
        return -np.inf
    m = a.max()
    if not np.isfinite(m):
        return m
    return m + np.log(np.exp(a - m).sum())


def top(row, k):
    """(values, ids) of the k largest, equal ones by the lower id, NaN first."""
    key = np.where(np.isnan(row), np.inf, row)
    order = np.lexsort((np.arange(row.size), -key, ~np.isnan(row)))[:k]
    values, ids = row[order], order
    if k > row.size:
        values, ids = np.append(values, np.full(k - row.size, -np.inf)), np.append(ids, np.full(k - row.size, -1))
    return values, ids


def sum_unit(n, reach):
    """Relative error of a sum of n fp32 exponentials whose exponents (natural) reach `reach`: 2^-22 of the exponential itself, the
    exponent's roundings, and at most n / 128 sequential additions."""
    return 2.0 ** -22 * (4 + 2 * reach + n / 512)


def distill(z, values, ids, lse_t, weight, t, scale):
    """One row: (loss, gradient, lse, log q_rest, error units).  z float64 [vocab]; ids as given (padding, repeats, out of range)."""
    vocab, zero = z.size, np.zeros(z.size)
    keep, seen = [], set()
    for k, j in enumerate(ids):
        if 0 <= j < vocab and j not in seen:
            seen.add(j)
            keep.append(k)
    if weight == 0 or not keep:
        return 0.0, zero, 0.0, 0.0, (0.0, zero)
    v, j = values[keep] / t, ids[keep]
    lse, f = log_sum_exp(z / t), weight * scale
    logq = z / t - lse
    out = np.ones(vocab, bool)
    out[j] = False
    log_rest = log_sum_exp(logq[out])
    logp = v - (log_sum_exp(v) if lse_t is None else lse_t)
    p = np.exp(logp)
    rest = 0.0 if lse_t is None else max(0.0, 1.0 - p.sum())
    use = p > 0
    loss = (p[use] * (logp[use] - logq[j][use])).sum()
    tail = rest > 0 and log_rest > -np.inf
    if tail:
        loss += rest * (np.log(rest) - log_rest)
    q = np.exp(logq)
    grad = q * np.where(out, 1 - rest * np.exp(-log_rest), 1) if tail else q.copy()
    grad[j] -= p
    # units: exponents reach |z|/T, |v|/T and the logs; p_rest is one minus a sum of such exponentials
    finite = np.abs(z[np.isfinite(z)] / t)
    reach = max(finite.max() if finite.size else 0.0, np.abs(v[np.isfinite(v)]).max(initial=0.0), abs(lse), 0.0 if lse_t is None else abs(lse_t))
    unit = 2 * sum_unit(vocab, reach)
    d_rest = unit if lse_t is not None else 0.0
    b_loss = abs(f) * (unit * (2 + reach) + (d_rest * (1 + abs(np.log(rest)) + abs(log_rest)) if tail else 0.0)) + U32 * abs(f * loss)
    b_grad = abs(f) / t * (unit * q + (np.where(out, q * np.exp(-log_rest) * (d_rest + 2 * unit * rest), 0) if tail else 0.0))
    b_grad[j] += abs(f) / t * unit * p
    return f * loss, f / t * grad, lse, log_rest if lse_t is not None else 0.0, (b_loss, b_grad)
