"""The operators of a language-model client's local step in 64 bits, from their definitions (numpy, test infrastructure).

Every function returns, beside its results, how far fp32 arithmetic may take them: `u` is fp32's unit roundoff 2^-24, a
sum over s terms by threads that each add every 64th of them at least is off by at most (s / 64 + 40) u times the sum of the
terms' magnitudes (a thread's share, then a few tree steps), an exponential by (3 |argument| + 4) u of its value.
Rounding to the output's type comes on top: see `half_step`.
"""
from __future__ import annotations

import numpy as np

U = 2.0 ** -24


def depth(terms: int) -> float:
    return terms / 64 + 40


def half_step(ref, eps: float, smallest: float):
    """Half a step of the type at `ref`: eps/2 of its value, and no less than half the smallest subnormal."""
    return np.maximum(np.abs(ref) * eps / 2, smallest / 2)


def embed(ids, table, scale):
    ids = np.asarray(ids)
    out = np.zeros((ids.size, table.shape[1]))
    ok = (ids >= 0) & (ids < table.shape[0])
    out[ok] = table[ids[ok]].astype(np.float64) * float(np.float32(scale))
    return out, np.abs(out) * U


def embed_grad(ids, dout, vocab, scale, start=None):
    ids, dout, scale = np.asarray(ids), dout.astype(np.float64), float(np.float32(scale))
    ok = (ids >= 0) & (ids < vocab)
    out, size = np.zeros((vocab, dout.shape[1])), np.zeros((vocab, dout.shape[1]))
    np.add.at(out, ids[ok], dout[ok])
    np.add.at(size, ids[ok], np.abs(dout[ok]))
    count = np.bincount(ids[ok], minlength=vocab)[:, None]
    out, tol = out * scale, (count + 2) * U * size * abs(scale)
    if start is not None:
        out = out + start
        tol = tol + np.abs(out) * U
    return out, tol


def layer_norm(x, gamma, beta, eps):
    """y, stats and how far off they may be."""
    x = x.astype(np.float64)
    n, dim = x.shape
    g = np.ones(dim) if gamma is None else gamma.astype(np.float64)
    b = np.zeros(dim) if beta is None else beta.astype(np.float64)
    mean = x.mean(1, keepdims=True)
    c = x - mean
    var = (c * c).mean(1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        r = 1.0 / np.sqrt(var + float(np.float32(eps)))
        off = (depth(dim) + 2) * U * np.abs(x).mean(1, keepdims=True)          # of the mean
        # the mean square around a mean that is off by `off` grows by off^2; its terms have the subtraction's rounding
        rel = 0.5 * ((depth(dim) + 6) * U + off * off * r * r + 2 * off * U * np.abs(c).max(1, keepdims=True) * r * r) + 4 * U
        y = c * r * g + b
        tol = np.abs(r * g) * (off + U * np.abs(c)) + np.abs(c * r * g) * (rel + 3 * U) + U * np.abs(y)
    return y, tol, np.concatenate([mean, r], 1), np.concatenate([off, np.abs(r) * rel], 1)


def layer_norm_grad(dy, x, stats, gamma):
    """dx, dgamma, dbeta and how far off they may be, from the statistics as given."""
    dy, x = dy.astype(np.float64), x.astype(np.float64)
    n, dim = x.shape
    mean, r = stats[:, :1].astype(np.float64), stats[:, 1:].astype(np.float64)
    g = dy if gamma is None else dy * gamma.astype(np.float64)
    h = (x - mean) * r
    mg, mgh = g.mean(1, keepdims=True), (g * h).mean(1, keepdims=True)
    dx = r * (g - mg - h * mgh)
    size = np.abs(g) + np.abs(mg) + np.abs(h * mgh)
    sums = np.abs(g).mean(1, keepdims=True) + np.abs(h) * np.abs(g * h).mean(1, keepdims=True)
    tol = np.abs(r) * (8 * U * size + (depth(dim) + 6) * U * sums)
    rows = (depth(n) + 6) * U
    return (dx, tol, (dy * h).sum(0), rows * np.abs(dy * h).sum(0) if n else np.zeros(dim), dy.sum(0), rows * np.abs(dy).sum(0) if n else np.zeros(dim))


def _list(ids, values, vocab, T, logprobs):
    """One row's list: the entries that are there, their p and ln p, and the relative error of p."""
    there = (ids >= 0) & (ids < vocab) & ~np.isneginf(values)
    ids, t = ids[there], values[there].astype(np.float64)
    if not ids.size:
        return ids, t, t, t
    if logprobs:
        return ids, np.exp(t), t, (3 * np.abs(t) + 4) * U
    d = (t - t.max()) / T
    e = np.exp(d)
    rel = (3 * np.abs(d) + 6) * U
    return ids, e / e.sum(), d - np.log(e.sum()), rel + (e * rel).sum() / e.sum() + (depth(ids.size) + 4) * U


def distill(logits, ids, values, T=1.0, weights=None, logprobs=False):
    """loss, stats (m, S), dlogits, and how far off each may be."""
    z = logits.astype(np.float64)
    n, vocab = z.shape
    T = float(np.float32(T))
    loss, loss_tol = np.zeros(n), np.zeros(n)
    stats, stats_tol = np.zeros((n, 2)), np.zeros((n, 2))
    grad, grad_tol = np.zeros((n, vocab)), np.zeros((n, vocab))
    for i in range(n):
        w = 1.0 if weights is None else float(weights[i])
        at, p, logp, rel_p = _list(ids[i], values[i], vocab, T, logprobs)
        P = p.sum() if logprobs or not p.size else 1.0
        if w == 0.0 or P == 0.0:
            continue
        m = z[i].max()
        masked = np.isneginf(m)
        d = np.full(vocab, -np.inf) if masked else (z[i] - m) / T
        e = np.exp(d)
        S = e.sum()
        live = np.where(np.isneginf(d), 0.0, d)
        rel_e = (3 * np.abs(live) + 4) * U
        rel_S = 0.0 if masked else (e * rel_e).sum() / S + (depth(vocab) + 4) * U
        q = np.zeros(vocab) if masked else e / S
        with np.errstate(divide="ignore"):
            logq = np.full(vocab, -np.inf) if masked else d - np.log(S)
        some = p > 0
        loss[i] = w * T * T * (p[some] * (logp[some] - logq[at[some]])).sum()
        if np.isfinite(loss[i]):
            far = np.abs(logp[some] - logq[at[some]])
            terms = p[some] * (far * (rel_p[some] + 3 * U) + rel_S + 3 * U * (1 + np.abs(logp[some]) + np.abs(live[at[some]]) + np.abs(np.log(S))))
            terms += p[some] * rel_p[some]                                    # ln p comes from the same sum as p
            loss_tol[i] = abs(w) * T * T * (terms.sum() + (depth(p.size) + 4) * U * (p[some] * far).sum()) + 4 * U * abs(loss[i])
        stats[i] = m if not masked else -np.finfo(np.float32).max, S
        stats_tol[i] = 0.0, S * rel_S
        grad[i] = P * q
        grad_tol[i] = P * q * (rel_e + rel_S + 6 * U + ((p * rel_p).sum() / P + depth(p.size) * U if logprobs else 0.0))
        np.subtract.at(grad[i], at, p)
        np.add.at(grad_tol[i], at, p * (rel_p + (depth(p.size) + 4) * U))
        grad[i] *= w * T
        grad_tol[i] = abs(w) * T * grad_tol[i] + 3 * U * np.abs(grad[i])
    return loss, loss_tol, stats, stats_tol, grad, grad_tol
