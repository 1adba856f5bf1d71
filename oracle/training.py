"""What a client trains with, in 64 bits, from the definitions (numpy, test infrastructure).

Every function returns, beside its results, how far fp32 arithmetic may take them; `U` is fp32's unit roundoff.
"""
from __future__ import annotations

import numpy as np

from .local_step import U, depth

# ----------------------------------------------------------------------------- AdamW
BLOCK, TOP, TINY = 256, 448.0, 2.0 ** -100
# the codes 0 ... 126 of e4m3: four bits of exponent (bias 7), three of fraction
CODES = np.array([(c % 8) * 2.0 ** -9 if c < 8 else (1 + (c % 8) / 8) * 2.0 ** (c // 8 - 7) for c in range(127)])


def values(codes):
    """What codes, as bytes, stand for."""
    codes = np.asarray(codes).astype(np.int64)
    return np.where(codes >= 128, -1.0, 1.0) * CODES[codes & 127]


def spread(scales, n):
    return np.repeat(np.asarray(scales, np.float64), BLOCK, 0)[:n]


def chances(n, seed, step, tensor, word=0):
    """Element i's 16 bits: Philox4x32-10 of (i / 8, word, step, tensor), the halves of its words, low ones first; word 1 is m's."""
    low = np.uint64(0xFFFFFFFF)
    c = [np.arange((n + 7) // 8, dtype=np.uint64)] + [np.full((n + 7) // 8, x, np.uint64) for x in (word, step, tensor)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), q & low, (p >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    halves = [h for w in c for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))]
    return np.stack(halves, 1).reshape(-1)[:n].astype(np.float64)


def nearest(y):
    """The codes nearest to y, 0 <= y <= 448, even ones where two are as near."""
    at = np.clip(np.searchsorted(CODES, y), 1, 126)
    below, above = y - CODES[at - 1], CODES[at] - y
    return np.where((below < above) | ((below == above) & ((at - 1) % 2 == 0)), at - 1, at)


def by_chance(y, chance, least=1):
    """The codes below y >= 0 or above it, above where the chance carries over; at least `least` unless y is 0 (m's: 0)."""
    at = np.clip(np.searchsorted(CODES, y, side="right") - 1, 0, 126)
    step = np.where(at < 126, CODES[np.minimum(at + 1, 126)] - CODES[at], 1.0)
    up = (y - CODES[at]) / step + chance * 2.0 ** -16 >= 1.0
    return np.where(y > 0, np.clip(at + up, least, 126), 0)


def adamw(param, grad, m, v, step, lr, betas, eps, decay, grad_scale=1.0, held=False):
    """param, m, v, sqrt v after the step and how far off each may be.  `held`: m and v come out of 8 bits, with a rounding
    (of v three) more.  An element whose gradient squared is beyond fp32 keeps what it has."""
    p, g, m, v = (np.asarray(x, np.float64) for x in (param, grad, m, v))
    (b1, b2), lr, scale = betas, float(lr), float(np.float32(grad_scale))
    with np.errstate(over="ignore", invalid="ignore"):
        gs = g * scale
        new_m, new_v = b1 * m + (1 - b1) * gs, b2 * v + (1 - b2) * gs * gs
        # a factor has a rounding, its product another, the sum a third
        off_m = (4 + held) * U * (np.abs(b1 * m) + np.abs((1 - b1) * gs)) + 2.0 ** -148
        off_v = (6 + 3 * held) * U * new_v + 2.0 ** -148
        fine = np.isfinite(gs) & (np.abs(gs) * np.abs(gs) < np.finfo(np.float32).max)
        new_m, new_v = np.where(fine, new_m, m), np.where(fine, new_v, v)
        root = np.sqrt(new_v)
        off_root = np.where(root > 0, off_v / np.maximum(2 * root, 1e-300), 0.0) + U * root
        rate = lr / (1 - b1 ** step)
        under = root / np.sqrt(1 - b2 ** step) + eps
        off_under = off_root / np.sqrt(1 - b2 ** step) + 3 * U * under
        move = new_m / under
        off_move = off_m / under + np.abs(move) * (off_under / under + U)
        to = p * (1 - lr * decay) - rate * move
        off = np.abs(p) * (3 * U * abs(lr * decay) + 2 * U) + abs(rate) * (off_move + 3 * U * np.abs(move)) + U * np.abs(to)
    return (np.where(fine, to, p), np.where(fine, off, 0.0), new_m, np.where(fine, off_m, 2 * U * np.abs(m)),
            new_v, np.where(fine, off_v, 4 * U * np.abs(v)), root, np.where(fine, off_root, 4 * U * root), fine)


def scales_of(x, off):
    """The blocks' scales of |x| and how far off; what lies about the border to zeros may go either way."""
    n = x.size
    blocks = -(-n // BLOCK)
    top, far = (np.pad(a, (0, blocks * BLOCK - n)).reshape(blocks, BLOCK) for a in (np.abs(x), off))
    top, far = top.max(1), far.max(1)
    return np.where(top >= TINY, top, 0.0) / TOP, far / TOP + 2 * U * top / TOP


# ----------------------------------------------------------------------------- the gated scan
def sigmoid(z):
    e = np.exp(-np.abs(z))
    return np.where(z >= 0, 1.0, e) / (1 + e), np.where(z >= 0, e, 1.0) / (1 + e)


def gated_scan(x, gate, bounds, h0=None):
    """h, the last states, and how far off each.  `bounds`: (first row, one behind the last) of every sequence.  A gate and
    its rest are off by at most 8 U of themselves; joined in any order a step adds no more than 16 U of what its terms'
    magnitudes would add up to."""
    f, rest = sigmoid(x * 0 + gate)
    h, off = np.full(x.shape, np.nan), np.zeros(x.shape)
    last, off_last = np.zeros((len(bounds), x.shape[1])), np.zeros((len(bounds), x.shape[1]))
    for s, (low, high) in enumerate(bounds):
        u = np.zeros(x.shape[1]) if h0 is None else h0[s].astype(np.float64)
        size, far = np.abs(u), np.zeros(x.shape[1])
        for t in range(low, high):
            u = f[t] * u + rest[t] * x[t]
            size = f[t] * size + rest[t] * np.abs(x[t])
            far = f[t] * far + 16 * U * size + 2.0 ** -126
            h[t], off[t] = u, far
        last[s], off_last[s] = u, far
    return h, off, last, off_last


def gated_scan_grad(dy, x, gate, h, bounds, h0=None, dlast=None):
    """dx, dgate, dh0, and how far off each."""
    f, rest = sigmoid(x * 0 + gate)
    dim = x.shape[1]
    dx, dgate, off_x, off_g = (np.full(x.shape, np.nan) for _ in range(4))
    dh0, off_0 = np.zeros((len(bounds), dim)), np.zeros((len(bounds), dim))
    for s, (low, high) in enumerate(bounds):
        c = np.zeros(dim) if dlast is None else dlast[s].astype(np.float64)
        size, far = np.abs(c), np.zeros(dim)
        for t in reversed(range(low, high)):
            before = h[t - 1] if t > low else (np.zeros(dim) if h0 is None else h0[s].astype(np.float64))
            d, whole = dy[t] + c, np.abs(dy[t]) + size
            off_d = far + U * whole
            dx[t], off_x[t] = rest[t] * d, rest[t] * (off_d + 10 * U * np.abs(d)) + 2.0 ** -126
            dgate[t] = d * (before - x[t]) * f[t] * rest[t]
            off_g[t] = f[t] * rest[t] * (np.abs(before - x[t]) * off_d + 24 * U * np.abs(d) * (np.abs(before) + np.abs(x[t]))) + 2.0 ** -126
            c = f[t] * d
            size = f[t] * whole
            far = f[t] * far + 16 * U * size + 2.0 ** -126
        dh0[s], off_0[s] = c, far
    return dx, off_x, dgate, off_g, dh0, off_0


# ----------------------------------------------------------------------------- the loss over a vocabulary
ROUNDS = {("f32", "f32"): 2.0 ** -23, ("bf16", "f32"): 2.0 ** -17, ("f16", "f32"): 2.0 ** -21, ("bf16", "bf16"): 2.0 ** -8, ("f16", "f16"): 2.0 ** -11}


def linear_xent(hidden, table, labels, scale=1.0, weights=None, cut=0.0):
    """Losses, stats (m, S), and what the gradients need; with how far off each.  `cut`: what of a product's term is left out.
    A logit is a sum of fp32 terms in any order."""
    h, t = hidden.astype(np.float64), table.astype(np.float64)
    n, vocab, dim = h.shape[0], t.shape[0], h.shape[1]
    s = float(np.float32(scale))
    labels = np.asarray(labels)
    w = np.ones(n) if weights is None else np.asarray(weights, np.float64)
    live = (labels >= 0) & (labels < vocab) & (w != 0)
    h = np.where(live[:, None], h, 0.0)
    z = s * (h @ t.T)
    far = abs(s) * (np.abs(h) @ np.abs(t).T) * ((dim + 2) * U + cut) + 2 * U * np.abs(z)
    if cut:                                                     # elements far below their matrix's largest
        far = far + abs(s) * 2.0 ** -38 * (np.abs(t).max() * np.abs(h).sum(1)[:, None] + np.abs(h).max() * np.abs(t).sum(1))
    m = z.max(1)
    off_m = far.max(1)
    d = z - m[:, None]
    rel = far + off_m[:, None] + (4 * np.abs(d) + 6) * U
    e = np.exp(d)
    S = e.sum(1)
    rel_S = (e * rel).sum(1) / S + (depth(vocab) + 8) * U
    at = np.where(live, labels, 0)
    rows = np.arange(n)
    loss = np.where(live, w * (np.log(S) - d[rows, at]), 0.0)
    tol = np.where(live, np.abs(w) * (rel_S + far[rows, at] + off_m + 4 * U * (np.abs(np.log(S)) + np.abs(d[rows, at]) + np.abs(m))) + 4 * U * np.abs(loss), 0.0)
    stats = np.where(live[:, None], np.stack([m, S], 1), 0.0)
    stats_tol = np.where(live[:, None], np.stack([off_m, S * (rel_S + off_m)], 1), 0.0)
    p = e / S[:, None]
    G = p.copy()
    G[rows, at] -= 1.0
    off_G = p * (rel + rel_S[:, None] + 4 * U) + 4 * U * np.abs(G)
    mask = (live * np.where(live, w, 0.0) * s)[:, None]
    return loss, tol, stats, stats_tol, G * mask, off_G * np.abs(mask), h, t


def linear_xent_grad(G, off_G, h, t, round_h, round_t, cut=0.0, start=None):
    """dh and dT and how far off: G is rounded (`round_h`, `round_t` of itself, beside what fp16 may lose below), terms are
    added in fp32 in any order, in pieces that are added in turn; results have steps of 2^-149."""
    n, vocab = G.shape
    lost = 2.0 ** -37 * np.abs(G).max() + 2.0 ** -150 if G.size else 0.0
    dh, dt = G @ t, G.T @ h
    size = np.abs(G)
    off_h = (off_G + round_h * size + lost) @ np.abs(t) + ((vocab + 8) * U + cut) * (size @ np.abs(t)) + 3 * U * np.abs(dh) + 2.0 ** -149
    off_t = (off_G + round_t * size + lost).T @ np.abs(h) + ((n + 8) * U + cut) * (size.T @ np.abs(h)) + 3 * U * np.abs(dt) + 2.0 ** -149
    if cut:
        off_h = off_h + 2.0 ** -38 * np.abs(t).max() * size.sum(1)[:, None]
        off_t = off_t + 2.0 ** -38 * np.abs(h).max() * size.sum(0)[:, None]
    if start is not None:
        dt = dt + start
        off_t = off_t + U * np.abs(dt)
    return dh, off_h, dt, off_t
