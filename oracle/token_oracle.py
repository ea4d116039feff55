"""The operators for token models in 64 bits on the CPU, from their definitions (test infrastructure; nothing here is
shared with the library).  Beside every result stands its magnitude: the same sum over absolute values, which rounding
errors are measured against.
"""
from __future__ import annotations

import numpy as np


def rotary(x, positions, frequencies, magnitude=1.0, interleaved=False, inverse=False):
    """(turned x, magnitudes); x (tokens, heads, numbers)."""
    x = np.asarray(x, np.float64)
    half = len(frequencies)
    angle = np.asarray(positions, np.float64)[:, None] * np.asarray(frequencies, np.float64)
    c = magnitude * np.cos(angle)[:, None]
    s = magnitude * np.sin(angle)[:, None] * (-1.0 if inverse else 1.0)
    first = np.arange(half) * 2 if interleaved else np.arange(half)
    second = first + 1 if interleaved else first + half
    y, size = x.copy(), np.abs(x)
    u, v = x[..., first], x[..., second]
    y[..., first], y[..., second] = u * c - v * s, v * c + u * s
    both = abs(magnitude) * (np.abs(u) + np.abs(v))
    size[..., first], size[..., second] = both, both
    return y, size


def frequencies(turned, base=10000.0, scaling=0, factor=1.0, context=0.0, low=1.0, high=32.0):
    i = np.arange(turned // 2, dtype=np.float64)
    if scaling == 2 and turned > 2:
        base = base * factor ** (turned / (turned - 2.0))
    f = base ** (-2.0 * i / max(turned, 1))
    if scaling == 1:
        return f / factor
    if scaling == 3:
        keep = np.clip((context * f / (2.0 * np.pi) - low) / (high - low), 0.0, 1.0)
        return f * keep + f / factor * (1.0 - keep)
    return f


def attention_sequence(q, k, v, rate, scale, state=None):
    """One head of one sequence: the recurrence token by token.  (y, last state, magnitudes of both)."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    keep = np.exp(-float(rate))
    S = np.zeros((q.shape[1], v.shape[1])) if state is None else np.asarray(state, np.float64).copy()
    M = np.abs(S)
    y, size = np.zeros(v.shape), np.zeros(v.shape)
    for t in range(q.shape[0]):
        S = keep * S + np.outer(k[t], v[t])
        M = keep * M + np.outer(np.abs(k[t]), np.abs(v[t]))
        y[t] = scale * (q[t] @ S)
        size[t] = scale * (np.abs(q[t]) @ M)
    return y, S, size, M


def _pair_weights(n, rate):
    t = np.arange(n, dtype=np.float64)
    with np.errstate(invalid="ignore"):
        w = np.where(t[:, None] == t, 1.0, np.exp(-float(rate) * np.abs(t[:, None] - t)))
    return np.tril(w)


def attention_sequence_backward(q, k, v, rate, scale, state, gy, gstate):
    """Gradients of sum(gy y) + sum(gstate last) for one head of one sequence: ((gq, gk, gv, g0), their magnitudes)."""
    q, k, v, gy = (np.asarray(t, np.float64) for t in (q, k, v, gy))
    n = q.shape[0]
    S0 = np.zeros((q.shape[1], v.shape[1])) if state is None else np.asarray(state, np.float64)
    G = np.zeros_like(S0) if gstate is None else np.asarray(gstate, np.float64)
    w = _pair_weights(n, rate)
    keep = np.exp(-float(rate))
    ahead = keep ** np.arange(1, n + 1)[:, None]
    behind = keep ** np.arange(n - 1, -1, -1)[:, None]

    def both(f):
        return f(q, k, v, gy, S0, G), f(*(np.abs(t) for t in (q, k, v, gy, S0, G)))

    def grads(q, k, v, gy, S0, G):
        back, map_ = w * (gy @ v.T), w * (q @ k.T)
        return (scale * (back @ k + ahead * (gy @ S0.T)), scale * (back.T @ q) + behind * (v @ G.T),
                scale * (map_.T @ gy) + behind * (k @ G), scale * ((q * ahead).T @ gy) + keep ** n * G)
    return both(grads)


def logprob(y, targets, tau=1.0, top=0):
    """dict of logp, lse, entropy, top_ids, top_logp of logits y (k, batch)."""
    z = tau * np.asarray(y, np.float64)
    k, t = z.shape
    out = dict(logp=np.zeros(t), lse=np.full(t, -np.inf), entropy=np.zeros(t), top_ids=np.zeros((top, t), np.int64), top_logp=np.zeros((top, t)))
    for c in range(t):
        col = z[:, c]
        odd = bool(np.isnan(col).any() or (col == np.inf).any())
        with np.errstate(all="ignore"):
            if odd:
                lse, ent = np.nan, np.nan
            elif k == 0 or not (col > -np.inf).any():
                lse, ent = -np.inf, 0.0
            else:
                m = col.max()
                lse = m + np.log(np.exp(col - m).sum())
                p = np.exp(col - lse)
                ent = -(p[p > 0] * (col - lse)[p > 0]).sum()
        of = lambda i: np.nan if odd else -np.inf if lse == -np.inf else col[i] - lse
        out["lse"][c], out["entropy"][c] = lse, ent
        if 0 <= targets[c] < k:
            out["logp"][c] = of(targets[c])
        order = sorted(range(k), key=lambda i: (-np.inf if np.isnan(col[i]) else -col[i] if col[i] != np.inf else -1e400, i)) if top else []
        order.sort(key=lambda i: 0 if np.isnan(col[i]) else 1)
        for r in range(top):
            out["top_ids"][r, c] = order[r]
            out["top_logp"][r, c] = of(order[r])
    return out


def logprob_backward(y, targets, glogp, gentropy, glse, tau=1.0):
    """Gradient of sum(glogp logp + gentropy entropy + glse lse) into y; columns with NaN or +inf are NaN."""
    z = tau * np.asarray(y, np.float64)
    k, t = z.shape
    f = logprob(y, targets, tau)
    g = np.zeros((k, t))
    for c in range(t):
        if np.isnan(f["lse"][c]):
            g[:, c] = np.nan
            continue
        if f["lse"][c] == -np.inf:
            continue
        logp = z[:, c] - f["lse"][c]
        p = np.exp(logp)
        if 0 <= targets[c] < k:
            g[:, c] -= glogp[c] * p
            g[targets[c], c] += glogp[c]
        some = p > 0
        g[some, c] -= gentropy[c] * (p[some] * (logp[some] + f["entropy"][c]))
        g[:, c] += glse[c] * p
    return tau * g
