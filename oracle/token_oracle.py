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


def layer_norm(x, weight, bias, eps):
    """(y, mean, rstd) over the last axis."""
    x = np.asarray(x, np.float64)
    mean = x.mean(-1, keepdims=True)
    rstd = 1.0 / np.sqrt(((x - mean) ** 2).mean(-1, keepdims=True) + eps)
    y = (x - mean) * rstd
    y = y * (1.0 if weight is None else weight) + (0.0 if bias is None else bias)
    return y, mean[..., 0], rstd[..., 0]


def layer_norm_backward(x, gy, weight, eps):
    """(gx, gweight, gbias) of sum(gy y), rows x (rows, width)."""
    x, gy = np.asarray(x, np.float64), np.asarray(gy, np.float64)
    mean = x.mean(-1, keepdims=True)
    rstd = 1.0 / np.sqrt(((x - mean) ** 2).mean(-1, keepdims=True) + eps)
    hat = (x - mean) * rstd
    g = gy * (1.0 if weight is None else weight)
    gx = rstd * (g - g.mean(-1, keepdims=True) - hat * (g * hat).mean(-1, keepdims=True))
    return gx, (gy * hat).sum(0), gy.sum(0)


def _softmax(z):
    z = np.asarray(z, np.float64)
    top = z.max() if len(z) else -np.inf
    if np.isnan(z).any() or not np.isfinite(top):
        return None, None
    e = np.exp(z - top)
    return e / e.sum(), z - top - np.log(e.sum())


def verify_drafts(y, z, drafts, starts, tau, draft_tau, chances, next_chances, greedy=False):
    """(accepted, next, logp, next_logp) sequence by sequence, column by column."""
    k, t = y.shape
    b = len(starts) - 1
    accepted, following = np.zeros(b, np.int64), np.full(b, -1, np.int64)
    logp, next_logp = np.zeros(t), np.zeros(b)
    for i in range(b):
        going = True
        for c in range(starts[i], starts[i + 1]):
            p, log = _softmax(tau * y[:, c])
            x = int(drafts[c]) if c + 1 < starts[i + 1] and 0 <= drafts[c] < k else None
            if x is not None:
                logp[c] = np.nan if p is None else log[x]
            if not going:
                continue
            if p is None:
                going = False
                continue
            if greedy:
                best = int(np.argmax(y[:, c]))
                if x == best:
                    accepted[i] += 1
                    continue
                following[i], next_logp[i], going = best, log[best], False
                continue
            q = None
            if x is not None:
                q = (np.arange(k) == x) * 1.0 if z is None else _softmax(draft_tau * z[:, c])[0]
            if q is not None and chances[c] * q[x] < p[x]:
                accepted[i] += 1
                continue
            left = p if q is None else np.maximum(p - q, 0.0)
            left = left if left.sum() > 0.0 else p
            run = np.cumsum(left)
            past = np.nonzero((run > next_chances[i] * run[-1]) & (left > 0.0))[0]
            at = int(past[0]) if len(past) else int(np.nonzero(left > 0.0)[0][-1])
            following[i], next_logp[i], going = at, log[at], False
    return accepted, following, logp, next_logp


def delta_sequence(q, k, v, rates, beta, scale, state=None):
    """One head of one sequence by the gated delta rule, token by token: (y, last state, sizes).  The update is a contraction for keys up to length 1 and beta from 0 to 2:
    errors do not grow, and are measured against sizes = the largest length of a column of the state, the largest |u|, of each column."""
    q, k, v, rates, beta = (np.asarray(t, np.float64) for t in (q, k, v, rates, beta))
    S = np.zeros((q.shape[1], v.shape[1])) if state is None else np.asarray(state, np.float64).copy()
    y, length, most = np.zeros(v.shape), np.sqrt((S ** 2).sum(0)), np.zeros(v.shape[1])
    for t in range(q.shape[0]):
        S = np.exp(-rates[t]) * S
        u = beta[t] * (v[t] - k[t] @ S)
        S = S + np.outer(k[t], u)
        y[t] = scale * (q[t] @ S)
        length = np.maximum(length, np.sqrt((S ** 2).sum(0)))
        most = np.maximum(most, np.abs(u) + np.abs(beta[t] * v[t]))
    return y, S, length + most


def delta_sequence_backward(q, k, v, rates, beta, scale, state, gy, gstate):
    """Gradients of sum(gy y) + sum(gstate last): (gq, gk, gv, grates, gbeta, g0), and the largest length of a column of the state's gradient."""
    q, k, v, rates, beta, gy = (np.asarray(t, np.float64) for t in (q, k, v, rates, beta, gy))
    n = q.shape[0]
    S = np.zeros((q.shape[1], v.shape[1])) if state is None else np.asarray(state, np.float64).copy()
    steps = []
    for t in range(n):
        before = np.exp(-rates[t]) * S
        miss = v[t] - k[t] @ before
        S = before + np.outer(k[t], beta[t] * miss)
        steps.append((before, miss, S))
    G = np.zeros_like(S) if gstate is None else np.asarray(gstate, np.float64).copy()
    gq, gk, gv, gr, gb = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape), np.zeros(n), np.zeros(n)
    length = np.sqrt((G ** 2).sum(0))
    for t in range(n - 1, -1, -1):
        before, miss, after = steps[t]
        gq[t] = scale * (after @ gy[t])
        G = G + scale * np.outer(q[t], gy[t])
        length = np.maximum(length, np.sqrt((G ** 2).sum(0)))
        gu = k[t] @ G
        gb[t] = gu @ miss
        gv[t] = beta[t] * gu
        gk[t] = G @ (beta[t] * miss) - before @ gv[t]
        G = G - np.outer(k[t], gv[t])
        gr[t] = -(G * before).sum()
        G = np.exp(-rates[t]) * G
    return (gq, gk, gv, gr, gb, G), length
