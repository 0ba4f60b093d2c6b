"""Plain 64-bit forms of the operators on logits and on updates, written from their definitions (include/pcm.h)."""
from __future__ import annotations

import numpy as np

NS_COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def _row(z, ok, temperature):
    """-> (ids of the allowed tokens, x - max x of them, log sum e^(x - max x), max x) of a row, x = z / temperature; the sum relative to
    the largest logit, so that logits of any size leave it what it is.  The sum is NaN where there is none, -inf where it is empty."""
    ids = np.flatnonzero(ok)
    z = z[ids]
    if np.isnan(z).any() or np.isposinf(z).any():
        return ids, np.full(len(ids), np.nan), np.nan, np.nan
    most = z.max() if len(ids) else -np.inf
    if most == -np.inf:
        return ids, np.full(len(ids), -np.inf), -np.inf, -np.inf
    a = (z - most) / temperature
    return ids, a, np.log(np.exp(a).sum()), most / temperature


def _allowed(allowed, r, V):
    ok = np.ones(V, bool) if allowed is None else np.asarray(allowed, bool)
    return ok if ok.ndim == 1 else ok[r]


def token_logprobs(logits, tokens, allowed=None, temperature=1.0, top=0):
    """-> dict(logp, lse, entropy [rows], top_ids, top_logp [rows, top]), row by row."""
    z = np.asarray(logits, dtype=np.float64)
    rows, V = z.shape
    out = dict(logp=np.zeros(rows), lse=np.zeros(rows), entropy=np.zeros(rows), top_ids=np.full((rows, top), -1, np.int32),
               top_logp=np.full((rows, top), -np.inf))
    for r in range(rows):
        ok = _allowed(allowed, r, V)
        ids, a, log_sum, most = _row(z[r], ok, temperature)
        logp = np.full(V, -np.inf)
        if log_sum == -np.inf:
            out["lse"][r], out["entropy"][r] = -np.inf, 0.0
        else:
            logp[ids] = a - log_sum
            out["lse"][r] = most + log_sum
            live = ~(logp[ids] == -np.inf)
            out["entropy"][r] = -(np.exp(logp[ids][live]) * logp[ids][live]).sum()
        t = int(tokens[r])
        if t >= 0:
            out["logp"][r] = logp[min(t, V - 1)]
        listed = ids[~np.isnan(z[r, ids])]
        best = listed[np.argsort(-z[r, listed], kind="stable")[:top]]
        out["top_ids"][r, :len(best)], out["top_logp"][r, :len(best)] = best, logp[best]
    return out


def token_logprobs_gradient(logits, tokens, dlogp, dentropy=None, allowed=None, temperature=1.0):
    """d logits of sum(dlogp * logp) + sum(dentropy * entropy)."""
    z = np.asarray(logits, dtype=np.float64)
    rows, V = z.shape
    g = np.zeros((rows, V))
    for r in range(rows):
        ok = _allowed(allowed, r, V)
        ids, a, log_sum, _ = _row(z[r], ok, temperature)
        if not np.isfinite(log_sum):
            continue
        ids, logp = ids[a > -np.inf], a[a > -np.inf] - log_sum
        p = np.exp(logp)
        t = int(tokens[r])
        d = 0.0 if t < 0 else float(dlogp[r])
        g[r, ids] -= d * p
        if t >= 0 and ok[min(t, V - 1)]:
            g[r, min(t, V - 1)] += d
        if dentropy is not None:
            g[r, ids] -= float(dentropy[r]) * p * (logp - (p * logp).sum())
    return g / temperature


def orthogonalise(update, ns_steps=5):
    """Newton-Schulz steps on update / its Frobenius norm."""
    a, b, c = NS_COEFFICIENTS
    x = np.asarray(update, dtype=np.float64)
    norm = np.sqrt((x * x).sum())
    if norm == 0.0:
        return np.zeros_like(x)
    x = x / norm
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.T
    for _ in range(ns_steps):
        gram = x @ x.T
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.T if tall else x


def muon_step(weights, grads, momentum, lr, momentum_coef=0.95, nesterov=True, weight_decay=0.0, ns_steps=5, scale="shape"):
    """-> (weights, momentum, the orthogonalised updates), lists of new arrays."""
    new_w, new_m, steps = [], [], []
    for w, g, m in zip(weights, grads, momentum):
        w, g, m = (np.asarray(x, dtype=np.float64) for x in (w, g, m))
        m = momentum_coef * m + g
        o = orthogonalise(g + momentum_coef * m if nesterov else m, ns_steps)
        rows, cols = w.shape
        s = np.sqrt(max(1.0, cols / rows)) if scale == "shape" else 0.2 * np.sqrt(max(rows, cols))
        new_w.append(w * (1.0 - lr * weight_decay) - lr * s * o)
        new_m.append(m)
        steps.append(o)
    return new_w, new_m, steps
