"""Plain 64-bit forms of the operators on logits and on updates, written from their definitions (include/pcm.h)."""
from __future__ import annotations

import numpy as np

NS_COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def token_logprobs(logits, tokens, allowed=None, temperature=1.0, top=0):
    """-> dict(logp, lse, entropy [rows], top_ids, top_logp [rows, top]), row by row."""
    z = np.asarray(logits, dtype=np.float64)
    rows, V = z.shape
    out = dict(logp=np.zeros(rows), lse=np.zeros(rows), entropy=np.zeros(rows), top_ids=np.full((rows, top), -1, np.int32),
               top_logp=np.full((rows, top), -np.inf))
    for r in range(rows):
        ok = np.ones(V, bool) if allowed is None else np.asarray(allowed, bool)
        ok = ok if ok.ndim == 1 else ok[r]
        ids = np.flatnonzero(ok)
        x = z[r, ids] / temperature
        broken = np.isnan(x).any() or np.isposinf(x).any()
        m = x.max() if len(x) else -np.inf
        empty = not broken and m == -np.inf
        if broken:
            lse = entropy = np.nan
        elif empty:
            lse, entropy = -np.inf, 0.0
        else:
            e = np.exp(x - m)
            lse = m + np.log(e.sum())
            p = e / e.sum()
            live = p > 0
            entropy = -(p[live] * (x[live] - lse)).sum()
        out["lse"][r], out["entropy"][r] = lse, entropy
        of = lambda j: -np.inf if empty else (np.nan if broken else z[r, j] / temperature - lse)
        t = int(tokens[r])
        if t >= 0:
            t = min(t, V - 1)
            out["logp"][r] = of(t) if ok[t] else -np.inf
        listed = [j for j in ids if not np.isnan(z[r, j])]
        for k, j in enumerate(sorted(listed, key=lambda j: (-z[r, j], j))[:top]):
            out["top_ids"][r, k], out["top_logp"][r, k] = j, of(j)
    return out


def token_logprobs_gradient(logits, tokens, dlogp, dentropy=None, allowed=None, temperature=1.0):
    """d logits of sum(dlogp * logp) + sum(dentropy * entropy)."""
    z = np.asarray(logits, dtype=np.float64)
    rows, V = z.shape
    got = token_logprobs(logits, tokens, allowed, temperature)
    g = np.zeros((rows, V))
    for r in range(rows):
        if not np.isfinite(got["lse"][r]):
            continue
        ok = np.ones(V, bool) if allowed is None else np.asarray(allowed, bool)
        ok = ok if ok.ndim == 1 else ok[r]
        ids = np.flatnonzero(ok & (z[r] > -np.inf))
        logp = z[r, ids] / temperature - got["lse"][r]
        p = np.exp(logp)
        t = int(tokens[r])
        d = 0.0 if t < 0 else float(dlogp[r])
        g[r, ids] -= d * p
        if t >= 0 and ok[min(t, V - 1)]:
            g[r, min(t, V - 1)] += d
        if dentropy is not None:
            g[r, ids] -= float(dentropy[r]) * p * (logp + got["entropy"][r])
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
