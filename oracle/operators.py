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


# ---- moments in 8 bits ---------------------------------------------------------------------------

MOMENT_BLOCK = 128
M_FIELD, V_FIELD = 15, 31            # largest exponent field of a code of m (with a sign) and of v


def _philox_groups(groups, step, seed):
    """Philox-4x32-10 of counters (group low, group high, step low, step high), as [groups, 8] numbers of 16 bits."""
    low = np.uint64(0xFFFFFFFF)
    g = np.asarray(groups, np.uint64)
    c = [g & low, g >> np.uint64(32), np.full_like(g, step & 0xFFFFFFFF), np.full_like(g, step >> 32)]
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), q & low, (p >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), p & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    words = np.stack(c, axis=1)
    return np.stack([words & np.uint64(0xFFFF), words >> np.uint64(16)], axis=2).reshape(len(g), 8).astype(np.int64)


def moment_codes(x, random, field):
    """-> (codes, block exponents) of fp32 values, whole blocks of them, with 16 random bits each; real arithmetic, value by value.

    The two neighbours of a value among (8 + k) 2^e, k = 0 .. 7, e whole: the upper one where the part behind the point and random / 2^16
    make one.  Below the block's reach the spacing stays what it is there."""
    x = np.asarray(x, np.float32).reshape(-1, MOMENT_BLOCK)
    u = np.asarray(random, np.int64).reshape(x.shape)
    codes, tops = np.zeros(x.shape, np.uint8), np.zeros(len(x), np.uint8)
    for b in range(len(x)):
        a = np.abs(x[b].astype(np.float64))
        if not np.all(np.isfinite(a)):
            tops[b] = 255
            continue
        a[a < 2.0 ** -126] = 0.0
        live = np.flatnonzero(a)
        if len(live) == 0:
            continue
        exponent = np.frexp(a[live])[1] - 1
        near = np.floor(a[live] / 2.0 ** (exponent - 3) + u[b, live] / 65536.0) * 2.0 ** (exponent - 3)
        top = int((np.frexp(near)[1] - 1).max()) + 127
        tops[b] = top
        if top >= 255:
            tops[b] = 255
            continue
        least = 2.0 ** (top - field - 129.0)
        for i, value in zip(live, near):
            if value < 8 * least:
                k = int(np.floor((np.floor(a[i] / least * 65536.0) + u[b, i]) / 65536.0))
            else:
                e = int(np.frexp(value)[1]) - 1
                k = 8 * (e + 127 - top + field) + int(round(value / 2.0 ** (e - 3))) - 8
            codes[b, i] = max(k, 1) if field == V_FIELD else (k + 128 if k and np.signbit(x[b, i]) else k)
    return codes.reshape(-1), tops


def moment_values(codes, tops, field):
    """The values that codes and block exponents stand for, in 64 bits."""
    codes = np.asarray(codes, np.int64).reshape(-1, MOMENT_BLOCK)
    top = np.asarray(tops, np.int64)[:, None]
    c = codes if field == V_FIELD else codes & 127
    x = np.where(c >= 8, (8.0 + c % 8) * 2.0 ** (top - field - 130.0 + c // 8), c * 2.0 ** (top - field - 129.0))
    x = np.where(top == 255, np.nan, x)
    return (x if field == V_FIELD else np.where(codes > 127, -x, x)).reshape(-1)


def adamw_many_eight(weights, grads, state, step, seed, lr, beta1, beta2, eps, weight_decay, max_grad_norm):
    """One step on moments in 8 bits, `state` = (m codes, v codes, m exponents, v exponents) of all tensors behind one another, each padded
    to whole blocks.  Norm and factor in 64 bits, moments in 32 (each operation rounded), the update in 64.
    -> (weights in 64 bits, state, norm)"""
    f = np.float32
    norm = np.sqrt(sum(float((np.asarray(g, np.float64) ** 2).sum()) for g in grads))
    scale = f(1.0) if max_grad_norm is None else f(np.minimum(1.0, max_grad_norm / (norm + 1e-6)))
    m_old = moment_values(state[0], state[2], M_FIELD).astype(f)
    v_old = moment_values(state[1], state[3], V_FIELD).astype(f)
    m, v, out, at = np.zeros_like(m_old), np.zeros_like(v_old), [], 0
    for w, g in zip(weights, grads):
        n = np.asarray(g).size
        x = np.asarray(g, f).reshape(-1) * scale
        part = slice(at, at + n)
        m[part] = f(beta1) * m_old[part] + f(1.0 - beta1) * x
        v[part] = f(beta2) * v_old[part] + f(1.0 - beta2) * (x * x)
        mh = m[part].astype(np.float64) / (1.0 - beta1 ** step)
        vh = v[part].astype(np.float64) / (1.0 - beta2 ** step)
        out.append(np.asarray(w, np.float64).reshape(-1) * (1.0 - lr * weight_decay) - lr * mh / (np.sqrt(vh) + eps))
        at += -(-n // MOMENT_BLOCK) * MOMENT_BLOCK
    random = _philox_groups(np.arange(len(m) // 8), step, seed).reshape(-1)
    mc, mt = moment_codes(m, random, M_FIELD)
    vc, vt = moment_codes(v, random, V_FIELD)
    return out, (mc, vc, mt, vt), norm


# ---- log-probabilities through a projection ------------------------------------------------------------

def linear_logprobs(hidden, weight, tokens, temperature=1.0):
    """-> dict(logp, lse, entropy [rows]) of the logits hidden @ weight; zeros for rows without a token (whatever they hold)."""
    hidden, weight = np.asarray(hidden, np.float64), np.asarray(weight, np.float64)
    rows = len(hidden)
    out = {k: np.zeros(rows) for k in ("logp", "lse", "entropy")}
    live = np.flatnonzero(np.asarray(tokens) >= 0)
    if len(live):
        got = token_logprobs(hidden[live] @ weight, np.asarray(tokens)[live], temperature=temperature)
        for k in out:
            out[k][live] = got[k]
    return out


def linear_logits_gradient(hidden, weight, tokens, dlogp, dentropy=None, temperature=1.0):
    """d of sum(dlogp * logp) + sum(dentropy * entropy) in hidden @ weight [rows, V]; zeros for rows without a token."""
    hidden, weight = np.asarray(hidden, np.float64), np.asarray(weight, np.float64)
    g = np.zeros((len(hidden), weight.shape[1]))
    live = np.flatnonzero(np.asarray(tokens) >= 0)
    if len(live):
        g[live] = token_logprobs_gradient(hidden[live] @ weight, np.asarray(tokens)[live], np.asarray(dlogp)[live],
                                          None if dentropy is None else np.asarray(dentropy)[live], temperature=temperature)
    return g


def linear_logprobs_gradient(hidden, weight, tokens, dlogp, dentropy=None, temperature=1.0):
    """-> (d hidden, d weight)."""
    g = linear_logits_gradient(hidden, weight, tokens, dlogp, dentropy, temperature)
    h = np.where(np.asarray(tokens)[:, None] >= 0, np.asarray(hidden, np.float64), 0.0)
    return g @ np.asarray(weight, np.float64).T, h.T @ g
