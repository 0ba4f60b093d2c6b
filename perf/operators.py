"""The operators around the actor step that work on a policy's logits and on its weight updates: log-probabilities of
given tokens (with entropy and the likeliest alternatives), their gradient, the orthogonalised update and the optimizer
step that applies it; the sizes they are timed at.

A case is a dict of plain values.  `listed()` names the fixed ones, `draw(rng)` makes one more of the same ranges;
`prepare(case, seed)` makes on the GPU what a training program holds before the call, `run(state)` is one pass,
`work(case)` the bytes and operations that the pass cannot do without and `exact(case, seed)` the pass in 64 bits.  With
`own` false, run() computes the operators from elementary torch operations in 32 bits; with `own` true it calls the library.

Four kinds of pass:
  logp   pcm_token_logprobs: log p(token), log-sum-exp and, as asked, entropy and the `top` likeliest tokens of each row
  grad   pcm_token_logprobs_backward: d logits from the gradients of log p and of the entropy
  orth   pcm_orthogonalise: Newton-Schulz iteration on a stack of matrices
  muon   pcm_muon_step: momentum, orthogonalisation and weight update of the head's matrices
"""
from __future__ import annotations

import math

import torch

own = False

# the quintic x -> a x + b x^3 + c x^5 of the singular values, and how often it is applied
NS_A, NS_B, NS_C = 3.4445, -4.7750, 2.0315
NS_STEPS = 5
MOMENTUM = 0.95
LR, WEIGHT_DECAY = 0.02, 0.01


# ---- the cases ---------------------------------------------------------------------------------

def _logp(name, rows, V, dtype, tokens="i32", entropy=True, top=0, mask="none", temperature=1.0, pad=0):
    return dict(name=name, kind="logp", rows=rows, V=V, dtype=dtype, tokens=tokens, entropy=entropy, top=top, mask=mask,
                temperature=temperature, pad=pad)


def _grad(name, rows, V, dtype, tokens="i32", entropy=True, mask="none", temperature=1.0, pad=0):
    return dict(name=name, kind="grad", rows=rows, V=V, dtype=dtype, tokens=tokens, entropy=entropy, mask=mask,
                temperature=temperature, pad=pad)


def _orth(name, rows, cols, dtype, batch=1):
    return dict(name=name, kind="orth", rows=rows, cols=cols, dtype=dtype, batch=batch)


def _muon(name, d, ff, V=256, nesterov=True, scale="shape", bf16=True):
    return dict(name=name, kind="muon", d=d, ff=ff, V=V, nesterov=nesterov, scale=scale, bf16=bf16)


def listed():
    return [
        # one decoding step of eight rollouts whose policy answers over a whole vocabulary: all latency
        _logp("logp-decode", 8, 131072, "bf16", top=8),
        # the old-policy pass over every action token of a masked batch (768 chunks of 56 tokens, 256 bins)
        _logp("logp-bins", 43008, 256, "bf16", tokens="u8"),
        # sampled with a temperature under a grammar that differs from row to row, logits a view of a wider matrix
        _logp("logp-masked", 777, 32003, "f32", tokens="i64", top=20, mask="rows", temperature=0.7, pad=5),
        # long sequences scored with their likeliest alternatives for the log
        _logp("logp-long", 4096, 65536, "bf16", top=5),
        # gradient of the clipped surrogate with an entropy bonus at the framework's own bins
        _grad("grad-bins", 43008, 256, "bf16", tokens="u8"),
        # fp32 logits, some tokens never allowed, no entropy bonus, an odd vocabulary
        _grad("grad-masked", 1111, 50021, "f32", entropy=False, mask="tokens", pad=3),
        # supervised warm start over a whole vocabulary, the largest pass over logits
        _grad("grad-wide", 4096, 131072, "bf16"),
        # one projection of the tiny instance: all launch latency
        _orth("orth-small", 256, 1024, "f32"),
        # a stack of odd-sized bf16 updates
        _orth("orth-odd", 1001, 2815, "bf16", batch=3),
        # one projection of the 7B policy's head
        _orth("orth-large", 4096, 11008, "f32"),
        # the head of the tiny instance
        _muon("muon-tiny-head", 256, 1024),
        # the head of the 7B policy: three projections and the logit projection
        _muon("muon-7b-head", 4096, 11008),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["logp", "logp", "grad", "grad", "orth", "orth", "muon"])
    if kind in ("logp", "grad"):
        V = rng.choice([256, _log_int(rng, 2, 131072), _log_int(rng, 2048, 131072)])
        rows = _log_int(rng, 1, min(43008, (1 << 28) // V))
        dtype = rng.choice(["bf16", "f32"])
        tokens = rng.choice(["u8", "i32"] if V <= 256 else ["i32", "i64"])
        mask, temperature, pad = rng.choice(["none", "tokens", "rows"]), rng.choice([1.0, 0.7, 1.3]), rng.choice([0, 0, 1, 8, 11])
        entropy = rng.random() < 0.6
        if kind == "logp":
            case = _logp("", rows, V, dtype, tokens, entropy, min(V, rng.choice([0, 1, 5, 20, 64])), mask, temperature, pad)
        else:
            case = _grad("", rows, V, dtype, tokens, entropy, mask, temperature, pad)
    elif kind == "orth":
        rows, cols = _log_int(rng, 16, 4096), _log_int(rng, 16, 11008)
        if rng.random() < 0.4:
            rows, cols = cols, rows
        most = max(1, min(4, 4096 * 4096 * 11008 // (min(rows, cols) * rows * cols)))
        case = _orth("", rows, cols, rng.choice(["bf16", "f32"]), rng.randint(1, most))
    else:
        case = _muon("", _log_int(rng, 64, 2048), _log_int(rng, 128, 5504), V=rng.choice([101, 256, 256, 512]),
                     nesterov=rng.random() < 0.7, scale=rng.choice(["shape", "rms"]), bf16=rng.random() < 0.7)
    del case["name"]
    return case


# ---- inputs ------------------------------------------------------------------------------------

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "u8": torch.uint8, "i32": torch.int32, "i64": torch.int64}


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _logit_inputs(case, seed):
    gen = _generator(seed)
    rows, V = case["rows"], case["V"]
    wide = torch.empty((rows, V + case["pad"]), dtype=TYPES[case["dtype"]], device="cuda")
    # rows from undecided to almost certain ones; the token is the one preferred by a draw on a part of the scale
    spread = 0.5 + 4.5 * torch.rand((rows, 1), generator=gen, device="cuda")
    block = max(1, (1 << 26) // (V + case["pad"]))
    for r in range(0, rows, block):
        wide[r:r + block] = spread[r:r + block] * torch.randn((min(block, rows - r), V + case["pad"]), generator=gen, device="cuda")
    logits = wide[:, :V]
    allowed = None
    if case["mask"] == "tokens":
        allowed = torch.rand(V, generator=gen, device="cuda") < 0.9
        allowed[V // 2] = True
    elif case["mask"] == "rows":
        share = torch.rand((rows, 1), generator=gen, device="cuda")
        share[torch.rand((rows, 1), generator=gen, device="cuda") < 0.01] = 0.0       # a grammar at its end allows nothing
        allowed = torch.rand((rows, V), generator=gen, device="cuda") < share
    guess = torch.randint(0, V, (rows, 16), generator=gen, device="cuda")
    best = torch.gather(logits, 1, guess).float().argmax(dim=1, keepdim=True)
    tokens = torch.gather(guess, 1, best)[:, 0].to(TYPES[case["tokens"]])
    return dict(logits=logits, tokens=tokens, allowed=allowed), gen


def _row_blocks(rows, V):
    block = max(1, (1 << 26) // V)
    return [(r, min(rows, r + block)) for r in range(0, rows, block)]


def _allowed_of(allowed, lo, hi):
    return allowed if allowed is None or allowed.dim() == 1 else allowed[lo:hi]


def _statistics(logits, allowed, temperature):
    """Log-sum-exp and entropy of the allowed tokens of each row in 64 bits (-inf and 0 where none is)."""
    lse, entropy = [], []
    for lo, hi in _row_blocks(*logits.shape):
        x = logits[lo:hi].double() / temperature
        if allowed is not None:
            x = x.masked_fill(~_allowed_of(allowed, lo, hi), -math.inf)
        s = torch.logsumexp(x, dim=1)
        p = torch.exp(x - torch.where(s > -math.inf, s, 0.0)[:, None])
        lse.append(s)
        entropy.append(-(p * torch.where(p > 0, x - s[:, None], 0.0)).sum(dim=1))
    return torch.cat(lse), torch.cat(entropy)


def _update_like(rows, cols, gen):
    """A matrix such as a gradient is: a few directions that matter, one less than the other, and noise."""
    r = min(64, rows, cols)
    left = torch.randn((rows, r), generator=gen, device="cuda") / torch.arange(1, r + 1, device="cuda")
    g = left @ torch.randn((r, cols), generator=gen, device="cuda")
    noise = torch.randn((rows, cols), generator=gen, device="cuda")
    return 1e-3 * (g + 0.3 * g.square().mean().sqrt() * noise)


def prepare(case, seed):
    kind = case["kind"]
    if kind in ("logp", "grad"):
        state, gen = _logit_inputs(case, seed)
        state.update(kind=kind, temperature=case["temperature"], want_entropy=case["entropy"], top=case.get("top", 0))
        if kind == "grad":
            rows = case["rows"]
            lse, entropy = _statistics(state["logits"], state["allowed"], case["temperature"])
            state.update(lse=lse.float(), dlogp=torch.randn(rows, generator=gen, device="cuda") / rows,
                         entropy=entropy.float() if case["entropy"] else None,
                         dentropy=0.1 * torch.rand(rows, generator=gen, device="cuda") / rows if case["entropy"] else None)
        return state
    gen = _generator(seed)
    if kind == "orth":
        update = torch.stack([_update_like(case["rows"], case["cols"], gen) for _ in range(case["batch"])])
        return dict(kind=kind, update=update.to(TYPES[case["dtype"]]))
    d, ff, V = case["d"], case["ff"], case["V"]
    shapes = ((d, ff), (d, ff), (ff, d), (d, V))
    weights = [0.02 * torch.randn(s, generator=gen, device="cuda") for s in shapes]
    return dict(kind=kind, weights=weights, grads=[_update_like(*s, gen) for s in shapes],
                momentum=[3.0 * _update_like(*s, gen) for s in shapes],
                weights_bf16=[w.to(torch.bfloat16) for w in weights] if case["bf16"] else None,
                nesterov=case["nesterov"], scale=case["scale"])


# ---- the plain forms ---------------------------------------------------------------------------

def _ordered(x):
    """fp32 values as integers of the same order."""
    bits = (x + 0.0).view(torch.int32)
    return bits ^ ((bits >> 31) & 0x7FFFFFFF)


def _plain_logp(s):
    z = s["logits"].float()
    rows, V = z.shape
    allowed = s["allowed"]
    x = z * (1.0 / s["temperature"])
    if allowed is not None:
        x = x.masked_fill(~allowed, -math.inf)
    top = x.max(dim=1, keepdim=True).values
    top = torch.where(top > -math.inf, top, 0.0)
    e = torch.exp(x - top)
    total = e.sum(dim=1, keepdim=True)
    lse = top + torch.log(total)
    given = torch.gather(x, 1, s["tokens"].long()[:, None])
    out = dict(lse=lse[:, 0], logp=torch.where(given > -math.inf, (given - top) - torch.log(total), -math.inf)[:, 0])
    if s["want_entropy"]:
        mean = (e * torch.where(e > 0, x - top, 0.0)).sum(dim=1, keepdim=True)
        out["entropy"] = torch.where(total > 0, torch.log(total) - mean / total, 0.0)[:, 0]
    if s["top"]:
        # the largest (logit, then the smaller index first), as one integer a token
        key = (_ordered(z).long() << 32) + (0xFFFFFFFF - torch.arange(V, device="cuda"))
        none = -(1 << 63)
        if allowed is not None:
            key = key.masked_fill(~allowed, none)
        best = torch.topk(key, s["top"], dim=1).values
        ids = torch.where(best == none, -1, 0xFFFFFFFF - (best & 0xFFFFFFFF))
        found = (torch.gather(x, 1, ids.clamp(min=0)) - top) - torch.log(total)
        out["top_ids"] = ids.int()
        out["top_logp"] = torch.where(ids >= 0, found, -math.inf)
    return out


def _plain_grad(s):
    z = s["logits"].float() * (1.0 / s["temperature"])
    lse = s["lse"][:, None]
    logp = z - torch.where(lse > -math.inf, lse, 0.0)
    p = torch.exp(logp)
    g = -s["dlogp"][:, None] * p
    if s["dentropy"] is not None:
        g = g - s["dentropy"][:, None] * p * (logp + s["entropy"][:, None])
    token = s["tokens"].long()[:, None]
    g.scatter_add_(1, token, s["dlogp"][:, None])
    if s["allowed"] is not None:
        g = g.masked_fill(~s["allowed"], 0.0)
    return (g * (1.0 / s["temperature"])).to(s["logits"].dtype)


def _plain_orth(update):
    g = update.float()
    x = g.mT.contiguous() if g.shape[-2] > g.shape[-1] else g
    norm = x.square().sum(dim=(-2, -1), keepdim=True).sqrt()
    x = torch.where(norm > 0, x / norm, 0.0)
    for _ in range(NS_STEPS):
        gram = x @ x.mT.contiguous()
        x = NS_A * x + (NS_B * gram + NS_C * (gram @ gram)) @ x
    return x.mT.contiguous() if g.shape[-2] > g.shape[-1] else x


def _shape_scale(rows, cols, rule):
    return math.sqrt(max(1.0, cols / rows)) if rule == "shape" else 0.2 * math.sqrt(max(rows, cols))


def _plain_muon(s):
    for i, (g, w, m) in enumerate(zip(s["grads"], s["weights"], s["momentum"])):
        m.mul_(MOMENTUM).add_(g)
        o = _plain_orth(g + MOMENTUM * m if s["nesterov"] else m)
        w.mul_(1.0 - LR * WEIGHT_DECAY).sub_(LR * _shape_scale(*w.shape, s["scale"]) * o)
        if s["weights_bf16"] is not None:
            s["weights_bf16"][i].copy_(w)


def run(state):
    kind = state["kind"]
    if own:
        import paper_2605_16154_amd as pcm
    if kind == "logp":
        if not own:
            return _plain_logp(state)
        return pcm.pcm_token_logprobs(state["logits"], state["tokens"], allowed=state["allowed"], temperature=state["temperature"],
                                      want_entropy=state["want_entropy"], top=state["top"])
    if kind == "grad":
        if not own:
            return _plain_grad(state)
        return pcm.pcm_token_logprobs_backward(state["logits"], state["tokens"], state["lse"], state["dlogp"], entropy=state["entropy"],
                                               dentropy=state["dentropy"], allowed=state["allowed"], temperature=state["temperature"])
    if kind == "orth":
        if not own:
            return _plain_orth(state["update"]).to(state["update"].dtype)
        return pcm.pcm_orthogonalise(state["update"], ns_steps=NS_STEPS)
    if own:
        pcm.pcm_muon_step(state["grads"], state["weights"], state["momentum"], lr=LR, momentum_coef=MOMENTUM, nesterov=state["nesterov"],
                          weight_decay=WEIGHT_DECAY, ns_steps=NS_STEPS, scale=state["scale"], weights_bf16=state["weights_bf16"])
    else:
        _plain_muon(state)
    return dict(weights=state["weights"], momentum=state["momentum"], weights_bf16=state["weights_bf16"])


# ---- what a pass needs, and its results in 64 bits -----------------------------------------------

def _ns_flops(rows, cols):
    """Multiply-adds (as two operations) of the iteration in the cheaper of two orders, symmetric products counted by
    half: every step on the matrix, or the steps on its Gram matrix and their product applied to the matrix once."""
    m, n = min(rows, cols), max(rows, cols)
    direct = NS_STEPS * (m * m * n + m * m * m + 2 * m * m * n)
    gram = m * m * n + (NS_STEPS + (NS_STEPS - 1) * 3) * m * m * m + 2 * m * m * n
    return min(direct, gram)


def work(case):
    kind = case["kind"]
    if kind in ("logp", "grad"):
        rows, V = case["rows"], case["V"]
        size = {"bf16": 2, "f32": 4}[case["dtype"]]
        mask = {"none": 0, "tokens": V, "rows": rows * V}[case["mask"]]
        token = {"u8": 1, "i32": 4, "i64": 8}[case["tokens"]]
        if kind == "logp":
            return {"bytes": rows * V * size + mask + rows * (token + 8 + 4 * case["entropy"] + 8 * case["top"]), "flops": 4 * rows * V}
        return {"bytes": 2 * rows * V * size + mask + rows * (token + 8 + 8 * case["entropy"]), "flops": 6 * rows * V}
    if kind == "orth":
        n = case["batch"] * case["rows"] * case["cols"]
        return {"bytes": 2 * n * {"bf16": 2, "f32": 4}[case["dtype"]], "flops": case["batch"] * _ns_flops(case["rows"], case["cols"])}
    d, ff, V = case["d"], case["ff"], case["V"]
    n = 3 * d * ff + d * V
    return {"bytes": n * (20 + 2 * case["bf16"]), "flops": 3 * _ns_flops(d, ff) + _ns_flops(d, V)}


def _exact_orth(update):
    """Every step is a polynomial of x x^T times x, so the steps are gathered there and applied at the end."""
    x = update.double()
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.t().contiguous()
    norm = torch.linalg.vector_norm(x)
    if norm > 0:
        x = x / norm
    gram = torch.matmul(x, x.t().contiguous())
    steps = torch.eye(x.shape[0], dtype=torch.float64, device=x.device)
    for k in range(NS_STEPS):
        one = NS_B * gram + NS_C * torch.matmul(gram, gram)
        one.diagonal().add_(NS_A)
        steps = torch.matmul(one, steps)
        if k + 1 < NS_STEPS:
            gram = torch.matmul(torch.matmul(one, gram), one)
    out = torch.matmul(steps, x)
    return out.t().contiguous() if tall else out


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "orth":
        return torch.stack([_exact_orth(u) for u in s["update"]])
    if kind == "muon":
        momentum = [MOMENTUM * m.double() + g.double() for m, g in zip(s["momentum"], s["grads"])]
        steps = [_exact_orth(g.double() + MOMENTUM * m if s["nesterov"] else m) for m, g in zip(momentum, s["grads"])]
        weights = [(1.0 - LR * WEIGHT_DECAY) * w.double() - LR * _shape_scale(*w.shape, s["scale"]) * o for w, o in zip(s["weights"], steps)]
        return dict(weights=weights, momentum=momentum, weights_bf16=weights if case["bf16"] else None)
    lse, entropy = _statistics(s["logits"], s["allowed"], s["temperature"])
    rows, V = s["logits"].shape
    token = s["tokens"].long()
    outs = []
    for lo, hi in _row_blocks(rows, V):
        logp = s["logits"][lo:hi].double() / s["temperature"] - torch.where(lse[lo:hi] > -math.inf, lse[lo:hi], 0.0)[:, None]
        if s["allowed"] is not None:
            logp = logp.masked_fill(~_allowed_of(s["allowed"], lo, hi), -math.inf)
        if kind == "logp":
            outs.append((torch.gather(logp, 1, token[lo:hi, None])[:, 0], torch.topk(logp, s["top"], dim=1).values))
            continue
        p = torch.exp(logp)
        one = torch.zeros_like(p).scatter_(1, token[lo:hi, None], 1.0)
        g = s["dlogp"][lo:hi, None].double() * (one - p)
        if s["dentropy"] is not None:
            g -= s["dentropy"][lo:hi, None].double() * p * (torch.where(p > 0, logp, 0.0) + entropy[lo:hi, None])
        outs.append((torch.where(logp > -math.inf, g, 0.0) / s["temperature"]).float() if rows * V > 1 << 27
                    else torch.where(logp > -math.inf, g, 0.0) / s["temperature"])
    if kind == "grad":
        return torch.cat(outs)
    got = dict(lse=lse, logp=torch.cat([a for a, _ in outs]))
    if s["want_entropy"]:
        got["entropy"] = entropy
    if s["top"]:
        got.update(top_ids=None, top_logp=torch.cat([b for _, b in outs]))
    return got
