"""The operators around the last layer of a policy and the update of all its parameters: log-probabilities of given tokens
through a vocabulary projection whose logits are never kept, their gradient in the hidden rows and in the projection, and
the optimizer step over many tensors with states in 32 or in 8 bits; the sizes they are timed at.

A case is a dict of plain values.  `listed()` names the fixed ones, `draw(rng)` makes one more of the same ranges;
`prepare(case, seed)` makes on the GPU what a training program holds before the call, `run(state)` is one pass,
`work(case)` the bytes and operations that the pass cannot do without and `exact(case, seed)` the pass in 64 bits.  With
`own` false, run() computes the operators from elementary torch operations in 32 bits; with `own` true it calls the library.

Three kinds of pass:
  logp   pcm_linear_logprobs: log p(token), log-sum-exp and, as asked, entropy of each row of hidden @ weight / temperature;
         rows without a token (a negative one: prompts, padding) are left out and get zeros
  grad   pcm_linear_logprobs_backward: d hidden and d weight from the gradients of log p and of the entropy
  adam   pcm_adamw_many_step: gradient clipping and AdamW over all tensors of a model; with states in 8 bits their values are
         read out behind it (pcm_adamw_many_states)
"""
from __future__ import annotations

import math

import torch

own = False

BETA1, BETA2, EPS, LR, WEIGHT_DECAY, MAX_NORM, STEP = 0.9, 0.999, 1e-8, 1e-3, 0.01, 2.0, 40
BLOCK = 128                              # elements that share an exponent of their 8-bit states
M_FIELD, V_FIELD = 15, 31                # largest exponent field of a code: m has a sign, 4 bits and 3, v has 5 bits and 3


# ---- the cases ---------------------------------------------------------------------------------

def _logp(name, rows, d, V, dtype, layout="in_out", tokens="i32", entropy=True, masked=0.0, temperature=1.0, pad=0):
    return dict(name=name, kind="logp", rows=rows, d=d, V=V, dtype=dtype, layout=layout, tokens=tokens, entropy=entropy,
                masked=masked, temperature=temperature, pad=pad)


def _grad(name, rows, d, V, dtype, layout="in_out", tokens="i32", entropy=True, masked=0.0, temperature=1.0, pad=0):
    return dict(_logp(name, rows, d, V, dtype, layout, tokens, entropy, masked, temperature, pad), kind="grad")


def _adam(name, layers, d, ff, V, bits, grads="f32", clip=True, packed=False, bf16=True):
    return dict(name=name, kind="adam", layers=layers, d=d, ff=ff, V=V, bits=bits, grads=grads, clip=clip, packed=packed, bf16=bf16)


def listed():
    return [
        # one decoding step of one rollout, whose own token is scored: the projection is read once
        _logp("linear-decode", 1, 4096, 131072, "bf16", layout="out_in"),
        # a few rollouts of a small policy in fp32, an odd vocabulary
        _logp("linear-few", 7, 1024, 32003, "f32", tokens="i64", temperature=0.7),
        # a batch of answers behind their prompts, hidden rows that are a view of wider ones
        _logp("linear-answers", 777, 2048, 50021, "bf16", layout="out_in", tokens="i64", masked=0.4, temperature=1.3, pad=8),
        # the old-policy pass over long sequences
        _logp("linear-long", 4096, 4096, 65536, "bf16"),
        # the tiny instance's last layer: all launch latency
        _grad("linear-grad-tiny", 256, 256, 1024, "bf16", tokens="u8"),
        # a policy kept in fp32, odd sizes throughout
        _grad("linear-grad-f32", 1111, 1001, 32003, "f32", entropy=False, masked=0.1),
        # demonstrations with masked prompts, entropy bonus, a vocabulary that fills no tile
        _grad("linear-grad-answers", 2072, 1536, 50021, "bf16", layout="out_in", masked=0.4),
        # supervised warm start over a whole vocabulary, the largest
        _grad("linear-grad-wide", 4096, 4096, 131072, "bf16"),
        # a small model of many small tensors: launches and latency
        _adam("adam-small", 32, 64, 172, 256, 32),
        # a whole model with fp32 master weights
        _adam("adam-model", 24, 1024, 2816, 32003, 32),
        # packed parameters of odd sizes, states in 8 bits, no clipping
        _adam("adam-eight-odd", 6, 257, 701, 1000, 8, clip=False, packed=True),
        # wide layers, bf16 gradients, states in 8 bits
        _adam("adam-eight-model", 4, 2048, 5504, 256, 8, grads="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["logp", "logp", "logp", "grad", "grad", "grad", "adam", "adam"])
    if kind == "adam":
        d = rng.choice([_log_int(rng, 16, 2048), 64 * _log_int(rng, 1, 32)])
        ff, V = rng.randint(d, 4 * d), rng.choice([256, _log_int(rng, 2, 32003)])
        most = max(1, (340000000 - d * V) // (4 * d * d + 3 * d * ff + 2 * d))
        case = _adam("", _log_int(rng, 1, min(48, most)), d, ff, V, rng.choice([32, 8]), rng.choice(["f32", "bf16"]), rng.random() < 0.7,
                     rng.random() < 0.4, rng.random() < 0.7)
    else:
        d = rng.choice([_log_int(rng, 16, 4096), 64 * _log_int(rng, 1, 64)])
        V = rng.choice([256, _log_int(rng, 2, 131072), _log_int(rng, 2048, 131072)])
        rows = _log_int(rng, 1, min(43008, 4096 * 4096 * 131072 // (d * V)))
        make = _logp if kind == "logp" else _grad
        case = make("", rows, d, V, rng.choice(["bf16", "bf16", "f32"]), rng.choice(["in_out", "out_in"]),
                    rng.choice(["u8", "i32"] if V <= 256 else ["i32", "i64"]), rng.random() < 0.6, rng.choice([0.0, 0.0, 0.1, 0.4, 0.9]),
                    rng.choice([1.0, 0.7, 1.3]), rng.choice([0, 0, 1, 8]))
        if case["tokens"] == "u8":
            case["masked"] = 0.0
    del case["name"]
    return case


def _sizes(case):
    """Shapes of a model's parameters: embedding, per layer four square matrices, three of the gated part and two norms, last norm."""
    d, ff = case["d"], case["ff"]
    layer = [(d, d)] * 4 + [(d, ff)] * 2 + [(ff, d)] + [(d,)] * 2
    return [(case["V"], d)] + layer * case["layers"] + [(d,)]


# ---- inputs ------------------------------------------------------------------------------------

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "u8": torch.uint8, "i32": torch.int32, "i64": torch.int64}


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _row_blocks(rows, V):
    block = max(1, (1 << 27) // V)
    return [(r, min(rows, r + block)) for r in range(0, rows, block)]


def _linear_inputs(case, seed):
    gen = _generator(seed)
    rows, d, V, dtype = case["rows"], case["d"], case["V"], TYPES[case["dtype"]]
    # hidden rows as a norm leaves them, from undecided to almost certain ones once they are projected
    spread = 0.3 + 2.7 * torch.rand((rows, 1), generator=gen, device="cuda")
    hidden = (spread * torch.randn((rows, d + case["pad"]), generator=gen, device="cuda")).to(dtype)[:, :d]
    shape = (V, d) if case["layout"] == "out_in" else (d, V)
    weight = (torch.randn(shape, generator=gen, device="cuda") * d ** -0.5).to(dtype)
    weight = weight.t() if case["layout"] == "out_in" else weight
    tokens = torch.randint(0, V, (rows,), generator=gen, device="cuda")
    if case["masked"]:
        tokens = torch.where(torch.rand(rows, generator=gen, device="cuda") < case["masked"], -1, tokens)
    if V <= 256 or case["tokens"] != "u8":
        tokens = tokens.to(TYPES[case["tokens"]])
    else:
        tokens = (tokens % 256).to(torch.uint8)
    return dict(hidden=hidden, weight=weight, tokens=tokens), gen


def _statistics(hidden, weight, tokens, temperature):
    """Log-sum-exp, log p of the token and entropy of each row in 64 bits; zeros where a row has no token."""
    w = weight.double()
    out = []
    for lo, hi in _row_blocks(hidden.shape[0], weight.shape[1]):
        x = torch.matmul(hidden[lo:hi].double(), w) / temperature
        lse = torch.logsumexp(x, dim=1)
        given = torch.gather(x, 1, tokens[lo:hi].long().clamp(min=0)[:, None])[:, 0]
        x -= lse[:, None]
        entropy = -(torch.exp(x) * x).sum(dim=1)
        has = (tokens[lo:hi].long() >= 0).double()
        out.append(torch.stack([lse * has, (given - lse) * has, entropy * has]))
    return torch.cat(out, dim=1)


def _power(e):
    """2^e in 64 bits, of whole numbers."""
    return ((e + 1023) << 52).view(torch.float64)


def _round_states(x, field, random):
    """The values near `x` (fp32, a multiple of BLOCK of them) that 8 bits hold: 3 bits behind the point and an exponent between 0
    and `field` below the exponent that the block's largest value gets; `random`, 16 bits of each value, says which of its
    two neighbours it goes to.  Values of x >= 0 that are not zero stay so if field is V_FIELD."""
    sign, bits = torch.signbit(x), x.abs().view(torch.int32).long()
    bits = torch.where(bits < 1 << 23, 0, bits)
    rounded = (bits + (random << 4)) >> 20
    top = (rounded >> 3).view(-1, BLOCK).max(dim=1, keepdim=True).values.expand(-1, BLOCK).reshape(-1)
    code = rounded - ((top - field) << 3)
    unit = top - 127 - (field - 1) - 3                       # exponent of the least value
    fine = torch.floor(bits.int().view(torch.float32).double() * _power(16 - unit)).clamp(max=float(1 << 20)).long()
    code = torch.where(code >= 8, code, (fine + random) >> 16)
    if field == V_FIELD:
        code = code.clamp(min=1)
    return torch.where(bits > 0, code, 0), top, sign


def _values(code, top, sign, field):
    exponent = (code >> 3).clamp(min=1) + top - field - 127 - 3
    x = (torch.where(code >= 8, 8 + (code & 7), code).double() * _power(exponent)).float()
    return torch.where(top == 255, math.nan, torch.where(sign, -x, x))


def _philox(groups, step, seed):
    """Philox4x32-10 of counters (group, group >> 32, step, step >> 32) and key `seed`: 8 times 16 bits per group, low half first."""
    low = 0xFFFFFFFF
    c = [groups & low, groups >> 32, torch.full_like(groups, step & low), torch.full_like(groups, step >> 32)]
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        # 32 x 32 bits in two halves, so that no product leaves 63 bits
        a_lo, a_hi = c[0] * 0x1F53, c[0] * 0xD251
        b_lo, b_hi = c[2] * 0x8D57, c[2] * 0xCD9E
        p = a_lo + ((a_hi & low) << 16)
        q = b_lo + ((b_hi & low) << 16)
        p_hi, q_hi = (p >> 32) + (a_hi >> 32 << 16), (q >> 32) + (b_hi >> 32 << 16)
        c = [q_hi ^ c[1] ^ k0, q & low, p_hi ^ c[3] ^ k1, p & low]
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack(c, dim=1)
    return torch.stack([words & 0xFFFF, words >> 16], dim=2).reshape(-1)


def _arena(case, dtype):
    """A flat buffer and the tensors in it: one behind the other, or each on a multiple of BLOCK elements."""
    sizes = _sizes(case)
    numel = [math.prod(s) for s in sizes]
    room = numel if case["packed"] else [-(-n // BLOCK) * BLOCK for n in numel]
    flat = torch.zeros(sum(room), dtype=dtype, device="cuda")
    return flat, [part[:n].view(s) for part, n, s in zip(flat.split(room), numel, sizes)]


def _adam_inputs(case, seed):
    gen = _generator(seed)
    weights, weight_list = _arena(case, torch.float32)
    grads, grad_list = _arena(case, TYPES[case["grads"]])
    lowp, lowp_list = _arena(case, torch.bfloat16) if case["bf16"] else (None, None)
    numel = [w.numel() for w in weight_list]
    # where each tensor begins among the states: on a multiple of BLOCK elements
    room = [-(-n // BLOCK) * BLOCK for n in numel]
    E = sum(room)
    size = torch.tensor(numel, device="cuda")
    start = torch.tensor(room, device="cuda").cumsum(0)
    spread = torch.exp(1.5 * torch.randn(len(numel), generator=gen, device="cuda"))
    which = torch.bucketize(torch.arange(E, device="cuda"), start, right=True)
    inside = torch.arange(E, device="cuda") - (start - torch.tensor(room, device="cuda"))[which]
    live = inside < size[which]
    # the state of step 39 and a gradient: as large as the tensor's place in the model makes them
    scale = 2e-4 * spread[which]
    v = torch.where(live, (scale * (0.2 + torch.rand(E, generator=gen, device="cuda"))).square(), 0.0)
    m = torch.where(live, 0.3 * scale * torch.randn(E, generator=gen, device="cuda"), 0.0)
    g = (scale * torch.randn(E, generator=gen, device="cuda"))[live]
    del scale, inside
    place = live.nonzero()[:, 0] if case["packed"] else None
    if case["packed"]:
        grads.copy_(g)
        weights.copy_(0.02 * torch.randn(weights.shape, generator=gen, device="cuda"))
    else:
        grads[live] = g.to(grads.dtype)
        weights[live] = 0.02 * torch.randn(g.shape, generator=gen, device="cuda")
    del which, live, g
    state = dict(kind="adam", weights=weights, grads=grads, weights_bf16=lowp, place=place, E=E, clip=case["clip"], bits=case["bits"],
                 seed=1000003 * (seed % 1000003) + 7)
    if case["bits"] == 32:
        state["opt"] = torch.cat([m, v]).view(torch.uint8)
    else:
        parts, tops = [], []
        for x, field in ((m, M_FIELD), (v, V_FIELD)):
            half = torch.full((BLOCK,), 1 << 15, device="cuda").repeat(E // BLOCK)
            code, top, sign = _round_states(x, field, half)
            parts.append((code + (sign & (code > 0) & (field == M_FIELD)) * 128).to(torch.uint8))
            tops.append(top.view(-1, BLOCK)[:, 0].to(torch.uint8))
        state["opt"] = torch.cat(parts + tops)
    return state, (grad_list, weight_list, lowp_list)


def prepare(case, seed):
    kind = case["kind"]
    if kind in ("logp", "grad"):
        state, gen = _linear_inputs(case, seed)
        state.update(kind=kind, temperature=case["temperature"], want_entropy=case["entropy"])
        if kind == "grad":
            rows = case["rows"]
            lse, _, entropy = _statistics(state["hidden"], state["weight"], state["tokens"], case["temperature"])
            state.update(lse=lse.float(), dlogp=torch.randn(rows, generator=gen, device="cuda") / rows,
                         entropy=entropy.float() if case["entropy"] else None,
                         dentropy=0.1 * torch.rand(rows, generator=gen, device="cuda") / rows if case["entropy"] else None)
        return state
    state, (grads, weights, lowp) = _adam_inputs(case, seed)
    if own:
        import paper_2605_16154_amd as pcm
        state["plan"] = pcm.pcm_adamw_many_plan(grads, weights, state_bits=case["bits"], weights_bf16=lowp, state=state["opt"])
    return state


# ---- the plain forms ---------------------------------------------------------------------------

def _plain_logp(s):
    x = (s["hidden"].float() @ s["weight"].float()) * (1.0 / s["temperature"])
    has = s["tokens"].long() >= 0
    top = x.max(dim=1, keepdim=True).values
    a = x - top
    e = torch.exp(a)
    total = e.sum(dim=1)
    given = torch.gather(a, 1, s["tokens"].long().clamp(min=0)[:, None])[:, 0]
    log_total = torch.log(total)
    out = dict(lse=torch.where(has, top[:, 0] + log_total, 0.0), logp=torch.where(has, given - log_total, 0.0))
    if s["want_entropy"]:
        out["entropy"] = torch.where(has, log_total - (e * a).sum(dim=1) / total, 0.0)
    return out


def _plain_grad(s):
    h, w = s["hidden"].float(), s["weight"].float()
    tokens = s["tokens"].long()
    has = tokens >= 0
    logp = (h @ w) * (1.0 / s["temperature"]) - s["lse"][:, None]
    p = torch.exp(logp)
    dlogp = torch.where(has, s["dlogp"], 0.0)
    g = -dlogp[:, None] * p
    if s["dentropy"] is not None:
        g -= torch.where(has, s["dentropy"], 0.0)[:, None] * p * (logp + s["entropy"][:, None])
    g.scatter_add_(1, tokens.clamp(min=0)[:, None], dlogp[:, None])
    g = torch.where(has[:, None], g, 0.0) * (1.0 / s["temperature"])
    return dict(dhidden=(g @ w.t()).to(s["hidden"].dtype), dweight=(h.t() @ g).to(s["weight"].dtype))


def _spread(x, s):
    """A packed buffer with its tensors on multiples of BLOCK elements."""
    return x if s["place"] is None else torch.zeros(s["E"], dtype=x.dtype, device="cuda").index_copy_(0, s["place"], x)


def _read_opt(s):
    """m and v in fp32 from the block that holds the states."""
    E = s["E"]
    if s["bits"] == 32:
        return s["opt"].view(torch.float32).split(E)
    m, v, tm, tv = s["opt"].long().split([E, E, E // BLOCK, E // BLOCK])
    return (_values(m & 127, tm.repeat_interleave(BLOCK), m > 127, M_FIELD),
            _values(v, tv.repeat_interleave(BLOCK), torch.zeros_like(v, dtype=torch.bool), V_FIELD))


def _plain_adam(s):
    g, w = _spread(s["grads"].float(), s), _spread(s["weights"], s)
    norm = None
    if s["clip"]:
        total = g.double().square().sum().sqrt()
        norm = total.float()[None]
        g = g * torch.clamp(MAX_NORM / (total + 1e-6), max=1.0).float()
    m, v = _read_opt(s)
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + (g * g) * (1.0 - BETA2)
    step_size, root = LR / (1.0 - BETA1 ** STEP), 1.0 / math.sqrt(1.0 - BETA2 ** STEP)
    w = w * (1.0 - LR * WEIGHT_DECAY) - step_size * (m / (torch.sqrt(v) * root + EPS))
    s["weights"].copy_(w if s["place"] is None else w[s["place"]])
    if s["weights_bf16"] is not None:
        s["weights_bf16"].copy_(s["weights"])
    if s["bits"] == 32:
        s["opt"].view(torch.float32).copy_(torch.cat([m, v]))
        return norm, m, v
    random = _philox(torch.arange(s["E"] // 8, device="cuda"), STEP, s["seed"])
    mc, mt, ms = _round_states(m, M_FIELD, random)
    vc, vt, vs = _round_states(v, V_FIELD, random)
    s["opt"].copy_(torch.cat([mc + (ms & (mc > 0)) * 128, vc, mt[::BLOCK], vt[::BLOCK]]))
    return norm, _values(mc, mt, ms, M_FIELD).to(torch.bfloat16), _values(vc, vt, vs, V_FIELD).to(torch.bfloat16)


def run(state):
    kind = state["kind"]
    if own:
        import paper_2605_16154_amd as pcm
    if kind == "logp":
        if not own:
            return _plain_logp(state)
        return pcm.pcm_linear_logprobs(state["hidden"], state["weight"], state["tokens"], temperature=state["temperature"],
                                       want_entropy=state["want_entropy"])
    if kind == "grad":
        if not own:
            return _plain_grad(state)
        return pcm.pcm_linear_logprobs_backward(state["hidden"], state["weight"], state["tokens"], state["lse"], state["dlogp"],
                                                entropy=state["entropy"], dentropy=state["dentropy"], temperature=state["temperature"])
    if own:
        norm = pcm.pcm_adamw_many_step(state["plan"], step=STEP, lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS, weight_decay=WEIGHT_DECAY,
                                       max_grad_norm=MAX_NORM if state["clip"] else None, seed=state["seed"])
        m, v = pcm.pcm_adamw_many_states(state["plan"])
    else:
        norm, m, v = _plain_adam(state)
    out = dict(weights=state["weights"], m=m, v=v)
    if state["weights_bf16"] is not None:
        out["weights_bf16"] = state["weights_bf16"]
    if state["clip"]:
        out["norm"] = norm
    return out


# ---- what a pass needs, and its results in 64 bits -----------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "adam":
        n = sum(math.prod(s) for s in _sizes(case))
        each = {"f32": 4, "bf16": 2}[case["grads"]] + 8 + 2 * case["bf16"]
        # states: read and written; those in 8 bits with two exponents per block, and their values in 16 bits
        states = 16 if case["bits"] == 32 else 4 + 4 / BLOCK + 4
        return {"bytes": int(n * (each + states)), "flops": 14 * n}
    rows, d, V = case["rows"], case["d"], case["V"]
    live = max(1, round(rows * (1.0 - case["masked"])))
    size = {"bf16": 2, "f32": 4}[case["dtype"]]
    token = {"u8": 1, "i32": 4, "i64": 8}[case["tokens"]]
    if kind == "logp":
        return {"bytes": (live + V) * d * size + rows * (token + 8 + 4 * case["entropy"]), "flops": 2 * live * d * V}
    return {"bytes": (2 * V + live + rows) * d * size + rows * (token + 8 + 8 * case["entropy"]), "flops": 6 * live * d * V}


def _exact_states(x, field, random):
    """The value of x's block-wise 8-bit form, from its definition with real numbers."""
    u = random.double() / 65536
    sign, a = torch.sign(x), x.abs()
    a = torch.where(a < 2.0 ** -126, 0.0, a)
    e = torch.frexp(a).exponent.long() - 1
    step = _power(e - 3)
    near = torch.floor(a / step + u) * step
    top = torch.where(near > 0, torch.frexp(near).exponent.long() - 1, -200).view(-1, BLOCK).max(dim=1, keepdim=True).values
    top = top.expand(-1, BLOCK).reshape(-1)
    least = _power(top - field + 1)              # below it steps no longer get smaller
    near = torch.where(near < least, torch.floor(a / (least / 8) + u) * (least / 8), near)
    if field == V_FIELD:
        near = torch.where(a > 0, torch.maximum(near, least / 8), near)
    return (sign * near).float()


def exact(case, seed):
    kind = case["kind"]
    if kind == "adam":
        s, _ = _adam_inputs(case, seed)
        place = s["place"] if s["place"] is not None else slice(None)
        m, v = (x.double()[place] for x in _read_opt(s))
        g, w = s["grads"].double(), s["weights"].double()
        norm = torch.linalg.vector_norm(g)
        if s["clip"]:
            g = g * min(1.0, MAX_NORM / (float(norm) + 1e-6))
        m.mul_(BETA1).add_(g, alpha=1 - BETA1)
        v.mul_(BETA2).addcmul_(g, g, value=1 - BETA2)
        w = (1 - LR * WEIGHT_DECAY) * w - LR * (m / (1 - BETA1 ** STEP)) / (torch.sqrt(v / (1 - BETA2 ** STEP)) + EPS)
        whole = [torch.zeros(s["E"], dtype=torch.float64, device="cuda") for _ in range(2)]
        for to, x in zip(whole, (m, v)):
            to[place] = x
        if case["bits"] == 8:
            random = _philox(torch.arange(s["E"] // 8, device="cuda"), STEP, s["seed"])
            whole = [_exact_states(x, field, random) for x, field in zip(whole, (M_FIELD, V_FIELD))]
        out = dict(weights=w, m=whole[0], v=whole[1])
        if case["bf16"]:
            out["weights_bf16"] = w
        if case["clip"]:
            out["norm"] = norm[None]
        return out
    s = prepare(case, seed)
    h, w, tokens = s["hidden"], s["weight"], s["tokens"].long()
    lse, logp, entropy = _statistics(h, w, tokens, case["temperature"])
    if kind == "logp":
        return dict(lse=lse, logp=logp, **(dict(entropy=entropy) if case["entropy"] else {}))
    # sums over rows and over tokens, block by block
    wd = w.double()
    dw = torch.zeros(wd.shape, dtype=torch.float64, device="cuda")
    dh = []
    for lo, hi in _row_blocks(h.shape[0], w.shape[1]):
        has = (tokens[lo:hi] >= 0).double()[:, None]
        x = torch.matmul(h[lo:hi].double(), wd) / case["temperature"] - lse[lo:hi, None]
        p = torch.exp(x)
        one = torch.zeros_like(p).scatter_(1, tokens[lo:hi].clamp(min=0)[:, None], 1.0)
        z = s["dlogp"][lo:hi, None].double() * (one - p)
        if case["entropy"]:
            z -= s["dentropy"][lo:hi, None].double() * p * (x + entropy[lo:hi, None])
        z = z * has / case["temperature"]
        dh.append(torch.matmul(z, wd.t().contiguous()))
        dw += torch.matmul(h[lo:hi].double().t().contiguous(), z)
    return dict(dhidden=torch.cat(dh), dweight=dw)
