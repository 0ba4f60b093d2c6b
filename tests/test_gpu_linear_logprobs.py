"""GPU parity of the log-probabilities through a vocabulary projection and of their gradient against the plain 64-bit form.

Tolerances, by arithmetic.  z: products of bf16 values are exact in fp32 and a sum of d terms in any order is off by at most d 2^-24 of the sum of
their sizes; fp32 values as pairs are off by 2^-22 each and leave a product of 2^-22 out, 2^-20 of the sum of sizes together, and by 2^-40 of
the largest value that shares their power of two.  x = z / temperature is off by E.  lse and logp: E and 2 E, the sum of the exponentials (a few
2^-24 relative, 2^-20 allowed), and roundings of 2^-23 of their sizes and of the largest x.  entropy: p moves by 2 E relative, so
sum p |log p + H| 2 E <= 2 E 2 log V.  The gradient takes log p = x - lse: E, 2^-23 |lse| and |x| and the exponential's 2^-20 make p wrong by
F relative, dz by F times its terms and by its own rounding (2^-8 for bf16; 2^-20 and 2^-38 of the row's bound for pairs); products then as above, over V and over
the rows, and the result's rounding."""
import numpy as np
import pytest
import torch

from oracle import operators as P

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
STEP = {BF16: 2.0 ** -8, F32: 2.0 ** -24}


def _inputs(rows, d, V, dtype, layout="in_out", tokens=torch.int32, masked=0.0, pad=0, scale=1.0, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(1000 * seed + rows + 7 * d + 13 * V)
    spread = 0.3 + 2.0 * torch.rand((rows, 1), generator=gen, device="cuda")
    hidden = (scale * spread * torch.randn((rows, d + pad), generator=gen, device="cuda")).to(dtype)[:, :d]
    shape = (V, d + pad) if layout == "out_in" else (d, V + pad)
    w = (torch.randn(shape, generator=gen, device="cuda") * d ** -0.5).to(dtype)
    w = w[:, :d].t() if layout == "out_in" else w[:, :V]
    t = torch.randint(0, V, (rows,), generator=gen, device="cuda")
    if masked:
        t[torch.rand(rows, generator=gen, device="cuda") < masked] = -1
    return hidden, w, t.to(tokens), gen


def _np(t):
    return t.double().cpu().numpy()


def _z_error(h, w, dtype, temperature):
    """Bound of |x - exact| per row and token."""
    d = h.shape[1]
    sizes = np.abs(h) @ np.abs(w)
    e = (d + 2) * 2.0 ** -24 * sizes
    if dtype == F32:
        top_h, top_w = np.abs(h).max(axis=1, keepdims=True), np.abs(w).max()
        e += 2.0 ** -20 * sizes + 2.0 ** -38 * (top_h * np.abs(w).sum(axis=0) + top_w * np.abs(h).sum(axis=1, keepdims=True))
    return e / temperature


def _forward(case, temperature=1.0):
    import paper_2605_16154_amd as pcm
    hidden, w, tokens, _ = case
    out = pcm.pcm_linear_logprobs(hidden, w, tokens, temperature=temperature)
    torch.cuda.synchronize()
    h, wn, t = _np(hidden), _np(w), tokens.cpu().numpy().astype(np.int64)
    live = t >= 0
    ref = P.linear_logprobs(h, wn, t, temperature)
    h = np.where(live[:, None], h, 0.0)
    E = _z_error(h, wn, hidden.dtype, temperature).max(axis=1)
    big = np.abs(h @ wn).max(axis=1) / temperature
    tol = {"lse": E + 2.0 ** -20 + 2.0 ** -23 * (np.abs(ref["lse"]) + big),
           "logp": 2 * E + 2.0 ** -20 + 2.0 ** -22 * (np.abs(ref["logp"]) + big),
           "entropy": (4 * E + 2.0 ** -19) * (1 + np.log(wn.shape[1]))}
    for k, v in out.items():
        got = _np(v)
        assert np.all(got[~live] == 0.0), k
        off = np.abs(got - ref[k])[live]
        assert np.all(off <= tol[k][live]), (k, off.max(), int(np.argmax(off - tol[k][live])))
    return out, ref


SIZES = [(1, 64, 300), (1, 1, 1), (2, 7, 2), (7, 96, 257), (16, 200, 1000), (17, 64, 255), (33, 65, 129), (100, 129, 1023), (128, 64, 256), (129, 320, 513),
         (257, 128, 64), (300, 72, 2050), (700, 256, 4099), (1100, 1000, 300)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", ["in_out", "out_in"])
@pytest.mark.parametrize("rows,d,V", SIZES)
def test_forward(rows, d, V, layout, dtype):
    tokens = torch.uint8 if V <= 256 else torch.int64 if rows % 2 else torch.int32
    _forward(_inputs(rows, d, V, dtype, layout, tokens))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,masked,pad,temperature,layout", [(9, 0.5, 3, 0.7, "in_out"), (300, 0.4, 1, 1.3, "out_in"), (300, 0.99, 8, 1.0, "in_out"),
                                                                (5000, 0.9, 0, 0.01, "out_in"), (40, 1.0, 0, 1.0, "in_out"), (5, 1.0, 0, 1.0, "out_in"),
                                                                (600, 0.5, 8, 100.0, "out_in")])
def test_forward_masks_strides_and_temperatures(rows, masked, pad, temperature, layout, dtype):
    _forward(_inputs(rows, 136, 520, dtype, layout, masked=masked, pad=pad), temperature)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [4, 200])
def test_what_masked_rows_hold_is_not_met(rows, dtype):
    import paper_2605_16154_amd as pcm
    hidden, w, tokens, gen = _inputs(rows, 64, 300, dtype, masked=0.4)
    tokens[0], tokens[1] = -1, 5
    junk = hidden.clone()
    junk[tokens < 0] = float("nan")
    junk[0] = float("inf")
    clean = pcm.pcm_linear_logprobs(hidden, w, tokens)
    got = pcm.pcm_linear_logprobs(junk, w, tokens)
    for k in clean:
        assert torch.equal(clean[k], got[k]), k
    g = torch.randn(rows, generator=gen, device="cuda")
    dirty = torch.where(tokens >= 0, g, float("nan"))
    a = pcm.pcm_linear_logprobs_backward(hidden, w, tokens, clean["lse"], g, clean["entropy"], g)
    b = pcm.pcm_linear_logprobs_backward(junk, w, tokens, clean["lse"], dirty, clean["entropy"], dirty)
    for k in a:
        assert torch.equal(a[k], b[k]), k
    assert not b["dhidden"][tokens < 0].any()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [6, 150])
def test_a_row_with_a_nan_is_nan_and_leaves_the_others(rows, dtype):
    import paper_2605_16154_amd as pcm
    hidden, w, tokens, _ = _inputs(rows, 64, 300, dtype)
    clean = pcm.pcm_linear_logprobs(hidden, w, tokens)
    hidden[3, 5] = float("nan")
    got = pcm.pcm_linear_logprobs(hidden, w, tokens)
    others = torch.arange(rows, device="cuda") != 3
    for k in clean:
        assert torch.isnan(got[k][3]) and torch.equal(clean[k][others], got[k][others]), k


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [3, 130])
def test_rows_of_very_different_sizes(rows, dtype):
    """Rows from 2^-30 to 2^4 of the usual size side by side, each as exact as alone."""
    hidden, w, tokens, gen = _inputs(rows, 96, 400, dtype)
    factor = torch.exp2(torch.linspace(-30, 4, rows, device="cuda").round())[:, None].to(dtype)
    _forward((hidden * factor, w * 8, tokens, gen))


def _bounds(case, g, e, temperature, out_dtype):
    """Plain gradients and elementwise bounds of the errors of both."""
    hidden, w, tokens, _ = case
    dtype = hidden.dtype
    t = tokens.cpu().numpy().astype(np.int64)
    live = t >= 0
    h, wn = np.where(live[:, None], np.nan_to_num(_np(hidden)), 0.0), _np(w)
    gn, en = np.where(live, _np(g), 0.0), None if e is None else np.where(live, _np(e), 0.0)
    dz = P.linear_logits_gradient(h, wn, t, gn, en, temperature)
    ref = P.linear_logprobs(h, wn, t, temperature)
    x = h @ wn / temperature
    logp = np.where(live[:, None], x - ref["lse"][:, None], 0.0)
    p = np.where(live[:, None], np.exp(logp), 0.0)
    E = _z_error(h, wn, dtype, temperature).max(axis=1, keepdims=True)
    F = 2 * E + 2.0 ** -20 + 2.0 ** -22 * (np.abs(x) + np.abs(ref["lse"])[:, None])
    terms = np.abs(gn)[:, None] * p
    size = np.abs(gn)[:, None] * p
    if en is not None:
        # p and the factor (log p + H) both move
        size = size + np.abs(en)[:, None] * p * (np.abs(logp) + ref["entropy"][:, None] + 1 + (1 + np.log(wn.shape[1])) * 4)
    dz_off = (np.expm1(F) * size + 2.0 ** -22 * np.abs(gn)[:, None] * (p > 0)) / temperature
    hit = np.zeros_like(p)
    hit[np.flatnonzero(live), np.minimum(t[live], wn.shape[1] - 1)] = 1
    dz_off += 2.0 ** -22 * np.abs(gn)[:, None] * hit / temperature
    row_bound = (np.abs(gn) + (0 if en is None else np.abs(en) * (0.5 + ref["entropy"])))[:, None] / temperature
    if dtype == BF16:
        dz_off += 2.0 ** -8 * np.abs(dz)
        extra = 0.0
    else:
        dz_off += 2.0 ** -22 * np.abs(dz) + 2.0 ** -38 * row_bound * live[:, None]
        extra = 2.0 ** -20
    V, rows = wn.shape[1], len(h)
    dh, dw = dz @ wn.T, h.T @ dz
    size_h, size_w = np.abs(dz) @ np.abs(wn).T, np.abs(h).T @ np.abs(dz)
    off_h = dz_off @ np.abs(wn).T + (V * 2.0 ** -24 + extra) * size_h
    off_w = np.abs(h).T @ dz_off + (rows * 2.0 ** -24 + extra) * size_w
    if dtype == F32:
        off_h += 2.0 ** -38 * np.abs(wn).max() * np.abs(dz).sum(axis=1, keepdims=True)
        # a row's power of two for dW is that of the largest product of a row of h and of dz
        off_w += 2.0 ** -36 * (np.abs(h).max(axis=1) * row_bound[:, 0]).max() * rows
    return (dh, off_h + 2 * STEP[dtype] * np.abs(dh) + 1e-37), (dw, off_w + 2 * STEP[out_dtype] * np.abs(dw) + 1e-37)


def _backward(case, temperature=1.0, entropy=True, seed=3, dweight_dtype=None, **kw):
    import paper_2605_16154_amd as pcm
    hidden, w, tokens, gen = case
    rows = hidden.shape[0]
    g = torch.randn(rows, generator=gen, device="cuda")
    e = 0.3 * torch.randn(rows, generator=gen, device="cuda") if entropy else None
    ref = P.linear_logprobs(np.nan_to_num(_np(hidden)), _np(w), tokens.cpu().numpy().astype(np.int64), temperature)
    to = lambda x: torch.from_numpy(x).float().cuda()
    out = pcm.pcm_linear_logprobs_backward(hidden, w, tokens, to(ref["lse"]), g, to(ref["entropy"]) if entropy else None, e, temperature=temperature,
                                           dweight_dtype=dweight_dtype, **kw)
    torch.cuda.synchronize()
    (dh, tol_h), (dw, tol_w) = _bounds(case, g, e, temperature, out["dweight"].dtype)
    for name, got, want, tol in (("dhidden", out["dhidden"], dh, tol_h), ("dweight", out["dweight"], dw, tol_w)):
        off = np.abs(_np(got) - want)
        assert np.all(off <= tol), (name, float((off / tol).max()), np.unravel_index(np.argmax(off / tol), off.shape))
    assert not out["dhidden"][tokens < 0].any()
    return out


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", ["in_out", "out_in"])
@pytest.mark.parametrize("rows,d,V", SIZES)
def test_gradient(rows, d, V, layout, dtype):
    out = _backward(_inputs(rows, d, V, dtype, layout, torch.uint8 if V <= 256 else torch.int32), entropy=rows % 3 != 0)
    assert out["dweight"].dtype == dtype and out["dhidden"].dtype == dtype


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,masked,pad,temperature,layout", [(9, 0.5, 3, 0.7, "in_out"), (300, 0.4, 1, 1.3, "out_in"), (300, 0.99, 8, 1.0, "in_out"),
                                                                (3000, 0.9, 0, 0.5, "out_in"), (40, 1.0, 0, 1.0, "in_out"), (600, 0.5, 8, 100.0, "out_in")])
def test_gradient_masks_strides_and_temperatures(rows, masked, pad, temperature, layout, dtype):
    _backward(_inputs(rows, 136, 520, dtype, layout, masked=masked, pad=pad), temperature)


def test_gradient_in_fp32_of_bf16_weights_and_added():
    import paper_2605_16154_amd as pcm
    for layout in ("in_out", "out_in"):
        case = _inputs(260, 136, 520, BF16, layout)
        out = _backward(case, dweight_dtype=F32)
        assert out["dweight"].dtype == F32
        hidden, w, tokens, gen = case
        fwd = pcm.pcm_linear_logprobs(hidden, w, tokens)
        g = torch.randn(260, generator=gen, device="cuda")
        once = pcm.pcm_linear_logprobs_backward(hidden, w, tokens, fwd["lse"], g, dweight_dtype=F32, want_dhidden=False)
        assert list(once) == ["dweight"]
        start = torch.randn_like(once["dweight"])
        added = {"dweight": start.clone()}
        pcm.pcm_linear_logprobs_backward(hidden, w, tokens, fwd["lse"], g, want_dhidden=False, accumulate=True, out=added)
        assert torch.equal(added["dweight"], start + once["dweight"])
        only = pcm.pcm_linear_logprobs_backward(hidden, w, tokens, fwd["lse"], g, want_dweight=False)
        assert list(only) == ["dhidden"]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", ["in_out", "out_in"])
def test_values_between_rows_are_left(layout, dtype):
    import paper_2605_16154_amd as pcm
    hidden, w, tokens, gen = _inputs(70, 136, 270, dtype, layout, masked=0.3)
    fwd = pcm.pcm_linear_logprobs(hidden, w, tokens)
    g = torch.randn(70, generator=gen, device="cuda")
    plain = pcm.pcm_linear_logprobs_backward(hidden, w, tokens, fwd["lse"], g)
    for pad in (1, 3, 8):
        dh = torch.full((72, 136 + pad), 7.0, dtype=dtype, device="cuda")
        shape = (272, 136 + pad) if layout == "out_in" else (138, 270 + pad)
        dw = torch.full(shape, 7.0, dtype=dtype, device="cuda")
        inner = dw[1:271, :136].t() if layout == "out_in" else dw[1:137, :270]
        pcm.pcm_linear_logprobs_backward(hidden, w, tokens, fwd["lse"], g, out={"dhidden": dh[1:71, :136], "dweight": inner})
        assert torch.equal(dh[1:71, :136], plain["dhidden"]) and torch.equal(inner, plain["dweight"])
        inner.fill_(7.0)
        dh[1:71, :136] = 7.0
        assert bool((dh == 7).all()) and bool((dw == 7).all())


def test_gradient_against_differences():
    """d loss / d hidden and d weight along random directions, from the forward call in fp32: the loss has values of order 1 known to about 2e-6
    (its rounding and that of z), a step of 1/64 makes 3e-4 of that in the quotient, and the third derivative, of order 1, a sixth of 2^-12."""
    import paper_2605_16154_amd as pcm
    hidden, w, tokens, gen = _inputs(40, 64, 200, F32, masked=0.2)
    g, e = torch.randn(40, generator=gen, device="cuda") / 6, torch.randn(40, generator=gen, device="cuda") / 6

    def loss(h, ww):
        out = pcm.pcm_linear_logprobs(h, ww, tokens, temperature=2.0)
        return float((g.double() * out["logp"].double() + e.double() * out["entropy"].double()).sum())

    fwd = pcm.pcm_linear_logprobs(hidden, w, tokens, temperature=2.0)
    grad = pcm.pcm_linear_logprobs_backward(hidden, w, tokens, fwd["lse"], g, fwd["entropy"], e, temperature=2.0)
    for k in range(4):
        u = torch.randn(hidden.shape, generator=gen, device="cuda")
        v = torch.randn(w.shape, generator=gen, device="cuda")
        u, v = u / u.norm(), v / v.norm()
        step = 1 / 64
        for du, dv, want in ((u, 0 * v, (grad["dhidden"] * u).double().sum()), (0 * u, v, (grad["dweight"] * v).double().sum())):
            got = (loss(hidden + step * du, w + step * dv) - loss(hidden - step * du, w - step * dv)) / (2 * step)
            assert abs(got - float(want)) <= 1e-3, (k, got, float(want))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_no_rows_and_no_tokens(dtype):
    import paper_2605_16154_amd as pcm
    w = torch.randn(64, 300, device="cuda").to(dtype)
    for layout in (w, torch.randn(300, 64, device="cuda").to(dtype).t()):
        none = torch.zeros(0, device="cuda")
        out = pcm.pcm_linear_logprobs(torch.zeros(0, 64, dtype=dtype, device="cuda"), layout, torch.zeros(0, dtype=torch.int32, device="cuda"))
        assert out["logp"].shape == (0,)
        grad = pcm.pcm_linear_logprobs_backward(torch.zeros(0, 64, dtype=dtype, device="cuda"), layout, torch.zeros(0, dtype=torch.int32, device="cuda"),
                                                none, none)
        assert grad["dhidden"].shape == (0, 64) and not grad["dweight"].any()


def test_tokens_beyond_the_vocabulary_are_its_last():
    import paper_2605_16154_amd as pcm
    for rows in (5, 50):
        hidden, w, tokens, _ = _inputs(rows, 64, 300, BF16, tokens=torch.int64)
        tokens[:] = 299
        a = pcm.pcm_linear_logprobs(hidden, w, tokens)
        tokens[1], tokens[2] = 300, 1 << 40
        b = pcm.pcm_linear_logprobs(hidden, w, tokens)
        assert torch.equal(a["logp"], b["logp"])


def test_replayed_graph_other_stream_and_same_bits():
    import paper_2605_16154_amd as pcm
    hidden, w, tokens, gen = _inputs(300, 200, 777, BF16, masked=0.3)
    g = torch.randn(300, generator=gen, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())

    def step():
        f = pcm.pcm_linear_logprobs(hidden, w, tokens)
        return f, pcm.pcm_linear_logprobs_backward(hidden, w, tokens, f["lse"], g, f["entropy"], g)

    with torch.cuda.stream(stream):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        captured = step()
    for turn in range(3):
        hidden.mul_(-0.9)
        tokens.copy_(torch.where(torch.rand(300, generator=gen, device="cuda") < 0.5, -1, torch.arange(300, device="cuda")))
        graph.replay()
        eager = step()
        again = step()
        torch.cuda.synchronize()
        for a, b, c in zip(captured, eager, again):
            for k in a:
                assert torch.equal(a[k], b[k]) and torch.equal(b[k], c[k]), (turn, k)


def test_binding_refuses():
    import paper_2605_16154_amd as pcm
    h, w, t, _ = _inputs(20, 64, 100, BF16)
    f = torch.zeros(20, device="cuda")
    for args in ((h.float(), w, t), (h, w[:32], t), (h, w, t[:10]), (h, w, t.float()), (h.cpu(), w, t), (h, w.cpu(), t), (h.half(), w.half(), t),
                 (h.t(), w, t), (h[:, ::2], w[:32], t), (h, w[:, ::2], t)):
        with pytest.raises(pcm.PcmError):
            pcm.pcm_linear_logprobs(*args)
    for kw in (dict(temperature=0.0), dict(temperature=float("nan")), dict(out={"logp": f[:5]}), dict(out={"lse": f.double()})):
        with pytest.raises(pcm.PcmError):
            pcm.pcm_linear_logprobs(h, w, t, **kw)
    for kw in (dict(lse=f[:5]), dict(dlogp=f.double()), dict(dentropy=f), dict(want_dhidden=False, want_dweight=False), dict(accumulate=True),
               dict(dweight_dtype=torch.float16), dict(out={"dweight": torch.zeros(100, 64, dtype=BF16, device="cuda").t()}),
               dict(out={"dhidden": h.float()}), dict(accumulate=True, out={"dweight": torch.zeros_like(w)}), dict(temperature=-1.0)):
        with pytest.raises(pcm.PcmError):
            pcm.pcm_linear_logprobs_backward(h, w, t, kw.pop("lse", f), kw.pop("dlogp", f), **kw)


@pytest.mark.parametrize("rows", [3, 40, 200, 5000])
@pytest.mark.parametrize("layout", ["in_out", "out_in"])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_with_a_gradient_of_zero_add_nothing(dtype, layout, rows):
    """However large what they hold is beside the gradients of the others; and no gradient at all is zeros."""
    import paper_2605_16154_amd as pcm
    hidden, w, tokens, gen = _inputs(rows, 72, 130, dtype, layout)
    idle = torch.arange(rows, device="cuda") % 3 == 1
    hidden[idle] *= 1000
    fwd = pcm.pcm_linear_logprobs(hidden, w, tokens)
    g = torch.where(idle, 0.0, 1e-5 * torch.randn(rows, generator=gen, device="cuda"))
    got = pcm.pcm_linear_logprobs_backward(hidden, w, tokens, fwd["lse"], g, fwd["entropy"], g)
    assert not got["dhidden"][idle].any() and bool(torch.isfinite(got["dweight"]).all())
    for name, want, tol in zip(("dhidden", "dweight"), *zip(*_bounds((hidden, w, tokens, gen), g, g, 1.0, dtype))):
        assert np.all(np.abs(_np(got[name]) - want) <= tol), name
    none = pcm.pcm_linear_logprobs_backward(hidden, w, tokens, fwd["lse"], 0 * g, fwd["entropy"], 0 * g)
    assert not none["dhidden"].any() and not none["dweight"].any()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", ["in_out", "out_in"])
@pytest.mark.parametrize("rows", [9, 150])
def test_what_lies_between_rows_is_not_met(rows, layout, dtype):
    import paper_2605_16154_amd as pcm
    for d, V, pad in ((136, 520, 8), (72, 200, 56), (64, 256, 8), (65, 129, 7)):
        hidden, w, tokens, gen = _inputs(rows, d, V, dtype, layout, pad=pad)
        g = torch.randn(rows, generator=gen, device="cuda")
        results = []
        for fill in (0.0, float("nan")):
            base = torch.full((rows, d + pad), fill, dtype=dtype, device="cuda")
            wide = torch.full((V, d + pad) if layout == "out_in" else (d, V + pad), fill, dtype=dtype, device="cuda")
            h = base[:, :d].copy_(hidden)
            ww = wide[:, :d].copy_(w.t()).t() if layout == "out_in" else wide[:, :V].copy_(w)
            f = pcm.pcm_linear_logprobs(h, ww, tokens)
            results.append({**f, **pcm.pcm_linear_logprobs_backward(h, ww, tokens, f["lse"], g, f["entropy"], g)})
        for k in results[0]:
            assert torch.equal(results[0][k], results[1][k]), (d, V, k)


@pytest.mark.parametrize("layout", ["in_out", "out_in"])
@pytest.mark.parametrize("rows,d,V,masked", [(1025, 1, 1, 0.0), (1030, 7, 2, 0.5), (1100, 65, 129, 0.0), (1279, 64, 255, 0.9), (1281, 320, 513, 0.3), (2000, 129, 1023, 0.99)])
def test_forward_of_more_fp32_rows_than_stream(rows, d, V, masked, layout):
    _forward(_inputs(rows, d, V, F32, layout, masked=masked, pad=1), 0.8)


def test_streamed_rows_and_rows_in_tiles_agree():
    """Rows on either side of where fp32 calls change from one to the other; the masked one that tells them apart is not met."""
    import paper_2605_16154_amd as pcm
    for layout, few in (("in_out", 96), ("out_in", 64)):
        hidden, w, tokens, _ = _inputs(few + 1, 1024, 8192, F32, layout)
        tokens[few] = -1
        a, b = pcm.pcm_linear_logprobs(hidden[:few], w, tokens[:few]), pcm.pcm_linear_logprobs(hidden, w, tokens)
        E = _z_error(_np(hidden), _np(w), F32, 1.0).max()
        for k in a:
            assert float((a[k] - b[k][:few]).abs().max()) <= 2 * (4 * E + 2.0 ** -19) * 11, k
