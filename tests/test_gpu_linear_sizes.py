"""Log-probabilities through a vocabulary projection and their gradient at the sizes where the work is cut otherwise: tiles of 256 x 256 in every product,
vocabularies that are taken in several pieces of which the last is shorter, gradients added to what is there in one part and in several.

Hidden rows are whole numbers up to 2 and weights are -1, 0 or 1 times a power of two, so that logits, with fewer than 24 significant bits, are exact in
either type.  What is left, by arithmetic: lse and log p, 2^-20 (sums of exponentials) and 2^-22 of |lse| and of the largest |x|; the entropy 2^-19 (1 + log V).
The gradient takes lse and entropy from the plain form, rounded to fp32: log p is off by F = 2^-20 + 2^-22 (|x| + |lse|), dz by expm1(F) times the sizes
of its terms, |g| p and |h| p (|log p| + H + 1), 2^-22 |g| where the token is, and its own rounding (2^-8; for pairs 2^-22 and 2^-38 of the row's bound); the
products by (terms 2^-24) of the sum of sizes, for pairs 2^-20 more and 2^-38 (of dhidden) and 2^-36 (of dweight) of the largest value that shares a power of two;
the results by their own rounding.  The plain form and the bounds are computed on the GPU in 64 bits, in products of matrices that are not batched."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
STEP = {BF16: 2.0 ** -8, F32: 2.0 ** -24}


def _inputs(rows, d, V, dtype, layout, masked=0.2):
    gen = torch.Generator(device="cuda").manual_seed(rows + 7 * d + 13 * V)
    hidden = torch.randint(-2, 3, (rows, d), generator=gen, device="cuda").to(dtype)
    shape = (V, d) if layout == "out_in" else (d, V)
    # a standard deviation of the logits of 1 to 2
    unit = 2.0 ** -round(math.log2(d ** 0.5))
    w = (torch.randint(-1, 2, shape, generator=gen, device="cuda") * unit).to(dtype)
    tokens = torch.randint(0, V, (rows,), generator=gen, device="cuda")
    # some where the pieces and the vocabulary end
    tokens[::7] = V - 1
    tokens[torch.rand(rows, generator=gen, device="cuda") < masked] = -1
    return hidden, w.t() if layout == "out_in" else w, tokens, gen


def _blocks(rows, V):
    step = max(1, (1 << 27) // V)
    return [slice(r, min(rows, r + step)) for r in range(0, rows, step)]


def _reference(hidden, w, tokens, g, e, temperature):
    """-> lse, logp, entropy, largest |x| per row; dhidden and dweight with the bounds of their errors but for the results' own rounding; in 64 bits."""
    dtype, (rows, d), V = hidden.dtype, hidden.shape, w.shape[1]
    live = tokens >= 0
    W = w.to(F64)
    absW = W.abs()
    out = {k: torch.zeros(rows, dtype=F64, device="cuda") for k in ("lse", "logp", "entropy", "big")}
    grads = {k: torch.zeros(s, dtype=F64, device="cuda") for k, s in (("dh", (rows, d)), ("dh_off", (rows, d)), ("dw", (d, V)), ("dw_off", (d, V)))}
    extra = 0.0 if dtype == BF16 else 2.0 ** -20
    gl, el = (torch.where(live, x.to(F64), 0.0) for x in (g, e))
    share = 0.0
    for s in _blocks(rows, V):
        keep = live[s][:, None]
        h = torch.where(keep, hidden[s].to(F64), 0.0)
        x = h @ W / temperature
        lse = torch.logsumexp(x, dim=1, keepdim=True)
        logp = x - lse
        p = logp.exp()
        H = -(p * logp).sum(dim=1, keepdim=True)
        at = tokens[s].clamp(min=0)[:, None]
        for k, v in (("lse", lse), ("logp", torch.gather(logp, 1, at)), ("entropy", H), ("big", x.abs().amax(dim=1, keepdim=True))):
            out[k][s] = torch.where(keep, v, 0.0)[:, 0]
        p = torch.where(keep, p, 0.0)
        gr, er = gl[s][:, None], el[s][:, None]
        hit = torch.zeros_like(p).scatter_(1, at, 1.0) * keep
        dz = (gr * hit - p * (gr + er * (logp + H))) / temperature
        size = p * (gr.abs() + er.abs() * (logp.abs() + H + 1))
        off = (torch.expm1(2.0 ** -20 + 2.0 ** -22 * (x.abs() + lse.abs())) * size + 2.0 ** -22 * gr.abs() * hit) / temperature
        bound = (gr.abs() + er.abs() * (0.5 + H)) / temperature
        if dtype == BF16:
            off += 2.0 ** -8 * dz.abs()
        else:
            off += 2.0 ** -22 * dz.abs() + 2.0 ** -38 * bound * keep
            share += float((h.abs().amax(dim=1, keepdim=True) * bound).max()) * h.shape[0]
        grads["dh"][s] = dz @ W.t()
        grads["dh_off"][s] = (off + (V * 2.0 ** -24 + extra) * dz.abs()) @ absW.t()
        if dtype == F32:
            grads["dh_off"][s] += 2.0 ** -38 * float(absW.max()) * dz.abs().sum(dim=1, keepdim=True)
        grads["dw"] += h.t() @ dz
        grads["dw_off"] += h.abs().t() @ (off + (rows * 2.0 ** -24 + extra) * dz.abs())
    grads["dw_off"] += 2.0 ** -36 * share
    return out, grads


def _check(rows, d, V, dtype, layout, temperature=1.0, masked=0.2, forward=True, accumulate=False, dweight_dtype=None, want_dhidden=True):
    import paper_2605_16154_amd as pcm
    hidden, w, tokens, gen = _inputs(rows, d, V, dtype, layout, masked)
    g = torch.randn(rows, generator=gen, device="cuda")
    e = 0.3 * torch.randn(rows, generator=gen, device="cuda")
    out_type = dweight_dtype or dtype
    shape = (V, d) if layout == "out_in" else (d, V)
    start = torch.randn(shape, generator=gen, device="cuda") if accumulate else torch.full(shape, 7.0, device="cuda", dtype=out_type)
    out = {"dweight": start.clone().t() if layout == "out_in" else start.clone()}
    start = start.t() if layout == "out_in" else start
    ref, grads = _reference(hidden, w, tokens, g, e, temperature)
    live = tokens >= 0
    if forward:
        got = pcm.pcm_linear_logprobs(hidden, w, tokens, temperature=temperature)
        size = ref["lse"].abs() + ref["big"]
        for k, tol in (("lse", 2.0 ** -20 + 2.0 ** -22 * size), ("logp", 2.0 ** -20 + 2.0 ** -22 * size),
                       ("entropy", torch.full_like(size, 2.0 ** -19 * (1 + math.log(V))))):
            off = (got[k].to(F64) - ref[k]).abs()
            assert bool((off <= tol)[live].all()), (k, float((off / tol)[live].max()), int((off - tol).argmax()))
            assert not got[k][~live].any(), k
    if want_dhidden:
        out["dhidden"] = torch.full((rows, d), 7.0, dtype=dtype, device="cuda")
    pcm.pcm_linear_logprobs_backward(hidden, w, tokens, ref["lse"].float(), g, ref["entropy"].float(), e, temperature=temperature, accumulate=accumulate, out=out,
                                     want_dhidden=want_dhidden)
    torch.cuda.synchronize()
    want = grads["dw"] + (start.to(F64) if accumulate else 0.0)
    results = [("dweight", out["dweight"], want, grads["dw_off"] + 2 * STEP[out_type] * (want.abs() + grads["dw"].abs() * accumulate))]
    if want_dhidden:
        results.append(("dhidden", out["dhidden"], grads["dh"], grads["dh_off"] + 2 * STEP[dtype] * grads["dh"].abs()))
        assert not out["dhidden"][~live].any()
    for name, x, y, tol in results:
        off = (x.to(F64) - y).abs() - tol - 1e-37
        worst = int(off.argmax())
        assert bool((off <= 0).all()), (name, divmod(worst, x.shape[1]), float(off.max()), float(tol.flatten()[worst]))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", ["in_out", "out_in"])
@pytest.mark.parametrize("rows,d,V", [(1100, 72, 8200), (1100, 4100, 8200), (2100, 2056, 4100), (4200, 2300, 2603)])
def test_large_tiles(rows, d, V, layout, dtype):
    _check(rows, d, V, dtype, layout, temperature=0.7)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", ["in_out", "out_in"])
@pytest.mark.parametrize("rows", [100, 300])
def test_pieces_of_a_copied_weight(rows, layout, dtype):
    """65535 x 2500: 2048 columns of bf16, or 1024 of pairs, are 256 MB."""
    _check(rows, 65535, 2500, dtype, layout)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", ["in_out", "out_in"])
def test_pieces_of_the_gradient_in_the_logits(layout, dtype):
    """70000 rows: 7424 columns of dz in bf16, or 3584 of pairs, are 1 GB."""
    _check(70000, 24, 8200, dtype, layout)


@pytest.mark.parametrize("layout", ["in_out", "out_in"])
@pytest.mark.parametrize("dtype,dweight_dtype", [(F32, F32), (BF16, F32)])
@pytest.mark.parametrize("rows,d,V", [(260, 136, 520), (260, 135, 521), (1100, 1000, 300), (70000, 24, 8200), (100, 65535, 2500)])
def test_a_gradient_that_is_added(rows, d, V, dtype, dweight_dtype, layout):
    _check(rows, d, V, dtype, layout, forward=False, accumulate=True, dweight_dtype=dweight_dtype)
    _check(rows, d, V, dtype, layout, forward=False, accumulate=True, dweight_dtype=dweight_dtype, want_dhidden=False)


@pytest.mark.parametrize("layout", ["in_out", "out_in"])
def test_fp32_dweight_of_bf16_weights_in_pieces(layout):
    _check(70000, 24, 8200, BF16, layout, forward=False, dweight_dtype=F32)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_no_rows_and_no_tokens_make_zeros_of_what_was_there(dtype):
    import paper_2605_16154_amd as pcm
    for layout, shape in (("in_out", (64, 300)), ("out_in", (300, 64))):
        for rows in (0, 5, 300):
            w = torch.randn(shape, device="cuda").to(dtype)
            full = torch.full((shape[0], shape[1] + 3), 7.0, dtype=dtype, device="cuda")
            dw, view = full[:, :shape[1]], (lambda x: x.t() if layout == "out_in" else x)
            tokens = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
            none = torch.zeros(rows, device="cuda")
            out = {"dweight": view(dw), "dhidden": torch.full((rows, 64), 7.0, dtype=dtype, device="cuda")}
            pcm.pcm_linear_logprobs_backward(torch.ones(rows, 64, dtype=dtype, device="cuda"), view(w), tokens, none, none, out=out)
            assert not dw.any() and not out["dhidden"].any() and bool((full[:, shape[1]:] == 7).all()), rows
            kept = torch.randn(shape, device="cuda")
            added = {"dweight": view(kept.clone())}
            pcm.pcm_linear_logprobs_backward(torch.ones(rows, 64, dtype=dtype, device="cuda"), view(w), tokens, none, none, out=added, accumulate=True,
                                             want_dhidden=False)
            assert torch.equal(added["dweight"], view(kept)), rows
