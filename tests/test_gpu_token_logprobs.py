"""pcm_token_logprobs and pcm_token_logprobs_backward against their plain 64-bit forms.

Tolerances, with x = logit / temperature and u = 2^-24: a term of the row's sum is 2 to an exponent that is the difference of two
fp32 numbers of the size of x log2 e, each rounded once or twice, so it is off by 6 u max|x| in relation to itself (and an ulp or
two of the exponential); the sum adds at most `chain` terms one after the other and then a few tens.  So lse, logp and top_logp
are within u (chain + 40 + 8 max|x|), in absolute terms; the entropy, a mean of |x - lse| <= 2 max|x| with such weights, within
(2 + 2 max|x|) times that.  A gradient is p times a bracket of |dlogp| + |dentropy| (|log p| + H): relative error of p, with lse
rounded to fp32 as well, u (chain + 60 + 12 max|x|) of the terms, and the rounding of the output type.
"""
import numpy as np
import pytest
import torch

from oracle import operators as P

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _pcm():
    import paper_2605_16154_amd as pcm
    return pcm


def _logits(rng, rows, V, dtype, scale=3.0):
    z = torch.from_numpy((scale * rng.standard_normal((rows, V))).astype(np.float32)).to(DTYPES[dtype])
    return z, z.double().numpy()


def _bound(z, temperature, V, allowed=None):
    x = np.where(np.isfinite(z), np.abs(z), 0.0) / temperature
    if allowed is not None:
        x = np.where(np.broadcast_to(np.asarray(allowed, bool), x.shape), x, 0.0)
    chain = V / 64 + 8                       # a row has at least 64 lanes
    return x.max(axis=1, initial=0.0), U * (chain + 40 + 8 * x.max(axis=1, initial=0.0))


def _close(got, want, tol):
    got = got.double().cpu().numpy()
    fine = np.isfinite(want)
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
    np.testing.assert_array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)])
    off = np.abs(np.where(fine, got, 0) - np.where(fine, want, 0))
    assert (off <= np.where(fine, tol, 1)).all(), (float(off.max()), off.shape)


def _check_forward(z, zd, tokens, allowed=None, temperature=1.0, top=0, entropy=True):
    pcm = _pcm()
    dev_allowed = None if allowed is None else torch.from_numpy(np.asarray(allowed, bool)).cuda()
    got = pcm.pcm_token_logprobs(z.cuda() if not z.is_cuda else z, tokens.cuda(), allowed=dev_allowed, temperature=temperature,
                                 want_entropy=entropy, top=top)
    want = P.token_logprobs(zd, tokens.numpy(), allowed, temperature, top)
    most, tol = _bound(zd, temperature, zd.shape[1], allowed)
    _close(got["lse"], want["lse"], tol)
    _close(got["logp"], want["logp"], tol)
    assert ("entropy" in got) == entropy
    if entropy:
        _close(got["entropy"], want["entropy"], (2 + 2 * most) * tol)
    if top:
        np.testing.assert_array_equal(got["top_ids"].cpu().numpy(), want["top_ids"])
        _close(got["top_logp"], want["top_logp"], tol[:, None])
    return got


def _check_backward(z, zd, tokens, dlogp, dentropy=None, allowed=None, temperature=1.0, out=None):
    pcm = _pcm()
    f = lambda x: torch.from_numpy(np.asarray(x, np.float32)).cuda()
    dev_allowed = None if allowed is None else torch.from_numpy(np.asarray(allowed, bool)).cuda()
    z, tok = z if z.is_cuda else z.cuda(), tokens.cuda()
    fwd = pcm.pcm_token_logprobs(z, tok, allowed=dev_allowed, temperature=temperature)
    got = pcm.pcm_token_logprobs_backward(z, tok, fwd["lse"], f(dlogp), entropy=fwd["entropy"],
                                          dentropy=None if dentropy is None else f(dentropy), allowed=dev_allowed,
                                          temperature=temperature, out=out)
    dlogp = np.asarray(dlogp, np.float32)
    dentropy = None if dentropy is None else np.asarray(dentropy, np.float32)
    want = P.token_logprobs_gradient(zd, tokens.numpy(), dlogp, dentropy, allowed, temperature)
    most, _ = _bound(zd, temperature, zd.shape[1], allowed)
    h = 0.0 if dentropy is None else np.abs(dentropy.astype(np.float64))
    x = np.where(np.isfinite(zd), zd, 0.0) / temperature
    lse = np.where(np.isfinite(fwd["lse"].double().cpu().numpy()), fwd["lse"].double().cpu().numpy(), 0.0)
    p = np.exp(np.minimum(x - lse[:, None], 1.0))
    size = p * (np.abs(dlogp.astype(np.float64)) + h * (3 + 4 * most))[:, None] / temperature
    tol = U * (zd.shape[1] / 64 + 60 + 12 * most)[:, None] * (2 + 2 * most)[:, None] * size
    tol = tol + 4 * U * (np.abs(want) + (np.abs(dlogp.astype(np.float64)) / temperature)[:, None]) + 1e-37
    if z.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (np.abs(want) + tol)
    _close(got, want, tol)
    return got


@pytest.mark.parametrize("dtype", ("f32", "bf16"))
@pytest.mark.parametrize("rows,V", ((1, 1), (3, 2), (2, 7), (5, 8), (4, 9), (1, 63), (9, 64), (6, 255), (70, 256), (7, 257), (3, 1000),
                                    (2, 2047), (2, 2049), (3, 5003), (1, 16384), (2, 40001), (1, 131072)))
def test_sizes(dtype, rows, V):
    rng = np.random.default_rng(rows * 1000 + V)
    z, zd = _logits(rng, rows, V, dtype)
    tokens = torch.from_numpy(rng.integers(0, V, rows).astype(np.int32))
    _check_forward(z, zd, tokens, top=5)
    _check_forward(z, zd, tokens, entropy=False)
    _check_backward(z, zd, tokens, rng.standard_normal(rows), rng.standard_normal(rows))
    _check_backward(z, zd, tokens, rng.standard_normal(rows))


@pytest.mark.parametrize("rows", (1, 2, 63, 64, 65, 1000))
def test_many_rows_of_the_action_bins(rows):
    rng = np.random.default_rng(rows)
    z, zd = _logits(rng, rows, 256, "bf16")
    tokens = torch.from_numpy(rng.integers(0, 256, rows).astype(np.uint8))
    _check_forward(z, zd, tokens)
    _check_forward(z, zd, tokens, top=3)
    _check_backward(z, zd, tokens, rng.standard_normal(rows), 0.1 * rng.random(rows))


@pytest.mark.parametrize("dtype", ("f32", "bf16"))
@pytest.mark.parametrize("V", (5, 64, 300, 4099, 33000))
@pytest.mark.parametrize("kind", ("tokens", "rows"))
def test_masks_over_anything_in_masked_places(dtype, V, kind):
    rng = np.random.default_rng(V)
    rows = 6
    z, zd = _logits(rng, rows, V, dtype)
    allowed = rng.random((rows, V)) < np.array([0.5, 0.0, 0.02, 1.0, 0.9, 0.3])[:, None]
    if kind == "tokens":
        allowed = rng.random(V) < 0.6
        allowed[V // 2] = True
    else:
        allowed[2, V - 1] = True                     # a row that may have no other
    full = np.broadcast_to(allowed, (rows, V))
    junk = torch.tensor([float("nan"), float("inf"), -float("inf"), torch.finfo(z.dtype).max, torch.finfo(z.dtype).min]).to(z.dtype)
    pick = torch.from_numpy(rng.integers(0, 5, (rows, V)))
    z = torch.where(torch.from_numpy(full.copy()), z, junk[pick])
    zd = z.double().numpy()
    tokens = torch.from_numpy(rng.integers(0, V, rows))
    for top in (0, 4, 64):
        _check_forward(z, zd, tokens, allowed, 0.7, top)
    _check_backward(z, zd, tokens, rng.standard_normal(rows), rng.standard_normal(rows), allowed, 0.7)
    _check_backward(z, zd, tokens, rng.standard_normal(rows), None, allowed)


def test_a_mask_that_allows_nothing():
    z, zd = _logits(np.random.default_rng(0), 3, 77, "f32")
    tokens = torch.tensor([0, 5, 76])
    got = _check_forward(z, zd, tokens, np.zeros(77, bool), top=3)
    assert (got["top_ids"] == -1).all()
    assert (_check_backward(z, zd, tokens, np.ones(3), np.ones(3), np.zeros(77, bool)) == 0).all()


@pytest.mark.parametrize("dtype", ("f32", "bf16"))
@pytest.mark.parametrize("V", (40, 256, 3001, 70001))
def test_extreme_logits(dtype, V):
    """-inf and the type's lowest value among allowed logits, one token far above all others, far apart scales, equal logits."""
    rng = np.random.default_rng(V)
    z, _ = _logits(rng, 8, V, dtype)
    low = torch.finfo(z.dtype).min
    z[0, rng.random(V) < 0.7] = -float("inf")
    z[1, rng.random(V) < 0.7] = low
    z[2] = low
    z[3] = -float("inf")
    z[4] = -300.0
    z[4, V - 1] = 400.0
    z[5] *= 100.0
    z[6] = 2.0
    z[7] = torch.linspace(-80, 80, V).to(z.dtype)      # rising: every logit is above all before it
    zd = z.double().numpy()
    tokens = torch.tensor([3, 4, 5, 6, V - 1, 0, 7, V - 2])
    got = _check_forward(z[:1], zd[:1], tokens[:1], top=7)
    for r in range(8):
        if r in (1, 2):
            continue
        _check_forward(z[r:r + 1], zd[r:r + 1], tokens[r:r + 1], top=7)
        if r != 3:
            _check_backward(z[r:r + 1], zd[r:r + 1], tokens[r:r + 1], [1.5], [-0.5])
    assert got["lse"].isfinite().all()
    # a row partly at the lowest value is one where those tokens are excluded, for all that can be seen
    keep = zd[1] > low
    a = _pcm().pcm_token_logprobs(z[1:2].cuda(), torch.tensor([int(np.flatnonzero(keep)[0])]).cuda(), top=3)
    b = P.token_logprobs(zd[1:2], [int(np.flatnonzero(keep)[0])], keep, top=3)
    _close(a["lse"], b["lse"], 1e-4)
    _close(a["entropy"], b["entropy"], 1e-3)
    np.testing.assert_array_equal(a["top_ids"].cpu().numpy(), b["top_ids"])
    # a row all at it is one of equal logits
    a = _pcm().pcm_token_logprobs(z[2:3].cuda(), tokens[2:3].cuda(), top=5)
    assert abs(a["entropy"].item() - np.log(V)) < 1e-4 and abs(a["logp"].item() + np.log(V)) < 1e-4
    assert a["top_ids"].tolist() == [[0, 1, 2, 3, 4]]


@pytest.mark.parametrize("bad", (float("nan"), float("inf")))
@pytest.mark.parametrize("V", (3, 256, 20000))
def test_nan_and_infinity_stay_in_their_row(bad, V):
    rng = np.random.default_rng(V)
    z, _ = _logits(rng, 3, V, "f32")
    z[1, V // 2] = bad
    zd = z.double().numpy()
    tokens = torch.tensor([0, 1, 2])
    got = _check_forward(z, zd, tokens, top=2)
    assert got["lse"][1].isnan() and got["entropy"][1].isnan() and got["logp"][1].isnan()
    g = _pcm().pcm_token_logprobs_backward(z.cuda(), tokens.cuda(), got["lse"], torch.ones(3, device="cuda"))
    assert g[1].isnan().all() and g[0].isfinite().all() and g[2].isfinite().all()


@pytest.mark.parametrize("dtype", ("f32", "bf16"))
@pytest.mark.parametrize("V", (10, 256, 1999, 50000))
@pytest.mark.parametrize("top", (1, 2, 17, 64))
def test_ties_go_to_the_lowest_index(dtype, V, top):
    rng = np.random.default_rng(top)
    z = torch.from_numpy(rng.integers(-3, 4, (4, V)).astype(np.float32)).to(DTYPES[dtype])
    z[1] = 0.0
    z[1, ::2] = -0.0                                   # equal to 0.0
    z[2] = -float("inf")
    z[2, V - 1] = 1.0
    zd = z.double().numpy()
    _check_forward(z, zd, torch.zeros(4, dtype=torch.int32), top=top)


@pytest.mark.parametrize("dtype", ("f32", "bf16"))
@pytest.mark.parametrize("V,ld,offset", ((256, 300, 3), (1000, 1001, 1), (33, 64, 5), (4099, 4200, 7)))
def test_views_of_wider_matrices(dtype, V, ld, offset):
    """Rows at any distance and any multiple of the type's size; what lies between the rows of the gradient is left alone."""
    rng = np.random.default_rng(V)
    rows = 5
    wide, _ = _logits(rng, rows, ld, dtype)
    wide = wide.cuda()
    z = wide[:, offset:offset + V]
    zd = z.double().cpu().numpy()
    tokens = torch.from_numpy(rng.integers(0, V, rows))
    allowed = torch.from_numpy(rng.random((rows, V + 3)) < 0.8).cuda()[:, 2:2 + V]
    _check_forward(z, zd, tokens, top=6)
    _check_forward(z, zd, tokens, allowed.cpu().numpy(), top=6)
    pcm = _pcm()
    fwd = pcm.pcm_token_logprobs(z, tokens.cuda(), allowed=allowed)
    want = P.token_logprobs(zd, tokens.numpy(), allowed.cpu().numpy())
    _close(fwd["lse"], want["lse"], _bound(zd, 1.0, V)[1])
    into = torch.full((rows, ld), 7.0, dtype=z.dtype, device="cuda")
    _check_backward(z, zd, tokens, rng.standard_normal(rows), out=into[:, offset:offset + V])
    assert (into[:, :offset] == 7).all() and (into[:, offset + V:] == 7).all()


def test_gradient_in_place_of_the_logits():
    rng = np.random.default_rng(5)
    z, zd = _logits(rng, 9, 777, "bf16")
    z, tokens, d = z.cuda(), torch.from_numpy(rng.integers(0, 777, 9)).cuda(), torch.randn(9, device="cuda")
    pcm = _pcm()
    lse = pcm.pcm_token_logprobs(z, tokens)["lse"]
    want = pcm.pcm_token_logprobs_backward(z, tokens, lse, d)
    got = pcm.pcm_token_logprobs_backward(z, tokens, lse, d, out=z)
    assert got is z and torch.equal(got, want)


@pytest.mark.parametrize("dtype", (torch.uint8, torch.int32, torch.int64))
def test_token_types_and_tokens_out_of_range(dtype):
    rng = np.random.default_rng(6)
    V = 100
    z, zd = _logits(rng, 6, V, "f32")
    values = [0, 99, 100, 255, 7, 8] if dtype == torch.uint8 else [0, 99, 100, 2 ** 31 - 1, -1, -(2 ** 31)]
    tokens = torch.tensor(values).to(dtype)
    if dtype == torch.int64:
        tokens[2], tokens[5] = 2 ** 40, -(2 ** 40)
    got = _check_forward(z, zd, tokens)
    if dtype != torch.uint8:
        assert got["logp"][4:].tolist() == [0.0, 0.0]
    _check_backward(z, zd, tokens, rng.standard_normal(6), rng.standard_normal(6))


def test_rows_beyond_32_bit_offsets():
    rng = np.random.default_rng(7)
    V, ld = 1000, (1 << 30) + 3
    big = torch.empty(3 * ld, dtype=torch.bfloat16, device="cuda")
    z = big.as_strided((3, V), (ld, 1))
    small, zd = _logits(rng, 3, V, "bf16")
    z.copy_(small.cuda())
    tokens = torch.from_numpy(rng.integers(0, V, 3))
    _check_forward(z, zd, tokens, top=3)
    _check_backward(z, zd, tokens, rng.standard_normal(3), out=z)


@pytest.mark.parametrize("top", (0, 2))
def test_more_rows_than_a_launch_takes(top):
    rows, V, tail = 2 ** 23 + 7, 4, 64
    gen = torch.Generator("cuda").manual_seed(4)
    z = torch.randn(rows, V, generator=gen, device="cuda")
    tokens = torch.randint(0, V, (rows,), generator=gen, device="cuda", dtype=torch.uint8)
    allowed = torch.rand(rows, V, generator=gen, device="cuda") < 0.8
    pcm = _pcm()
    whole = pcm.pcm_token_logprobs(z, tokens, allowed=allowed, top=top)
    dlogp, dentropy = torch.randn(2, rows, generator=gen, device="cuda").unbind()
    grad = pcm.pcm_token_logprobs_backward(z, tokens, whole["lse"], dlogp, whole["entropy"], dentropy, allowed=allowed)
    for part in (slice(0, tail), slice(rows - tail, rows)):
        zs, ts, ok = z[part].contiguous(), tokens[part].cpu(), allowed[part].cpu().numpy()
        alone = _check_forward(zs, zs.double().cpu().numpy(), ts, ok, top=top)
        for k, v in alone.items():
            assert torch.equal(whole[k][part], v), k
        got = _check_backward(zs, zs.double().cpu().numpy(), ts, dlogp[part].cpu().numpy(), dentropy[part].cpu().numpy(), ok)
        if top == 0:                                   # (lse and entropy come from the same launch shape)
            assert torch.equal(grad[part], got)
    assert torch.isfinite(grad).all()


def test_rows_do_not_depend_on_one_another_and_repeat_bit_for_bit():
    rng = np.random.default_rng(8)
    pcm = _pcm()
    for rows, V in ((50, 256), (20, 3000), (4, 60000)):
        z, _ = _logits(rng, rows, V, "bf16")
        z, tokens = z.cuda(), torch.from_numpy(rng.integers(0, V, rows)).cuda()
        first = pcm.pcm_token_logprobs(z, tokens, top=4)
        again = pcm.pcm_token_logprobs(z, tokens, top=4)
        for k in first:
            assert torch.equal(first[k], again[k]), k


def test_no_rows():
    pcm = _pcm()
    z, tokens = torch.empty((0, 40), device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    got = pcm.pcm_token_logprobs(z, tokens, top=3)
    assert got["logp"].shape == (0,) and got["top_ids"].shape == (0, 3)
    assert pcm.pcm_token_logprobs_backward(z, tokens, got["lse"], got["logp"]).shape == (0, 40)


def test_on_another_stream_and_in_a_graph():
    """The calls go to the current stream; a graph of them gives the eager results on every replay, with new logits too."""
    rng = np.random.default_rng(9)
    pcm = _pcm()
    rows, V = 4, 50000
    z = _logits(rng, rows, V, "bf16")[0].cuda()
    other = _logits(rng, rows, V, "bf16")[0].cuda()
    tokens, d = torch.from_numpy(rng.integers(0, V, rows)).cuda(), torch.randn(rows, device="cuda")

    def both(x):
        f = pcm.pcm_token_logprobs(x, tokens, top=3)
        return [*f.values(), pcm.pcm_token_logprobs_backward(x, tokens, f["lse"], d)]

    want, want_other = both(z), both(other)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = both(z)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    x = z.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = both(x)
    for k in range(4):
        x.copy_(other if k % 2 else z)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, want_other if k % 2 else want)), k
        both(other)                                    # eager work between the replays
        torch.cuda.synchronize()


def test_the_gradient_moves_the_loss_as_it_says():
    """A step against the gradient of mean(-logp) - 0.1 mean(entropy) lowers it by step |g|^2, to first order (fp32 losses of
    about 5 are known to 1e-6, the fall is 1e-2 and its second-order part below a tenth of it)."""
    rng = np.random.default_rng(10)
    pcm = _pcm()
    rows, V = 32, 200
    z = _logits(rng, rows, V, "f32")[0].cuda()
    tokens = torch.from_numpy(rng.integers(0, V, rows)).cuda()

    def loss(x):
        f = pcm.pcm_token_logprobs(x, tokens)
        return (-f["logp"].double().mean() - 0.1 * f["entropy"].double().mean()).item(), f

    before, f = loss(z)
    ones = torch.ones(rows, device="cuda")
    g = pcm.pcm_token_logprobs_backward(z, tokens, f["lse"], -ones / rows, entropy=f["entropy"], dentropy=-0.1 * ones / rows)
    sq = g.double().square().sum().item()
    step = 1e-2 / sq
    after, _ = loss(z - step * g)
    assert abs((before - after) / 1e-2 - 1) < 0.2, (before, after, sq)


def test_refusals():
    pcm = _pcm()
    z = torch.zeros((4, 10), device="cuda")
    t = torch.zeros(4, dtype=torch.int32, device="cuda")
    lse = torch.zeros(4, device="cuda")
    for kw in (dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=float("nan")), dict(temperature=float("inf")),
               dict(temperature=1e-45), dict(top=-1), dict(top=65), dict(allowed=torch.ones(9, dtype=torch.bool, device="cuda")),
               dict(allowed=torch.ones((4, 9), dtype=torch.bool, device="cuda")), dict(allowed=torch.ones(10, device="cuda")),
               dict(allowed=torch.ones(10, dtype=torch.bool)), dict(out=dict(logp=torch.zeros(3, device="cuda"))),
               dict(out=dict(lse=torch.zeros(4, dtype=torch.float64, device="cuda")))):
        with pytest.raises(pcm.PcmError):
            pcm.pcm_token_logprobs(z, t, **kw)
    for bad in (z.cpu(), z.half(), z.T, z[0], z[:, ::2], z[:1].expand(4, 10)):
        with pytest.raises(pcm.PcmError):
            pcm.pcm_token_logprobs(bad, t[:bad.shape[0]])
    for bad in (t.cpu(), t.float(), t[:3], t[:, None]):
        with pytest.raises(pcm.PcmError):
            pcm.pcm_token_logprobs(z, bad)
    for args, kw in (((lse[:3], lse), {}), ((lse, lse.double()), {}), ((lse, lse), dict(dentropy=lse)),
                     ((lse, lse), dict(out=z[:3])), ((lse, lse), dict(out=z.to(torch.bfloat16)))):
        with pytest.raises(pcm.PcmError):
            pcm.pcm_token_logprobs_backward(z, t, *args, **kw)
