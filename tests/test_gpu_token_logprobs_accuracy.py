"""How exact pcm_token_logprobs is, against the plain 64-bit form: rows that are all but certain, and ordinary ones.

With a_j = (z_j - max z) / temperature, p_j = e^(a_j) / s, s = sum e^(a_j), E = sum p |a|, E2 = sum p a^2, u = 2^-24 and `adds` the additions that a
lane makes one after the other (a chunk of eight logits each; a row of more than 4096 has 256 lanes, others 64): every addition and each of some 20 levels of
sums and joins rounds by at most u of s, and a term by (4 + 4 |a|) u of itself.  The largest term is exactly one.  So log s is off by u (adds + 20) +
4 u (E + the weight of the other terms), and the entropy log s + E by (1 + E) u (adds + 20) + 4 u (E + E2) at most.  Single roundings are as often up as
down, and of u / 2 on average, so over rows the root mean square is that of sqrt(adds + 30) roundings in place of their sum, with the rounding of log2 e (a factor on
all a alike: 2 u E on log s, 2 u (E2 - E^2) on the entropy) and of the results.
"""
import numpy as np
import pytest
import torch

from oracle import operators as P

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _both(z, tokens, top=0):
    """-> results, 64-bit results, adds, E, E2"""
    import paper_2605_16154_amd as pcm
    got = {k: v.double().cpu().numpy() for k, v in pcm.pcm_token_logprobs(z.cuda(), tokens.cuda(), top=top).items()}
    zd = z.double().numpy()
    a = zd - zd.max(axis=1, keepdims=True)
    p = np.exp(a)
    p /= p.sum(axis=1, keepdims=True)
    V = z.shape[1]
    return got, P.token_logprobs(zd, tokens.numpy(), top=top), V / (8 * (256 if V > 4096 else 64)), -(p * a).sum(axis=1), (p * a * a).sum(axis=1)


def _signs(got):
    assert (got["logp"] <= 0).all() and (got["entropy"] >= 0).all() and ("top_logp" not in got or (got["top_logp"] <= 0).all())


@pytest.mark.parametrize("dtype", ("f32", "bf16"))
@pytest.mark.parametrize("above", (12.0, 20.0, 30.0, 40.0, 60.0))
@pytest.mark.parametrize("V", (256, 1000, 3001, 32003, 100000))
@pytest.mark.parametrize("top", (0, 4))
def test_rows_that_are_all_but_certain(dtype, above, V, top):
    rng = np.random.default_rng(int(V + above))
    rows = 40
    z = rng.standard_normal((rows, V))
    at = rng.integers(0, V, rows)
    at[:4] = 0, V - 1, V - 8, min(V - 1, 2050)
    z[np.arange(rows), at] = above + 0.37 * rng.random(rows)
    z[20:, rng.integers(0, V, 3)] = above - 7.0            # a few others that count
    z = torch.from_numpy(z.astype(np.float32)).to(DTYPES[dtype])
    got, want, adds, E, E2 = _both(z, torch.from_numpy(at), top)
    off = lambda k: np.abs(got[k] - want[k])
    d = U * (adds + 20) + 4 * U * (E + np.minimum(E, 1.0))
    assert (off("logp") <= d + 6 * U * np.abs(want["logp"])).all(), (off("logp") / U).max()
    assert (off("entropy") <= U * (adds + 20) * (1 + E) + 4 * U * (E + E2)).all(), (off("entropy") / U).max()
    assert (off("lse") <= d + 2 * U * np.abs(want["lse"])).all(), (off("lse") / U).max()
    _signs(got)


@pytest.mark.parametrize("dtype", ("f32", "bf16"))
@pytest.mark.parametrize("spread", (0.0, 1.0, 3.0))
@pytest.mark.parametrize("rows,V", ((64, 256), (64, 1000), (50, 4096), (24, 32003), (300, 10007), (30, 131072)))
def test_ordinary_rows(dtype, spread, rows, V):
    rng = np.random.default_rng(V)
    z = torch.from_numpy((0.25 + spread * rng.standard_normal((rows, V))).astype(np.float32)).to(DTYPES[dtype])
    tokens = torch.from_numpy(rng.integers(0, V, rows))
    for top in (0, 3):
        got, want, adds, E, E2 = _both(z, tokens, top)
        rms = lambda x: float(np.sqrt(np.mean(np.square(x))))
        log_s, n = want["entropy"] - E, np.sqrt(adds + 30)
        d = U * (n + 2 * E + log_s)
        assert rms(got["lse"] - want["lse"]) <= rms(d + U * np.abs(want["lse"])), rms(got["lse"] - want["lse"]) / U
        assert rms(got["logp"] - want["logp"]) <= rms(d + 4 * U * np.abs(want["logp"])), rms(got["logp"] - want["logp"]) / U
        h = U * ((1 + E) * n + 2 * (E2 - E * E) + 2 * E + 2 * want["entropy"])
        assert rms(got["entropy"] - want["entropy"]) <= rms(h), rms(got["entropy"] - want["entropy"]) / U
        _signs(got)


@pytest.mark.parametrize("rows,V,top", ((50, 256, 0), (50, 256, 4), (20, 3000, 0), (4, 60000, 3), (700, 9000, 2)))
def test_a_row_does_not_depend_on_what_others_hold(rows, V, top):
    """The same row among others of any kind, and at another place: the same bits.  Alone: the same but for its last ones."""
    import paper_2605_16154_amd as pcm
    gen = torch.Generator("cuda").manual_seed(V)
    z = 2.0 * torch.randn((rows, V), generator=gen, device="cuda")
    tokens = torch.randint(0, V, (rows,), generator=gen, device="cuda")
    want = pcm.pcm_token_logprobs(z, tokens, top=top)
    other = 1e30 * torch.randn((rows, V), generator=gen, device="cuda")
    other[1::3] = float("nan")
    other[2::3] = -float("inf")
    d = torch.randn(rows, generator=gen, device="cuda")
    grad = pcm.pcm_token_logprobs_backward(z, tokens, want["lse"], d, want["entropy"], d)
    for keep, to in ((0, rows - 1), (rows - 1, 1), (rows // 2, rows // 2)):
        x, t = other.clone(), tokens.clone()
        x[to], t[to] = z[keep], tokens[keep]
        got = pcm.pcm_token_logprobs(x, t, top=top)
        for k in want:
            assert torch.equal(got[k][to], want[k][keep]), k
        dx = d.clone()
        dx[to] = d[keep]
        assert torch.equal(pcm.pcm_token_logprobs_backward(x, t, got["lse"], dx, got["entropy"], dx)[to], grad[keep])
    alone = pcm.pcm_token_logprobs(z[3:4], tokens[3:4], top=top)
    zd = z[3:4].double().cpu().numpy()
    a = zd - zd.max()
    p = np.exp(a) / np.exp(a).sum()
    E, E2 = -(p * a).sum(), (p * a * a).sum()
    d_s = 2 * (U * (V / (8 * (256 if V > 4096 else 64)) + 20) + 4 * U * (E + 1))
    for k, tol in (("lse", d_s + 4 * U * 20), ("logp", d_s + 8 * U * 20), ("entropy", d_s * (2 + E) + 8 * U * E2)):
        assert abs(alone[k].item() - want[k][3].item()) <= tol, k
    if top:
        assert torch.equal(alone["top_ids"][0], want["top_ids"][3])
