"""pcm_token_logprobs over the whole range of finite logits and temperatures, against the plain 64-bit form.

Tolerances, with u = 2^-24, m the largest logit, a_j = (z_j - m) / temperature and p_j = e^(a_j) / s, s = sum e^(a_j): the difference of two logits
is rounded once, its product with log2 e / temperature (two roundings of its own) once more, the exponential is good to an ulp or two: a
term is off by (4 + 4 |a|) u of itself.  A lane adds up the sums of its chunks of eight, V / 512 at most, and about 40 levels of sums and
joins follow, each with a rounding or two.  So s is off by d = u (V / 512 + 50 + 4 E), E = sum p |a|, in relation to itself; log s by d in
absolute terms; logp = a - log s by d + 6 u |a| + 2 u |logp|; lse by d + 4 u |lse|; the entropy log s + E by d (2 + E) + 4 u E2, E2 = sum p a^2.
None of it grows with the size of the logits (but u |lse|).
"""
import numpy as np
import pytest
import torch

from oracle import operators as P

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
FILLS = (-1e9, -1e10, -1e12, -1e15, -1e20, -1e30, -1e38, None)         # None: the type's lowest value


def _pcm():
    import paper_2605_16154_amd as pcm
    return pcm


def _spread(z, allowed, temperature):
    """d, E and E2 of each row as above."""
    z = np.where(allowed, z, -np.inf)
    most = z.max(axis=1, keepdims=True)
    a = np.where(z > -np.inf, (z - np.where(most > -np.inf, most, 0.0)) / temperature, -np.inf)
    p = np.exp(a)
    p = p / np.maximum(p.sum(axis=1, keepdims=True), 1e-300)
    size = np.where(p > 0, -a, 0.0)
    E, E2 = (p * size).sum(axis=1), (p * size * size).sum(axis=1)
    return U * (z.shape[1] / 512 + 50 + 4 * E), E, E2


def _close(name, got, want, tol):
    got = got.double().cpu().numpy()
    with np.errstate(over="ignore"):
        want = np.where(np.isfinite(want.astype(np.float32)), want, want.astype(np.float32))       # beyond fp32: infinite
    fine = np.isfinite(want)
    np.testing.assert_array_equal(got[~fine], want[~fine], err_msg=name)
    off = np.abs(np.where(fine, got, 0.0) - np.where(fine, want, 0.0)) / np.broadcast_to(tol, want.shape)
    assert (off <= 1.0).all(), (name, np.argwhere(~(off <= 1.0))[:5].tolist(), float(off.max()))


def _check(z, tokens, temperature=1.0, top=0, allowed=None):
    zd = z.double().numpy()
    dev = None if allowed is None else torch.from_numpy(allowed).cuda()
    got = _pcm().pcm_token_logprobs(z.cuda(), tokens.cuda(), allowed=dev, temperature=temperature, top=top)
    want = P.token_logprobs(zd, tokens.numpy(), allowed, temperature, top)
    d, E, E2 = _spread(zd, np.ones(zd.shape, bool) if allowed is None else np.broadcast_to(allowed, zd.shape), temperature)
    finite = lambda x: np.where(np.isfinite(x), np.abs(x), 0.0)
    _close("lse", got["lse"], want["lse"], d + 4 * U * finite(want["lse"]))
    _close("logp", got["logp"], want["logp"], d + 8 * U * finite(want["logp"]))
    _close("entropy", got["entropy"], want["entropy"], d * (2 + E) + 4 * U * E2)
    if top:
        np.testing.assert_array_equal(got["top_ids"].cpu().numpy(), want["top_ids"])
        _close("top_logp", got["top_logp"], want["top_logp"], d[:, None] + 8 * U * finite(want["top_logp"]))
    return got


def _filled(rng, V, dtype, fill):
    """Rows of ordinary logits of which some hold a value that stands for an excluded token: shares of it at random, the first chunk of a lane, the first
    chunk of every lane, all but one logit, all."""
    z = 3.0 * rng.standard_normal((8, V))
    fill = torch.finfo(DTYPES[dtype]).min if fill is None else fill
    for r, share in enumerate((0.3, 0.5, 0.7, 0.99)):
        z[r, rng.random(V) < share] = fill
    z[4, 8:16] = fill
    z[5, :2048] = fill
    z[5, -1] = z[6, V // 2] = 0.5
    z[6, np.arange(V) != V // 2] = fill
    z[7] = fill
    return torch.from_numpy(z.astype(np.float32)).to(DTYPES[dtype])


@pytest.mark.parametrize("dtype", ("f32", "bf16"))
@pytest.mark.parametrize("temperature", (1.0, 0.7, 1.3, 1e-9))
@pytest.mark.parametrize("V", (100, 256, 1000, 3001, 32003))
def test_values_that_stand_for_excluded_tokens(dtype, temperature, V):
    rng = np.random.default_rng(V)
    z = torch.cat([_filled(rng, V, dtype, fill) for fill in FILLS])
    best = z.float().argmax(dim=1).int()
    some = torch.from_numpy(rng.integers(0, V, z.shape[0]).astype(np.int32))
    _check(z, torch.where(torch.arange(z.shape[0]) % 2 == 0, best, some), temperature)
    _check(z, best, temperature, top=3)
    _check(z, some, temperature, top=2, allowed=rng.random(V) < 0.9)


@pytest.mark.parametrize("dtype", ("f32", "bf16"))
@pytest.mark.parametrize("temperature", (1.0, 0.7, 0.3, 1e-9, 1e9))
@pytest.mark.parametrize("V", (7, 256, 3001, 40001))
def test_forced_tokens_and_logits_of_any_size(dtype, temperature, V):
    """One logit far above all, two equal ones, rows all near one large value, rows of a large scale."""
    rng = np.random.default_rng(V)
    rows = []
    for force in (1e9, 1e10, 1e20, 1e30, 9e37, 3e38):
        z = 3.0 * rng.standard_normal((5, V))
        z[0, V - 2] = z[1, 1] = force
        z[2, [V // 3, V - 1]] = force
        z[3] = -force
        z[3, V // 2] = force
        z[4] *= 1e-5 * force
        rows.append(z)
    z = torch.from_numpy(np.concatenate(rows).astype(np.float32)).to(DTYPES[dtype])
    best = z.float().argmax(dim=1).int()
    got = _check(z, best, temperature, top=2)
    one = torch.arange(z.shape[0]) % 5 == 0
    assert (got["logp"].cpu()[one] == 0).all() and (got["entropy"].cpu()[one] == 0).all() if temperature <= 1.0 else True
    _check(z, best, temperature)
    _check(z, torch.zeros(z.shape[0], dtype=torch.int32), temperature, allowed=np.arange(V) != V - 2)


@pytest.mark.parametrize("temperature", (2.0 ** -126, 1e-30, 1e-3, 1e6, 1e30, 3e38))
@pytest.mark.parametrize("V", (200, 5000))
def test_any_temperature(temperature, V):
    rng = np.random.default_rng(V)
    z = torch.from_numpy(np.concatenate([s * rng.standard_normal((3, V)) for s in (1e-36, 1e-5, 1.0, 1e4, 1e20, 5e36)]).astype(np.float32))
    tokens = torch.from_numpy(rng.integers(0, V, z.shape[0]).astype(np.int32))
    _check(z, tokens, temperature, top=4)
    _check(z, tokens, temperature)
    with pytest.raises(_pcm().PcmError):
        _pcm().pcm_token_logprobs(z.cuda(), tokens.cuda(), temperature=2.0 ** -127)
