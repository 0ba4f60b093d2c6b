"""pcm_token_logprobs_backward over the whole range of finite logits and temperatures, against the plain 64-bit form.

Tolerances, with u = 2^-24, a = (z - max z) / temperature, E = sum p |a|: where |lse| is below 1024 log p is x - lse with x and lse rounded, off by
u (3 |lse| + 6 |log p|); beyond, it comes from a sum over the row, off by u (V / 64 + 50 + 4 E) (a narrow row has as few as four lanes of two chunks, a wide one 256:
V / 64 additions at most), and from a, off by 6 u |log p|.  p has that as its relative error.  d x = [j = token] dlogp - p (dlogp + dentropy (log p + H)), where H is off by
the forward pass' d (2 + E) + 4 u E2 (E2 = sum p a^2).  Then come the roundings of the terms, 4 u of each, and of the result to its type; what is below 1e-37 may be zero.
"""
import numpy as np
import pytest
import torch

from oracle import operators as P

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _check(z, tokens, temperature=1.0, allowed=None, entropy=True, exact_lse=False, in_place=False, seed=0):
    import paper_2605_16154_amd as pcm
    rng = np.random.default_rng(seed)
    rows, V = z.shape
    dlogp = rng.standard_normal(rows).astype(np.float32)
    dentropy = rng.standard_normal(rows).astype(np.float32) if entropy else None
    dev = lambda x: None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()
    zc, tok, ok = z.cuda(), tokens.cuda(), dev(allowed)
    zd = z.double().numpy()
    plain = P.token_logprobs(zd, tokens.numpy(), allowed, temperature)
    fwd = pcm.pcm_token_logprobs(zc, tok, allowed=ok, temperature=temperature)
    with np.errstate(over="ignore"):
        lse = dev(plain["lse"].astype(np.float32)) if exact_lse else fwd["lse"]
    got = pcm.pcm_token_logprobs_backward(zc, tok, lse, dev(dlogp), entropy=fwd["entropy"] if entropy else None, dentropy=dev(dentropy), allowed=ok,
                                          temperature=temperature, out=zc if in_place else None)
    want = P.token_logprobs_gradient(zd, tokens.numpy(), dlogp, dentropy, allowed, temperature)
    full = np.ones(zd.shape, bool) if allowed is None else np.broadcast_to(allowed, zd.shape)
    x = np.where(full, zd, -np.inf)
    most = x.max(axis=1, keepdims=True)
    a = np.where(x > -np.inf, (x - np.where(most > -np.inf, most, 0.0)) / temperature, -np.inf)
    p = np.exp(a)
    s = np.maximum(p.sum(axis=1, keepdims=True), 1e-300)
    p = p / s
    size, logp = np.where(p > 0, -a, 0.0), np.where(p > 0, np.log(s) - a, 0.0)
    E, E2 = (p * size).sum(axis=1, keepdims=True), (p * size * size).sum(axis=1, keepdims=True)
    d = U * (V / 64 + 50 + 4 * E)
    known = np.abs(np.where(np.isfinite(plain["lse"]), plain["lse"], 1e9))[:, None]
    rel = np.where(known < 1100.0, 3 * U * np.minimum(known, 1100.0) + d, d) + 6 * U * logp + 6 * U
    h = np.zeros((rows, 1)) if dentropy is None else np.abs(dentropy.astype(np.float64))[:, None]
    g = np.abs(dlogp.astype(np.float64))[:, None]
    H = plain["entropy"][:, None]
    tol = p * (rel * (g + h * (logp + H + 1)) + h * (d * (2 + E) + 4 * U * E2 + 4 * U * (logp + H))) + 4 * U * g * (np.abs(want) > 0) * p
    tol = tol / temperature + 4 * U * np.abs(want) + 1e-37 * (1 + 1 / temperature)
    if z.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (np.abs(want) + tol)
    got = got.double().cpu().numpy()
    off = np.abs(got - want) / tol
    assert (off <= 1.0).all(), (np.argwhere(~(off <= 1.0))[:4].tolist(), got[~(off <= 1.0)][:4], want[~(off <= 1.0)][:4])
    if allowed is not None:
        assert (got[~full] == 0).all()


def _rows(rng, V, dtype):
    """Ordinary logits with a value that stands for excluded tokens in some of them, in all but one, in all; a forced token, two of them; large scales."""
    rows = []
    for size in (1e3, 3e4, 1e9, 1e10, 1e20, 1e38, float(torch.finfo(DTYPES[dtype]).max)):
        z = 3.0 * rng.standard_normal((8, V))
        z[0, rng.random(V) < 0.5] = -size
        z[1, np.arange(V) != V // 2] = -size
        z[2] = -size
        z[3, V - 1] = size
        z[4, [V // 3, V - 2]] = size
        z[5] *= size * 1e-4
        z[6] += size
        z[7, :8] = -size
        rows.append(z)
    return torch.from_numpy(np.clip(np.concatenate(rows), -3.4028234e38, 3.4028234e38).astype(np.float32)).clamp(
        torch.finfo(DTYPES[dtype]).min, torch.finfo(DTYPES[dtype]).max).to(DTYPES[dtype])


@pytest.mark.parametrize("dtype", ("f32", "bf16"))
@pytest.mark.parametrize("temperature", (1.0, 0.7, 1.3, 0.01, 1e9))
@pytest.mark.parametrize("V", (7, 60, 256, 700, 1500, 9001, 40001))
def test_logits_of_any_size(dtype, temperature, V):
    """Rows in one part and in several, with and without a mask, the lse of the forward call and one rounded from 64 bits, in place of the logits."""
    rng = np.random.default_rng(V)
    z = _rows(rng, V, dtype)
    best = z.float().argmax(dim=1).int()
    some = torch.from_numpy(rng.integers(-1, V, z.shape[0]).astype(np.int32))
    tokens = torch.where(torch.arange(z.shape[0]) % 2 == 0, best, some)
    _check(z, tokens, temperature)
    _check(z, some, temperature, entropy=False, in_place=True)
    _check(z, best, temperature, exact_lse=True)
    allowed = rng.random(z.shape) < 0.8
    allowed[3] = False
    _check(z, tokens, temperature, allowed=allowed, in_place=True)


@pytest.mark.parametrize("temperature", (1.0, 0.7, 1.3))
@pytest.mark.parametrize("force", (1e9, 1e10, 1e30))
@pytest.mark.parametrize("V", (200, 6000))
def test_a_certain_token_leaves_nothing_to_move(temperature, force, V):
    import paper_2605_16154_amd as pcm
    z = torch.randn((3, V), generator=torch.Generator().manual_seed(0)).cuda()
    z[:, 5] = force
    tokens = torch.tensor([5, 5, -1], device="cuda")
    f = pcm.pcm_token_logprobs(z, tokens, temperature=temperature)
    one = torch.ones(3, device="cuda")
    assert (pcm.pcm_token_logprobs_backward(z, tokens, f["lse"], one, f["entropy"], one, temperature=temperature) == 0).all()
