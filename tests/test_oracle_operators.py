"""The plain 64-bit forms of the operators on logits and updates against what they are defined by: scipy's log-softmax and
entropy, central differences of the scalar losses, and singular values."""
import numpy as np
import pytest
from scipy.special import log_softmax
from scipy.stats import entropy as scipy_entropy

from oracle import operators as P


def _case(seed, rows=5, V=9):
    rng = np.random.default_rng(seed)
    return rng, 2.0 * rng.standard_normal((rows, V)), rng.integers(0, V, rows)


@pytest.mark.parametrize("temperature", (1.0, 0.7))
def test_logprobs_against_scipy(temperature):
    rng, z, tokens = _case(0)
    got = P.token_logprobs(z, tokens, temperature=temperature, top=3)
    want = log_softmax(z / temperature, axis=1)
    np.testing.assert_allclose(got["logp"], want[np.arange(5), tokens], rtol=0, atol=1e-13)
    np.testing.assert_allclose(got["entropy"], scipy_entropy(np.exp(want), axis=1), rtol=0, atol=1e-13)
    order = np.argsort(-z, axis=1, kind="stable")[:, :3]
    np.testing.assert_array_equal(got["top_ids"], order)
    np.testing.assert_allclose(got["top_logp"], np.take_along_axis(want, order, 1), rtol=0, atol=1e-13)


def test_an_excluded_token_is_as_one_that_is_not_there():
    rng, z, tokens = _case(1)
    allowed = np.array([True, False, True, True, False, True, True, True, True])
    z[:, 1], z[:, 4] = np.nan, np.inf
    tokens = np.flatnonzero(allowed)[tokens % 7]
    got = P.token_logprobs(z, tokens, allowed, top=9)
    want = P.token_logprobs(z[:, allowed], np.searchsorted(np.flatnonzero(allowed), tokens), top=7)
    for k in ("logp", "lse", "entropy"):
        np.testing.assert_array_equal(got[k], want[k])
    assert (got["top_ids"][:, 7:] == -1).all() and np.isneginf(got["top_logp"][:, 7:]).all()
    assert np.isneginf(P.token_logprobs(z, np.full(5, 4), allowed)["logp"]).all()


def test_rows_without_a_choice_and_without_a_token():
    z = np.array([[-np.inf, -np.inf], [0.5, -0.5], [0.5, -0.5]])
    allowed = np.array([[1, 1], [0, 0], [1, 1]])
    got = P.token_logprobs(z, [0, 0, -1], allowed)
    assert np.isneginf(got["lse"][:2]).all() and (got["entropy"][:2] == 0).all() and np.isneginf(got["logp"][:2]).all()
    assert got["logp"][2] == 0
    g = P.token_logprobs_gradient(z, [0, 0, -1], np.ones(3), None, allowed)
    assert (g == 0).all()


@pytest.mark.parametrize("masked", (False, True))
@pytest.mark.parametrize("temperature", (1.0, 1.3))
def test_gradient_against_differences(masked, temperature):
    rng, z, tokens = _case(2)
    allowed = None
    if masked:
        allowed = rng.random(z.shape) < 0.7
        allowed[np.arange(5), tokens] = True
    dlogp, dentropy = rng.standard_normal(5), rng.standard_normal(5)
    g = P.token_logprobs_gradient(z, tokens, dlogp, dentropy, allowed, temperature)

    def loss(x):
        got = P.token_logprobs(x, tokens, allowed, temperature)
        return (dlogp * got["logp"]).sum() + (dentropy * got["entropy"]).sum()

    h = 1e-6
    for r in range(z.shape[0]):
        for j in range(z.shape[1]):
            up, down = z.copy(), z.copy()
            up[r, j] += h
            down[r, j] -= h
            assert abs((loss(up) - loss(down)) / (2 * h) - g[r, j]) < 1e-8, (r, j)


@pytest.mark.parametrize("shape", ((6, 6), (4, 11), (11, 4), (1, 5)))
def test_orthogonalise_moves_singular_values_only(shape):
    rng = np.random.default_rng(3)
    x = rng.standard_normal(shape)
    u, s, vt = np.linalg.svd(x / np.linalg.norm(x), full_matrices=False)
    counts = s > 0.002
    for _ in range(5):
        s = 3.4445 * s - 4.7750 * s**3 + 2.0315 * s**5
    np.testing.assert_allclose(P.orthogonalise(x), (u * s) @ vt, rtol=0, atol=1e-12)
    assert (s[counts] > 0.68).all() and (s < 1.21).all()


def test_muon_step_is_momentum_then_an_orthogonal_step():
    rng = np.random.default_rng(4)
    w, g, m = (rng.standard_normal((4, 16)) for _ in range(3))
    (nw,), (nm,), _ = P.muon_step([w], [g], [m], lr=0.1, weight_decay=0.5)
    np.testing.assert_allclose(nm, 0.95 * m + g)
    np.testing.assert_allclose(nw, w * 0.95 - 0.1 * 2.0 * P.orthogonalise(g + 0.95 * nm))
    (nw,), _, _ = P.muon_step([w], [g], [m], lr=0.1, nesterov=False, scale="rms")
    np.testing.assert_allclose(nw, w - 0.1 * 0.8 * P.orthogonalise(nm))
