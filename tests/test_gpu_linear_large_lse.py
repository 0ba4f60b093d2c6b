"""Gradient through a vocabulary projection where the log-sum-exp of a row is large beside 1: low temperatures, rows that are all but certain.

log p = z / temperature - lse is then the difference of two large numbers, each rounded, and is known up to
  D = 2^-22 (|x| + |lse|) + 2 E,   E the error of a logit in either direction (tests/test_gpu_linear_logprobs.py),
so p is between e^-D times what it is and the smaller of e^D times that and 1.  The inputs leave the second largest logit of a row so far behind
(more than 2 D + 200) that all probabilities but the largest are nothing: the gradient in the logits is g in the token's place and -g p in the largest one's.
With |p - 1| <= 1 - e^-D the results are off by that times |g| / temperature times the weight's column, or the hidden row; and by the roundings of what
is computed, which is as large as the exact value and that error together: a value of dz (2^-8 of it; 2^-20 for pairs), a sum of n terms (n 2^-24), the
product's operands (2^-20 for pairs), the result (2^-8, 2^-24 of its size)."""
import numpy as np
import pytest
import torch

from tests.test_gpu_linear_logprobs import _np, _z_error

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def _case(rows, d, V, dtype, layout, temperature):
    gen = torch.Generator().manual_seed(11)
    hidden = (4.0 * torch.randn((rows, d), generator=gen)).to(dtype)
    w = torch.randn((d, V), generator=gen).mul(d ** -0.5).to(dtype)
    best = torch.randint(0, V, (rows,), generator=gen)
    hidden = (hidden.float() + 2.0 * w.float().t()[best]).to(dtype)
    z = _np(hidden) @ _np(w)
    E = _z_error(_np(hidden), _np(w), dtype, temperature).max(axis=1)
    best = z.argmax(axis=1)
    lse = z.max(axis=1) / temperature                       # exactly, up to log(1 + e^-200)
    D = 2.0 ** -22 * 2 * np.abs(lse) + 2 * E
    second = np.sort(z, axis=1)[:, -2] / temperature
    clear = lse - second > 2 * D + 200                      # the others are left out of the call
    tokens = np.where(np.arange(rows) % 2 == 0, best, (best + 1) % V)
    tokens = torch.from_numpy(np.where(clear, tokens, -1))
    assert clear.sum() >= 3
    w = w.t().contiguous().cuda().t() if layout == "out_in" else w.cuda()
    return hidden.cuda(), w, tokens.cuda(), best, D


@pytest.mark.parametrize("entropy", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", ["in_out", "out_in"])
@pytest.mark.parametrize("temperature", [1e-2, 1e-4, 1e-6, 1e-9, 2.0 ** -60])
@pytest.mark.parametrize("rows,d,V", [(40, 64, 300), (300, 72, 130)])
def test_rows_that_are_certain(rows, d, V, temperature, layout, dtype, entropy):
    import paper_2605_16154_amd as pcm
    hidden, w, tokens, best, D = _case(rows, d, V, dtype, layout, temperature)
    t = tokens.cpu().numpy()
    live = t >= 0
    forward = pcm.pcm_linear_logprobs(hidden, w, tokens, temperature=temperature)
    g = torch.randn(rows, generator=torch.Generator().manual_seed(5)).cuda()
    e = 0.3 * g.flip(0).contiguous() if entropy else None
    out = pcm.pcm_linear_logprobs_backward(hidden, w, tokens, forward["lse"], g, forward["entropy"] if entropy else None, e, temperature=temperature)
    gn = np.where(live, _np(g), 0.0) / temperature
    one = np.zeros((rows, V))
    one[np.arange(rows), np.where(live, best, 0)] = live
    hit = np.zeros((rows, V))
    hit[np.arange(rows), np.where(live, t, 0)] = live
    dz = gn[:, None] * (hit - one)
    # p log p and p H, H what the forward call gave: each at most D or 1 / e away from 0, and the entropy is 0 up to its own error of 4 E (1 + log V)
    off = np.abs(gn)[:, None] * (-np.expm1(-D))[:, None] * one
    if entropy:
        en = np.abs(np.where(live, _np(e), 0.0))[:, None] / temperature
        off += en * one * (np.minimum(D, np.exp(-1.0))[:, None] + np.abs(_np(forward["entropy"]))[:, None])
    # what is rounded from here on is a value that is off by that already: roundings are relative to a size of |dz| + off
    size = np.abs(dz) + off + (en * one if entropy else 0.0)
    step = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
    off += size * (2.0 ** -8 if dtype == BF16 else 2.0 ** -20) + 2.0 ** -38 * size.max(axis=1, keepdims=True) * live[:, None]
    h, wn = np.where(live[:, None], _np(hidden), 0.0), _np(w)
    more = (0.0 if dtype == BF16 else 2.0 ** -20)
    for name, want, tol in (("dhidden", dz @ wn.T, off @ np.abs(wn.T) + (V * 2.0 ** -24 + more) * (size @ np.abs(wn.T))),
                            ("dweight", h.T @ dz, np.abs(h.T) @ off + (rows * 2.0 ** -24 + more) * (np.abs(h.T) @ size)
                             + 2.0 ** -36 * np.abs(h).max() * size.max() * rows)):
        got = _np(out[name])
        assert np.all(np.isfinite(got)), (name, "not finite")
        tol = tol + 2 * step * (np.abs(want) + tol)
        assert np.all(np.abs(got - want) <= tol), (name, float((np.abs(got - want) / np.maximum(tol, 1e-300)).max()))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_logits_that_cancel(dtype):
    """One column whose logit is a small difference of terms of 2^22: p is 1 up to the error of the logit, 2^-20 of the terms' sizes, and the gradient
    of the only token nothing, up to all of g times what p may be less than 1."""
    import paper_2605_16154_amd as pcm
    rows, d = 300, 64
    gen = torch.Generator().manual_seed(3)
    w = torch.randn((d, 1), generator=gen).to(dtype)
    hidden = (torch.randn((rows, d), generator=gen) * 2.0 ** 20).to(dtype).cuda()
    w, tokens = w.cuda(), torch.zeros(rows, dtype=torch.int64, device="cuda")
    forward = pcm.pcm_linear_logprobs(hidden, w, tokens)
    g = torch.ones(rows, device="cuda")
    # the lse of a call that rounds its products otherwise: within the logit's error
    lse = (hidden.double() @ w.double())[:, 0]
    for x in (forward["lse"], lse.float()):
        out = pcm.pcm_linear_logprobs_backward(hidden, w, tokens, x, g)
        for k in out:
            assert bool(torch.isfinite(out[k].float()).all()), k
        assert float((out["dhidden"].double().abs() / (w.double().abs()[:, 0] + 1e-30)).max()) <= 1.0 + 2.0 ** -7
