"""The optimizer step over many tensors where the norm of the gradients is no number, is infinite, or is asked for without clipping."""
import pytest
import torch

pytestmark = pytest.mark.gpu

HP = dict(lr=1e-2, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01)
SIZES = (1000, 5000, 130)


def _plan(bits, half=False):
    import paper_2605_16154_amd as pcm
    gen = torch.Generator().manual_seed(1)
    grads = [(10 * torch.randn(n, generator=gen)).to(torch.bfloat16 if half and i == 1 else torch.float32).cuda() for i, n in enumerate(SIZES)]
    weights = [torch.randn(n, generator=gen).cuda() for n in SIZES]
    copies = [torch.zeros(n, dtype=torch.bfloat16, device="cuda") for n in SIZES]
    return pcm, pcm.pcm_adamw_many_plan(grads, weights, state_bits=bits, weights_bf16=copies), grads, weights, copies


def _moments(pcm, plan):
    return [torch.cat([x[at:at + n] for at, n in zip(plan.offsets, SIZES)]).float() for x in pcm.pcm_adamw_many_states(plan)]


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("bits", [32, 8])
def test_a_nan_among_the_gradients_reaches_every_weight(bits, half):
    """The clip factor is max / norm, so NaN: no gradient is taken at its full size because another one is no number."""
    pcm, plan, grads, weights, copies = _plan(bits, half)
    grads[1][4321] = float("nan")
    norm = pcm.pcm_adamw_many_step(plan, 1, max_grad_norm=1.0, **HP)
    assert bool(torch.isnan(norm).all())
    for x in (*weights, *copies, *_moments(pcm, plan)):
        assert bool(torch.isnan(x).all())


@pytest.mark.parametrize("bits", [32, 8])
def test_without_clipping_a_nan_stays_where_it_is(bits):
    pcm, plan, grads, weights, copies = _plan(bits)
    grads[1][4321] = float("nan")
    norm = torch.zeros(1, device="cuda")
    before = [w.clone() for w in weights]
    for out in (norm, None):
        pcm.pcm_adamw_many_step(plan, 1, max_grad_norm=None, grad_norm_out=out, **HP)
        w = torch.cat(weights)
        assert int(torch.isnan(w).sum()) == 1 + (127 if bits == 8 and out is None else 0)
        for x, y in zip(weights, before):
            assert not bool((x == y).any())
    assert bool(torch.isnan(norm).all())


@pytest.mark.parametrize("bits", [32, 8])
def test_an_infinite_gradient_makes_the_others_nothing(bits):
    """max / inf is 0: the finite gradients count as zeros, the infinite one is NaN (with it, in 8 bits, its block of moments)."""
    pcm, plan, grads, weights, copies = _plan(bits)
    grads[1][4321] = float("inf")
    before = torch.cat(weights)
    norm = pcm.pcm_adamw_many_step(plan, 1, max_grad_norm=1.0, **HP)
    assert bool(torch.isinf(norm).all())
    w = torch.cat(weights)
    at = SIZES[0] + 4321
    others = torch.arange(len(w), device="cuda") != at
    assert bool(torch.isnan(w[at]))
    # decay alone: the product's rounding and that of its factor
    want = before.double() * (1 - HP["lr"] * HP["weight_decay"])
    assert float(((w.double() - want).abs() / want.abs())[others].max()) <= 2.0 ** -23
    m, v = _moments(pcm, plan)
    gone = torch.isnan(m)
    assert bool(gone[at]) and int(gone.sum()) == (1 if bits == 32 else 128) and torch.equal(gone, torch.isnan(v))
    assert not m[~gone].any() and not v[~gone].any()


def test_a_norm_that_has_no_place_is_refused():
    pcm, plan, grads, weights, copies = _plan(32)
    before = torch.cat(weights)
    for clip in (None, 1.0):
        for out in (torch.empty(0, device="cuda"), torch.empty(1)):
            with pytest.raises(pcm.PcmError):
                pcm.pcm_adamw_many_step(plan, 1, max_grad_norm=clip, grad_norm_out=out, **HP)
    assert torch.equal(torch.cat(weights), before)
