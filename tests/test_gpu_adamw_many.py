"""GPU parity of the optimizer step over many tensors against its plain forms.

Tolerances.  32-bit moments: as for the step over few tensors (tests/test_gpu_optimizer.py): v relative 2e-6, m relative to its terms 2e-6, a weight
three of its own roundings and 1e-5 of the step.  8-bit moments: their codes are defined bit by bit, so they are the plain form's; the plain form
takes fp32 moments as they are rounded, so a weight is off by its own last rounding (with the decay's product and the sum: three of 2^-24) and
the step's few fp32 operations (a root, a division and four products: 1e-6 of the step)."""
import numpy as np
import pytest
import torch

from oracle import operators as P
from oracle import pcm_oracle as O

pytestmark = pytest.mark.gpu

HP = dict(lr=1e-2, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, max_grad_norm=2.0)
SHAPES = [(1,), (7,), (128,), (40, 100), (4096,), (4097,), (3, 5, 11), (0,), (10007,), (129,), (64, 192)]


def _tensors(seed, shapes, dtypes, offset=0, scale=0.1):
    """Tensors of all shapes in one buffer, one right behind the other from element `offset` on, and what lies around them."""
    rng = np.random.default_rng(seed)
    total = offset + sum(int(np.prod(s)) for s in shapes) + 8
    flat = {t: torch.from_numpy((scale * rng.standard_normal(total)).astype(np.float32)).cuda().to(t) for t in set(dtypes)}
    out, at = [], offset
    for s, t in zip(shapes, dtypes):
        n = int(np.prod(s))
        out.append(flat[t][at:at + n].view(s))
        at += n
    return out, flat


def _host(ts):
    return [t.detach().float().cpu().numpy().reshape(-1) for t in ts]


def _case(seed, bits, shapes=SHAPES, offset=0, half=True, lowp=True, gscale=0.1):
    import paper_2605_16154_amd as pcm
    dtypes = [torch.bfloat16 if half and i % 2 else torch.float32 for i in range(len(shapes))]
    grads, _ = _tensors(seed, shapes, dtypes, offset, gscale)
    weights, w_flat = _tensors(seed + 1, shapes, [torch.float32] * len(shapes), offset)
    copies, b_flat = _tensors(seed + 2, shapes, [torch.bfloat16] * len(shapes), offset)
    copies = [c if i % 3 else None for i, c in enumerate(copies)] if lowp else None
    plan = pcm.pcm_adamw_many_plan(grads, weights, state_bits=bits, weights_bf16=copies)
    return pcm, plan, grads, weights, copies, w_flat[torch.float32], b_flat[torch.bfloat16]


def _parts(plan, flat):
    x = flat.detach().double().cpu().numpy()
    return [x[at:at + w.numel()] for at, w in zip(plan.offsets, plan.weights)]


def _padding(plan, flat):
    keep = torch.ones(flat.numel(), dtype=torch.bool)
    for at, w in zip(plan.offsets, plan.weights):
        keep[at:at + w.numel()] = False
    return flat.cpu()[keep]


def _check_copies(weights, copies):
    for w, c in zip(weights, copies or []):
        if c is not None:
            assert torch.equal(c, w.to(torch.bfloat16))


@pytest.mark.parametrize("offset", [0, 1, 2, 3, 7])
@pytest.mark.parametrize("clip", [2.0, None])
def test_states_in_32_bits(offset, clip):
    pcm, plan, grads, weights, copies, w_flat, b_flat = _case(3 + offset, 32, offset=offset)
    around = w_flat[:offset].clone(), w_flat[-8:].clone()
    w, m, v = _host(weights), [np.zeros(t.numel()) for t in weights], [np.zeros(t.numel()) for t in weights]
    for step in (1, 2, 3):
        g = _host(grads)
        norm = pcm.pcm_adamw_many_step(plan, step, **{**HP, "max_grad_norm": clip})
        w0, m0 = w, m
        w, m, v, ref_norm = O.adamw_step(w, g, m, v, step, **{**HP, "max_grad_norm": clip or 1e30})
        if clip:
            assert abs(float(norm) - ref_norm) <= 2e-7 * ref_norm
        else:
            assert norm is None
        scale = min(1.0, (clip or 1e30) / (ref_norm + 1e-6))
        got_m, got_v = (_parts(plan, x) for x in pcm.pcm_adamw_many_states(plan))
        for i, got in enumerate(_host(weights)):
            terms = HP["beta1"] * np.abs(m0[i]) + (1 - HP["beta1"]) * np.abs(g[i].astype(np.float64)) * scale
            assert np.all(np.abs(got_m[i] - m[i]) <= 2e-6 * step * terms + 1e-30)
            np.testing.assert_allclose(got_v[i], v[i], rtol=2e-6 * step, atol=1e-35)
            size = HP["lr"] / (1 - HP["beta1"] ** step) * terms / (np.sqrt(v[i] / (1 - HP["beta2"] ** step)) + HP["eps"])
            assert np.all(np.abs(got - w[i]) <= step * (3 * np.spacing(np.abs(w0[i]).astype(np.float32)).astype(np.float64) + 1e-5 * size))
        w, m, v = [x.astype(np.float64) for x in _host(weights)], got_m, got_v
        _check_copies(weights, copies)
    assert torch.equal(w_flat[:offset], around[0]) and torch.equal(w_flat[-8:], around[1])
    for x in pcm.pcm_adamw_many_states(plan):
        assert not _padding(plan, x).any()


def _eight(plan):
    E = plan.layout.elements
    x = plan.state.cpu().numpy()
    return x[:E], x[E:2 * E], x[2 * E:2 * E + E // 128], x[2 * E + E // 128:]


@pytest.mark.parametrize("offset,clip,gscale", [(0, 2.0, 0.1), (1, None, 0.1), (5, 0.5, 30.0), (2, 2.0, 1e-12), (0, None, 1e-17)])
def test_states_in_8_bits(offset, clip, gscale):
    hp = {**HP, "max_grad_norm": clip}
    pcm, plan, grads, weights, copies, w_flat, b_flat = _case(20 + offset, 8, offset=offset, gscale=gscale)
    seed = (5 << 32) + 11 + offset
    for step in (1, 2, 3, 4):
        before, w, g = tuple(x.copy() for x in _eight(plan)), _host(weights), _host(grads)
        norm = pcm.pcm_adamw_many_step(plan, step, seed=seed, **hp)
        ref_w, ref_state, ref_norm = P.adamw_many_eight(w, g, before, step, seed, **hp)
        if clip:
            assert abs(float(norm) - ref_norm) <= 2e-7 * ref_norm
        for name, got, want in zip(("m", "v", "exponents of m", "exponents of v"), _eight(plan), ref_state):
            assert np.array_equal(got, want), (step, name, np.flatnonzero(got != want)[:5])
        for got, want, old in zip(_host(weights), ref_w, w):
            size = np.abs(want - old.astype(np.float64) * (1 - hp["lr"] * hp["weight_decay"]))
            assert np.all(np.abs(got - want) <= 3 * 2.0 ** -24 * (np.abs(old) + np.abs(want)) + 1e-6 * size)
        _check_copies(weights, copies)
        for g_t in grads:                                  # another gradient
            g_t.mul_(-0.7)
    m, v = pcm.pcm_adamw_many_states(plan)
    assert m.dtype == torch.bfloat16
    state = _eight(plan)
    for got, codes, tops, field in ((m, state[0], state[2], P.M_FIELD), (v, state[1], state[3], P.V_FIELD)):
        want = P.moment_values(codes, tops, field)
        want = np.where(np.abs(want) < 2.0 ** -126, np.float32(want), want)
        big = np.abs(want) >= 2.0 ** -126
        assert np.array_equal(got.double().cpu().numpy()[big], want[big])
    m32, v32 = pcm.pcm_adamw_many_states(plan, dtype=torch.float32)
    assert torch.equal(m32.to(torch.bfloat16), m) and torch.equal(v32.to(torch.bfloat16), v)
    assert not _padding(plan, m).any() and not _padding(plan, v).any()


def test_8_bits_hold_blocks_that_leave_the_range():
    """A block with an infinity or a NaN is NaN, its neighbours are not; a block of zeros stays zero."""
    import paper_2605_16154_amd as pcm
    g = torch.randn(1024, device="cuda")
    g[130], g[300], g[512:640] = float("inf"), float("nan"), 0.0
    w = torch.zeros(1024, device="cuda")
    plan = pcm.pcm_adamw_many_plan([g], [w], state_bits=8)
    pcm.pcm_adamw_many_step(plan, 1, max_grad_norm=None)
    for x in pcm.pcm_adamw_many_states(plan):
        nan = torch.isnan(x).view(8, 128)
        assert nan[1].all() and nan[2].all() and not nan[[0, 3, 4, 5, 6, 7]].any()
        assert not x[512:640].any()
    finite = torch.isfinite(w)
    assert int((~finite).sum()) == 2 and not finite[130] and not finite[300]
    assert not w[512:640].any()


def test_8_bit_moments_follow_32_bit_ones():
    """Over 400 steps of noisy gradients of a fixed mean the 8-bit second moment stays around the 32-bit one: rounding to nearest would leave it
    where the first steps put it.  Its mean over 20,000 elements: each step adds an error without bias of at most the spacing (an eighth), which
    decays with 1 - beta2 = 0.01: a deviation of at most 0.125 / 2 / sqrt(2 * 0.01) = 0.45 per element, 0.0032 of the mean, of which five are
    allowed."""
    import paper_2605_16154_amd as pcm
    gen = torch.Generator(device="cuda").manual_seed(4)
    n = 20000
    g = torch.empty(n, device="cuda")
    w = [torch.zeros(n, device="cuda") for _ in range(2)]
    plans = [pcm.pcm_adamw_many_plan([g], [x], state_bits=b) for x, b in zip(w, (32, 8))]
    for step in range(1, 401):
        g.copy_((3.0 if step < 100 else 1.0) * torch.randn(n, generator=gen, device="cuda"))
        for plan in plans:
            pcm.pcm_adamw_many_step(plan, step, lr=1e-3, beta2=0.99, max_grad_norm=None, seed=9)
    v32, v8 = (pcm.pcm_adamw_many_states(p)[1].double()[:n] for p in plans)
    assert abs(float(v8.mean() / v32.mean()) - 1) <= 5 * 0.0032
    assert float(v32.mean()) < 2.0                          # the large gradients of the beginning are forgotten


def test_same_bits_again_and_many_small_tensors():
    import paper_2605_16154_amd as pcm
    shapes = [(1 + 37 * i % 301,) for i in range(400)]
    states = []
    for _ in range(2):
        pcm_, plan, grads, weights, copies, w_flat, _b = _case(50, 8, shapes)
        pcm.pcm_adamw_many_step(plan, 1, seed=1, **HP)
        pcm.pcm_adamw_many_step(plan, 2, seed=1, **HP)
        states.append((plan.state.clone(), w_flat.clone()))
    assert torch.equal(states[0][0], states[1][0]) and torch.equal(states[0][1], states[1][1])


@pytest.mark.parametrize("bits", [32, 8])
def test_more_than_a_launch_holds_at_once(bits):
    """More chunks than workgroups, and enough elements for the accesses that stream past the cache: the same bits as the same tensor's parts on
    their own plans."""
    import paper_2605_16154_amd as pcm
    n = (20 << 20) + 128 * 40 + 64
    gen = torch.Generator(device="cuda").manual_seed(1)
    g = torch.randn(n, generator=gen, device="cuda")
    w = torch.randn(n, generator=gen, device="cuda")
    whole = pcm.pcm_adamw_many_plan([g], [w.clone()], state_bits=bits)
    pcm.pcm_adamw_many_step(whole, 1, lr=1e-3, max_grad_norm=None, seed=2)
    cut = 4096 * 1000
    parts = pcm.pcm_adamw_many_plan([g[:cut]], [w.clone()[:cut]], state_bits=bits)
    pcm.pcm_adamw_many_step(parts, 1, lr=1e-3, max_grad_norm=None, seed=2)
    assert torch.equal(whole.weights[0][:cut], parts.weights[0])
    for a, b in zip(pcm.pcm_adamw_many_states(whole), pcm.pcm_adamw_many_states(parts)):
        assert torch.equal(a[:cut], b)
    # the last elements, against the definition
    tail = slice(n - 200, n)
    m = np.float32(0.1) * g[tail].cpu().numpy()
    if bits == 32:
        got = pcm.pcm_adamw_many_states(whole)[0][tail].cpu().numpy()
        np.testing.assert_allclose(got, m, rtol=1e-6)
    norm = pcm.pcm_adamw_many_step(whole, 2, lr=1e-3, max_grad_norm=1.0, seed=2)
    ref = float(g.double().square().sum().sqrt())
    assert abs(float(norm) - ref) <= 2.0 ** -23 * ref


def test_replayed_graph_and_another_stream():
    import paper_2605_16154_amd as pcm
    make = lambda: _case(70, 8, SHAPES)
    _, eager, g_e, *_ = make()
    _, captured, g_c, *_ = make()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    norm = torch.zeros(1, device="cuda")
    with torch.cuda.stream(stream):
        pcm.pcm_adamw_many_step(captured, 1, seed=3, grad_norm_out=norm, **HP)       # scratch for the capture
        pcm.pcm_adamw_many_step(eager, 1, seed=3, **HP)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        pcm.pcm_adamw_many_step(captured, 2, seed=3, grad_norm_out=norm, **HP)
    for turn in range(3):
        for a, b in zip(g_e, g_c):
            a.mul_(1.0 + 0.5 * turn)
            b.copy_(a)
        graph.replay()
        ref = pcm.pcm_adamw_many_step(eager, 2, seed=3, **HP)
        torch.cuda.synchronize()
        assert torch.equal(ref, norm) and torch.equal(eager.state, captured.state), turn
        for a, b in zip(eager.weights, captured.weights):
            assert torch.equal(a, b)


def test_a_copied_state_goes_on_where_it_was():
    import paper_2605_16154_amd as pcm
    _, a, _, weights, *_ = _case(80, 8)
    pcm.pcm_adamw_many_step(a, 1, **HP)
    others = [w.clone() for w in weights]
    b = pcm.pcm_adamw_many_plan(a.grads, others, state_bits=8, state=a.state.clone())
    for plan in (a, b):
        pcm.pcm_adamw_many_step(plan, 2, **HP)
    assert torch.equal(a.state, b.state) and all(torch.equal(x, y) for x, y in zip(weights, others))


def test_binding_refuses():
    import paper_2605_16154_amd as pcm
    g, w = torch.zeros(8, device="cuda"), torch.zeros(8, device="cuda")
    for args in (([], []), ([g], []), ([g], [w[:4]]), ([g.half()], [w]), ([g], [w.double()]), ([g.cpu()], [w]), ([g, g], [w, w]), ([w], [w]),
                 ([torch.zeros(4, 8, device="cuda").t()], [torch.zeros(8, 4, device="cuda")])):
        with pytest.raises(pcm.PcmError):
            pcm.pcm_adamw_many_plan(*args)
    with pytest.raises(pcm.PcmError):
        pcm.pcm_adamw_many_plan([g], [w], state_bits=16)
    with pytest.raises(pcm.PcmError):
        pcm.pcm_adamw_many_plan([g], [w], state=torch.zeros(8, dtype=torch.uint8, device="cuda"))
    with pytest.raises(pcm.PcmError):
        pcm.pcm_adamw_many_plan([g], [w], weights_bf16=[torch.zeros(4, dtype=torch.bfloat16, device="cuda")])
    plan = pcm.pcm_adamw_many_plan([g], [w], state_bits=8)
    for bad in (dict(step=0), dict(step=1, eps=0.0), dict(step=1, max_grad_norm=-1.0), dict(step=1, grad_norm_out=torch.zeros(1))):
        with pytest.raises(pcm.PcmError):
            pcm.pcm_adamw_many_step(plan, **bad)
    with pytest.raises(pcm.PcmError):
        pcm.pcm_adamw_many_states(plan, dtype=torch.float16)
