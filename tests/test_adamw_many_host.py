"""The optimizer step over many tensors, without a GPU: sizes, plans, refusals, and the plain form of moments in 8 bits."""
import ctypes as C
import os

import numpy as np
import pytest

from oracle import operators as P
from oracle import pcm_oracle as O

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2605_16154_amd", "libpcm.so")
OK, EINVAL, EWORKSPACE = 0, -1, -2
vp, i32, i64, u64, f64, sz = C.c_void_p, C.c_int, C.c_int64, C.c_uint64, C.c_double, C.c_size_t
A = 1 << 30                                  # an address that is only looked at
CHUNK = 2048                                 # elements of a chunk of a plan


class Layout(C.Structure):
    _fields_ = [("chunks", i64), ("elements", i64), ("plan_bytes", sz), ("state_bytes", sz), ("state_bits", i32)]


@pytest.fixture(scope="module")
def cdll():
    if not os.path.exists(LIB):
        import __graft_entry__
        __graft_entry__.build()
    lib = C.CDLL(LIB)
    lib.pcm_adamw_many_describe.argtypes = [i32, vp, i32, vp]
    lib.pcm_adamw_many_plan.argtypes = [i32, vp, vp, vp, vp, vp, vp, sz]
    lib.pcm_adamw_many_step.argtypes = [vp, vp, vp, i64, f64, f64, f64, f64, f64, f64, u64, vp, vp, sz, vp]
    lib.pcm_adamw_many_states.argtypes = [vp, vp, i32, vp, vp, vp]
    lib.pcm_adamw_many_step_workspace_bytes.argtypes = [vp]
    lib.pcm_adamw_many_step_workspace_bytes.restype = sz
    return lib


def _describe(cdll, numel, bits=32):
    out = Layout()
    rc = cdll.pcm_adamw_many_describe(len(numel), (i64 * len(numel))(*numel), bits, C.byref(out))
    return rc, out


def _plan(cdll, numel, grads, dtypes, weights, lowp=None, short=0):
    n = len(numel)
    rc, layout = _describe(cdll, numel)
    assert rc == OK
    table = (C.c_char * max(1, layout.plan_bytes))()
    ptrs = lambda xs: (vp * n)(*xs)
    rc = cdll.pcm_adamw_many_plan(n, (i64 * n)(*numel), ptrs(grads), (i32 * n)(*dtypes), ptrs(weights), ptrs(lowp) if lowp else None,
                                  C.addressof(table), layout.plan_bytes - short)
    return rc, bytes(table), layout


@pytest.mark.parametrize("numel", [[1], [128], [129, 0, 7], [4096, 4097], [3, 10007, 1]])
def test_layout(cdll, numel):
    blocks = sum(-(-n // 128) for n in numel)
    for bits, per_block in ((32, 128 * 8), (8, 128 * 2 + 2)):
        rc, layout = _describe(cdll, numel, bits)
        assert (rc, layout.elements, layout.state_bytes, layout.state_bits) == (OK, 128 * blocks, per_block * blocks, bits)
        assert layout.chunks == sum(-(-n // CHUNK) for n in numel) and layout.plan_bytes == 40 * layout.chunks
        assert cdll.pcm_adamw_many_step_workspace_bytes(C.byref(layout)) == 8192


def test_plan_holds_every_element_once(cdll):
    numel, dtypes = [5, 0, 9000, 4096, 130], [0, 1, 1, 0, 1]
    grads, weights = [A + (i << 22) + 2 * d for i, d in enumerate(dtypes)], [2 * A + (i << 22) + 4 for i in range(5)]
    lowp = [3 * A, None, 3 * A + (1 << 22) + 2, None, None]
    rc, table, layout = _plan(cdll, numel, grads, dtypes, weights, lowp)
    assert rc == OK
    chunks = np.frombuffer(table, dtype=np.dtype([("g", "u8"), ("w", "u8"), ("b", "u8"), ("at", "i8"), ("count", "i4"), ("half", "i4")]))
    assert len(chunks) == layout.chunks
    at, k = 0, 0
    for n, d, g, w, b in zip(numel, dtypes, grads, weights, lowp):
        for first in range(0, n, CHUNK):
            c = chunks[k]
            assert (c["g"], c["w"], c["b"]) == (g + first * (2 if d else 4), w + first * 4, b + first * 2 if b else 0)
            assert (c["at"], c["count"], c["half"]) == (at + first, min(CHUNK, n - first), d)
            k += 1
        at += -(-n // 128) * 128
    assert at == layout.elements


def test_plan_refuses(cdll):
    two = ([100, 200], [A, 2 * A], [0, 1], [3 * A, 4 * A], [5 * A, 6 * A])
    assert _plan(cdll, *two)[0] == OK
    assert _plan(cdll, *two, short=1)[0] == EWORKSPACE
    for where, what in ((1, [None, 2 * A]), (1, [A + 2, 2 * A]), (1, [A, 2 * A + 1]), (2, [0, 2]), (2, [-1, 1]), (3, [3 * A, None]),
                        (3, [3 * A + 2, 4 * A]), (4, [5 * A + 1, None]),
                        (3, [3 * A, 3 * A]), (3, [3 * A, 3 * A + 396]), (3, [A, 4 * A]), (3, [3 * A, A - 796]), (4, [5 * A, 5 * A]),
                        (4, [3 * A, 6 * A]), (4, [2 * A + 398, None])):
        args = list(two)
        args[where] = what
        assert _plan(cdll, *args)[0] == EINVAL, (where, what)
    # neighbours without a gap, gradients that are shared, and tensors of no elements are fine
    assert _plan(cdll, [100, 200], [A, A], [0, 0], [3 * A, 3 * A + 400])[0] == OK
    assert _plan(cdll, [100, 0], [A, None], [0, 0], [3 * A, None])[0] == OK
    many = 300
    order = np.random.default_rng(0).permutation(many)
    assert _plan(cdll, [64] * many, [A + 256 * int(i) for i in order], [0] * many, [2 * A + 256 * int(i) for i in order])[0] == OK
    assert _plan(cdll, [64] * many, [A + 256 * int(i) for i in order], [0] * many, [2 * A + 252 * int(i) for i in order])[0] == EINVAL


def test_describe_refuses(cdll):
    out = Layout()
    assert _describe(cdll, [-1])[0] == EINVAL and _describe(cdll, [1 << 43])[0] == EINVAL and _describe(cdll, [5], 16)[0] == EINVAL
    assert cdll.pcm_adamw_many_describe(0, (i64 * 1)(5), 32, C.byref(out)) == EINVAL
    assert cdll.pcm_adamw_many_describe(1, None, 32, C.byref(out)) == EINVAL
    assert cdll.pcm_adamw_many_describe(1, (i64 * 1)(5), 32, None) == EINVAL


def test_step_refuses(cdll):
    _, layout = _describe(cdll, [1000], 8)
    base = dict(plan=A, layout=C.addressof(layout), state=A, step=1, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, wd=0.0, clip=1.0, seed=0,
                norm=None, ws=A, ws_bytes=8192, stream=None)
    for change in (dict(plan=None), dict(plan=A + 4), dict(layout=None), dict(state=None), dict(state=A + 8), dict(step=0), dict(lr=-1.0),
                   dict(beta1=1.0), dict(beta2=-0.1), dict(eps=0.0), dict(wd=-1.0), dict(clip=0.0), dict(clip=float("nan")), dict(norm=A + 2)):
        assert cdll.pcm_adamw_many_step(*{**base, **change}.values()) == EINVAL, change
    for change in (dict(ws=None), dict(ws=A + 8), dict(ws_bytes=8191), dict(ws=None, clip=float("inf"), norm=A)):
        assert cdll.pcm_adamw_many_step(*{**base, **change}.values()) == EWORKSPACE, change
    bad = Layout(layout.chunks + 100, layout.elements, layout.plan_bytes, layout.state_bytes, 8)
    assert cdll.pcm_adamw_many_step(*{**base, "layout": C.addressof(bad)}.values()) == EINVAL
    bad = Layout(layout.chunks, layout.elements + 1, layout.plan_bytes, layout.state_bytes, 8)
    assert cdll.pcm_adamw_many_step(*{**base, "layout": C.addressof(bad)}.values()) == EINVAL
    bad = Layout(layout.chunks, layout.elements, layout.plan_bytes, layout.state_bytes, 16)
    assert cdll.pcm_adamw_many_step(*{**base, "layout": C.addressof(bad)}.values()) == EINVAL
    _, none = _describe(cdll, [0], 8)
    assert cdll.pcm_adamw_many_step(*{**base, "layout": C.addressof(none), "plan": None, "state": None}.values()) == OK


def test_states_refuses(cdll):
    _, layout = _describe(cdll, [1000], 8)
    _, wide = _describe(cdll, [1000], 32)
    at = C.addressof(layout)
    for args in ((None, A, 1, A, A), (C.addressof(wide), A, 1, A, A), (at, None, 1, A, A), (at, A, 2, A, A), (at, A, 1, None, A), (at, A, 1, A, None),
                 (at, A + 8, 1, A, A), (at, A, 1, A + 1, A), (at, A, 0, A, A + 2)):
        assert cdll.pcm_adamw_many_states(*args, None) == EINVAL, args


# ---- the plain form of moments in 8 bits ------------------------------------------------------------

def test_random_bits_are_those_of_the_published_generator(golden_dir):
    step, seed = (3 << 32) + 41, (7 << 32) + 5
    got = P._philox_groups([9, (2 << 32) + 1], step, seed)
    for g, row in zip((9, (2 << 32) + 1), got):
        words = O.philox4x32_10((g & 0xFFFFFFFF, g >> 32, 41, 3), (5, 7))
        assert [int(x) for x in row] == [h for w in words for h in (w & 0xFFFF, w >> 16)]


@pytest.mark.parametrize("field,signed", [(P.M_FIELD, True), (P.V_FIELD, False)])
def test_codes_stand_for_themselves_and_round_to_a_neighbour(field, signed):
    every = np.arange(256)
    if signed:
        every[128] = 0                                    # a zero has no sign
    codes, tops = np.concatenate([every, every[::-1]]), np.full(4, 120)
    codes[[0, 200, 300, 500]] = 127 if signed else 255    # every block reaches its exponent
    values = P.moment_values(codes, tops, field)
    for random in (0, 1, 40000, 65535):
        back, back_tops = P.moment_codes(values, np.full(512, random), field)
        assert np.array_equal(back, codes) and np.array_equal(back_tops, tops)
    rng = np.random.default_rng(1)
    x = (rng.standard_normal(1280) * np.exp(3 * rng.standard_normal(1280))).astype(np.float32)
    x = x if signed else np.abs(x)
    low = P.moment_values(*P.moment_codes(x, np.zeros(1280, int), field), field)
    high = P.moment_values(*P.moment_codes(x, np.full(1280, 65535), field), field)
    assert np.all(np.abs(low) <= np.abs(x) * (1 if signed else 1 + 1e-9) + (0 if signed else np.abs(low).max() * 2.0 ** -30)) and np.all(np.abs(high) >= np.abs(x) * (1 - 2.0 ** -15))
    grid = np.abs(x) > np.abs(x).reshape(-1, 128).max(axis=1).repeat(128) * 2.0 ** (2 - field)
    assert np.all(np.abs(high - low)[grid] <= np.abs(x)[grid] / 8)


def test_rounding_is_right_on_average():
    x = np.float32([0.3, -1.7, 1e-3, 2.0 ** -20, -0.9, 3.3] + [0.0] * 122)
    total = np.zeros(128)
    turns = 256                                           # the random numbers i / 256 + 1 / 512
    for i in range(turns):
        total += P.moment_values(*P.moment_codes(x, np.full(128, 256 * i + 128), P.M_FIELD), P.M_FIELD)
    spacing = np.maximum(np.abs(x) / 8, 2.0 ** (1 - 17))
    assert np.all(np.abs(total / turns - x) <= spacing / turns)


def test_step_follows_the_moments_in_64_bits():
    """The plain step on moments of 8 bits is AdamW's but for the rounding of the moments, which its own codes undo."""
    rng = np.random.default_rng(2)
    w, g = [rng.standard_normal(200), rng.standard_normal(5)], [rng.standard_normal(200).astype(np.float32), rng.standard_normal(5).astype(np.float32)]
    state = (np.zeros(384, np.uint8), np.zeros(384, np.uint8), np.zeros(3, np.uint8), np.zeros(3, np.uint8))
    hp = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1, max_grad_norm=2.0)
    new, state, norm = P.adamw_many_eight(w, g, state, 1, 3, **hp)
    ref, m, v, ref_norm = O.adamw_step(w, g, [0 * x for x in w], [0 * x for x in w], 1, **hp)
    assert abs(norm - ref_norm) <= 1e-12 * norm
    for a, b in zip(new, ref):
        # m and v carry a factor, two products and a sum of 2^-24 each; their quotient is of order one
        np.testing.assert_allclose(a, b, atol=1e-2 * 8 * 2.0 ** -24, rtol=1e-12)
    got_m, got_v = P.moment_values(state[0], state[2], P.M_FIELD), P.moment_values(state[1], state[3], P.V_FIELD)
    for got, want in ((got_m, m), (got_v, v)):
        for part, x in ((got[:200], want[0]), (got[256:261], want[1])):
            top = np.abs(x).max()
            assert np.all(np.abs(part - x) <= np.abs(x) / 8 + top * 2.0 ** -16)
        assert not got[200:256].any() and not got[261:].any()
