"""Host-side checks and workspace queries of the log-probabilities through a projection: no GPU work is issued."""
import ctypes as C
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2605_16154_amd", "libpcm.so")
OK, EINVAL, EWORKSPACE, EUNSUPPORTED = 0, -1, -2, -4
P = 1 << 20                                  # an address that is only looked at
vp, i32, i64, f32, sz = C.c_void_p, C.c_int, C.c_int64, C.c_float, C.c_size_t
HEAD = [vp, i64, vp, i64, i32, i32, vp, i32, i64, i32, i32, f32]


@pytest.fixture(scope="module")
def cdll():
    if not os.path.exists(LIB):
        import __graft_entry__
        __graft_entry__.build()
    lib = C.CDLL(LIB)
    lib.pcm_linear_logprobs.argtypes = HEAD + [vp, vp, vp, vp, sz, vp]
    lib.pcm_linear_logprobs_backward.argtypes = HEAD + [vp, vp, vp, vp, vp, i64, vp, i64, i32, i32, vp, sz, vp]
    for f in (lib.pcm_linear_logprobs_workspace_bytes, lib.pcm_linear_logprobs_backward_workspace_bytes):
        f.argtypes, f.restype = [i64, i32, i32, i32, i32, vp, i64], sz
    return lib


BASE = dict(hidden=P, hidden_ld=64, weight=P, weight_ld=200, layout=0, dtype=1, tokens=P, token_type=1, rows=40, d=64, V=200, temperature=1.0)
FORWARD = {**BASE, **dict(logp=P, lse=P, entropy=P, ws=P, ws_bytes=1 << 40, stream=None)}
BACKWARD = {**BASE, **dict(lse=P, dlogp=P, entropy=P, dentropy=P, dhidden=P, dhidden_ld=64, dweight=P, dweight_ld=200, dweight_dtype=1, accumulate=0, ws=P,
                           ws_bytes=1 << 40, stream=None)}
BOTH = [dict(hidden=None), dict(weight=None), dict(tokens=None), dict(lse=None), dict(hidden_ld=63), dict(weight_ld=199), dict(layout=2), dict(layout=-1),
        dict(layout=1, weight_ld=63), dict(dtype=2), dict(dtype=-1), dict(token_type=3), dict(token_type=-1), dict(rows=-1), dict(d=0), dict(V=0), dict(d=-3),
        dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=float("nan")), dict(temperature=float("inf")), dict(temperature=1e-44),
        dict(hidden=P + 1), dict(weight=P + 1), dict(tokens=P + 2), dict(dtype=0, hidden=P + 2), dict(dtype=0, weight=P + 2), dict(lse=P + 2),
        dict(entropy=P + 1)]


@pytest.mark.parametrize("change", BOTH + [dict(logp=None), dict(logp=P + 3)])
def test_forward_refuses(cdll, change):
    assert cdll.pcm_linear_logprobs(*{**FORWARD, **change}.values()) == EINVAL


@pytest.mark.parametrize("change", BOTH + [dict(dlogp=None), dict(dlogp=P + 1), dict(entropy=None), dict(dentropy=None), dict(dentropy=P + 2),
                                           dict(dhidden=None, dweight=None), dict(dhidden_ld=63), dict(dhidden=P + 1), dict(dweight_ld=199), dict(dweight=P + 1),
                                           dict(dweight_dtype=2), dict(dweight_dtype=0, dweight=P + 2), dict(accumulate=1), dict(dtype=0, dweight_dtype=1),
                                           dict(layout=1, weight_ld=64, dweight_ld=63)])
def test_backward_refuses(cdll, change):
    assert cdll.pcm_linear_logprobs_backward(*{**BACKWARD, **change}.values()) == EINVAL


def test_workspace(cdll):
    for query, call, base in ((cdll.pcm_linear_logprobs_workspace_bytes, cdll.pcm_linear_logprobs, FORWARD),
                              (cdll.pcm_linear_logprobs_backward_workspace_bytes, cdll.pcm_linear_logprobs_backward, BACKWARD)):
        for rows in (3, 40):
            need = query(rows, 64, 200, 1, 0, P, 200)
            assert need > 0 and need % 256 == 0
            for change in (dict(ws_bytes=need - 1), dict(ws=None), dict(ws=P + 16)):
                assert call(*{**base, "rows": rows, "ws_bytes": need, **change}.values()) == EWORKSPACE
        for bad in ((0, 64, 200, 1, 0, P, 200), (40, 0, 200, 1, 0, P, 200), (40, 64, 200, 1, 0, P, 199), (40, 64, 200, 3, 0, P, 200), (40, 64, 200, 1, 2, P, 200),
                    ((1 << 24) + 1, 64, 200, 1, 0, P, 200), (40, (1 << 16) + 1, 200, 1, 0, P, 200), (40, 64, (1 << 22) + 1, 1, 0, P, 1 << 23)):
            assert query(*bad) == 0, bad


def test_limits(cdll):
    for change in (dict(rows=(1 << 24) + 1), dict(d=(1 << 16) + 1, hidden_ld=1 << 17, dhidden_ld=1 << 17), dict(V=(1 << 22) + 1, weight_ld=1 << 23, dweight_ld=1 << 23)):
        pick = lambda base: {**base, **{k: v for k, v in change.items() if k in base}}
        assert cdll.pcm_linear_logprobs(*pick(FORWARD).values()) == EUNSUPPORTED
        assert cdll.pcm_linear_logprobs_backward(*pick(BACKWARD).values()) == EUNSUPPORTED


def test_no_rows(cdll):
    none = {**FORWARD, "rows": 0, "hidden": None, "tokens": None, "weight": None, "logp": None, "lse": None, "entropy": None, "ws": None, "ws_bytes": 0}
    assert cdll.pcm_linear_logprobs(*none.values()) == OK
    none = {**BACKWARD, "rows": 0, "hidden": None, "tokens": None, "weight": None, "lse": None, "dlogp": None, "entropy": None, "dentropy": None, "dweight": None,
            "ws": None, "ws_bytes": 0}
    assert cdll.pcm_linear_logprobs_backward(*none.values()) == OK


def test_no_rows_of_sizes_beyond_the_limits(cdll):
    for change in (dict(d=1 << 30, hidden_ld=1 << 30, dhidden_ld=1 << 30), dict(V=1 << 30, weight_ld=1 << 30, dweight_ld=1 << 30)):
        pick = lambda base: {**base, "rows": 0, **{k: v for k, v in change.items() if k in base}}
        assert cdll.pcm_linear_logprobs(*pick(FORWARD).values()) == EUNSUPPORTED
        assert cdll.pcm_linear_logprobs_backward(*pick({**BACKWARD, "dweight": None}).values()) == EUNSUPPORTED


def test_logits_are_never_kept(cdll):
    """The forward call takes 16 bytes per row and 128 columns beside its rows, a copy of at most 256 MB, the gradient one GB of dz besides."""
    rows, d, V = 4096, 4096, 131072
    forward = cdll.pcm_linear_logprobs_workspace_bytes(rows, d, V, 1, 0, P, V)
    assert forward <= rows * d * 2 + rows * V // 128 * 16 + (1 << 20)
    assert cdll.pcm_linear_logprobs_workspace_bytes(rows, d, V, 1, 0, P + 2, V) <= forward + (256 << 20) + 4096
    for big in (1 << 20, V):
        backward = cdll.pcm_linear_logprobs_backward_workspace_bytes(rows, d, big, 1, 0, P, big)
        assert backward <= rows * d * 2 + (1 << 30) + (256 << 20) + 3 * (1 << 26) + (1 << 20)
