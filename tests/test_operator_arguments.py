"""Host-side checks and workspace queries of the operators on logits and updates: no GPU work is issued."""
import ctypes as C
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2605_16154_amd", "libpcm.so")
OK, EINVAL, EWORKSPACE, EUNSUPPORTED = 0, -1, -2, -4
P = 1 << 20                                  # an address that is only looked at
vp, i32, i64, f32, f64, sz = C.c_void_p, C.c_int, C.c_int64, C.c_float, C.c_double, C.c_size_t


@pytest.fixture(scope="module")
def cdll():
    if not os.path.exists(LIB):
        import __graft_entry__
        __graft_entry__.build()
    lib = C.CDLL(LIB)
    lib.pcm_token_logprobs.argtypes = [vp, i64, i32, vp, i32, vp, i64, i64, i32, f32, i32, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.pcm_token_logprobs_backward.argtypes = [vp, i64, i32, vp, i32, vp, i64, i64, i32, f32, vp, vp, vp, vp, vp, i64, vp]
    lib.pcm_orthogonalise.argtypes = [vp, i64, i64, vp, i64, i64, i32, i32, i32, i32, i32, vp, sz, vp]
    lib.pcm_muon_step.argtypes = [i32] + [vp] * 6 + [f64, f64, i32, f64, i32, i32, vp, sz, vp]
    lib.pcm_token_logprobs_workspace_bytes.argtypes = [i64, i32, i32]
    lib.pcm_orthogonalise_workspace_bytes.argtypes = [i32] * 3
    lib.pcm_muon_step_workspace_bytes.argtypes = [i32, vp, vp]
    for f in (lib.pcm_token_logprobs_workspace_bytes, lib.pcm_orthogonalise_workspace_bytes, lib.pcm_muon_step_workspace_bytes):
        f.restype = sz
    return lib


FORWARD = dict(logits=P, ld=100, dtype=0, tokens=P, token_type=1, allowed=None, allowed_ld=0, rows=4, V=100, temperature=1.0, top=0,
               logp=P, lse=P, entropy=P, top_ids=None, top_logp=None, ws=None, ws_bytes=0, stream=None)
BACKWARD = dict(logits=P, ld=100, dtype=1, tokens=P, token_type=2, allowed=None, allowed_ld=0, rows=4, V=100, temperature=1.0, lse=P,
                dlogp=P, entropy=P, dentropy=P, dlogits=P, dlogits_ld=100, stream=None)
BOTH = [dict(logits=None), dict(tokens=None), dict(lse=None), dict(ld=99), dict(dtype=2), dict(dtype=-1), dict(token_type=3), dict(token_type=-1),
        dict(rows=-1), dict(V=0), dict(V=-5), dict(temperature=0.0), dict(temperature=float("nan")), dict(temperature=float("inf")),
        dict(temperature=-2.0), dict(temperature=1e-44), dict(allowed=P, allowed_ld=99), dict(allowed=P, allowed_ld=-1), dict(logits=P + 1),
        dict(tokens=P + 2), dict(lse=P + 2), dict(entropy=P + 1)]


@pytest.mark.parametrize("change", BOTH + [dict(top=-1), dict(top=65), dict(top=1), dict(top=1, top_ids=P), dict(top=1, top_ids=P + 2, top_logp=P),
                                           dict(logp=None), dict(logp=P + 1)])
def test_forward_refuses(cdll, change):
    assert cdll.pcm_token_logprobs(*{**FORWARD, **change}.values()) == EINVAL


@pytest.mark.parametrize("change", BOTH + [dict(dlogp=None), dict(dlogits=None), dict(dlogits_ld=99), dict(entropy=None), dict(dentropy=None),
                                           dict(dlogits=P + 1), dict(dlogp=P + 1), dict(dentropy=P + 3)])
def test_backward_refuses(cdll, change):
    assert cdll.pcm_token_logprobs_backward(*{**BACKWARD, **change}.values()) == EINVAL


def test_no_rows_is_a_call_that_does_nothing(cdll):
    none = dict(rows=0, logits=None, tokens=None, lse=None, logp=None, entropy=None, dlogp=None, dentropy=None, dlogits=None)
    pick = lambda base: {**base, **{k: v for k, v in none.items() if k in base}}
    assert cdll.pcm_token_logprobs(*pick(FORWARD).values()) == OK
    assert cdll.pcm_token_logprobs_backward(*pick(BACKWARD).values()) == OK
    assert cdll.pcm_token_logprobs(*{**FORWARD, "rows": 1 << 31}.values()) == EUNSUPPORTED
    assert cdll.pcm_token_logprobs_backward(*{**BACKWARD, "rows": 1 << 31}.values()) == EUNSUPPORTED


ORTH = dict(update=P, ld=30, stride=600, out=P, out_ld=30, out_stride=600, batch=2, rows=20, cols=30, dtype=0, steps=5, ws=P,
            ws_bytes=1 << 40, stream=None)


@pytest.mark.parametrize("change", [dict(update=None), dict(out=None), dict(update=P + 2), dict(out=P + 1), dict(ld=29), dict(out_ld=29),
                                    dict(stride=-1), dict(out_stride=599), dict(batch=-1), dict(rows=0), dict(cols=0), dict(dtype=2),
                                    dict(steps=0), dict(steps=11)])
def test_orthogonalise_refuses(cdll, change):
    assert cdll.pcm_orthogonalise(*{**ORTH, **change}.values()) == EINVAL


def test_orthogonalise_workspace(cdll):
    assert cdll.pcm_orthogonalise(*{**ORTH, "ws": None}.values()) == EWORKSPACE
    assert cdll.pcm_orthogonalise(*{**ORTH, "ws": P + 128}.values()) == EWORKSPACE
    need = cdll.pcm_orthogonalise_workspace_bytes(2, 20, 30)
    assert need > 0 and cdll.pcm_orthogonalise(*{**ORTH, "ws_bytes": need - 1}.values()) == EWORKSPACE
    assert cdll.pcm_orthogonalise(*{**ORTH, "batch": 0, "update": None, "out": None}.values()) == OK
    q = cdll.pcm_orthogonalise_workspace_bytes
    assert q(0, 4, 4) == q(1, 0, 4) == q(1, 4, 0) == q(-1, 4, 4) == 0
    assert q(1, 1 << 15, 1 << 20) > 0 and q(1, 1 << 20, 1 << 15) > 0
    assert q(1, (1 << 15) + 1, 1 << 16) == q(1, 1, (1 << 20) + 1) == 0
    assert cdll.pcm_orthogonalise(*{**ORTH, "rows": 1 << 16, "cols": 1 << 16, "ld": 1 << 16, "out_ld": 1 << 16, "out_stride": 1 << 32}.values()) == EUNSUPPORTED
    assert q(100, 64, 64) == q(8, 64, 64)                        # more matrices than share a launch take no more
    assert q(1, 4096, 11008) < 6 * 4 * 4096 * 11008              # six matrices of pairs at most


def _muon(cdll, n=2, null=None, **change):
    arr = lambda v: (vp * 9)(*[v] * 9)
    a = dict(rows=(i32 * 9)(*[20] * 9), cols=(i32 * 9)(*[30] * 9), grads=arr(P), weights=arr(P), momentum=arr(P), lowp=None, lr=0.1, mu=0.9,
             nesterov=1, wd=0.0, steps=5, rule=0, ws=P, ws_bytes=1 << 40, stream=None)
    a.update(change)
    return cdll.pcm_muon_step(n, *a.values())


def test_muon_step_refuses(cdll):
    bad = lambda v: (vp * 9)(P, v)
    for change in (dict(n=0), dict(n=9), dict(grads=None), dict(weights=None), dict(momentum=None), dict(rows=None), dict(cols=None),
                   dict(grads=bad(None)), dict(weights=bad(None)), dict(momentum=bad(None)), dict(grads=bad(P + 2)), dict(weights=bad(P + 1)),
                   dict(momentum=bad(P + 3)), dict(lowp=bad(P + 1)), dict(rows=(i32 * 9)(20, 0)), dict(cols=(i32 * 9)(20, -1)), dict(lr=-0.1),
                   dict(lr=float("nan")), dict(mu=1.0), dict(mu=-0.1), dict(wd=-1.0), dict(steps=0), dict(steps=11), dict(rule=2), dict(rule=-1)):
        assert _muon(cdll, **change) == EINVAL, change
    assert _muon(cdll, ws=None) == EWORKSPACE
    assert _muon(cdll, rows=(i32 * 9)(*[1 << 16] * 9), cols=(i32 * 9)(*[1 << 16] * 9)) == EUNSUPPORTED
    q = cdll.pcm_muon_step_workspace_bytes
    rows, cols = (i32 * 2)(20, 300), (i32 * 2)(30, 10)
    need = q(2, rows, cols)
    assert need > 0 and q(0, rows, cols) == q(9, rows, cols) == q(2, None, cols) == 0
    assert _muon(cdll, rows=rows, cols=cols, ws_bytes=need - 1) == EWORKSPACE
