"""The operators on logits at the ends of what they accept, on the CPU: temperatures, and the plain 64-bit form on logits of any size."""
import ctypes as C
import os

import numpy as np
import pytest

from oracle import operators as P
from paper_2605_16154_amd import build

OK, EINVAL = 0, -1


@pytest.fixture(scope="module")
def cdll():
    if not os.path.exists(build.LIB):
        build.build_library()
    lib = C.CDLL(build.LIB)
    vp, i32, i64, f32, sz = C.c_void_p, C.c_int, C.c_int64, C.c_float, C.c_size_t
    lib.pcm_token_logprobs.argtypes = [vp, i64, i32, vp, i32, vp, i64, i64, i32, f32, i32, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.pcm_token_logprobs_backward.argtypes = [vp, i64, i32, vp, i32, vp, i64, i64, i32, f32, vp, vp, vp, vp, vp, i64, vp]
    return lib


@pytest.mark.parametrize("temperature,rc", ((2.0 ** -126, OK), (2.0 ** -127, EINVAL), (3.4e38, OK), (1.0, OK)))
def test_temperatures(cdll, temperature, rc):
    """No rows, so a call that is not refused does nothing."""
    assert cdll.pcm_token_logprobs(None, 9, 0, None, 1, None, 0, 0, 9, temperature, 0, *[None] * 6, 0, None) == rc
    assert cdll.pcm_token_logprobs_backward(None, 9, 0, None, 1, None, 0, 0, 9, temperature, *[None] * 5, 9, None) == rc


@pytest.mark.parametrize("size", (1e9, 1e20, 1e38, -1e9, -1e38))
def test_plain_form_on_large_logits(size):
    """Equal logits are equally likely whatever their size; one that stands alone is certain."""
    z = np.full((2, 6), size)
    z[1, 4] = 3.0 * abs(size)
    got = P.token_logprobs(z, [2, 4], temperature=0.5, top=2)
    np.testing.assert_allclose(got["logp"], [-np.log(6), 0.0], rtol=0, atol=1e-14)
    np.testing.assert_allclose(got["entropy"], [np.log(6), 0.0], rtol=0, atol=1e-14)
    np.testing.assert_allclose(got["lse"], [2.0 * size, 6.0 * abs(size)], rtol=1e-8)
    g = P.token_logprobs_gradient(z, [2, 4], np.ones(2), np.ones(2), temperature=0.5)
    np.testing.assert_allclose(g[0], 2.0 * ((np.arange(6) == 2) - 1 / 6), rtol=0, atol=1e-13)
    assert (g[1] == 0).all()
