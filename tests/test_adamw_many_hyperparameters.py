"""Hyper-parameters that the optimizer step over many tensors cannot hold in fp32 are refused: no GPU work is issued."""
import ctypes as C
import os

import pytest

from paper_2605_16154_amd.binding import AdamwManyLayout

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2605_16154_amd", "libpcm.so")
OK, EINVAL = 0, -1
GOOD = dict(step=1, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, max_grad_norm=float("inf"))


@pytest.fixture(scope="module")
def call():
    if not os.path.exists(LIB):
        import __graft_entry__
        __graft_entry__.build()
    lib = C.CDLL(LIB)
    lib.pcm_adamw_many_step.argtypes = [C.c_void_p, C.POINTER(AdamwManyLayout), C.c_void_p, C.c_int64] + [C.c_double] * 6 + [
        C.c_uint64, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]

    def step(bits, **change):
        layout = AdamwManyLayout()
        numel = (C.c_int64 * 1)(0)                         # no elements: a valid call does nothing
        assert lib.pcm_adamw_many_describe(1, numel, bits, C.byref(layout)) == OK
        p = {**GOOD, **change}
        return lib.pcm_adamw_many_step(None, C.byref(layout), None, *p.values(), 0, None, None, 0, None)

    return step


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("eps", [1e-50, 1e-46, 1e-40, 2.0 ** -127])
def test_an_eps_that_fp32_has_not_is_refused(call, bits, eps):
    """Elements that no gradient has reached yet would be 0 / 0."""
    assert call(bits, eps=eps) == EINVAL


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("eps", [2.0 ** -126, 1e-30, 1e-8, 1.0])
def test_others_are_taken(call, bits, eps):
    assert call(bits, eps=eps) == OK
