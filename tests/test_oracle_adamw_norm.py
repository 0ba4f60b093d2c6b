"""The plain form of the optimizer step with 8-bit moments where the norm of the gradients is no number: the clip factor max / norm is none either."""
import numpy as np

from oracle import operators as P


def test_a_nan_among_the_gradients_reaches_every_weight():
    w, g = [np.ones(300, np.float32)], [np.full(300, 3.0, np.float32)]
    g[0][7] = np.nan
    state = tuple(np.zeros(n, np.uint8) for n in (384, 384, 3, 3))
    hp = dict(lr=1e-2, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01)
    out, (mc, vc, mt, vt), norm = P.adamw_many_eight(w, g, state, 1, 0, max_grad_norm=1.0, **hp)
    assert np.isnan(norm) and np.isnan(out[0]).all() and (mt == 255).all() and (vt == 255).all()
    out, _, norm = P.adamw_many_eight(w, g, state, 1, 0, max_grad_norm=None, **hp)
    assert np.isnan(norm) and int(np.isnan(out[0]).sum()) == 1
