"""The tolerance of routing weights tells right from wrong: mistakes planted in the oracle's answer."""
import numpy as np
import pytest

import oracle.ops as ops
from ops_tolerance import route_weights


@pytest.mark.parametrize("sigmoid", [False, True])
def test_the_tolerance_of_weights_finds_wrong_ones(sigmoid):
    rng = np.random.default_rng(3)
    z = rng.standard_normal((20, 48))
    z[0, ::3] = -np.inf
    z[1, 1::2] = np.nan
    z[2, 7] = np.inf
    z[3, ::2] = np.finfo(np.float32).min
    z[4] = -120 - 10 * rng.random(48)
    kw = dict(sigmoid=sigmoid, renorm=True)
    r = ops.route_scores(z, None, 4, **kw)
    want, tol = r["w"], route_weights(z, r["ids"], r["w"], sigmoid)
    assert (tol < 1e-4 * want + 2e-37).all()
    plain = ops.route_scores(z, None, 4, sigmoid=sigmoid)["w"]
    for row in (0, 1, 3, 4, 10):
        assert (np.abs(want[row][::-1] - want[row]) > tol[row]).any()                       # weights of the wrong experts
        assert (np.abs(want[row] * (1 + 2e-5) - want[row]) > tol[row]).any()                # slightly off
        assert (np.abs(plain[row] - want[row]) > tol[row]).any()     # not divided by their sum
