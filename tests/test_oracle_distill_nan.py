"""The oracle of the distillation loss keeps NaN and infinities as the formulas have them."""
import math

import numpy as np
import pytest

from oracle import distill_oracle as D

HOWS = [(d, s, 1.0) for d in (0, 1) for s in (0, 1, 2)] + [(0, 1, 2.5), (1, 1, 0.5)]


@pytest.mark.parametrize("how", HOWS)
def test_a_nan_is_a_nan(how):
    lt, lq = np.log([0.5, 0.2, 0.1]), np.log([0.3, 0.3, 0.2])
    assert math.isfinite(D.divergence_ref(lt, lq, *how)[0])
    for side in (0, 1):
        for k in range(3):
            rows = [lt.copy(), lq.copy()]
            rows[side][k] = math.nan
            loss, grad = D.divergence_ref(rows[0], rows[1], *how)
            assert math.isnan(loss) and np.isnan(grad).all()
    # behind an absent slot it is not looked at
    loss, grad = D.divergence_ref(np.array([lt[0], -np.inf, lt[2]]), np.array([lq[0], np.nan, lq[2]]), *how)
    assert math.isfinite(loss) and np.isfinite(grad).all() and grad[1] == 0.0


def test_terms_of_probability_zero():
    """0 log 0 = 0; a zero of the student under a teacher's mass is an infinity in one direction."""
    lt, lq = np.array([0.0, -800.0]), np.array([-0.5, -np.inf])
    assert math.isfinite(D.divergence_ref(lt, lq, 0, 0)[0])
    assert D.divergence_ref(np.log([0.5, 0.5]), np.array([0.0, -np.inf]), 0, 0)[0] == math.inf
    assert D.divergence_ref(np.log([0.5, 0.5]), np.array([0.0, -np.inf]), 0, 1)[0] == math.inf
    assert math.isnan(D.divergence_ref(np.log([0.5, 0.5]), np.array([-np.inf, -np.inf]), 0, 1)[0])
    assert math.isnan(D.divergence_ref(np.log([0.5, 0.5]), np.array([-np.inf, -np.inf]), 1, 1)[0])
