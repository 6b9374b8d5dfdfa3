"""The oracle of the preference loss keeps NaN and infinities as the formulas have them."""
import math

import numpy as np
import pytest

from oracle import distill_oracle as D


@pytest.mark.parametrize("kind", [0, 1, 2])
def test_a_nan_score(kind):
    got = D.preference_loss_ref([math.nan, -1.0, -1.0, -2.0], None, np.arange(5), kind=kind, beta=1.0)
    assert math.isnan(got["pair_loss"][0]) and math.isfinite(got["pair_loss"][1]) and math.isnan(got["loss"])
    assert np.isnan(got["dlogp"][:2]).all() and np.isfinite(got["dlogp"][2:]).all()


@pytest.mark.parametrize("kind,eps", [(0, 0.0), (0, 0.25), (1, 0.0), (2, 0.0)])
def test_responses_of_probability_zero(kind, eps):
    got = D.preference_loss_ref([-math.inf, -1.0, -1.0, -math.inf], None, np.arange(5), kind=kind, beta=1.0, label_smoothing=eps)
    assert not np.isnan(got["pair_loss"]).any() and not np.isnan(got["dlogp"]).any()
    assert got["pair_loss"][0] == math.inf
    assert got["pair_loss"][1] == (math.inf if kind == 1 or eps else 0.0)
