"""Undefined and infinite scores in the preference loss."""
import numpy as np
import pytest

from oracle import distill_oracle as D
from test_gpu_preference import call

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2507_01663_b200 import binding as B
    c = B.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("kind", [0, 1, 2])
def test_a_nan_score_has_a_nan_gradient(ctx, kind, layout):
    """Both sequences of its pair, and no other pair."""
    logp = np.full(12, -0.75, np.float32)
    cu = np.arange(0, 13, 2, dtype=np.int32)
    clean = call(ctx, logp, None, cu, kind=kind, beta=0.5, pair_layout=layout)
    logp[5] = np.nan                              # in sequence 2
    res, pair, score, g = call(ctx, logp, None, cu, kind=kind, beta=0.5, pair_layout=layout)
    pair_of = np.arange(6) % 3 if layout else np.arange(6) // 2
    hit = pair_of == pair_of[2]
    assert np.isnan(pair[pair_of[2]]) and np.isnan(score[2]) and np.isnan(res["loss"])
    assert np.isnan(g.reshape(6, 2)[hit]).all()
    assert np.array_equal(g.reshape(6, 2)[~hit], clean[3].reshape(6, 2)[~hit])
    assert np.array_equal(np.delete(pair, pair_of[2]), np.delete(clean[1], pair_of[2]))


@pytest.mark.parametrize("eps", [0.0, 0.1, 0.5])
@pytest.mark.parametrize("kind", [0, 1, 2])
def test_infinite_scores(ctx, kind, eps):
    """A response of probability 0 on either side: the loss is the formula's limit, infinite or not."""
    eps = float(np.float32(eps)) if kind == 0 else 0.0
    logp = np.array([-np.inf, -1.0, -1.0, -np.inf, -1.0, -2.0], np.float32)      # chosen, rejected; x = -inf, inf, 1
    cu = np.arange(7, dtype=np.int32)
    want = D.preference_loss_ref(logp, None, cu, kind=kind, beta=1.0, label_smoothing=eps)
    res, pair, score, g = call(ctx, logp, None, cu, kind=kind, beta=1.0, label_smoothing=eps)
    assert np.array_equal(score, want["seq_score"])
    assert not np.isnan(want["pair_loss"]).any() and np.array_equal(np.isinf(pair), np.isinf(want["pair_loss"]))
    assert pair == pytest.approx(want["pair_loss"], rel=1e-6, abs=1e-12)
    assert g == pytest.approx(want["dlogp"], rel=1e-6, abs=1e-12)
    assert res["loss"] == pytest.approx(want["loss"], rel=1e-6)
