"""The renormalised distillation loss where the student has no distribution over the present slots."""
import numpy as np
import pytest

from distill_util import U, teacher_lists
from test_gpu_distill import loss_call

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2507_01663_b200 import binding as B
    c = B.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("K", [2, 3, 20, 64, 130])
@pytest.mark.parametrize("how", [(0, 1, 1.0), (1, 1, 1.0), (0, 1, 2.5), (1, 1, 0.5)])
def test_a_student_with_nothing_on_the_present_slots(ctx, how, K):
    """No distribution of the student over these slots exists: NaN.  Absent slots must not stand in for them."""
    T, row = 30, 11
    lt, lq = teacher_lists(np.random.default_rng(K), T, K, short=False)
    keep = (K + 1) // 2
    lt[row, keep:] = -np.inf
    clean = loss_call(ctx, lq, lt, [0, T], how)
    lq[row, :keep] = -np.inf
    res, token, g = loss_call(ctx, lq, lt, [0, T], how)
    others = np.arange(T) != row
    assert np.isnan(token[row]) and np.isnan(g[row, :keep]).all() and np.isnan(res["loss"])
    assert np.array_equal(token[others], clean[1][others]) and np.array_equal(g[others], clean[2][others])
    on = ~np.isneginf(lt)
    want = np.exp(lq.astype(np.float64), where=on, out=np.zeros(lq.shape)).sum() / T
    assert abs(res["student_mass"] - want) <= 128 * U * want
    assert ctx.check_device_errors() == 0
