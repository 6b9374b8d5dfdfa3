"""The renormalised distillation loss at the ends of its temperatures."""
import numpy as np
import pytest
import torch

from distill_util import U, np_of, teacher_lists
from gpu_util import device
from oracle import distill_oracle as D
from test_gpu_distill import loss_call

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2507_01663_b200 import binding as B
    c = B.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("K", [3, 7, 50, 64, 100, 200])
@pytest.mark.parametrize("direction", [0, 1])
@pytest.mark.parametrize("tau", [1e-4, 1e4])
def test_both_ends_of_the_temperature(ctx, tau, direction, K):
    """Short lists and lists that leave lanes idle: what is absent keeps no weight.

    A log ratio d = (lt - lq) / tau + log of the ratio of the sums is off by at most e = c (1 + |x| + |y|) absolutely, c the
    relative error of a probability (see row_scales), x and y the scaled inputs, and so is a probability, relatively.  A
    term of the loss, a log(a / b) + b - a, then moves by at most (a + b) (|d| + e) e, and as much again by the
    probabilities' own error; the gradients tau (b - a) and tau b (d - mean) by tau (a + b) e and tau b (|d| + mean + 2) e.
    Probabilities below 2^-126 come out as 0."""
    T = 60
    lt, lq = teacher_lists(np.random.default_rng(K), T, K)
    tau = float(np.float32(tau))
    res, token, g = loss_call(ctx, lq, lt, [0, T], (direction, 1, tau), 1)
    for t in range(T):
        want, wg = D.divergence_ref(lt[t], lq[t], direction, 1, tau)
        on = np.flatnonzero(~np.isneginf(lt[t]))
        assert not np.delete(g[t], on).any()
        if on.size == 0:
            assert token[t] == 0.0
            continue
        x, y = lt[t, on].astype(np.float64) / tau, lq[t, on].astype(np.float64) / tau
        a, b = np.exp(x - x.max()), np.exp(y - y.max())
        d = np.abs((x - np.log(a.sum()) - x.max()) - (y - np.log(b.sum()) - y.max()))
        a, b = a / a.sum(), b / b.sum()
        e = 20 * U * (1 + np.abs(x).max() + np.abs(y).max())
        assert abs(token[t] - want) <= 2 * tau * tau * ((a + b) * (d + e) * e).sum() + 4 * U * abs(want)
        mean = (b * d).sum()
        tol = tau * ((a + b) if direction == 0 else b * (d + mean + 2)) * e
        tol = tol + tau * 2.0 ** -126 * (d + mean + 2)
        assert (np.abs(g[t, on] - wg[on] / T) <= tol / T + 6 * U * np.abs(wg[on]) / T).all()
    assert ctx.check_device_errors() == 0


def test_temperatures_past_the_ends_are_refused(ctx):
    """Far from 1 an absent slot's stand-in would gain weight, or the inverse overflow."""
    from paper_2507_01663_b200 import binding as B
    dev = device()
    x, cu = torch.full((4, 3), -1.0, device=dev), torch.tensor([0, 4], dtype=torch.int32, device=dev)
    for tau in (9.9e-5, 1e-39, 1.01e4, 1e30, 3e38):
        out, g = B.new_distill_out(dev), torch.full((4, 3), 5.0, device=dev)
        with pytest.raises(B.AfError) as e:
            ctx.distill_loss(x, x, cu, out, dcand=g, support=1, temperature=tau)
        assert e.value.status == -1 and bool((g == 5.0).all())
    assert np_of(out).any() == 0 and ctx.check_device_errors() == 0
