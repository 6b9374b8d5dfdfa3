"""A NaN in the distillation loss: the whole token it stands in, and no other."""
import numpy as np
import pytest
import torch

from distill_util import dev_of, model, np_of, teacher_lists
from gpu_util import device
from test_gpu_distill import HOWS, loss_call

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2507_01663_b200 import binding as B
    c = B.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("side", ["teacher", "student", "student where the teacher has nothing left"])
@pytest.mark.parametrize("K", [1, 4, 20, 100])
@pytest.mark.parametrize("how", HOWS, ids=[f"div{d}-sup{s}-t{t}" for d, s, t in HOWS])
def test_a_nan_reaches_its_whole_token(ctx, how, K, side):
    """Loss, gradients of every slot and the record are NaN; every other token has the bits of a clean batch."""
    T, row, slot = 40, 17, K // 2
    lt, lq = teacher_lists(np.random.default_rng(K), T, K, short=False)
    if side.endswith("left"):
        lt[row, slot] = -200.0                   # present, but its probability is 0 in 32 bits
    clean = loss_call(ctx, lq, lt, [0, 25, T], how)
    (lt if side == "teacher" else lq)[row, slot] = np.nan
    res, token, g = loss_call(ctx, lq, lt, [0, 25, T], how)
    others = np.arange(T) != row
    assert np.isnan(token[row]) and np.isnan(g[row]).all() and np.isnan(res["loss"])
    assert np.isfinite(clean[1]).all() and np.array_equal(token[others], clean[1][others])
    assert np.array_equal(g[others], clean[2][others])
    assert ctx.check_device_errors() == 0


@pytest.mark.parametrize("how", HOWS, ids=[f"div{d}-sup{s}-t{t}" for d, s, t in HOWS])
@pytest.mark.parametrize("T", [9, 50])
def test_an_id_outside_the_vocabulary_shows_in_the_update(ctx, T, how):
    """The slot's log-prob is NaN, so the token's loss and the record are, whichever divergence is taken."""
    from paper_2507_01663_b200 import binding as B
    dev = device()
    d, V, K, row = 64, 520, 6, 3
    H, W, cand = model(5, T, d, V, K)
    lt, _ = teacher_lists(np.random.default_rng(6), T, K, short=False)
    cand[row] = [5, 9, V, 12, 0, 1]
    lt[cand < 0] = -np.inf
    token, lq, lse = torch.zeros(T, device=dev), torch.zeros(T, K, device=dev), torch.zeros(T, device=dev)
    out = B.new_distill_out(dev)
    ctx.distill_update(H.to(dev), W.to(dev), dev_of(cand), dev_of(lt.astype(np.float32)), dev_of(np.array([0, T], np.int32)), out,
                       lq, lse, torch.empty_like(H, device=dev), None, token_loss=token, divergence=how[0], support=how[1],
                       temperature=how[2])
    assert ctx.check_device_errors() == B.DEVERR_TARGET_RANGE
    t = np_of(token)
    assert np.isnan(t[row]) and np.isfinite(np.delete(t, row)).all() and np.isnan(B.read_distill_out(out)["loss"])
