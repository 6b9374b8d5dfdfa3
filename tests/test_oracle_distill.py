"""Pins of the distillation and preference oracle: finite differences, closed forms, invariances."""
import math

import numpy as np
import pytest
import torch

from oracle import distill_oracle as D
from oracle import grpo_oracle as O


def to_bits(x):
    t = torch.as_tensor(np.asarray(x, dtype=np.float32)).to(torch.bfloat16)
    return t.view(torch.int16).numpy().view(np.uint16)


def lists(rng, T, K, short=True):
    lt = np.log(rng.dirichlet(np.full(K + 1, 0.7), size=T))[:, :K]
    lq = np.log(rng.dirichlet(np.full(K + 1, 0.9), size=T))[:, :K]
    if short and T > 2 and K > 1:
        lt[1, K // 2:] = -math.inf
        lt[2, :] = -math.inf
    return lt, lq


def test_one_candidate_is_the_single_target_path():
    rng = np.random.default_rng(0)
    T, d, V = 5, 8, 11
    H, W = to_bits(rng.standard_normal((T, d))), to_bits(rng.standard_normal((V, d)))
    y = rng.integers(0, V, T)
    lp, ent, lse = O.token_logprob_ref(H, W, y)
    lq, ent2, lse2 = D.candidate_logprob_ref(H, W, y[:, None])
    assert np.allclose(lq[:, 0], lp, atol=1e-13) and np.allclose(ent, ent2) and np.allclose(lse, lse2)
    g = rng.standard_normal(T)
    a = O.policy_loss_backward_ref(H, W, y, lse, g)
    b = D.candidate_backward_ref(H, W, y[:, None], lse, g[:, None])
    assert np.allclose(a[0], b[0], atol=1e-12) and np.allclose(a[1], b[1], atol=1e-12)


def test_candidate_slots_without_an_id():
    rng = np.random.default_rng(1)
    H, W = to_bits(rng.standard_normal((2, 8))), to_bits(rng.standard_normal((9, 8)))
    cand = np.array([[3, -1, 3], [9, 0, -5]])
    lq, _, lse = D.candidate_logprob_ref(H, W, cand)
    assert lq[0, 1] == -math.inf and lq[1, 2] == -math.inf and math.isnan(lq[1, 0]) and lq[0, 0] == lq[0, 2]
    g = rng.standard_normal((2, 3))
    g2 = g.copy()
    g2[0, 1], g2[1, 0], g2[1, 2] = 7.0, math.nan, -3.0
    a, b = D.candidate_backward_ref(H, W, cand, lse, g), D.candidate_backward_ref(H, W, cand, lse, g2)
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])


def test_candidate_backward_by_differences():
    """d_hidden against central differences of sum(g * cand_logp) in H, taken in fp64 without bf16."""
    rng = np.random.default_rng(2)
    T, d, V, K = 3, 8, 10, 4
    H, W = to_bits(rng.standard_normal((T, d))), to_bits(rng.standard_normal((V, d)))
    cand, g = rng.integers(0, V, (T, K)), rng.standard_normal((T, K))
    _, _, lse = D.candidate_logprob_ref(H, W, cand)
    dH, dW = D.candidate_backward_ref(H, W, cand, lse, g)
    Hf, Wf = O.bf16_bits_to_f64(H), O.bf16_bits_to_f64(W)

    def objective(h, w):
        z = h @ w.T
        l = z - np.log(np.exp(z).sum(1, keepdims=True))
        return float((g * np.take_along_axis(l, cand, 1)).sum())

    e = 1e-6
    for idx in [(0, 0), (1, 3), (2, 7)]:
        up, dn = Hf.copy(), Hf.copy()
        up[idx] += e
        dn[idx] -= e
        assert dH[idx] == pytest.approx((objective(up, Wf) - objective(dn, Wf)) / (2 * e), abs=1e-7)
    for idx in [(0, 0), (int(cand[1, 0]), 5), (9, 2)]:
        up, dn = Wf.copy(), Wf.copy()
        up[idx] += e
        dn[idx] -= e
        assert dW[idx] == pytest.approx((objective(Hf, up) - objective(Hf, dn)) / (2 * e), abs=1e-7)


@pytest.mark.parametrize("divergence", [0, 1])
@pytest.mark.parametrize("support,tau", [(0, 1.0), (1, 1.0), (1, 2.5), (2, 1.0)])
@pytest.mark.parametrize("agg", [0, 1])
def test_distill_gradient_by_differences(divergence, support, tau, agg):
    rng = np.random.default_rng(3)
    T, K = 6, 5
    lt, lq = lists(rng, T, K)
    cu = [0, 2, 2, 6]
    got = D.distill_loss_ref(lq, lt, cu, divergence, support, tau, agg, 1.7)
    e = 1e-6
    for t in range(T):
        for k in range(K):
            up, dn = lq.copy(), lq.copy()
            up[t, k] += e
            dn[t, k] -= e
            num = (D.distill_loss_ref(up, lt, cu, divergence, support, tau, agg, 1.7)["loss"]
                   - D.distill_loss_ref(dn, lt, cu, divergence, support, tau, agg, 1.7)["loss"]) / (2 * e)
            assert got["dcand"][t, k] == pytest.approx(num, abs=2e-8)
    assert not got["dcand"][2].any() and got["token_loss"][2] == 0.0      # a token without a list
    assert got["teacher_mass"] == pytest.approx(np.exp(lt).sum() / T)


def test_distill_closed_forms():
    # equal distributions: every divergence that is one is zero, and so is its gradient
    lt = np.log(np.array([[0.5, 0.2, 0.1]]))
    for divergence in (0, 1):
        for support, tau in ((1, 1.0), (1, 3.0), (2, 1.0)):
            r = D.distill_loss_ref(lt, lt, [0, 1], divergence, support, tau)
            assert abs(r["loss"]) < 1e-15 and np.abs(r["dcand"]).max() < 1e-15
    # two outcomes by hand: teacher (3/4, 1/4), student (1/2, 1/2), renormalised
    r = D.distill_loss_ref(np.log([[0.3, 0.3]]), np.log([[0.6, 0.2]]), [0, 1], 0, 1)
    assert r["loss"] == pytest.approx(0.75 * math.log(1.5) + 0.25 * math.log(0.5))
    assert r["dcand"][0] == pytest.approx([0.5 - 0.75, 0.5 - 0.25])
    # renormalised: a shift of the student's log-probs changes nothing
    rng = np.random.default_rng(4)
    a, b = lists(rng, 4, 6)
    for divergence in (0, 1):
        x = D.distill_loss_ref(b, a, [0, 4], divergence, 1, 2.0)
        y = D.distill_loss_ref(b - 3.0, a, [0, 4], divergence, 1, 2.0)
        assert x["loss"] == pytest.approx(y["loss"], rel=1e-12) and np.allclose(x["dcand"], y["dcand"], atol=1e-14)
    # the tail is one more outcome: the same as listing it and leaving (almost) nothing
    lt, lq = np.log([[0.5, 0.3]]), np.log([[0.4, 0.1]])
    full_t, full_q = np.log([[0.5, 0.3, 0.2]]), np.log([[0.4, 0.1, 0.5]])
    for divergence in (0, 1):
        assert D.distill_loss_ref(lq, lt, [0, 1], divergence, 2)["loss"] == pytest.approx(
            D.distill_loss_ref(full_q, full_t, [0, 1], divergence, 0)["loss"])


@pytest.mark.parametrize("kind", [0, 1, 2])
@pytest.mark.parametrize("norm,layout,nll,with_ref", [(False, 0, 0.0, True), (True, 1, 0.3, True), (True, 0, 0.2, False)])
def test_preference_gradient_by_differences(kind, norm, layout, nll, with_ref):
    rng = np.random.default_rng(5)
    cu = [0, 3, 8, 8, 10]                     # one sequence is empty
    logp = -rng.random(10)
    ref = logp + 0.3 * rng.standard_normal(10) if with_ref else None
    how = dict(kind=kind, beta=0.7, label_smoothing=0.1, margin=0.2, nll_coef=nll, length_norm=norm, pair_layout=layout,
               loss_scale=1.3)
    got = D.preference_loss_ref(logp, ref, cu, **how)
    e = 1e-6
    for t in range(10):
        up, dn = logp.copy(), logp.copy()
        up[t] += e
        dn[t] -= e
        num = (D.preference_loss_ref(up, ref, cu, **how)["loss"] - D.preference_loss_ref(dn, ref, cu, **how)["loss"]) / (2 * e)
        assert got["dlogp"][t] == pytest.approx(num, abs=2e-8)


def test_preference_closed_forms():
    # equal log ratios: log 2, half the slope; the pair's order does not matter without smoothing or margin
    r = D.preference_loss_ref([-1.0, -2.0], [-1.0, -2.0], [0, 1, 2], beta=0.5)
    assert r["loss"] == pytest.approx(math.log(2.0)) and r["dlogp"] == pytest.approx([-0.25, 0.25]) and r["accuracy"] == 0.0
    # far apart in either direction: 0 and the (negative) score difference itself
    r = D.preference_loss_ref([0.0, -1000.0], None, [0, 1, 2], beta=1.0)
    assert r["loss"] == 0.0 and r["accuracy"] == 1.0
    r = D.preference_loss_ref([-1000.0, 0.0], None, [0, 1, 2], beta=1.0)
    assert r["loss"] == pytest.approx(1000.0) and r["dlogp"] == pytest.approx([-1.0, 1.0])
    # squared: zero where the log ratio is 1 / (2 beta)
    r = D.preference_loss_ref([5.0, 0.0], [0.0, 0.0], [0, 1, 2], kind=1, beta=0.1)
    assert r["loss"] == pytest.approx(0.0, abs=1e-20)
    # both layouts hold the same pairs
    a = D.preference_loss_ref([-1.0, -2.0, -3.0, -5.0], None, [0, 1, 2, 3, 4], beta=1.0, pair_layout=0)
    b = D.preference_loss_ref([-1.0, -3.0, -2.0, -5.0], None, [0, 1, 2, 3, 4], beta=1.0, pair_layout=1)
    assert a["loss"] == pytest.approx(b["loss"]) and a["pair_loss"] == pytest.approx(b["pair_loss"])


def test_a_mask_of_the_lowest_value_is_absent():
    lt = np.array([-1.0, -np.inf, -2.0], np.float64)
    lq = np.array([-1.5, -0.5, -0.7], np.float64)
    for div in (0, 1):
        for support in (0, 1, 2):
            want = D.divergence_ref(lt, lq, div, support)
            for low in (np.finfo(np.float32).min, -1e30, -3.0e38):
                got = D.divergence_ref(np.where(np.isneginf(lt), np.float32(low), lt), lq, div, support)
                assert got[0] == want[0] and np.array_equal(got[1], want[1])
    assert D.divergence_ref(np.full(3, -3.4e38), lq, 0, 1)[0] == 0.0
