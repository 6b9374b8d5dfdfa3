"""CPU oracle of the distillation and preference operators.  TEST INFRASTRUCTURE ONLY.

Plain, slow, fp64 restatements (numpy, one token / one pair at a time) of what the candidate, distillation
and preference calls compute; see the header of the C library for the formulas.  Nothing here is shared with
the CUDA path.  Pins: tests/test_oracle_distill.py (finite differences of every gradient, closed forms,
invariances, K = 1 against the single-target oracle).
"""
from __future__ import annotations

import math

import numpy as np

from .grpo_oracle import bf16_bits_to_f64

TAIL_FLOOR = 2.0 ** -16
ABSENT = float(np.float32(-1e30))      # teacher values down from here mark an absent slot


def _logits(H_bits, W_bits):
    return bf16_bits_to_f64(H_bits) @ bf16_bits_to_f64(W_bits).T


def candidate_logprob_ref(H_bits, W_bits, cand):
    """cand [T, K] ids -> (cand_logp [T, K], entropy [T], lse [T]); ids < 0 give -inf, ids >= V NaN."""
    z = _logits(H_bits, W_bits)
    T, V = z.shape
    cand = np.asarray(cand, dtype=np.int64)
    out = np.empty(cand.shape)
    ent, lse = np.empty(T), np.empty(T)
    for t in range(T):
        m = z[t].max()
        e = np.exp(z[t] - m)
        lse[t] = m + math.log(e.sum())
        ent[t] = lse[t] - float((e * z[t]).sum() / e.sum())
        for k, c in enumerate(cand[t]):
            out[t, k] = -math.inf if c < 0 else math.nan if c >= V else z[t, c] - lse[t]
    return out, ent, lse


def candidate_backward_ref(H_bits, W_bits, cand, lse, dcand):
    """(d_hidden [T, d], d_W [V, d]) for dL/dcand_logp = dcand; slots without a valid id are skipped."""
    H, W = bf16_bits_to_f64(H_bits), bf16_bits_to_f64(W_bits)
    z = H @ W.T
    T, V = z.shape
    dz = np.zeros((T, V))
    for t in range(T):
        G = 0.0
        for c, g in zip(np.asarray(cand)[t], np.asarray(dcand, dtype=np.float64)[t]):
            if 0 <= c < V:
                dz[t, c] += g
                G += g
        dz[t] -= G * np.exp(z[t] - float(lse[t]))
    return dz @ W, dz.T @ H


def divergence_ref(lt, lq, divergence, support, temperature=1.0):
    """One token: (loss, gradient in lq) over the slots with lt > -1e30; with a NaN among them all of it is NaN."""
    lt, lq = np.asarray(lt, dtype=np.float64), np.asarray(lq, dtype=np.float64)
    grad = np.zeros(lt.shape)
    on = np.flatnonzero(~(lt <= ABSENT))
    if support == 1:
        if on.size == 0:
            return 0.0, grad
        tau = temperature

        def log_softmax(v):
            m = v.max()
            return v - m - math.log(np.exp(v - m).sum())

        la, lb = log_softmax(lt[on] / tau), log_softmax(lq[on] / tau)
        a, b = np.exp(la), np.exp(lb)
        if divergence == 0:
            grad[on] = tau * (b - a)
            loss = tau * tau * sum(x * (u - v) for x, u, v in zip(a, la, lb) if not (x == 0 and not math.isnan(v)))
        else:
            r = sum(y * (v - u) for y, u, v in zip(b, la, lb) if not (y == 0 and not math.isnan(u)))
            grad[on] = [0.0 if y == 0 else tau * y * ((v - u) - r) for y, u, v in zip(b, la, lb)]
            loss = tau * tau * r
        if math.isnan(loss):
            grad[on] = math.nan
        return loss, grad
    loss = ps = qs = 0.0
    for i in on:
        p, q = math.exp(lt[i]), math.exp(lq[i])
        ps, qs = ps + p, qs + q
        if divergence == 0:
            loss += 0.0 if p == 0 and not math.isnan(lq[i]) else p * (lt[i] - lq[i])
            grad[i] = -p
        elif not (q == 0 and not math.isnan(lt[i])):
            loss += q * (lq[i] - lt[i])
            grad[i] = q * (lq[i] - lt[i] + 1.0)
    if support == 2:
        pr, qr = (TAIL_FLOOR if 1.0 - s < TAIL_FLOOR else 1.0 - s for s in (ps, qs))      # a NaN stays one
        # qr = 1 - sum q, so d qr / d lq_i = -q_i unless it is held at the floor
        slope = 0.0 if 1.0 - qs <= TAIL_FLOOR else (-pr / qr if divergence == 0 else math.log(qr / pr) + 1.0)
        loss += pr * math.log(pr / qr) if divergence == 0 else qr * math.log(qr / pr)
        for i in on:
            grad[i] += slope * -math.exp(lq[i])
    if math.isnan(loss):                   # a NaN of one slot is the whole token's
        grad[on] = math.nan
    return loss, grad


def token_weights(cu, T, agg_mode, loss_scale):
    """Weight of every token in the aggregation of the policy loss."""
    w = np.zeros(T)
    B = len(cu) - 1
    for j in range(B):
        n = int(cu[j + 1]) - int(cu[j])
        for t in range(int(cu[j]), int(cu[j + 1])):
            w[t] = loss_scale / (B * n) if agg_mode == 0 else loss_scale / T
    return w


def distill_loss_ref(cand_logp, teacher_logp, cu, divergence=0, support=1, temperature=1.0, agg_mode=0, loss_scale=1.0):
    """dict: loss, teacher_mass, student_mass, n_tokens, token_loss [T], dcand [T, K]."""
    lq, lt = np.asarray(cand_logp, dtype=np.float64), np.asarray(teacher_logp, dtype=np.float64)
    T = lq.shape[0]
    w = token_weights(cu, T, agg_mode, loss_scale)
    token, grad = np.zeros(T), np.zeros(lq.shape)
    mt = ms = 0.0
    for t in range(T):
        token[t], g = divergence_ref(lt[t], lq[t], divergence, support, temperature)
        grad[t] = w[t] * g
        on = ~(lt[t] <= ABSENT)
        mt += np.exp(lt[t][on]).sum()
        ms += np.exp(lq[t][on]).sum()
    return {"loss": float((w * token).sum()), "teacher_mass": mt / T if T else 0.0, "student_mass": ms / T if T else 0.0,
            "n_tokens": T, "token_loss": token, "dcand": grad}


def preference_loss_ref(logp, ref_logp, cu, kind=0, beta=0.1, label_smoothing=0.0, margin=0.0, nll_coef=0.0,
                        length_norm=False, pair_layout=0, loss_scale=1.0):
    """dict: the record's means, pair_loss [P], seq_score [B], dlogp [T]."""
    logp = np.asarray(logp, dtype=np.float64)
    ref = np.zeros(logp.shape) if ref_logp is None else np.asarray(ref_logp, dtype=np.float64)
    B = len(cu) - 1
    P = B // 2
    score, dlogp, pair = np.zeros(B), np.zeros(logp.shape), np.zeros(P)
    rows = [slice(int(cu[j]), int(cu[j + 1])) for j in range(B)]
    n = [int(cu[j + 1]) - int(cu[j]) for j in range(B)]
    share = [1.0 / max(n[j], 1) if length_norm else 1.0 for j in range(B)]
    for j in range(B):
        score[j] = beta * share[j] * math.fsum(logp[rows[j]] - ref[rows[j]])
    ls, nlls, wins = [], [], []
    for p in range(P):
        c, r = (p, P + p) if pair_layout else (2 * p, 2 * p + 1)
        x = score[c] - score[r] - margin
        if kind == 0:
            def log_sigmoid(v):
                return -math.log1p(math.exp(-v)) if v > 0 else v - math.log1p(math.exp(v))

            s = math.exp(log_sigmoid(x))
            value = -(1 - label_smoothing) * log_sigmoid(x) - (label_smoothing * log_sigmoid(-x) if label_smoothing else 0.0)
            slope = -(1 - label_smoothing) * (1 - s) + label_smoothing * s
        elif kind == 1:
            value, slope = ((x - 0.5) / beta) ** 2, 2.0 * (x - 0.5) / beta ** 2
        else:
            value, slope = (1.0 - x, -1.0) if x < 1.0 else (0.0, 0.0) if x >= 1.0 else (x, x)      # a NaN stays one
        nll = -math.fsum(logp[rows[c]]) / n[c] if n[c] else 0.0
        pair[p] = value + (nll_coef * nll if nll_coef else 0.0)
        dlogp[rows[c]] += loss_scale / P * (slope * beta * share[c] - nll_coef / max(n[c], 1))
        dlogp[rows[r]] -= loss_scale / P * slope * beta * share[r]
        ls.append(value), nlls.append(nll), wins.append(score[c] > score[r])
    first = list(range(P)) if pair_layout else list(range(0, B, 2))
    second = list(range(P, B)) if pair_layout else list(range(1, B, 2))

    def mean(v):
        return float(np.mean(v)) if len(v) else 0.0

    return {"loss": loss_scale * mean(pair), "pair_loss_mean": mean(ls), "nll": mean(nlls), "accuracy": mean(wins),
            "chosen_score": mean(score[first]), "rejected_score": mean(score[second]), "n_pairs": P, "pair_loss": pair,
            "seq_score": score, "dlogp": dlogp}
