"""Inputs and derived tolerances of the candidate / distillation / preference tests.

Rounding model (u = 2^-24, half a step of fp32; bf16 half step 2^-8):
  * a logit is a sum of exact bf16 products on the tensor core.  Every K = 16 step may drop up to one place
    of the accumulator (2^-23 of at most A = sum |h w|), so after n steps a logit is off by at most
    n 2^-23 A;  with promoted accumulation a part has 16 steps on its own share of A, and adding `parts`
    parts rounds `parts` times:  (16 + parts) 2^-23 A in all, A over the whole sum.
  * ex2.approx is good to 2^-22 relative; its argument x log2 e is rounded once, which is |x| 2^-23 relative
    in the result.
  * a chain of n fp32 additions of non-negative terms is off by at most n u relative.
"""
import math

import numpy as np
import torch

from gpu_util import device, np_of
from paper_2507_01663_b200 import workloads as wl

U = 2.0 ** -24
BF = 2.0 ** -8


def model(seed, T, d, V, K, scale=1.0):
    """Hidden rows and head with logits of a few units, lists with repeats and unused slots."""
    rng = np.random.default_rng(seed)
    H = torch.as_tensor(rng.standard_normal((T, d)).astype(np.float32)).to(torch.bfloat16)
    W = torch.as_tensor((rng.standard_normal((V, d)) * scale * 1.5 / math.sqrt(d)).astype(np.float32)).to(torch.bfloat16)
    cand = rng.integers(0, V, (T, K)).astype(np.int32)
    if T > 3 and K > 1:
        cand[1, K // 2:] = -1               # a short list
        cand[2, :] = -1                     # an empty one
        cand[3, :] = cand[3, 0]             # one id in every slot
    if T > 4 and K > 2:
        cand[4, 0], cand[4, 1], cand[4, 2] = V - 1, 0, -7
    return H, W, cand


def abs_product(H, W):
    """max over the batch of A = sum_k |h_k w_k|."""
    return float((H.double().abs() @ W.double().abs().T).max()) if H.shape[0] else 0.0


def logit_tol(H, W, promoted):
    d = H.shape[1]
    steps = (d + 15) // 16
    n = 16 + (d + 255) // 256 if promoted else steps
    return min(n, steps + 1) * 2 * U * abs_product(H, W)


def lse_tol(H, W, z_max, promoted=True):
    """lse = m + log sum exp(z - m): the logits', the exponentials' and the additions' share.  A thread adds 32
    terms in each of four chains, joins them per tile (V / 256 of them at most), then parts are joined."""
    V = W.shape[0]
    adds = 32 + 2 + (V + 255) // 256 + 8 + 10
    return logit_tol(H, W, promoted) + 4 * U + 2 * z_max * 2 * U + adds * U + 4 * U * (z_max + math.log(V) + 1)


def bits(t):
    return wl.bf16_bits(t.contiguous())


def teacher_lists(rng, T, K, short=True):
    """(teacher, student) float32 log-probs of listed ids, with short and empty lists."""
    lt = np.log(rng.dirichlet(np.full(K + 1, 0.7), size=T) + 1e-7)[:, :K]
    lq = np.log(rng.dirichlet(np.full(K + 1, 0.9), size=T) + 1e-7)[:, :K]
    lt, lq = np.minimum(lt, -1e-3).astype(np.float32), np.minimum(lq, -1e-3).astype(np.float32)
    if short:
        for t in range(0, T, 5):
            lt[t, rng.integers(0, K + 1):] = -np.inf
        if T > 1:
            lt[1] = -np.inf
    # -inf entries of the teacher hide the student's value, whatever it is
    lq[np.isneginf(lt) & (rng.random(lt.shape) < 0.5)] = -np.inf
    hidden_nan = np.isneginf(lt) & (rng.random(lt.shape) < 0.2)
    lq[hidden_nan] = np.nan
    return lt, lq


def cuts(rng, B, T):
    """cu_seqlens of B sequences with T tokens, empty ones among them."""
    cu = np.zeros(B + 1, dtype=np.int32)
    cu[1:B] = np.sort(rng.integers(0, T + 1, B - 1))
    cu[B] = T
    return cu


def dev_of(x):
    return torch.as_tensor(np.ascontiguousarray(x), device=device())


__all__ = ["U", "BF", "model", "abs_product", "logit_tol", "lse_tol", "bits", "teacher_lists", "cuts", "dev_of", "np_of"]
