"""Inputs and derived tolerances of the rollout tests.

u = 2^-24, half a step of fp32.  2^-22 is the error bound of ex2.approx.
"""
import math

import numpy as np
import torch

from gpu_util import device

U = 2.0 ** -24


def bf16(x):
    return torch.as_tensor(np.asarray(x, dtype=np.float32)).to(torch.bfloat16)


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def dev_of(x):
    return torch.as_tensor(np.ascontiguousarray(x), device=device())


def i32(x):
    return torch.as_tensor(np.asarray(x, dtype=np.int32), device=device())


def f32(x):
    return torch.as_tensor(np.asarray(x, dtype=np.float32), device=device())


def logits_tol(d, magnitude, exact, bf16_out):
    """Products of a bf16 and a digit are exact in fp32 (8 + 4 bits).  Every sum of at most d terms, in whatever order and
    split, adds d - 1 times at most; an addition, also a truncating one, is off by at most 2^-23 of the absolute terms.  A scale is
    applied once more per partial sum (u).  The sums are far shorter than d in a row: tensor-core steps take 16 terms at a time
    and chains are split over lanes, so d / 16 + 64 additions bound every order used.  A bf16 result adds half a step."""
    tol = (d / 16 + 64) * 2 * U * magnitude
    return tol + (2.0 ** -8 * np.abs(exact) if bf16_out else 0.0)


def logp_tol(V, spread):
    """log-prob of a token whose row's sum is taken in fp32 by 256 threads or more: V / 256 + 1 additions in a chain, 40 in
    joining, an exponential good to 2^-22 whose argument (up to `spread`, in halvings) is rounded twice, and the result's
    rounding to fp32, of up to `spread` too."""
    return (V / 256 + 41) * U + 2.0 ** -22 + 2 * spread * 2 * U + 2 * U * (spread + math.log(V) + 1)


def spans(rng, R, most):
    n = rng.integers(0, most + 1, R)
    return np.concatenate([[0], np.cumsum(n)]).astype(np.int32)


def verify_case(seed, R, most, V, mode="dense", ttype=torch.float32, dtype=torch.float32, masked=True, noise=0.7):
    """Target and draft logits (CPU tensors of their types), ids drawn from the draft, uniforms."""
    rng = np.random.default_rng(seed)
    cu = spans(rng, R, most)
    D = int(cu[-1])
    z = rng.standard_normal((D + R, V)) * 1.5
    for row in z:
        at = rng.integers(0, V, 4)
        row[at] += np.array([6.0, 5.0, 4.0, 3.0])
    if masked and V > 3:
        z[:, V - V // 4:] = -np.inf
    target = torch.as_tensor(z.astype(np.float32)).to(ttype)
    zq = np.empty((D, V))
    ids = np.empty(D, dtype=np.int32)
    for r in range(R):
        for i in range(cu[r + 1] - cu[r]):
            k = cu[r] + i
            zq[k] = z[k + r] + noise * rng.standard_normal(V)
    draft = torch.as_tensor(zq.astype(np.float32)).to(dtype)
    zq = f64(draft)
    for k in range(D):
        if mode == "greedy":
            ids[k] = zq[k].argmax()
            continue
        g = zq[k] * (2.0 if mode == "lookup" else 1.0) - np.log(-np.log(rng.random(V)))
        ids[k] = np.nan_to_num(g, nan=-np.inf).argmax()
    return {"target": target, "draft": draft if mode == "dense" else None, "ids": ids, "cu": cu,
            "ua": rng.random(D).astype(np.float32), "us": rng.random(R).astype(np.float32)}
