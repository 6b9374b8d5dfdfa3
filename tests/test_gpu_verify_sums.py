"""af_draft_verify's row sums on rows that are hard to sum in 32 bits: long flat ones, where all roundings go one way, taken by one
slice (a call of at least four rows to an SM; here by an upper bound of the drafts that no request uses)."""
import math

import numpy as np
import pytest
import torch

from gpu_util import device
from rollout_util import U
from test_gpu_draft_verify import ctx, run  # noqa: F401  (ctx is a fixture)

pytestmark = pytest.mark.gpu

ONE_SLICE = 1023                                   # max_draft


def sum_bound(V):
    """Of a row's sum in 32 bits, relative.  An exponential's argument e is rounded three times (difference, 1 / temperature, product),
    3 u |e| ln 2, and by their weights the terms are log2 V halvings below the largest on average at most (Gibbs), and 4 more
    where a part is summed about less than its maximum;  ex2.approx is good to 4 u, and used once for the term, at most twice
    where the maximum moves, and three times where parts are joined;  20 additions: chains of eight, and those that join 256 threads."""
    return (3 * math.log(2) * (math.log2(V) + 4) + 6 * 4 + 20) * U


def exact_logp(V, tail, x, tau):
    """A row of one token at 0 (the first) and all others at `tail`."""
    tau = float(np.float32(tau))
    return (tail / tau if x else 0.0) - math.log1p((V - 1) * math.exp(tail / tau))


def passed(ctx, row, x, tau, u=0.0):  # noqa: F811
    """log-prob of a draft x that u lets pass, or None."""
    two = torch.stack([row, row])
    c = {"target": two, "draft": None, "ids": np.array([x], np.int32), "cu": np.array([0, 1], np.int32), "ua": np.array([u], np.float32),
         "us": np.array([0.5], np.float32)}
    token, lp, n = run(ctx, c, tau, max_draft=ONE_SLICE)
    assert ctx.check_device_errors() == 0 and n[0] in (1, 2)
    return lp[0] if n[0] == 2 else None


def flat(V, tail, dtype):
    row = torch.full((V,), -tail, device=device()).to(dtype)
    row[0] = 0.0
    return row, float(row[-1])


TAILS = [0.7, 1.1, 1.5, 2.7, 5.1, 5.9, 7.5, 8.3, 8.7, 9.1, 9.9, 10.1, 11.1]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [152064, 1 << 20, 1 << 22])
def test_log_probs_of_flat_rows(ctx, V, dtype):  # noqa: F811
    for tail in TAILS:
        row, z = flat(V, tail, dtype)
        for tau in (0.8, 1.0):
            want = exact_logp(V, z, V // 2, tau)
            assert abs(passed(ctx, row, V // 2, tau) - want) <= sum_bound(V) + 2 * U * abs(want), (tail, tau)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1 << 20, 1 << 22])
def test_comparisons_on_flat_rows(ctx, V, dtype):  # noqa: F811
    """u 2e-6 to 1e-4 to either side of p: decided as 64 bits decide it."""
    for tail in TAILS:
        row, z = flat(V, tail, dtype)
        for tau in (0.8, 1.0):
            p = math.exp(exact_logp(V, z, 0, tau))
            for off in (-1e-4, -3e-5, -1e-5, -2e-6, 2e-6, 1e-5, 3e-5, 1e-4):
                u = np.float32(p * (1 + off))
                assert (passed(ctx, row, 0, tau, u) is not None) == (float(u) < p), (tail, tau, off)


def ramp(V, width, order):
    """Logits that rise by `width` from the first looked at to the last: over the row, the other way, or from one group of eight to the
    next of the same thread (256 threads of eight neighbours) and back down within the groups."""
    x = torch.arange(V, device=device(), dtype=torch.float64)
    if order == "down":
        x = x.flip(0)
    elif order == "threads":
        x = (x // 2048) * 2048 + (x % 2048).flip(0)
    return (x * (width / V)).float()


@pytest.mark.parametrize("order", ["up", "down", "threads"])
@pytest.mark.parametrize("V", [152064, 1 << 20, 1 << 22])
@pytest.mark.parametrize("greedy", [False, True])
def test_log_probs_of_rising_rows(ctx, V, order, greedy):  # noqa: F811
    """Every new maximum scales what was added up before."""
    for width in (1e-3, 0.03, 0.3, 1.0, 3.0, 20.0):
        row = ramp(V, width, order)
        z = row.double()
        x = int(row.argmax()) if greedy else V // 2 + 5
        for max_draft in (1, ONE_SLICE):
            two = torch.stack([row, row])
            c = {"target": two, "draft": None, "ids": np.array([x], np.int32), "cu": np.array([0, 1], np.int32),
                 "ua": np.zeros(1, np.float32), "us": np.array([0.5], np.float32)}
            token, lp, n = run(ctx, c, 0.0 if greedy else 1.0, max_draft=max_draft)
            want = float(z[x] - z.max() - (z - z.max()).exp().sum().log())
            assert ctx.check_device_errors() == 0 and n[0] == 2 and token[0] == x
            assert abs(lp[0] - want) <= sum_bound(V) + 20 * U + 2 * U * abs(want), (width, max_draft)      # 20 more additions join slices
            if greedy:
                assert token[1] == x and lp[1] == lp[0]
