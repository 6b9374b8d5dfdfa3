"""af_draft_verify on rows whose maximum is of any magnitude a finite logit can have: the distribution is that of the differences, so
the lowest value of a type, alone or between masked entries, is as good a maximum as 0."""
import math

import numpy as np
import pytest
import torch

from oracle import rollout_oracle as O
from rollout_util import U
from test_gpu_draft_verify import ctx, reference, run  # noqa: F401  (ctx is a fixture)

pytestmark = pytest.mark.gpu

V = 1000
TYPES = [torch.float32, torch.bfloat16]
# of fp32, and "lowest" and "largest" of the row's type
VALUES = ["lowest", "largest", -1e30, 1e30, -1e20, -1e18, -1e12]
TEMPERATURES = [0.55, 0.7, 0.8, 1.0, 1.3]


def number(value, dtype):
    info = torch.finfo(dtype)
    return {"lowest": info.min, "largest": info.max}.get(value, value)


def masked(dtype, value, tokens):
    row = torch.full((V,), -math.inf)
    row[list(tokens)] = number(value, dtype)
    return row


def compare(ctx, c, temperature, tokens=None, **how):
    """Tokens (the oracle's, or these) and counts exactly.  A drawn token's log-prob is rounded once to fp32, from 64 bits with powers good to 2^-42; a passed one's
    row sum here has a few equal terms, exact in any order, whose logarithm is exact as well."""
    token, lp, n = run(ctx, c, temperature, **how)
    want = reference(c, temperature)
    if tokens is None:
        assert want["margin"] > 1e-11
        tokens = want["token"]
    assert not want["flags"] and np.array_equal(n, want["n_emitted"]) and np.array_equal(token, tokens)
    assert (np.abs(lp - want["logp"]) <= U * np.abs(want["logp"]) + 1e-11).all()
    assert ctx.check_device_errors() == 0
    return want


def case(rows, drafts=None, ids=(), cu=None, ua=(), us=(), dtype=torch.float32, draft_type=torch.float32):
    return {"target": torch.stack(rows).to(dtype), "draft": None if drafts is None else torch.stack(drafts).to(draft_type),
            "ids": np.array(ids, np.int32), "cu": np.array([0] * (len(rows) + 1) if cu is None else cu, np.int32),
            "ua": np.array(ua, np.float32), "us": np.array(us, np.float32)}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("value", VALUES)
@pytest.mark.parametrize("temperature", TEMPERATURES)
def test_a_draw_from_the_target(ctx, value, temperature, dtype):  # noqa: F811
    at = number(value, dtype)
    below = torch.full((V,), torch.finfo(dtype).min if at > 0 else -math.inf)       # finite ones, far below, have no weight either
    below[700:703] = at
    rows = [torch.full((V,), at), masked(dtype, value, range(300, V)), masked(dtype, value, [517]), masked(dtype, value, [3, 4, 900]), below]
    # all weights are 1: C_v is a whole number, and the second draw's u C = 175 a border, which C = 175 does not pass
    compare(ctx, case(rows, us=[0.6171, 0.25, 0.9, 0.5, 0.7], dtype=dtype), temperature, tokens=[617, 475, 517, 4, 702])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("value", VALUES)
@pytest.mark.parametrize("temperature", TEMPERATURES)
def test_drafts_without_a_distribution(ctx, value, temperature, dtype):  # noqa: F811
    """p = 1/3 at three tokens: the floats on both sides of 1/3 are told apart by the sums that are made again."""
    three = masked(dtype, value, [5, 90, 411])
    third = np.float32(1 / 3)                                  # above 1/3
    last = masked(dtype, value, [600, 601])
    c = case([three, last] * 3, ids=[90, 90, 5], cu=[0, 1, 2, 3], ua=[third, np.nextafter(third, np.float32(0)), 0.75], us=[0.3, 0.6, 0.6], dtype=dtype)
    want = compare(ctx, c, temperature, max_draft=1)
    assert want["n_emitted"].tolist() == [1, 2, 1] and want["token"].tolist() == [5, -1, 90, 601, 411, -1]


@pytest.mark.parametrize("dtype,draft_type", [(a, b) for a in TYPES for b in TYPES])
@pytest.mark.parametrize("value", VALUES)
@pytest.mark.parametrize("temperature", TEMPERATURES)
def test_drafts_with_a_distribution(ctx, value, temperature, dtype, draft_type):  # noqa: F811
    ordinary = torch.as_tensor(np.random.default_rng(5).standard_normal(V).astype(np.float32)).to(torch.bfloat16).float()
    last = masked(dtype, value, [7, 8])
    # requests: the draft's row is extreme; the target's; both, where the draft has no mass in the target
    rows = [ordinary, last, masked(dtype, value, [5, 90, 411]), last, masked(dtype, value, [5, 90, 411]), last]
    drafts = [masked(draft_type, value, [20, 30, 40]), ordinary, masked(draft_type, value, [90, 777])]
    c = case(rows, drafts, ids=[30, 90, 777], cu=[0, 1, 2, 3], ua=[0.75, 0.75, 0.25], us=[0.43, 0.75, 0.75], dtype=dtype, draft_type=draft_type)
    with np.errstate(all="ignore"):
        p = O.softmax(ordinary.double().numpy(), float(np.float32(temperature)))
    assert p[30] < 0.25 * 0.75
    token, lp, n = run(ctx, c, temperature, max_draft=1)
    want = reference(c, temperature)
    assert want["margin"] > 1e-11 and not want["flags"] and want["n_emitted"].tolist() == [1, 2, 1]
    assert np.array_equal(n, want["n_emitted"]) and np.array_equal(token, want["token"])
    assert want["token"][2:].tolist() == [90, 8, 411, -1] and want["token"][0] not in (20, 30, 40)
    assert (np.abs(lp - want["logp"]) <= U * np.abs(want["logp"]) + 1e-11).all()
    assert ctx.check_device_errors() == 0
