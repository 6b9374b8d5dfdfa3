"""af_draft_verify where u_sample is 0 (one fp32 uniform in 2^24 is): the first token that has any mass, however many masked ones
stand before it."""
import math

import numpy as np
import pytest
import torch

from test_gpu_draft_verify import ctx, reference, run  # noqa: F401  (ctx is a fixture)

pytestmark = pytest.mark.gpu

SIZES = [(7, 1), (7, 6), (600, 31), (600, 299), (4099, 1), (4099, 3000), (70001, 128), (70001, 9999), (152064, 1024), (152064, 152063)]


@pytest.mark.parametrize("kind", ["plain", "lookup", "dense", "nothing left"])
@pytest.mark.parametrize("mask", [-math.inf, "lowest"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,before", SIZES)
def test_the_first_token_with_mass(ctx, V, before, dtype, mask, kind):  # noqa: F811
    rng = np.random.default_rng(V + before)
    row = torch.as_tensor(rng.standard_normal((2, V)).astype(np.float32)).to(dtype)
    row[:, :before] = torch.finfo(dtype).min if mask == "lowest" else mask
    us = np.zeros(1, np.float32)
    if kind == "plain":
        c = {"target": row[:1], "draft": None, "ids": np.zeros(0, np.int32), "cu": np.array([0, 0], np.int32), "ua": np.zeros(0, np.float32), "us": us}
    else:
        # the draft is a token before the mask's end, or, where something has to be left over, the last one; it never passes
        draft = row[:1].clone()
        if kind == "dense":
            draft[0, before:] -= (torch.arange(V - before) % 2 * 0.5).to(dtype)      # even places have less of the target than of the draft
            draft[0, V - 1] += 2
        c = {"target": row, "draft": None if kind == "lookup" else draft, "ids": np.array([0 if kind == "lookup" else V - 1], np.int32),
             "cu": np.array([0, 1], np.int32), "ua": np.array([1e9], np.float32), "us": us}
    want = reference(c)
    token, lp, n = run(ctx, c)
    assert n[0] == 1 and token[0] == want["token"][0] >= before, (token[0], want["token"][0])
    if kind != "dense":
        assert token[0] == before
    assert abs(lp[0] - want["logp"][0]) <= 2.0 ** -24 * abs(want["logp"][0]) + 1e-11
    assert ctx.check_device_errors() == 0
