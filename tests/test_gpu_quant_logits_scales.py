"""af_quant_logits with scales of every kind the header takes: more than five significant bits at each token count and group size, and the
ends of bf16's range."""
import numpy as np
import pytest
import torch

from oracle import rollout_oracle as O
from rollout_util import bf16, f64, logits_tol
from test_gpu_quant_logits import ctx, head, run  # noqa: F401  (ctx is a fixture)

pytestmark = pytest.mark.gpu


def check(ctx, H, words, scale, group):  # noqa: F811
    got = run(ctx, H, words, scale, group)
    want, mag = O.quant_logits_ref(f64(H), words.numpy(), f64(scale), group)
    assert np.isfinite(want).all() and (np.abs(got - want) <= logits_tol(H.shape[1], mag, want, False)).all(), float((np.abs(got - want) / mag).max())


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("T", [1, 16, 17, 32, 33, 64, 65, 128, 129, 320])
def test_scales_of_eight_bits(ctx, T, group):  # noqa: F811
    check(ctx, *head(T + group, T, 416, 517, group, any_scale=True), group)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("T", [3, 20, 50])
@pytest.mark.parametrize("mixed", [False, True])
def test_rows_of_both_kinds_in_one_warp(ctx, T, group, mixed):  # noqa: F811
    """One row of other scales among rows of five bits; or one scale among those of a row."""
    H, words, scale = head(7, T, 512, 300, group)
    scale[100, 0 if mixed else slice(None)] = 0.01171875 * (1 + 1 / 128)
    check(ctx, H, words, scale, group)


@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("T", [2, 18, 40])
@pytest.mark.parametrize("bits", [4, 7])                       # of a scale's fraction: products of a digit and five bits are exact
@pytest.mark.parametrize("exponent", [-133, -130, -127, -126, -125, -120, 0, 119, 120, 121, 122, 123])
def test_ends_of_the_range(ctx, exponent, bits, T, group):  # noqa: F811
    """8 times the largest scale is finite; tokens are scaled the other way, so that the logits are ordinary numbers."""
    rng = np.random.default_rng(exponent + 200)
    _, words, scale = head(9, T, 256, 200, group)
    fraction = 1 + rng.integers(0, 1 << bits, scale.shape) / (1 << bits)
    scale = bf16(np.ldexp(fraction, exponent))                 # below -126: rounded to what bf16 has there
    H = bf16(np.ldexp(rng.standard_normal((T, 256)), np.clip(-exponent, -110, 110)))
    check(ctx, H, words, scale, group)
