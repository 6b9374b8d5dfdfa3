"""af_candidate_logprob and its backward against the fp64 oracle, element by element."""
import math

import numpy as np
import pytest
import torch

from distill_util import BF, U, bits, dev_of, logit_tol, lse_tol, model, np_of
from gpu_util import device
from oracle import distill_oracle as D

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2507_01663_b200 import binding as B
    c = B.Context(0)
    yield c
    c.close()


def score(ctx, H, W, cand, **kw):
    dev = device()
    T, K = cand.shape
    lq, ent, lse = torch.full((T, K), 5.0, device=dev), torch.full((T,), 5.0, device=dev), torch.full((T,), 5.0, device=dev)
    ctx.candidate_logprob(H.to(dev), W.to(dev), dev_of(cand), lq, ent, lse, **kw)
    return lq, ent, lse


def check_scores(H, W, cand, got):
    want = D.candidate_logprob_ref(bits(H), bits(W), cand)
    z_max = float(np.abs(want[2]).max()) + float(np.abs(want[0][np.isfinite(want[0])]).max(initial=0.0))
    lq, ent, lse = (np_of(t).astype(np.float64) for t in got)
    tz, tl = logit_tol(H, W, True), lse_tol(H, W, z_max)
    assert np.array_equal(np.isfinite(lq), np.isfinite(want[0])) and np.array_equal(np.isnan(lq), np.isnan(want[0]))
    ok = np.isfinite(want[0])
    assert np.abs(lse - want[2]).max() <= tl
    assert np.abs(lq - want[0])[ok].max(initial=0.0) <= tz + tl + 2 * U * z_max
    # entropy = lse - sum p z: an error e of every p (relative) and z moves it by at most tl + e max|z - mean| + tz
    assert np.abs(ent - want[1]).max() <= 2 * tl + tz + 2 * (tl + 8 * U) * 2 * z_max
    return want


SHAPES = [(1, 8, 1, 1), (1, 256, 4096, 20), (2, 24, 129, 2), (5, 64, 127, 3), (37, 128, 300, 31), (64, 264, 1000, 32),
          (255, 256, 4104, 33), (256, 640, 520, 64), (257, 320, 8200, 65), (300, 192, 2051, 128), (70, 512, 4099, 129),
          (513, 1000, 777, 256), (100, 64, 30000, 40), (33, 72, 45001, 7), (128, 136, 20011, 12), (129, 64, 20011, 12),
          (9, 200, 5003, 30), (16, 4096, 300, 9), (8, 6144, 200, 5), (17, 8, 700, 3)]


@pytest.mark.parametrize("T,d,V,K", SHAPES)
def test_scores_match_the_oracle(ctx, T, d, V, K):
    H, W, cand = model(T + d, T, d, V, K)
    check_scores(H, W, cand, score(ctx, H, W, cand))
    assert ctx.check_device_errors() == 0


@pytest.mark.parametrize("v_splits,variant", [(1, 0), (3, 0), (7, 2), (500, 0), (0, 1), (0, 2)])
def test_scores_with_other_splits_and_dealing(ctx, v_splits, variant):
    H, W, cand = model(9, 900, 256, 5000, 40)
    ctx.set_tuning(v_splits, 0, variant)
    try:
        check_scores(H, W, cand, score(ctx, H, W, cand))
        assert ctx.check_device_errors() == 0
    finally:
        ctx.set_tuning(0, 0)


def test_scores_are_closer_than_the_plain_accumulation(ctx):
    """d = 3584: the parts' sums keep what the tensor core's accumulator drops over 224 steps."""
    dev = device()
    H, W, cand = model(3, 200, 3584, 2000, 4, scale=3.0)
    cand = np.where(cand < 0, 0, cand).astype(np.int32)
    got = score(ctx, H, W, cand)
    want = check_scores(H, W, cand, got)
    lp, ent, lse = (torch.empty(200, device=dev) for _ in range(3))
    ctx.token_logprob(H.to(dev), W.to(dev), dev_of(cand[:, 0].copy()), lp, ent, lse)
    mine = np.abs(np_of(got[2]) - want[2]).mean()
    plain = np.abs(np_of(lse) - want[2]).mean()
    assert mine < plain


def test_no_probability_mass_is_lost(ctx):
    """Listing the whole vocabulary gives a distribution."""
    H, W, _ = model(4, 50, 128, 200, 3)
    cand = np.tile(np.random.default_rng(0).permutation(200).astype(np.int32), (50, 1))
    lq, _, _ = score(ctx, H, W, cand)
    assert np.abs(np.exp(np_of(lq).astype(np.float64)).sum(1) - 1).max() <= 1e-5


def test_slots_without_an_id_and_outside_the_vocabulary(ctx):
    from paper_2507_01663_b200 import binding as B
    H, W, cand = model(5, 20, 64, 500, 6)
    cand[7, 2], cand[8, 0] = 500, 2 ** 31 - 1
    cand[9, 1], cand[9, 2] = -2 ** 31, 2 ** 24
    got = score(ctx, H, W, cand)
    check_scores(H, W, cand, got)
    assert ctx.check_device_errors() == B.DEVERR_TARGET_RANGE
    lq = np_of(got[0])
    assert np.isnan(lq[7, 2]) and np.isnan(lq[8, 0]) and np.isnan(lq[9, 2]) and lq[9, 1] == -np.inf
    assert np.isfinite(lq[7, [0, 1, 3]]).all()


def test_rows_behind_the_batch_and_optional_outputs(ctx):
    dev = device()
    H, W, cand = model(6, 40, 64, 300, 5)
    lq = torch.full((40, 5), 7.0, device=dev)
    ent = torch.full((40,), 7.0, device=dev)
    ctx.candidate_logprob(H.to(dev), W.to(dev), dev_of(cand), lq, T=33)
    full, _, _ = score(ctx, H, W, cand)
    assert torch.equal(lq[:33], full[:33]) and bool((lq[33:] == 7.0).all())
    ctx.candidate_logprob(H.to(dev), W.to(dev), dev_of(cand), lq, entropy=ent, T=33)
    assert bool((ent[33:] == 7.0).all())
    ctx.candidate_logprob(H.to(dev), W.to(dev), dev_of(cand), lq, T=0)
    assert ctx.check_device_errors() == 0


def test_repeated_calls_give_the_same_bits(ctx):
    H, W, cand = model(7, 700, 256, 3000, 50)
    a = score(ctx, H, W, cand)
    b = score(ctx, H, W, cand)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_values_past_two_to_the_31_elements(ctx):
    """T * K > 2^31: the last rows of the lists are addressed with 64 bits."""
    dev = device()
    T, d, V, K = 8_400_000, 8, 64, 256
    g = torch.Generator(device=dev).manual_seed(1)
    H = torch.randn(T, d, generator=g, device=dev, dtype=torch.bfloat16)
    W = torch.randn(V, d, generator=g, device=dev, dtype=torch.bfloat16)
    cand = torch.randint(0, V, (T, K), generator=g, device=dev, dtype=torch.int32)
    lq = torch.empty(T, K, device=dev)
    ctx.candidate_logprob(H, W, cand, lq)
    assert ctx.check_device_errors() == 0
    rows = [0, T // 2, T - 2, T - 1]
    want, _, _ = D.candidate_logprob_ref(bits(H[rows]), bits(W), np_of(cand[rows]))
    tol = logit_tol(H[rows].cpu(), W.cpu(), True) + lse_tol(H[rows].cpu(), W.cpu(), float(np.abs(want).max()))
    assert np.abs(np_of(lq[rows]) - want).max() <= tol + 2 * U * float(np.abs(want).max())


# ------------------------------------------------------------------------------------------- backward
def gradient(ctx, H, W, cand, lse, g, dW_dtype=torch.float32, accumulate=False, start=None):
    dev = device()
    dH = torch.full(H.shape, 7.0, dtype=torch.bfloat16, device=dev)
    dW = None if dW_dtype is None else torch.full(W.shape, 7.0, dtype=dW_dtype, device=dev) if start is None else start.clone()
    ctx.candidate_logprob_backward(H.to(dev), W.to(dev), dev_of(cand), dev_of(lse), dev_of(g), dH, dW, accumulate)
    return dH, dW


def check_gradient(H, W, cand, lse, g, dH, dW, blocks=1):
    """dZ is rounded to bf16 once (half a step, 2^-8 of each value), carries the recomputed logits' error, and the
    products drop a place per K = 16 step; the result is rounded to its type."""
    Hf, Wf = H.double().numpy(), W.double().numpy()
    T, V = Hf.shape[0], Wf.shape[0]
    z = Hf @ Wf.T
    q = np.exp(z - np.asarray(lse, dtype=np.float64)[:, None])
    G = np.zeros(T)
    mag = np.zeros((T, V))                       # |terms| of dZ
    for t in range(T):
        for c, x in zip(cand[t], g[t]):
            if 0 <= c < V:
                G[t] += float(x)
                mag[t, c] += abs(float(x))
    dense = np.abs(G)[:, None] * q
    rel_q = logit_tol(H, W, False) + 8 * U + 2 * U * float(np.abs(z).max() + np.abs(lse).max())
    dz_err = BF * (mag + dense) + dense * rel_q + 1e-37 + 4 * U * (mag + dense)
    dz_mag = mag + dense
    wantH, wantW = D.candidate_backward_ref(bits(H), bits(W), cand, lse, g)
    # G itself is rounded to fp32 from a 64-bit sum of at most 256 gradients
    steps_v, steps_t = (V + 15) // 16 + 1, (T + 15) // 16 + 1 + blocks
    tolH = dz_err @ np.abs(Wf) + steps_v * 2 * U * (dz_mag @ np.abs(Wf)) + BF * np.abs(wantH) + 1e-37
    gotH = np_of(dH.float()).astype(np.float64)
    assert (np.abs(gotH - wantH) <= tolH).all(), float((np.abs(gotH - wantH) / tolH).max())
    if dW is not None:
        half = BF if dW.dtype == torch.bfloat16 else U
        tolW = dz_err.T @ np.abs(Hf) + steps_t * 2 * U * (dz_mag.T @ np.abs(Hf)) + half * np.abs(wantW) + 1e-37
        gotW = np_of(dW.float()).astype(np.float64)
        assert (np.abs(gotW - wantW) <= tolW).all(), float((np.abs(gotW - wantW) / tolW).max())


def backward_inputs(seed, T, d, V, K):
    H, W, cand = model(seed, T, d, V, K)
    rng = np.random.default_rng(seed + 1)
    g = (rng.standard_normal((T, K)) / max(T, 1)).astype(np.float32)
    _, _, lse = D.candidate_logprob_ref(bits(H), bits(W), cand)
    g[cand < 0] = np.nan                          # unused slots are not looked at
    return H, W, cand, lse.astype(np.float32), g


BWD_SHAPES = [(1, 8, 8, 1), (1, 256, 4096, 20), (3, 24, 136, 2), (130, 64, 304, 31), (257, 264, 1000, 33), (300, 320, 4104, 64),
              (256, 128, 2048, 129), (65, 512, 520, 256)]


@pytest.mark.parametrize("variant", [0, 1], ids=["pair", "cta"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, None], ids=["f32", "bf16", "frozen"])
@pytest.mark.parametrize("T,d,V,K", BWD_SHAPES)
def test_gradient_matches_the_oracle(ctx, T, d, V, K, dtype, variant):
    H, W, cand, lse, g = backward_inputs(T + V, T, d, V, K)
    ctx.set_tuning(0, 0, variant)
    try:
        dH, dW = gradient(ctx, H, W, cand, lse, g, dtype)
        assert ctx.check_device_errors() == 0
    finally:
        ctx.set_tuning(0, 0)
    check_gradient(H, W, cand, lse, np.nan_to_num(g), dH, dW)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_gradient_over_several_token_blocks(ctx, dtype):
    H, W, cand, lse, g = backward_inputs(11, 700, 128, 520, 12)
    ctx.set_tuning(0, 128)
    try:
        dH, dW = gradient(ctx, H, W, cand, lse, g, dtype)
        assert ctx.check_device_errors() == 0
    finally:
        ctx.set_tuning(0, 0)
    check_gradient(H, W, cand, lse, np.nan_to_num(g), dH, dW, blocks=6)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("T,d,V", [(1, 264, 20008), (2, 3584, 264), (29, 136, 19000), (129, 520, 4104), (300, 1032, 1160), (520, 8, 40)])
def test_gradient_of_few_tokens(ctx, T, d, V, dtype):
    """Products whose work is to write d_W, ragged in both directions; and fp32 sums on top of what was there."""
    H, W, cand, lse, g = backward_inputs(T + d, T, d, V, 9)
    dH, dW = gradient(ctx, H, W, cand, lse, g, dtype)
    check_gradient(H, W, cand, lse, np.nan_to_num(g), dH, dW)
    if dtype == torch.float32:
        base = torch.randn(V, d, device=device())
        _, more = gradient(ctx, H, W, cand, lse, g, accumulate=True, start=base)
        assert float((more - (base + dW)).abs().max()) <= 2 * U * float(base.abs().max() + dW.abs().max())
    assert ctx.check_device_errors() == 0


def test_gradient_accumulates_in_fp32_only(ctx):
    from paper_2507_01663_b200 import binding as B
    dev = device()
    H, W, cand, lse, g = backward_inputs(12, 100, 64, 200, 6)
    base = torch.randn(200, 64, device=dev)
    _, dW0 = gradient(ctx, H, W, cand, lse, g)
    _, dW1 = gradient(ctx, H, W, cand, lse, g, accumulate=True, start=base)
    assert float((dW1 - (base + dW0)).abs().max()) <= 2 * U * float(base.abs().max() + dW0.abs().max())
    with pytest.raises(B.AfError) as e:
        gradient(ctx, H, W, cand, lse, g, torch.bfloat16, accumulate=True)
    assert e.value.status == -1


def test_gradient_by_differences(ctx):
    """d_hidden against differences of the scores themselves, taken by the device: steps of a whole unit in a
    bf16 coordinate with exactly representable ends."""
    dev = device()
    T, d, V, K = 4, 64, 96, 5
    H, W, cand, _, g = backward_inputs(13, T, d, V, K)
    H = (H.float() * 8).round().div(8).to(torch.bfloat16)          # eighths: +- 1/64 stays exact for |h| < 4
    g = np.nan_to_num(g)

    def objective(h):
        lq, _, _ = score(ctx, h, W, cand)
        v = np_of(lq).astype(np.float64)
        v[~np.isfinite(v)] = 0.0
        return float((g * v).sum())

    _, _, lse = score(ctx, H, W, cand)
    dH, _ = gradient(ctx, H, W, cand, np_of(lse), g, None)
    h = 1.0 / 64
    for t, k in [(0, 0), (1, 5), (3, 63)]:
        up, dn = H.clone(), H.clone()
        up[t, k] += h
        dn[t, k] -= h
        assert float(up[t, k]) - float(dn[t, k]) == 2 * h
        num = (objective(up) - objective(dn)) / (2 * h)
        scale = float(np.abs(g[t]).sum()) * float(W.float().abs().max())
        # central differences are off by h^2 / 6 third derivatives (at most 6 |w|^3 sum |g|), dH by its roundings
        w = float(W.float().abs().max())
        tol = h * h * w ** 3 * float(np.abs(g[t]).sum()) + 2 * BF * scale + 2 * lse_tol(H, W, 10.0) * np.abs(g[t]).sum() / h
        assert abs(float(dH[t, k]) - num) <= tol


def test_gradient_of_an_empty_batch(ctx):
    dev = device()
    H, W = torch.zeros(0, 64, dtype=torch.bfloat16, device=dev), torch.zeros(16, 64, dtype=torch.bfloat16, device=dev)
    cand, f = torch.zeros(0, 3, dtype=torch.int32, device=dev), torch.zeros(0, 3, device=dev)
    for dtype in (torch.float32, torch.bfloat16):
        dW = torch.full((16, 64), 3.0, dtype=dtype, device=dev)
        ctx.candidate_logprob_backward(H, W, cand, torch.zeros(0, device=dev), f, torch.zeros_like(H), dW)
        assert not dW.any()
    dW = torch.full((16, 64), 3.0, device=dev)
    ctx.candidate_logprob_backward(H, W, cand, torch.zeros(0, device=dev), f, torch.zeros_like(H), dW, accumulate_dW=True)
    assert bool((dW == 3.0).all())


def test_refusals(ctx):
    from paper_2507_01663_b200 import binding as B
    dev = device()
    H, W = torch.zeros(4, 16, dtype=torch.bfloat16, device=dev), torch.zeros(24, 16, dtype=torch.bfloat16, device=dev)
    cand, lq = torch.zeros(4, 3, dtype=torch.int32, device=dev), torch.zeros(4, 3, device=dev)
    v = torch.zeros(4, device=dev)

    def status(f):
        with pytest.raises(B.AfError) as e:
            f()
        return e.value.status

    wide = torch.zeros(4, 257, dtype=torch.int32, device=dev)
    assert status(lambda: ctx.candidate_logprob(H, W, wide, torch.zeros(4, 257, device=dev))) == -2       # K > 256
    odd = torch.zeros(4, 12, dtype=torch.bfloat16, device=dev)
    assert status(lambda: ctx.candidate_logprob(odd, torch.zeros(24, 12, dtype=torch.bfloat16, device=dev), cand, lq)) == -3
    assert status(lambda: ctx.candidate_logprob(H, W, cand, None if False else lq, T=-1)) == -1
    assert status(lambda: ctx.candidate_logprob(H.view(-1)[1:1 + 48].view(3, 16), W, cand, lq, T=3)) == -3   # misaligned
    W12 = torch.zeros(12, 16, dtype=torch.bfloat16, device=dev)
    ctx.candidate_logprob(H, W12, cand, lq)                                                # fine without a backward
    assert status(lambda: ctx.candidate_logprob_backward(H, W12, cand, v, lq, torch.zeros_like(H),
                                                         torch.zeros(12, 16, device=dev))) == -3
    with pytest.raises(ValueError):
        ctx.candidate_logprob_backward(H, W, cand, v, lq, torch.zeros_like(H), torch.zeros(24, 16, dtype=torch.float16, device=dev))
    with pytest.raises(ValueError):                                                        # other list width
        ctx.candidate_logprob(H, W, cand, torch.zeros(4, 4, device=dev))
    with pytest.raises(ValueError):                                                        # strided
        ctx.candidate_logprob(H, W, torch.zeros(4, 6, dtype=torch.int32, device=dev)[:, ::2], lq)
    with pytest.raises(ValueError):                                                        # lists of 64-bit ids
        ctx.candidate_logprob(H, W, cand.long(), lq)
    with pytest.raises(ValueError):
        ctx.candidate_logprob(H, W, cand, lq.double())
    # the C entry itself: null pointers, vocabulary and token limits, types
    lib, h = ctx.lib, ctx.handle
    p = [t.data_ptr() for t in (H, W, cand, lq, v)]
    assert lib.af_candidate_logprob(None, p[0], p[1], p[2], 4, 3, 16, 24, p[3], None, None, None) == -1
    assert lib.af_candidate_logprob(h, None, p[1], p[2], 4, 3, 16, 24, p[3], None, None, None) == -1
    assert lib.af_candidate_logprob(h, p[0], p[1], p[2], 4, 3, 16, 24, None, None, None, None) == -1
    assert lib.af_candidate_logprob(h, p[0], p[1], p[2], 4, 0, 16, 24, p[3], None, None, None) == -1
    assert lib.af_candidate_logprob(h, p[0], p[1], p[2], 4, 3, 16, 1 << 24, p[3], None, None, None) == -2
    assert lib.af_candidate_logprob(h, p[0], p[1], p[2], 1 << 31, 3, 16, 24, p[3], None, None, None) == -2
    assert lib.af_candidate_logprob_backward(h, p[0], p[1], p[2], p[4], p[3], 4, 3, 16, 24, p[0], p[1], 2, 0, None) == -1
    assert lib.af_candidate_logprob_backward(h, p[0], p[1], p[2], None, p[3], 4, 3, 16, 24, p[0], p[1], 0, 0, None) == -1
    assert lib.af_reserve_candidates(h, 4, 3, 16, 24, 3, 0) == -1
    assert lib.af_reserve_candidates(h, 4, 300, 16, 24, 0, 0) == -2
    assert ctx.check_device_errors() == 0
