"""af_distill_loss and af_distill_update against the fp64 oracle, and the calls as one training step."""
import math

import numpy as np
import pytest
import torch

from distill_util import BF, U, bits, cuts, dev_of, logit_tol, lse_tol, model, np_of, teacher_lists
from gpu_util import device
from oracle import distill_oracle as D
from test_gpu_candidate import check_gradient

pytestmark = pytest.mark.gpu

HOWS = [(0, 0, 1.0), (1, 0, 1.0), (0, 1, 1.0), (1, 1, 1.0), (0, 1, 2.5), (1, 1, 0.5), (0, 2, 1.0), (1, 2, 1.0)]


@pytest.fixture(scope="module")
def ctx():
    from paper_2507_01663_b200 import binding as B
    c = B.Context(0)
    yield c
    c.close()


def loss_call(ctx, lq, lt, cu, how, agg=0, scale=1.0, offset=0, **kw):
    """The call on device copies; offset > 0 puts the [T, K] tensors that many floats past a 16-byte boundary."""
    from paper_2507_01663_b200 import binding as B
    dev = device()
    T, K = lq.shape

    def place(x):
        buf = torch.full((T * K + 8,), 3.0, device=dev)
        view = buf[offset:offset + T * K].view(T, K)
        if x is not None:
            view.copy_(torch.as_tensor(x))
        return buf, view

    _, a = place(lq)
    _, b = place(lt)
    gbuf, g = place(None)
    out, token = B.new_distill_out(dev), torch.full((T,), 3.0, device=dev)
    ctx.distill_loss(a, b, dev_of(np.asarray(cu, np.int32)), out, token_loss=token, dcand=g, divergence=how[0], support=how[1], temperature=how[2],
                     agg_mode=agg, loss_scale=scale, **kw)
    res = B.read_distill_out(out)
    assert bool((gbuf[:offset] == 3.0).all()) and bool((gbuf[offset + T * K:] == 3.0).all())
    return res, np_of(token).astype(np.float64), np_of(g).astype(np.float64)


def row_scales(lq, lt, how):
    """Per token: what the relative errors of p, q (or a, b) act on -- for the loss and for the gradient.
    exp is off by (2^-22 + |x| 2^-23) relative and a row's sums add up to 256 terms in a tree (12 u): c below."""
    T, K = lq.shape
    sl, sg = np.zeros(T), np.zeros((T, K))
    tau = how[2] if how[1] == 1 else 1.0
    for t in range(T):
        on = np.flatnonzero(~np.isneginf(lt[t]))
        if on.size == 0:
            continue
        x, y = lt[t, on].astype(np.float64) / tau, lq[t, on].astype(np.float64) / tau
        c = 4 * U + (np.abs(x).max() + np.abs(y).max() + 1) * 2 * U + 16 * U
        a, b = np.exp(x), np.exp(y)
        if how[1] == 1:
            a, b = a / a.sum(), b / b.sum()
            d = np.abs(np.log(a) - np.log(b)) + 1 + np.abs(x) + np.abs(y)
            mean = (b * d).sum()
            # an error of the sums moves a log ratio by c absolutely; the loss and its parts by c times their size
            sl[t] = 4 * c * tau * tau * ((a + b) * d).sum()
            sg[t, on] = 4 * c * tau * (a + b * (d + mean))
        else:
            d = np.abs(x - y) + 1
            sl[t] = 4 * c * ((a + b) * d).sum()
            sg[t, on] = 4 * c * (a + b * d)
            if how[1] == 2:
                pr, qr = max(1 - a.sum(), D.TAIL_FLOOR), max(1 - b.sum(), D.TAIL_FLOOR)
                ratio = abs(math.log(pr / qr)) + 1
                # the masses are off by c absolutely.  d(pr log(pr / qr)) = (log(pr / qr) + 1) dpr - (pr / qr) dqr, and
                # for the other direction the same with pr and qr exchanged: either ratio can be the large one
                sl[t] += 8 * c * (ratio + pr / qr + qr / pr + 1)
                sg[t, on] += 8 * c * b * (ratio + 1 / qr + 1 / pr + pr / qr * (1 + 1 / qr))
    return sl, sg


def check_loss(lq, lt, cu, how, agg, scale, got):
    res, token, g = got
    want = D.distill_loss_ref(lq, lt, cu, how[0], how[1], how[2], agg, scale)
    sl, sg = row_scales(lq, lt, how)
    w = D.token_weights(cu, lq.shape[0], agg, scale)
    assert (np.abs(token - want["token_loss"]) <= sl + 2 * U * np.abs(want["token_loss"])).all()
    assert (np.abs(g - want["dcand"]) <= np.abs(w)[:, None] * sg + 6 * U * np.abs(want["dcand"])).all()
    assert not g[np.isneginf(lt)].any()
    assert abs(res["loss"] - want["loss"]) <= float((np.abs(w) * sl).sum()) + 8 * U * float((np.abs(w * want["token_loss"])).sum())
    for k in ("teacher_mass", "student_mass"):
        assert abs(res[k] - want[k]) <= 64 * U * max(1.0, want[k]) * 2
    assert res["n_tokens"] == lq.shape[0]


@pytest.mark.parametrize("how", HOWS, ids=[f"div{d}-sup{s}-t{t}" for d, s, t in HOWS])
@pytest.mark.parametrize("T,K", [(1, 1), (7, 2), (40, 3), (33, 8), (65, 9), (129, 16), (50, 31), (64, 50), (300, 64), (21, 65),
                                 (40, 100), (17, 128), (9, 129), (12, 255), (30, 256)])
def test_loss_matches_the_oracle(ctx, T, K, how):
    rng = np.random.default_rng(T * 1000 + K)
    lt, lq = teacher_lists(rng, T, K)
    cu = cuts(rng, min(5, T + 1), T)
    for agg, scale, offset in [(0, 1.0, 0), (1, 0.7, 0), (0, 1.0, 1), (1, 1.0, 2)]:
        got = loss_call(ctx, lq, lt, cu, how, agg, scale, offset)
        check_loss(lq, lt, cu, how, agg, scale, got)
    assert ctx.check_device_errors() == 0


def test_loss_with_many_sequences_and_rows(ctx):
    """More rows than one step of the grid, sequences of zero to a few tokens, and again with the same bits."""
    rng = np.random.default_rng(1)
    T, K = 60001, 10
    lt, lq = teacher_lists(rng, T, K)
    cu = cuts(rng, 20000, T)
    how = (1, 2, 1.0)
    a = loss_call(ctx, lq, lt, cu, how)
    b = loss_call(ctx, lq, lt, cu, how)
    assert a[0] == b[0] and np.array_equal(a[1], b[1]) and np.array_equal(a[2], b[2])
    sub = np.arange(0, T, 97)
    want_token = np.array([D.divergence_ref(lt[t], lq[t], *how)[0] for t in sub])
    sl, _ = row_scales(lq[sub], lt[sub], how)
    assert (np.abs(a[1][sub] - want_token) <= sl + 2 * U * np.abs(want_token)).all()
    n = np.diff(cu)
    w = np.repeat(1.0 / (np.maximum(n, 1) * float(len(n))), n)
    assert abs(a[0]["loss"] - float((w * a[1]).sum())) <= 4 * U * float((w * np.abs(a[1])).sum())
    assert ctx.check_device_errors() == 0


def test_loss_edges(ctx):
    from paper_2507_01663_b200 import binding as B
    dev = device()
    # no token at all
    out = B.new_distill_out(dev)
    e = torch.zeros(0, 4, device=dev)
    ctx.distill_loss(e, e, torch.zeros(1, dtype=torch.int32, device=dev), out, dcand=e, B=0)
    assert B.read_distill_out(out) == {"loss": 0.0, "teacher_mass": 0.0, "student_mass": 0.0, "n_tokens": 0}
    # certainty on either side: masses of exactly 1 leave the floor of the tail; zero probabilities
    lt = np.array([[0.0, -np.inf, -np.inf], [np.log(0.5), np.log(0.5), -np.inf], [0.0, -200.0, -300.0]], dtype=np.float32)
    lq = np.array([[0.0, -1.0, np.nan], [0.0, -np.inf, -3.0], [-0.5, -250.0, -1e30]], dtype=np.float32)
    for how in HOWS:
        res, token, g = loss_call(ctx, lq, lt, [0, 1, 3], how, 1)
        for t in range(3):
            want, wg = D.divergence_ref(lt[t], lq[t], *how)
            if math.isinf(want):
                assert token[t] == want
            else:
                assert token[t] == pytest.approx(want, abs=2e-5, rel=1e-5) or (math.isnan(want) and math.isnan(token[t]))
    # a NaN of the student in a present slot reaches its own token only
    lt, lq = teacher_lists(np.random.default_rng(2), 6, 4, short=False)
    lq[3, 1] = np.nan
    _, token, g = loss_call(ctx, lq, lt, [0, 6], (0, 1, 1.0), 1)
    assert np.isnan(token[3]) and np.isfinite(np.delete(token, 3)).all() and np.isfinite(np.delete(g, 3, 0)).all()
    ctx.check_device_errors()


def test_masks_of_the_lowest_value(ctx):
    """Absent slots marked by the lowest float32 or bf16 value instead of -inf, whole rows of them too: the same bits."""
    lt, lq = teacher_lists(np.random.default_rng(8), 60, 20)
    lq = np.where(np.isfinite(lq), lq, np.float32(-4.0))
    for how in HOWS:
        want = loss_call(ctx, lq, lt, [0, 25, 60], how)
        for low in (np.finfo(np.float32).min, torch.finfo(torch.bfloat16).min, -1e30):
            for under in (lq, np.where(np.isneginf(lt), np.float32(low), lq)):
                got = loss_call(ctx, under.astype(np.float32), np.where(np.isneginf(lt), np.float32(low), lt), [0, 25, 60], how)
                assert got[0] == want[0] and np.array_equal(got[1], want[1]) and np.array_equal(got[2], want[2])
    assert ctx.check_device_errors() == 0


def test_loss_leaves_rows_behind_the_batch(ctx):
    from paper_2507_01663_b200 import binding as B
    dev = device()
    lt, lq = teacher_lists(np.random.default_rng(3), 20, 6, short=False)
    g, token = torch.full((20, 6), 9.0, device=dev), torch.full((20,), 9.0, device=dev)
    ctx.distill_loss(dev_of(lq), dev_of(lt), dev_of(np.array([0, 13], np.int32)), B.new_distill_out(dev), token_loss=token,
                     dcand=g, T=13)
    assert bool((g[13:] == 9.0).all()) and bool((token[13:] == 9.0).all()) and bool((token[:13] != 9.0).all())
    assert ctx.check_device_errors() == 0


def test_loss_flags_bad_sequences(ctx):
    from paper_2507_01663_b200 import binding as B
    lt, lq = teacher_lists(np.random.default_rng(4), 8, 3, short=False)
    for cu in ([0, 5, 3, 8], [1, 8], [0, 7]):
        loss_call(ctx, lq, lt, np.array(cu, np.int32), (0, 1, 1.0))
        assert ctx.check_device_errors() & B.DEVERR_CU_SEQLENS
    loss_call(ctx, lq, lt, np.array([0, 8], np.int32), (0, 1, 1.0))
    assert ctx.check_device_errors() == 0


def test_loss_past_two_to_the_31_elements(ctx):
    from paper_2507_01663_b200 import binding as B
    dev = device()
    T, K = 8_400_000, 256
    gen = torch.Generator(device=dev).manual_seed(5)
    lt = torch.rand(T, K, generator=gen, device=dev).neg_().sub_(5.0)
    lq = torch.rand(T, K, generator=gen, device=dev).neg_().sub_(5.2)
    g, token = torch.empty(T, K, device=dev), torch.empty(T, device=dev)
    ctx.distill_loss(lq, lt, torch.tensor([0, T], dtype=torch.int32, device=dev), B.new_distill_out(dev), token_loss=token,
                     dcand=g, divergence=1, support=1, agg_mode=1)
    rows = [0, T // 2, T - 1]
    a, b = np_of(lt[rows]), np_of(lq[rows])
    sl, sg = row_scales(b, a, (1, 1, 1.0))
    for i, r in enumerate(rows):
        want, wg = D.divergence_ref(a[i], b[i], 1, 1)
        assert abs(float(token[r]) - want) <= sl[i] + 2 * U * abs(want)
        assert (np.abs(np_of(g[r]) - wg / T) <= sg[i] / T + 6 * U * np.abs(wg) / T).all()
    assert ctx.check_device_errors() == 0


def test_loss_refusals(ctx):
    from paper_2507_01663_b200 import binding as B
    dev = device()
    x, cu, out = torch.zeros(4, 3, device=dev), torch.tensor([0, 4], dtype=torch.int32, device=dev), B.new_distill_out(dev)

    def status(**kw):
        with pytest.raises(B.AfError) as e:
            ctx.distill_loss(x, x, cu, out, **kw)
        return e.value.status

    assert status(divergence=2) == -1 and status(divergence=-1) == -1 and status(support=3) == -1 and status(agg_mode=2) == -1
    assert status(temperature=0.0) == -1 and status(temperature=-1.0) == -1 and status(temperature=math.inf) == -1
    assert status(temperature=math.nan) == -1 and status(support=2, temperature=2.0) == -1 and status(support=0, temperature=2.0) == -1
    assert status(B=0) == -1 and status(T=-1) == -1
    with pytest.raises(B.AfError) as e:
        w = torch.zeros(4, 257, device=dev)
        ctx.distill_loss(w, w, cu, out)
    assert e.value.status == -2
    with pytest.raises(ValueError):
        ctx.distill_loss(x, torch.zeros(4, 4, device=dev), cu, out)
    with pytest.raises(ValueError):
        ctx.distill_loss(x, x.half(), cu, out)
    with pytest.raises(ValueError):
        ctx.distill_loss(x, x, cu, out, dcand=torch.zeros(3, 3, device=dev))
    lib, h = ctx.lib, ctx.handle
    prm = B.DistillParams(0, 1, 0, 1.0, 1.0)
    import ctypes
    assert lib.af_distill_loss(h, x.data_ptr(), None, cu.data_ptr(), 1, 4, 3, ctypes.byref(prm), out.data_ptr(), None, None, None) == -1
    assert lib.af_distill_loss(h, x.data_ptr(), x.data_ptr(), cu.data_ptr(), 1, 4, 3, ctypes.byref(prm), None, None, None, None) == -1
    assert lib.af_distill_loss(h, x.data_ptr(), x.data_ptr(), cu.data_ptr(), 1, 2 ** 31 - 65535, 3, ctypes.byref(prm), out.data_ptr(),
                               None, None, None) == -2
    assert ctx.check_device_errors() == 0


# --------------------------------------------------------------------------------------------- update
def update_inputs(seed, T, d, V, K, B):
    H, W, cand = model(seed, T, d, V, K)
    rng = np.random.default_rng(seed + 7)
    lt, _ = teacher_lists(rng, T, K, short=False)
    lt[cand < 0] = -np.inf
    return H, W, cand, lt.astype(np.float32), cuts(rng, B, T)


def update_call(ctx, H, W, cand, lt, cu, how, agg=0, scale=1.0, dtype=torch.float32, want=True, start=None):
    from paper_2507_01663_b200 import binding as B
    dev = device()
    T, K = cand.shape
    o = {"lq": torch.full((T, K), 5.0, device=dev), "lse": torch.full((T,), 5.0, device=dev),
         "dH": torch.full(H.shape, 5.0, dtype=torch.bfloat16, device=dev), "out": B.new_distill_out(dev),
         "dW": None if dtype is None else start.clone() if start is not None else torch.full(W.shape, 5.0, dtype=dtype, device=dev),
         "ent": torch.full((T,), 5.0, device=dev) if want else None,
         "token": torch.full((T,), 5.0, device=dev) if want else None,
         "g": torch.full((T, K), 5.0, device=dev) if want else None}
    ctx.distill_update(H.to(dev), W.to(dev), dev_of(cand), dev_of(lt), dev_of(cu), o["out"], o["lq"], o["lse"], o["dH"], o["dW"],
                       entropy=o["ent"], token_loss=o["token"], dcand=o["g"], divergence=how[0], support=how[1],
                       temperature=how[2], agg_mode=agg, loss_scale=scale, accumulate_dW=start is not None)
    o["res"] = B.read_distill_out(o["out"])
    return o


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, None], ids=["f32", "bf16", "frozen"])
@pytest.mark.parametrize("T,d,V,K,block,how,agg", [
    (1, 64, 136, 4, 0, (0, 1, 1.0), 0), (130, 64, 304, 31, 0, (1, 2, 1.0), 1), (300, 264, 1000, 33, 128, (0, 1, 2.0), 0),
    (257, 256, 4104, 64, 0, (0, 2, 1.0), 0), (500, 128, 520, 16, 128, (1, 0, 1.0), 1), (40, 320, 2048, 256, 0, (1, 1, 1.0), 0)])
def test_update_matches_the_oracle_stage_by_stage(ctx, T, d, V, K, block, how, agg, dtype):
    H, W, cand, lt, cu = update_inputs(T + K, T, d, V, K, min(4, T + 1))
    ctx.set_tuning(0, block)
    try:
        o = update_call(ctx, H, W, cand, lt, cu, how, agg, 1.3, dtype)
        assert ctx.check_device_errors() == 0
    finally:
        ctx.set_tuning(0, 0)
    want, went, wlse = D.candidate_logprob_ref(bits(H), bits(W), cand)
    z_max = float(np.abs(wlse).max()) + float(np.abs(want[np.isfinite(want)]).max())
    tz, tl = logit_tol(H, W, True), lse_tol(H, W, z_max)
    lq = np_of(o["lq"])
    ok = np.isfinite(want)
    assert np.array_equal(np.isfinite(lq), ok)
    assert np.abs(np_of(o["lse"]) - wlse).max() <= tl and np.abs(lq - want)[ok].max() <= tz + tl + 2 * U * z_max
    assert np.abs(np_of(o["ent"]) - went).max() <= 2 * tl + tz + 2 * (tl + 8 * U) * 2 * z_max
    # the loss and the gradients from the device's own log-probs, then the backward from its gradients
    check_loss(lq, lt, cu, how, agg, 1.3, (o["res"], np_of(o["token"]).astype(np.float64), np_of(o["g"]).astype(np.float64)))
    check_gradient(H, W, cand, np_of(o["lse"]), np_of(o["g"]), o["dH"], o["dW"], blocks=4)


@pytest.mark.parametrize("T,d,V,K", [(1, 64, 20008, 30), (5, 256, 9000, 256), (16, 136, 12000, 7), (17, 64, 2056, 3), (90, 128, 6152, 64)])
def test_update_of_few_tokens(ctx, T, d, V, K):
    """Rows cut into ranges of columns for dZ; scoring in one pass over W up to 16 tokens."""
    H, W, cand, lt, cu = update_inputs(T + V, T, d, V, K, 2)
    o = update_call(ctx, H, W, cand, lt, cu, (1, 2, 1.0), 1, 1.0, torch.bfloat16)
    assert ctx.check_device_errors() == 0
    want, went, wlse = D.candidate_logprob_ref(bits(H), bits(W), cand)
    ok = np.isfinite(want)
    z_max = float(np.abs(wlse).max()) + float(np.abs(want[ok]).max(initial=0.0))
    tz, tl = logit_tol(H, W, True), lse_tol(H, W, z_max)
    assert np.abs(np_of(o["lse"]) - wlse).max() <= tl
    assert np.array_equal(np.isfinite(np_of(o["lq"])), ok) and np.abs(np_of(o["lq"])[ok] - want[ok]).max(initial=0.0) <= tz + tl + 2 * U * z_max
    check_gradient(H, W, cand, np_of(o["lse"]), np_of(o["g"]), o["dH"], o["dW"])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, None], ids=["f32", "bf16", "frozen"])
def test_update_whose_last_block_is_a_few_tokens(ctx, dtype):
    H, W, cand, lt, cu = update_inputs(264, 264, 136, 4104, 21, 5)
    ctx.set_tuning(0, 128)
    try:
        o = update_call(ctx, H, W, cand, lt, cu, (0, 1, 1.0), 0, 1.0, dtype)
    finally:
        ctx.set_tuning(0, 0)
    assert ctx.check_device_errors() == 0
    want, _, wlse = D.candidate_logprob_ref(bits(H), bits(W), cand)
    ok = np.isfinite(want)
    z_max = float(np.abs(wlse).max()) + float(np.abs(want[ok]).max())
    tl = lse_tol(H, W, z_max)
    assert np.abs(np_of(o["lse"]) - wlse).max() <= tl
    assert np.abs(np_of(o["lq"])[ok] - want[ok]).max() <= logit_tol(H, W, True) + tl + 2 * U * z_max
    check_loss(np_of(o["lq"]), lt, cu, (0, 1, 1.0), 0, 1.0,
               (o["res"], np_of(o["token"]).astype(np.float64), np_of(o["g"]).astype(np.float64)))
    check_gradient(H, W, cand, np_of(o["lse"]), np_of(o["g"]), o["dH"], o["dW"], blocks=3)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_update_equals_the_three_calls(ctx, dtype):
    from paper_2507_01663_b200 import binding as B
    dev = device()
    H, W, cand, lt, cu = update_inputs(21, 400, 256, 2048, 24, 6)
    how = (0, 1, 1.5)
    o = update_call(ctx, H, W, cand, lt, cu, how, 0, 1.0, dtype)
    lq, ent, lse = torch.empty(400, 24, device=dev), torch.empty(400, device=dev), torch.empty(400, device=dev)
    Hd, Wd, cd = H.to(dev), W.to(dev), dev_of(cand)
    ctx.candidate_logprob(Hd, Wd, cd, lq, ent, lse)
    assert torch.equal(lq, o["lq"]) and torch.equal(lse, o["lse"]) and torch.equal(ent, o["ent"])
    out, token, g = B.new_distill_out(dev), torch.empty(400, device=dev), torch.empty(400, 24, device=dev)
    ctx.distill_loss(lq, dev_of(lt), dev_of(cu), out, token_loss=token, dcand=g, divergence=0, support=1, temperature=1.5)
    assert torch.equal(token, o["token"]) and torch.equal(g, o["g"]) and B.read_distill_out(out) == o["res"]
    dH, dW = torch.empty_like(o["dH"]), torch.empty_like(o["dW"])
    ctx.candidate_logprob_backward(Hd, Wd, cd, lse, g, dH, dW)
    # both round dZ and the result once; the recomputed logits differ in the last places
    assert float((dH.float() - o["dH"].float()).norm()) <= 2 * BF * float(dH.float().norm())
    assert float((dW.float() - o["dW"].float()).norm()) <= 2 * BF * float(dW.float().norm())
    assert ctx.check_device_errors() == 0


def test_update_without_the_optional_outputs_and_in_parts(ctx):
    """Nothing optional asked for gives the same required outputs; two half batches accumulate to the whole."""
    H, W, cand, lt, _ = update_inputs(22, 300, 128, 520, 9, 3)
    cu = np.array([0, 150, 300], np.int32)
    how = (1, 2, 1.0)
    a = update_call(ctx, H, W, cand, lt, cu, how)
    b = update_call(ctx, H, W, cand, lt, cu, how, want=False)
    assert a["res"] == b["res"] and all(torch.equal(a[k], b[k]) for k in ("lq", "lse", "dH", "dW"))
    half = np.array([0, 150], np.int32)
    first = update_call(ctx, H[:150], W, cand[:150], lt[:150], half, how, scale=0.5)
    both = update_call(ctx, H[150:], W, cand[150:], lt[150:], half, how, scale=0.5, start=first["dW"])
    assert float((both["dW"] - a["dW"]).norm()) <= 2 * BF * float(a["dW"].norm())
    assert first["res"]["loss"] + both["res"]["loss"] == pytest.approx(a["res"]["loss"], rel=1e-5)
    assert ctx.check_device_errors() == 0


def test_update_of_nothing_and_refusals(ctx):
    from paper_2507_01663_b200 import binding as B
    dev = device()
    W = torch.zeros(16, 64, dtype=torch.bfloat16, device=dev)
    z = lambda *s: torch.zeros(*s, device=dev)   # noqa: E731
    H0 = torch.zeros(0, 64, dtype=torch.bfloat16, device=dev)
    c0 = torch.zeros(0, 3, dtype=torch.int32, device=dev)
    out, dW = B.new_distill_out(dev), torch.full((16, 64), 2.0, dtype=torch.bfloat16, device=dev)
    ctx.distill_update(H0, W, c0, z(0, 3), torch.zeros(1, dtype=torch.int32, device=dev), out, z(0, 3), z(0), H0.clone(), dW, B=0)
    assert not dW.any() and B.read_distill_out(out)["n_tokens"] == 0
    H, c, cu = torch.zeros(4, 64, dtype=torch.bfloat16, device=dev), torch.zeros(4, 3, dtype=torch.int32, device=dev), \
        torch.tensor([0, 4], dtype=torch.int32, device=dev)

    def status(W=W, dW=None, **kw):
        with pytest.raises(B.AfError) as e:
            ctx.distill_update(H, W, c, z(4, 3), cu, out, z(4, 3), z(4), torch.zeros_like(H), dW, **kw)
        return e.value.status

    assert status(divergence=5) == -1 and status(support=2, temperature=3.0) == -1 and status(B=0) == -1
    assert status(W=torch.zeros(12, 64, dtype=torch.bfloat16, device=dev)) == -3
    assert status(dW=torch.zeros(16, 64, dtype=torch.bfloat16, device=dev), accumulate_dW=True) == -1
    assert ctx.check_device_errors() == 0
