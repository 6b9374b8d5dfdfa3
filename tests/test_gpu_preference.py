"""af_preference_loss against the fp64 oracle."""
import ctypes
import math

import numpy as np
import pytest
import torch

from distill_util import U, cuts, dev_of, np_of
from gpu_util import device
from oracle import distill_oracle as D

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2507_01663_b200 import binding as B
    c = B.Context(0)
    yield c
    c.close()


def call(ctx, logp, ref, cu, offset=0, T=None, **how):
    from paper_2507_01663_b200 import binding as B
    dev = device()
    n = len(logp)
    P = (len(cu) - 1) // 2

    def place(x):
        buf = torch.full((n + 8,), 3.0, device=dev)
        v = buf[offset:offset + n]
        if x is not None:
            v.copy_(torch.as_tensor(x))
        return buf, v

    a = place(logp)[1]
    b = None if ref is None else place(ref)[1]
    gbuf, g = place(None)
    out, pair, score = B.new_preference_out(dev), torch.full((P,), 3.0, device=dev), torch.full((2 * P,), 3.0, device=dev)
    ctx.preference_loss(a, b, dev_of(np.asarray(cu, np.int32)), out, pair, score, g, T=T, **how)
    used = n if T is None else T
    assert bool((gbuf[:offset] == 3.0).all()) and bool((gbuf[offset + used:] == 3.0).all())
    return B.read_preference_out(out), np_of(pair).astype(np.float64), np_of(score).astype(np.float64), np_of(g)[:used].astype(np.float64)


def f(x):
    return float(np.float32(x))


def check(logp, ref, cu, got, **how):
    """Sums, pairs and coefficients are taken in 64 bits from the fp32 inputs: what is left is one rounding of
    each output to fp32 (u), and of the sums in fp64 (n 2^-53 of their absolute terms)."""
    how = {k: (f(v) if isinstance(v, float) else v) for k, v in how.items()}
    want = D.preference_loss_ref(logp, ref, cu, **how)
    res, pair, score, g = got
    n = max(len(logp), 1)
    mass = float(np.abs(np.asarray(logp, np.float64)).sum() + (0 if ref is None else np.abs(np.asarray(ref, np.float64)).sum()))
    slack = n * 2.0 ** -52 * (mass + 1) * how.get("beta", 0.1)
    rel = 2 * U
    assert (np.abs(score - want["seq_score"]) <= rel * np.abs(want["seq_score"]) + slack).all()
    steep = 1 + (2.0 / how.get("beta", 0.1) ** 2 * (1 + np.abs(want["seq_score"]).max(initial=0)) if how.get("kind") == 1 else 0)
    assert (np.abs(pair - want["pair_loss"]) <= rel * np.abs(want["pair_loss"]) + slack * steep + 1e-12).all()
    gm = np.abs(want["dlogp"]).max(initial=0.0)
    assert (np.abs(g - want["dlogp"]) <= rel * np.abs(want["dlogp"]) + slack * steep * gm + 1e-14 * gm).all()
    for k, name in (("loss", "loss"), ("pair_loss", "pair_loss_mean"), ("nll", "nll"), ("chosen_score", "chosen_score"),
                    ("rejected_score", "rejected_score")):
        assert abs(res[k] - want[name]) <= rel * abs(want[name]) + slack * steep + 1e-12, k
    assert abs(res["accuracy"] - want["accuracy"]) <= 2 * U and res["n_pairs"] == want["n_pairs"]


def data(seed, T, B):
    rng = np.random.default_rng(seed)
    logp = (-2.0 * rng.random(T)).astype(np.float32)
    ref = (logp + 0.2 * rng.standard_normal(T)).astype(np.float32)
    return logp, ref, cuts(rng, B, T)


SIZES = [(1, 2), (2, 2), (255, 2), (256, 2), (257, 2), (300, 8), (1024, 4), (5000, 10), (20000, 400), (2049, 3000), (70000, 6)]


@pytest.mark.parametrize("kind", [0, 1, 2])
@pytest.mark.parametrize("T,B", SIZES)
def test_matches_the_oracle(ctx, T, B, kind):
    logp, ref, cu = data(T + B, T, B)
    for i, (r, norm, layout, nll, eps) in enumerate([(ref, False, 0, 0.0, 0.0), (ref, True, 1, 0.5, 0.1), (None, True, 0, 0.0, 0.2),
                                                     (None, False, 1, 0.25, 0.0)]):
        how = dict(kind=kind, beta=0.1 if not norm else 2.0, label_smoothing=eps if kind == 0 else 0.0, margin=0.3 * i, nll_coef=nll,
                   length_norm=norm, pair_layout=layout, loss_scale=1.0 + i)
        got = call(ctx, logp, r, cu, offset=i % 3, **how)
        check(logp, r, cu, got, **how)
    assert ctx.check_device_errors() == 0


def test_sequences_at_every_offset_of_a_slice(ctx):
    """Borders just before, on and after multiples of 256, and sequences that span many of them."""
    edges = [0, 1, 255, 256, 257, 511, 511, 512, 1024, 1025, 2047, 2048, 2304, 4095, 4096, 9000, 9001]
    cu = np.array(edges, np.int32)
    logp, ref, _ = data(3, 9001, 2)
    for layout in (0, 1):
        check(logp, ref, cu, call(ctx, logp, ref, cu, pair_layout=layout), pair_layout=layout)
    assert ctx.check_device_errors() == 0


def test_empty_sequences_and_batches(ctx):
    logp, ref, _ = data(4, 600, 2)
    for cu in ([0, 0, 0, 600, 600], [0, 600, 600, 600, 600], [0] * 5 + [300, 300, 300, 600], [0, 300] + [300] * 2000 + [600]):
        cu = np.array(cu, np.int32)
        how = dict(length_norm=True, nll_coef=0.5, margin=0.1)
        check(logp, ref, cu, call(ctx, logp, ref, cu, **how), **how)
    none = np.zeros(0, np.float32)
    check(none, none, np.zeros(5, np.int32), call(ctx, none, none, np.zeros(5, np.int32)))     # two pairs, no token
    got = call(ctx, none, none, np.zeros(1, np.int32))
    assert got[0]["n_pairs"] == 0 and got[0]["loss"] == 0.0
    assert ctx.check_device_errors() == 0


def test_same_bits_and_optional_outputs(ctx):
    from paper_2507_01663_b200 import binding as B
    dev = device()
    logp, ref, cu = data(5, 30000, 50)
    a, b = call(ctx, logp, ref, cu), call(ctx, logp, ref, cu)
    assert a[0] == b[0] and all(np.array_equal(x, y) for x, y in zip(a[1:], b[1:]))
    out = B.new_preference_out(dev)
    ctx.preference_loss(dev_of(logp), dev_of(ref), dev_of(cu), out)
    assert B.read_preference_out(out) == a[0]
    got = call(ctx, logp, ref, np.array([0, 100, 213], np.int32), T=213)         # rows behind the batch stay
    check(logp[:213], ref[:213], [0, 100, 213], got)


def test_extremes(ctx):
    """Scores far apart, and infinities and NaN that stay in their own pair."""
    logp = np.array([-1e4, 0.0, 0.0, -1e4, -1.0, -1.0], np.float32)
    cu = np.arange(7, dtype=np.int32)
    for kind in (0, 1, 2):
        check(logp, None, cu, call(ctx, logp, None, cu, kind=kind, beta=1.0), kind=kind, beta=1.0)
    logp[0], logp[2] = np.nan, -np.inf
    res, pair, score, g = call(ctx, logp, None, cu, beta=1.0)
    assert np.isnan(pair[0]) and np.isnan(g[0]) and pair[1] == np.inf and g[2] == pytest.approx(-1 / 3) and np.isfinite(pair[2])
    assert np.isfinite(g[2:]).all() and pair[2] == pytest.approx(math.log(2.0))


def test_infinities_stay_in_their_own_short_sequence(ctx):
    """Sequences of 0 to 9 tokens, some with an infinity, a NaN or 1e30: the others are as if those were not there."""
    rng = np.random.default_rng(12)
    lengths = rng.integers(0, 10, 4000)
    cu = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    T = int(cu[-1])
    logp = (-2.0 * rng.random(T)).astype(np.float32)
    ref = (logp + 0.2 * rng.standard_normal(T)).astype(np.float32)
    spoilt = logp.copy()
    at = rng.choice(T, 300, replace=False)
    spoilt[at] = rng.choice(np.array([np.nan, -np.inf, -1e30], np.float32), 300)
    hit = np.zeros(2000, bool)
    hit[(np.searchsorted(cu, at, side="right") - 1) // 2] = True
    a, b = call(ctx, logp, ref, cu), call(ctx, spoilt, ref, cu)
    check(logp, ref, cu, a)
    assert 100 < hit.sum() < 500 and np.array_equal(a[1][~hit], b[1][~hit])
    assert np.array_equal(a[2].reshape(-1, 2)[~hit], b[2].reshape(-1, 2)[~hit])
    token = np.repeat(~hit, lengths.reshape(-1, 2).sum(1))
    assert np.array_equal(a[3][token], b[3][token])


def test_long_batch_against_float64_sums(ctx):
    """2^26 tokens in sequences of very uneven length."""
    from paper_2507_01663_b200 import binding as B
    dev = device()
    T = (1 << 26) + 13
    g = torch.Generator(device=dev).manual_seed(3)
    logp = -torch.rand(T, generator=g, device=dev)
    ref = logp + 0.1 * torch.randn(T, generator=g, device=dev)
    rng = np.random.default_rng(6)
    cu = np.concatenate([[0, T // 2], np.sort(rng.integers(T // 2, T, 1997)), [T]]).astype(np.int32)
    B_ = len(cu) - 1
    cu = cu if B_ % 2 == 0 else np.delete(cu, 5)
    score = torch.empty(len(cu) - 1, device=dev)
    d = torch.empty(T, device=dev)
    ctx.preference_loss(logp, ref, dev_of(cu), B.new_preference_out(dev), seq_score=score, dlogp=d, beta=0.5)
    run = torch.nn.functional.pad(torch.cumsum(logp.double() - ref.double(), 0), (1, 0))
    at = torch.as_tensor(cu.astype(np.int64), device=dev)
    want = 0.5 * (run[at[1:]] - run[at[:-1]])
    assert float((score.double() - want).abs().max()) <= 1e-5 * float(want.abs().max()) * 1e-2 + 2 * U * float(want.abs().max())
    x = want[0::2] - want[1::2]
    coef = torch.empty(len(cu) - 1, dtype=torch.float64, device=dev)
    coef[0::2] = -0.5 * torch.sigmoid(-x) / x.numel()
    coef[1::2] = 0.5 * torch.sigmoid(-x) / x.numel()
    full = torch.repeat_interleave(coef, at[1:] - at[:-1])
    assert float((d.double() - full).abs().max()) <= 4 * U * float(full.abs().max())
    assert ctx.check_device_errors() == 0


def test_flags_and_refusals(ctx):
    from paper_2507_01663_b200 import binding as B
    dev = device()
    logp, ref, _ = data(7, 40, 2)
    for cu in ([0, 30, 20, 35, 40], [0, 10, 20, 30, 39], [2, 10, 20, 30, 40], [0, -5, 50, 30, 40]):
        call(ctx, logp, ref, np.array(cu, np.int32))
        assert ctx.check_device_errors() & B.DEVERR_CU_SEQLENS
    check(logp, ref, [0, 30, 40], call(ctx, logp, ref, [0, 30, 40]))
    assert ctx.check_device_errors() == 0
    x, cu, out = dev_of(logp), torch.tensor([0, 20, 40], dtype=torch.int32, device=dev), B.new_preference_out(dev)

    def status(cu=cu, **kw):
        with pytest.raises(B.AfError) as e:
            ctx.preference_loss(x, None, cu, out, **kw)
        return e.value.status

    assert status(kind=3) == -1 and status(kind=-1) == -1 and status(pair_layout=2) == -1
    assert status(beta=0.0) == -1 and status(beta=-1.0) == -1 and status(beta=math.nan) == -1 and status(beta=math.inf) == -1
    assert status(label_smoothing=1.0) == -1 and status(label_smoothing=-0.1) == -1 and status(label_smoothing=math.nan) == -1
    assert status(B=1) == -2 and status(B=0) == -1 and status(T=-1) == -1
    prm = B.PreferenceParams(0, 0, 0, 0.1, 0.0, 0.0, 0.0, 1.0)
    lib, h = ctx.lib, ctx.handle
    assert lib.af_preference_loss(h, None, None, cu.data_ptr(), 2, 40, ctypes.byref(prm), out.data_ptr(), None, None, None, None) == -1
    assert lib.af_preference_loss(h, x.data_ptr(), None, None, 2, 40, ctypes.byref(prm), out.data_ptr(), None, None, None, None) == -1
    assert lib.af_preference_loss(h, x.data_ptr(), None, cu.data_ptr(), 2, 2 ** 31 - 65535, ctypes.byref(prm), out.data_ptr(),
                                  None, None, None, None) == -2
    assert lib.af_reserve_preference(h, -1, 2) == -1 and lib.af_reserve_preference(h, 10, 3) == -2
    with pytest.raises(ValueError):
        ctx.preference_loss(x.double(), None, cu, out)
    assert ctx.check_device_errors() == 0
