"""Pins of the rollout oracle: closed forms, brute force, frequencies, invariants."""
import math
from fractions import Fraction

import numpy as np
import pytest

from oracle import rollout_oracle as O


def bf16_values(rng, shape, spread=1.0):
    x = (rng.standard_normal(shape) * spread).astype(np.float32)
    return (x.view(np.uint32) & 0xffff0000).view(np.float32).astype(np.float64)


def test_five_bits_by_fractions():
    rng = np.random.default_rng(0)
    for x in [1.0, 31.0, 33.0, 35.0, 1 / 7.0, 2.0 ** -90 * 33] + list(rng.random(200) * 10.0 ** rng.integers(-20, 20, 200)):
        got = Fraction(O.five_bits(x))
        e = math.frexp(x)[1] - 5
        low = math.floor(Fraction(x) / Fraction(2) ** e)
        lo, hi = low * Fraction(2) ** e, (low + 1) * Fraction(2) ** e
        d = Fraction(x) - lo, hi - Fraction(x)
        want = lo if d[0] < d[1] or (d[0] == d[1] and low % 2 == 0) else hi
        assert got == want


@pytest.mark.parametrize("group", [32, 64, 128])
def test_quantized_values_are_nearest_and_bf16(group):
    W = bf16_values(np.random.default_rng(group), (5, 224), 0.02)
    W[1, :32] = 0.0
    q, s, v = O.quantize_head_ref(W, group)
    assert np.abs(q).max() == 7 and (q[1, :32] == 0).all()
    unit = np.repeat(s, group, axis=1)[:, :224]
    assert (np.abs(W - v) <= unit / 2 * (1 + 1e-15)).all()                     # the nearest multiple, also at the largest weight
    bits = v.astype(np.float32).view(np.uint32)
    assert (bits & 0xffff == 0).all() and np.array_equal(v.astype(np.float32).astype(np.float64), v)
    assert np.array_equal(O.unpack_digits(O.pack_digits(q)), q)


def test_halves_go_away_from_zero_and_odd_groups():
    w = np.zeros(32)
    w[:5] = [7.0, 2.5, -2.5, 0.5, -0.5]                                        # scale 1
    q, s = O.quantize_group(w)
    assert s == 1.0 and list(q[:5]) == [7, 3, -3, 1, -1]
    assert O.quantize_group(np.full(32, 2.0 ** -101))[1] == 0.0
    for bad in (math.nan, math.inf, -2.0 ** 121):
        w[9] = bad
        q, s = O.quantize_group(w)
        assert math.isnan(s) and (q == 0).all()


def test_logits_by_hand():
    q = np.zeros((1, 32), dtype=np.int64)
    q[0, :8] = [1, -2, 3, -4, 5, -6, 7, -8]
    H = np.zeros((2, 32))
    H[0, :8] = 1.0
    H[1, 3] = 2.0
    z, mag = O.quant_logits_ref(H, O.pack_digits(q), np.array([[0.5]]), 32)
    assert z.tolist() == [[-2.0], [-4.0]] and mag.tolist() == [[18.0], [4.0]]


def test_weights_are_rounded_to_bf16():
    import torch
    x = np.random.default_rng(5).standard_normal(4000) * 10.0 ** np.random.default_rng(6).integers(-20, 20, 4000)
    x = np.concatenate([x.astype(np.float32), np.float32([1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8, -1 - 2.0 ** -8, 0.0])])
    assert np.array_equal(O.to_bf16(x), torch.as_tensor(x).to(torch.bfloat16).double().numpy())


def test_verification_has_the_targets_law():
    """Rejection sampling gives the target's distribution whatever the draft's is: exact, by integrating over the uniforms on a
    grid that their borders fall on."""
    p, q = np.array([1, 3, 4, 0, 8.0]) / 16, np.array([8, 2, 2, 4, 0.0]) / 16
    with np.errstate(divide="ignore"):
        target, draft = np.log(np.stack([p, p])), np.log(q)[None]
    mass = np.zeros(5)
    n = 11 * 16                     # what is left of p - q holds 1, 2 and 8 elevenths: each border lies between two grid points
    us = (np.arange(n) + 0.5) / n
    for x in range(5):
        if q[x] == 0:
            continue
        ratio = min(1.0, p[x] / q[x])
        for u, w in ((ratio / 2, ratio), ((1 + ratio) / 2, 1 - ratio)):        # passes, does not
            if w == 0:
                continue
            if u < ratio:
                mass[x] += q[x] * w
                continue
            out = [O.draft_verify_ref(target, draft, [x], [0, 1], [u], [v])["token"][0] for v in us]
            mass += q[x] * w * np.bincount(out, minlength=5) / n
    assert np.abs(mass - p).max() < 1e-12


def test_lookup_and_greedy_and_edges():
    z = np.log(np.array([[1, 2, 1.0], [2, 1, 1]]) / 4)
    ref = lambda x, u, v, **k: O.draft_verify_ref(z, None, [x], [0, 1], [u], [v], **k)
    assert ref(1, 0.49, 0.0)["token"].tolist() == [1, 0]                       # passes, then the second row's first token
    out = ref(1, 0.51, 0.6)
    assert out["token"].tolist() == [2, -1] and out["n_emitted"].tolist() == [1]    # without 1: halves for 0 and 2
    assert abs(out["logp"][0] - math.log(0.25)) < 1e-15 and out["logp"][1] == 0.0
    assert ref(1, 0.0, 0.0, temperature=0)["token"].tolist() == [1, 0]
    assert ref(2, 0.0, 0.0, temperature=0)["token"].tolist() == [1, -1]
    assert ref(9, 0.0, 0.0)["flags"] == {"range"} and ref(-1, 0.0, 0.3)["token"][0] == 1
    bad = z.copy()
    bad[1, 0] = math.nan
    out = O.draft_verify_ref(bad, None, [1], [0, 1], [0.1], [0.0])
    assert out["token"].tolist() == [1, -1] and out["n_emitted"][0] == 1 and "distribution" in out["flags"]
    # the same distribution twice: what is not let through has nothing left, the target itself is drawn from
    out = O.draft_verify_ref(z, z[:1], [1], [0, 1], [1.0], [0.3])
    assert out["token"].tolist() == [1, -1]


@pytest.mark.parametrize("seed", range(20))
def test_blocks_are_neither_lost_nor_shared(seed):
    rng = np.random.default_rng(seed)
    R, bs, per, n = 9, int(rng.integers(1, 6)), 8, 40
    table, free = np.full((R, per), -1), list(range(n))
    length, held, count = np.zeros(R, int), np.zeros(R, int), n
    for step in range(30):
        grow = rng.integers(0, 7, R)
        grow = np.minimum(grow, per * bs - length)
        out = O.block_slots_ref(length, grow, held, table, free, count, bs, 200)
        table, free, count, held = out["table"], out["free"], out["free_count"], np.array(out["held"])
        mine = [int(b) for r in range(R) for b in table[r, :held[r]]]
        assert sorted(mine + free[:count]) == list(range(n))
        slots = [s for s in out["slot"] if s is not None and s >= 0]
        assert len(set(slots)) == len(slots)
        for r in range(R):
            if out["granted"][r]:
                assert held[r] * bs >= length[r] + grow[r]
                kept = rng.integers(0, grow[r] + 1)
                length[r] += kept
                if rng.random() < 0.15:
                    length[r] = 0
    assert out["cu"][-1] == grow.sum()
