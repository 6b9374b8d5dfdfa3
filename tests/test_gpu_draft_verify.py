"""af_draft_verify against the oracle: tokens and counts exactly, log-probs within a derived tolerance."""
import math

import numpy as np
import pytest
import torch

from gpu_util import device
from oracle import rollout_oracle as O
from rollout_util import f32, f64, i32, logp_tol, verify_case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2507_01663_b200 import binding as B
    c = B.Context(0)
    yield c
    c.close()


def place(t, pad, offset):
    """The rows of a CPU matrix on the device, `pad` apart, from an address that is only aligned to the type."""
    n, V = t.shape
    buf = torch.full((n * (V + pad) + offset,), float("nan"), dtype=t.dtype, device=device())     # between rows lies what may not be read
    rows = buf[offset:].view(n, V + pad)[:, :V]
    rows.copy_(t)
    return rows


def run(ctx, c, temperature=1.0, max_draft=None, pad=0, offset=0, logp=True, spare=3):
    dev = device()
    R, D = len(c["cu"]) - 1, len(c["ids"])
    token, lp, n = (torch.full((D + R + spare,), -7, dtype=torch.int32, device=dev), torch.full((D + R + spare,), -7.0, device=dev),
                    torch.full((R + spare,), -7, dtype=torch.int32, device=dev))
    ctx.draft_verify(place(c["target"], pad, offset), None if c["draft"] is None else place(c["draft"], pad, offset), i32(c["ids"]),
                     i32(c["cu"]), f32(c["ua"]), f32(c["us"]), token, n, logp=lp if logp else None, max_draft=max_draft,
                     temperature=temperature, R=R, D=D)
    torch.cuda.synchronize()
    for t in (token[D + R:], lp[D + R:], n[R:]):
        assert bool((t == -7).all())
    return token[:D + R].cpu().numpy(), lp[:D + R].cpu().numpy().astype(np.float64), n[:R].cpu().numpy()


def reference(c, temperature=1.0, max_draft=None):
    with np.errstate(all="ignore"):
        return O.draft_verify_ref(f64(c["target"]), None if c["draft"] is None else f64(c["draft"]), c["ids"], c["cu"], c["ua"], c["us"],
                                  temperature, max_draft)


def check(ctx, c, temperature=1.0, flags=0, max_draft=None, **how):
    from paper_2507_01663_b200 import binding as B
    token, lp, n = run(ctx, c, temperature, max_draft, **how)
    want = reference(c, temperature, max_draft)
    assert want["margin"] > 1e-11                  # sums in 64 bits decide as the oracle's do
    w = want["written"]
    assert np.array_equal(token[w], want["token"][w]) and np.array_equal(n, want["n_emitted"])
    assert (token[~w] == -7).all() and (lp[~w] == -7.0).all()
    exact = want["logp"]
    assert np.array_equal(np.isnan(lp[w]), np.isnan(exact[w]))
    z = f64(c["target"])
    z = z[np.isfinite(z)]
    spread = (z.max() - z.min()) / (temperature or 1.0) if z.size else 0.0
    ok = w & np.isfinite(exact)
    assert np.abs(lp[ok] - exact[ok]).max(initial=0.0) <= logp_tol(c["target"].shape[1], spread)
    bits = {"cu": B.DEVERR_CU_SEQLENS, "range": B.DEVERR_TARGET_RANGE, "distribution": B.DEVERR_DISTRIBUTION}
    assert ctx.check_device_errors() == sum(bits[f] for f in want["flags"]) == flags
    return want


MODES = ["dense", "lookup", "greedy"]


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("V", [1, 2, 3, 7, 8, 33, 255, 256, 257, 1000, 2047, 4099, 8200, 32000])
def test_vocabularies(ctx, V, mode):
    want = check(ctx, verify_case(V, 6, 4, V, mode), 0.0 if mode == "greedy" else 1.0)
    assert (want["n_emitted"] > 0).all()


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("R,most", [(1, 0), (1, 1), (1, 7), (2, 3), (9, 8), (37, 5), (150, 3), (333, 1), (700, 2)])
def test_requests(ctx, R, most, mode):
    check(ctx, verify_case(R * 10 + most, R, most, 517, mode), 0.0 if mode == "greedy" else 0.9, max_draft=most)


@pytest.mark.parametrize("ttype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pad,offset", [(0, 0), (1, 0), (3, 1), (8, 7), (13, 5)])
def test_types_pitches_and_alignment(ctx, ttype, dtype, pad, offset):
    check(ctx, verify_case(pad, 8, 4, 2501, "dense", ttype, dtype), pad=pad, offset=offset)
    check(ctx, verify_case(pad, 8, 4, 2501, "lookup", ttype, dtype), pad=pad, offset=offset)


@pytest.mark.parametrize("mode", MODES)
def test_a_whole_vocabulary_in_many_slices(ctx, mode):
    check(ctx, verify_case(1, 3, 4, 152064, mode, torch.float32, torch.bfloat16), 0.0 if mode == "greedy" else 1.0)
    check(ctx, verify_case(2, 1, 0, 151643, mode, torch.bfloat16, torch.float32), 0.0 if mode == "greedy" else 0.7)


@pytest.mark.parametrize("temperature", [1e-4, 0.01, 0.3, 1.0, 7.0, 1e4])
@pytest.mark.parametrize("mode", ["dense", "lookup"])
def test_temperatures(ctx, temperature, mode):
    check(ctx, verify_case(5, 20, 3, 700, mode), temperature)


def test_without_log_probs(ctx):
    c = verify_case(6, 12, 4, 900)
    token, lp, n = run(ctx, c, logp=False)
    want = reference(c)
    assert np.array_equal(token, want["token"]) and np.array_equal(n, want["n_emitted"]) and (lp == -7.0).all()


def uniform_case(V, ids, ua, us, draft=None):
    n = len(ids)
    return {"target": torch.zeros(n + 1, V), "draft": draft, "ids": np.array(ids, np.int32), "cu": np.array([0, n], np.int32),
            "ua": np.array(ua, np.float32), "us": np.array([us], np.float32)}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_borders_exactly(ctx, dtype):
    """Weights that are powers of two: both sides of every comparison are exact, and a tie decides as the definition says."""
    step = 2.0 ** -24
    for V in (4, 256, 4096):
        for u, passes in ((1 / V, False), (1 / V - step, True), (1 / V + step, False), (0.0, True)):
            c = uniform_case(V, [V // 2], [u], 0.5)
            c["target"] = c["target"].to(dtype)
            token, _, n = run(ctx, c)
            assert n[0] == 1 + passes and (token[0] == V // 2) == passes
        for k in (0, 1, V // 2, V - 1):                        # C_v = v + 1
            token, _, _ = run(ctx, {**uniform_case(V, [], [], k / V), "target": torch.zeros(1, V, dtype=dtype)})
            assert token[0] == k
            if k:
                token, _, _ = run(ctx, uniform_case(V, [], [], k / V - step))
                assert token[0] == k - 1
    assert ctx.check_device_errors() == 0


def test_uniforms_outside_their_range(ctx):
    for u, y in ((-1.0, 0), (1.0, 255), (7.0, 255), (float("nan"), 0)):
        token, _, _ = run(ctx, uniform_case(256, [], [], u))
        assert token[0] == y
    token, _, n = run(ctx, uniform_case(256, [3], [float("nan")], 0.0))
    assert n[0] == 1 and token[0] == 0


def test_near_ties_are_decided_in_64_bits(ctx):
    """u at the float below, at and above p / q: fp32 sums could not tell."""
    c = verify_case(11, 40, 3, 3001, "dense")
    z, zq = f64(c["target"]), f64(c["draft"])
    for r in range(40):
        for i in range(c["cu"][r + 1] - c["cu"][r]):
            k = c["cu"][r] + i
            ratio = O.softmax(z[k + r], 1.0)[c["ids"][k]] / O.softmax(zq[k], 1.0)[c["ids"][k]]
            if ratio < 1.0:
                u = np.float32(ratio)
                u = np.nextafter(u, np.float32(r % 2), dtype=np.float32) if r % 3 == 0 else u
                c["ua"][k] = u
    token, _, n = run(ctx, c)
    want = reference(c)
    assert 1e-13 < want["margin"] < 1e-7 and np.array_equal(token, want["token"]) and np.array_equal(n, want["n_emitted"])
    assert ctx.check_device_errors() == 0


def test_masks_that_leave_one_token_or_share_none(ctx):
    c = verify_case(12, 6, 1, 600, masked=False)
    c = verify_case(12, 6, 1, 600, masked=False) if c["cu"][-1] else c
    c["cu"] = np.arange(7, dtype=np.int32)
    c["target"], c["draft"] = torch.randn(12, 600), torch.randn(6, 600)
    c["ids"], c["ua"], c["us"] = np.arange(6, dtype=np.int32) * 90 + 5, np.full(6, 0.5, np.float32), np.linspace(0, 0.99, 6).astype(np.float32)
    c["target"][0], c["target"][0, 5] = -math.inf, 0.0            # only the draft is left: passes
    c["target"][2, 95] = -math.inf                                # the draft is masked: does not
    c["target"][4, ::2], c["draft"][2, 1::2] = -math.inf, -math.inf     # disjoint supports; the draft has no mass of its own
    c["draft"][3] = c["target"][6]                                # the same distribution
    c["target"][8], c["target"][8, 7] = torch.finfo(torch.float32).min, 3.0     # a mask of the type's lowest value
    c["draft"][5], c["draft"][5, 455] = -math.inf, -1e30          # one token of the draft, far below zero
    want = check(ctx, c)
    assert want["token"][0] == 5 and want["token"][2] != 95 and want["token"][8] == 7
    lookup = dict(c, draft=None)
    check(ctx, lookup)
    check(ctx, lookup, 0.0)


def test_nothing_left_after_a_certain_draft(ctx):
    """p = 1 at the draft: it passes whatever u is below 1; where u is not, what is left is nothing, and p is drawn from."""
    c = uniform_case(300, [17], [1.0], 0.9)
    c["target"][0], c["target"][0, 17] = -math.inf, 2.0
    token, lp, n = run(ctx, c)
    assert token.tolist() == [17, -1] and n[0] == 1 and lp[0] == 0.0
    c["draft"] = c["target"][:1].clone()
    token, lp, n = run(ctx, c)
    assert token.tolist() == [17, -1] and n[0] == 1
    assert ctx.check_device_errors() == 0


@pytest.mark.parametrize("what", [float("nan"), math.inf, "masked"])
@pytest.mark.parametrize("mode", MODES)
def test_rows_that_are_no_distribution(ctx, what, mode):
    from paper_2507_01663_b200 import binding as B
    c = verify_case(13, 5, 3, 400, mode)
    c["cu"] = np.array([0, 3, 6, 9, 12, 15], np.int32)
    rng = np.random.default_rng(1)
    c["target"], c["ids"] = torch.as_tensor(rng.standard_normal((20, 400)).astype(np.float32)), rng.integers(0, 400, 15).astype(np.int32)
    c["draft"] = None if mode != "dense" else torch.as_tensor(rng.standard_normal((15, 400)).astype(np.float32))
    c["ua"], c["us"] = np.zeros(15, np.float32), rng.random(5).astype(np.float32)       # u = 0: everything passes
    if mode == "greedy":
        for r in range(5):
            for i in range(3):
                c["ids"][3 * r + i] = int(c["target"][4 * r + i].argmax())

    def spoil(t, row):
        if what == "masked":
            t[row] = -math.inf
        else:
            t[row, 399] = what
    spoil(c["target"], 0)                                      # first draft of request 0
    spoil(c["target"], 4 + 2)                                  # last draft of request 1
    spoil(c["target"], 8 + 3)                                  # the row behind request 2's drafts
    if mode == "greedy":
        c["ids"][9] = (c["ids"][9] + 1) % 400                  # request 3 stops before its spoiled row
    else:
        c["ua"][9] = 1e9
    spoil(c["target"], 12 + 1)
    if mode == "dense":
        spoil(c["draft"], 13)                                  # second draft of request 4
    want = check(ctx, c, 0.0 if mode == "greedy" else 1.0, flags=B.DEVERR_DISTRIBUTION)
    assert want["n_emitted"].tolist() == [0, 2, 3, 1, 1 if mode == "dense" else 4]


@pytest.mark.parametrize("mode", MODES)
def test_drafts_outside_the_vocabulary(ctx, mode):
    from paper_2507_01663_b200 import binding as B
    c = verify_case(14, 6, 3, 300, mode)
    c["ids"][::2] = [-1, 300, 2 ** 31 - 1, -2 ** 31][0]
    if len(c["ids"]) > 2:
        c["ids"][2] = 300
    check(ctx, c, 0.0 if mode == "greedy" else 1.0, flags=B.DEVERR_TARGET_RANGE)


def test_parts_of_cu_that_cannot_be(ctx):
    from paper_2507_01663_b200 import binding as B
    base = verify_case(15, 5, 3, 200)
    for cu in ([0, 2, 1, 3, 4, 4], [0, 1, 2, 3, 9, 4], [0, -3, 1, 2, 3, 4], [1, 1, 2, 3, 4, 4], [0, 1, 2, 3, 4, 3], [0, 4, 4, 4, 4, 4]):
        rng = np.random.default_rng(2)
        c = dict(base, cu=np.array(cu, np.int32), target=torch.as_tensor(rng.standard_normal((9, 200)).astype(np.float32)),
                 draft=torch.as_tensor(rng.standard_normal((4, 200)).astype(np.float32)), ids=rng.integers(0, 200, 4).astype(np.int32),
                 ua=rng.random(4).astype(np.float32), us=rng.random(5).astype(np.float32))
        token, lp, n = run(ctx, c, max_draft=3)
        want = reference(c, max_draft=3)
        assert "cu" in want["flags"] and ctx.check_device_errors() == B.DEVERR_CU_SEQLENS
        ok = [r for r in range(5) if want["n_emitted"][r] > 0]
        assert np.array_equal(n, want["n_emitted"]) and (token[~want["written"]] == -7).all()
        assert ok or cu == [0, 4, 4, 4, 4, 4]


def test_results_repeat_bit_for_bit(ctx):
    c = verify_case(16, 50, 4, 9000)
    first = run(ctx, c)
    for _ in range(4):
        assert all(np.array_equal(a, b) for a, b in zip(first, run(ctx, c)))


def test_rows_past_2_31_elements(ctx):
    """Row offsets past 32 bits: the last requests of a batch of 3e9 logits."""
    dev = device()
    V, R, most = 152064, 6600, 2
    rows, D = R * 3, R * 2
    target = torch.empty(rows, V, dtype=torch.bfloat16, device=dev)
    target.normal_(0.0, 2.0)
    cu = np.arange(R + 1, dtype=np.int32) * 2
    rng = np.random.default_rng(4)
    ids = target[: 1].float().argmax().item() * np.ones(D, np.int32)
    tail = 4                                                   # requests that are checked
    for k in range(D - 2 * tail, D):
        ids[k] = int(target[k + k // 2].float().argmax())
    ua, us = rng.random(D).astype(np.float32) * 0.02, rng.random(R).astype(np.float32)
    token, n = torch.empty(rows, dtype=torch.int32, device=dev), torch.empty(R, dtype=torch.int32, device=dev)
    ctx.draft_verify(target, None, i32(ids), i32(cu), f32(ua), f32(us), token, n, max_draft=most)
    want = O.draft_verify_ref(f64(target[-3 * tail:]), None, ids[-2 * tail:], np.arange(tail + 1) * 2, ua[-2 * tail:], us[-tail:])
    assert np.array_equal(token[-3 * tail:].cpu().numpy(), want["token"]) and np.array_equal(n[-tail:].cpu().numpy(), want["n_emitted"])
    assert ctx.check_device_errors() == 0
    del target
    torch.cuda.empty_cache()


def test_refusals(ctx):
    dev = device()
    c = verify_case(17, 3, 2, 64)
    R, D = 3, len(c["ids"])
    t, q, ids, cu, ua, us = c["target"].to(dev), c["draft"].to(dev), i32(c["ids"]), i32(c["cu"]), f32(c["ua"]), f32(c["us"])
    token, n = torch.zeros(D + R, dtype=torch.int32, device=dev), torch.zeros(R, dtype=torch.int32, device=dev)
    p = lambda x: x.data_ptr()
    ok = dict(t=p(t), tt=0, tp=64, q=p(q), qt=0, qp=64, ids=p(ids), cu=p(cu), ua=p(ua), us=p(us), R=R, D=D, V=64, most=2, tau=1.0, token=p(token), lp=None, n=p(n))
    call = lambda **k: ctx.lib.af_draft_verify(ctx.handle, *{**ok, **k}.values(), None)
    assert call() == 0 and call(R=0, D=0) == 0 and call(tau=0.0, ua=None, us=None, q=None) == 0
    for name in ("t", "ids", "cu", "ua", "us", "token", "n"):
        assert call(**{name: None}) == -1
    assert call(R=-1) == -1 and call(D=-1) == -1 and call(V=0) == -1 and call(most=-1) == -1
    assert call(tt=2) == -1 and call(qt=-1) == -1
    for tau in (-1.0, 5e-5, 2e4, math.inf, math.nan):
        assert call(tau=tau) == -1
    assert call(tp=63) == -2 and call(qp=63) == -2 and call(most=1024) == -2 and call(D=7) == -2 and call(R=(1 << 24) // 3 + 1) == -2
    assert call(t=p(t) + 2) == -3 and call(q=p(q) + 1, qt=1) == -3
    torch.cuda.synchronize()
    with pytest.raises(ValueError):
        ctx.draft_verify(t[:-1], q, ids, cu, ua, us, token, n)
