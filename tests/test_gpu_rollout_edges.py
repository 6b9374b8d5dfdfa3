"""Calls of the rollout operators that end somewhere: ids at the ends of int32, streams that have to be waited for, stores without blocks,
heads whose CTAs have an odd number of tiles."""
import numpy as np
import pytest
import torch

from gpu_util import device
from oracle import rollout_oracle as O
from rollout_util import f64, logits_tol, verify_case
from test_gpu_block_slots import case as blocks_case
from test_gpu_block_slots import check as check_blocks
from test_gpu_draft_verify import check as check_verify
from test_gpu_draft_verify import ctx  # noqa: F401  (a fixture)
from test_gpu_quant_logits import head
from test_gpu_quant_logits import run as run_logits
from test_gpu_rollout_step import Step, same

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mode", ["dense", "lookup", "greedy"])
@pytest.mark.parametrize("bad", [-1, 300, 2 ** 31 - 1, -2 ** 31])
def test_drafts_at_the_ends_of_their_type(ctx, bad, mode):  # noqa: F811
    """Every other draft; the requests that reach one stop there."""
    from paper_2507_01663_b200 import binding as B
    c = verify_case(21, 8, 4, 300, mode)
    c["ids"][::2] = bad
    want = check_verify(ctx, c, 0.0 if mode == "greedy" else 1.0, flags=B.DEVERR_TARGET_RANGE)
    assert (want["token"] != bad).all() or bad == -1


@pytest.mark.parametrize("given", ["current", "argument"])
def test_inputs_that_arrive_on_the_same_stream(ctx, given):  # noqa: F811
    """The buffers hold another step's inputs until the side stream, behind much work, copies the right ones in."""
    st, other = Step(ctx, 11, 9, 30), Step(ctx, 11, 9, 30)
    other.load(40)
    other.run()
    want = other.results()
    other.check(want)
    other.restore()
    st.run()
    assert not torch.equal(st.results()["token"], want["token"])
    st.load(12)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    names = "H Hd cu ids ua us length held table free count".split()
    with torch.cuda.stream(side):
        x = torch.randn(8192, 8192, device=device())
        for _ in range(8):
            x = x @ x * 1e-2
        for k in names:
            getattr(st, k).copy_(getattr(other, k))
        if given == "current":
            st.run()
    if given == "argument":
        plain, ctx_of = {}, st.ctx
        for name in ("quant_logits", "draft_verify", "block_slots"):
            plain[name] = getattr(ctx_of, name)
        st.ctx = type("OnSide", (), {k: staticmethod(lambda *a, f=f, **kw: f(*a, stream=side, **kw)) for k, f in plain.items()})
        st.run()
        st.ctx = ctx_of
    with torch.cuda.stream(side):
        got = {k: getattr(st, k).clone() for k in want}
    side.synchronize()
    same(want, got)
    assert ctx.check_device_errors() == 0


@pytest.mark.parametrize("R", [5, 60, 300, 1100])
@pytest.mark.parametrize("spare", ["none", "some"])
@pytest.mark.parametrize("shrink", [0.0, 0.2])
def test_a_store_without_enough_blocks(ctx, R, spare, shrink):  # noqa: F811
    c = blocks_case(R, R, 4, 9, 0 if spare == "none" else R // 2, shrink=shrink, most=20)
    want = check_blocks(ctx, c, in_place=R % 2 == 0)
    wants = [-(-int(l + g) // 4) > h for l, g, h in zip(c["length"], c["grow"], c["held"])]
    refused = [w and not g for w, g in zip(wants, want["granted"])]
    assert "blocks" in want["flags"] and sum(refused) > R // 10
    if spare == "some" and R > 5:                              # of five requests the first one wants more than there is
        assert any(w and g for w, g in zip(wants, want["granted"]))


@pytest.mark.parametrize("V", [37889, 38000, 50000, 56832])
@pytest.mark.parametrize("T", [1, 33, 64])
@pytest.mark.parametrize("group", [32, 128])
def test_ctas_with_two_and_three_boxes(ctx, V, T, group):  # noqa: F811
    """Above 32 tokens two boxes of 128 rows share a tile; on 148 SMs these heads leave some CTAs or all with a third."""
    H, words, scale = head(V, T, 192, V, group, any_scale=True)
    got = run_logits(ctx, H, words, scale, group)
    want, mag = O.quant_logits_ref(f64(H), words.numpy(), f64(scale), group)
    assert (np.abs(got - want) <= logits_tol(192, mag, want, False)).all()


@pytest.mark.parametrize("T", [1000, 65536])
def test_as_many_tokens_as_the_call_takes(ctx, T):  # noqa: F811
    H, words, scale = head(3, T, 64, 40, 32, any_scale=True)
    got = run_logits(ctx, H, words, scale, 32)
    want, mag = O.quant_logits_ref(f64(H), words.numpy(), f64(scale), 32)
    assert (np.abs(got - want) <= logits_tol(64, mag, want, False)).all()


@pytest.mark.parametrize("mode", ["dense", "lookup", "greedy"])
@pytest.mark.parametrize("passes", [False, True])
def test_requests_of_a_thousand_drafts(ctx, mode, passes):  # noqa: F811
    """Up to 1023 of one request; nearly equal distributions, so that many pass, or uniforms of 0 and first maxima, so that all do."""
    c = verify_case(31, 4, 1023, 60, mode, masked=False, noise=0.02)
    if passes:
        c["ua"][:] = 0.0
        if mode == "greedy":
            z = f64(c["target"])
            for r in range(4):
                for i in range(c["cu"][r + 1] - c["cu"][r]):
                    c["ids"][c["cu"][r] + i] = z[c["cu"][r] + r + i].argmax()
    want = check_verify(ctx, c, 0.0 if mode == "greedy" else 1.0, max_draft=1023)
    if passes:
        assert np.array_equal(want["n_emitted"], np.diff(c["cu"]) + 1) and want["n_emitted"].max() > 500
