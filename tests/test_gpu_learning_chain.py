"""The candidate, distillation and preference calls as they are used together: from the store to the gradients, in
graphs of one context, on streams of their own, and beside what a context's other calls leave in its workspace."""
import numpy as np
import pytest
import torch

from distill_util import BF, U, bits, cuts, dev_of, logit_tol, lse_tol, model, np_of, teacher_lists
from gpu_util import GRAD_RTOL, LOGP_TOL, device
from oracle import distill_oracle as D
from oracle import grpo_oracle as O
from test_gpu_candidate import check_gradient
from test_gpu_distill import check_loss
from test_gpu_preference import check as check_preference

pytestmark = pytest.mark.gpu


@pytest.fixture()
def ctx():
    from paper_2507_01663_b200 import binding as B
    c = B.Context(0)
    yield c
    c.close()


def store(seed, lengths, d, V, K):
    """Samples with hidden rows, listed ids and a teacher's log-probs of them, as a data store keeps them."""
    off = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)
    H, W, cand = model(seed, int(off[-1]), d, V, K)
    lt, _ = teacher_lists(np.random.default_rng(seed + 1), int(off[-1]), K, short=False)
    lt[cand < 0] = -np.inf
    return off, H, W, cand, lt.astype(np.float32)


def test_distillation_step_from_the_store(ctx):
    """Index list -> packed rows, ids and teacher columns (the lists travel as rows of 4 K bytes) -> scores -> loss ->
    gradients -> per-token losses written back; one sample is listed twice, one is empty."""
    from paper_2507_01663_b200 import binding as B
    dev = device()
    d, V, K = 128, 1000, 8
    off, H, W, cand, lt = store(31, [40, 0, 97, 3, 130, 61], d, V, K)
    idx = np.array([4, 2, 1, 0, 2], np.int32)
    rows = np.concatenate([np.arange(off[i], off[i + 1]) for i in idx])
    T = len(rows)
    Hs, cs, ls, Wd = H.to(dev), dev_of(cand), dev_of(lt), W.to(dev)

    def pack(column):                             # [sum L, n] bf16, or 4-byte lists seen as twice as many
        column = column if column.dtype == torch.bfloat16 else column.view(torch.bfloat16)
        out = {"cu_seqlens": torch.zeros(len(idx) + 1, dtype=torch.int32, device=dev),
               "hidden": torch.zeros(T, column.shape[1], dtype=torch.bfloat16, device=dev)}
        assert ctx.pack_microbatch({"tok_offset_host": off, "d": column.shape[1], "hidden": column}, idx, out) == T
        return out["hidden"], out["cu_seqlens"]

    h, cu = pack(Hs)
    ids, t = pack(cs)[0].view(torch.int32), pack(ls)[0].view(torch.float32)
    assert np.array_equal(np_of(ids), cand[rows]) and np.array_equal(np_of(t), lt[rows])
    lq, lse, token, g = (torch.empty(s, device=dev) for s in ((T, K), (T,), (T,), (T, K)))
    out, dH, dW = B.new_distill_out(dev), torch.empty(T, d, dtype=torch.bfloat16, device=dev), torch.empty(V, d, device=dev)
    how = (0, 1, 1.5)
    ctx.candidate_logprob(h, Wd, ids, lq, lse=lse)
    ctx.distill_loss(lq, t, cu, out, token_loss=token, dcand=g, divergence=0, support=1, temperature=1.5)
    ctx.candidate_logprob_backward(h, Wd, ids, lse, g, dH, dW)
    column = torch.full((int(off[-1]),), 7.0, device=dev)
    ctx.unpack_microbatch(off, idx[:4], [token], [column])
    assert ctx.check_device_errors() == 0

    Hp = H[torch.as_tensor(rows)]
    want, _, wlse = D.candidate_logprob_ref(bits(Hp), bits(W), cand[rows])
    ok = np.isfinite(want)
    z_max = float(np.abs(wlse).max() + np.abs(want[ok]).max())
    tz, tl = logit_tol(Hp, W, True), lse_tol(Hp, W, z_max)
    assert np.array_equal(np.isfinite(np_of(lq)), ok) and np.abs(np_of(lq)[ok] - want[ok]).max() <= tz + tl + 2 * U * z_max
    check_loss(np_of(lq), lt[rows], np_of(cu), how, 0, 1.0,
               (B.read_distill_out(out), np_of(token).astype(np.float64), np_of(g).astype(np.float64)))
    check_gradient(Hp, W, cand[rows], np_of(lse), np_of(g), dH, dW)
    back = np.full(int(off[-1]), 7.0, np.float32)
    back[rows[:T - 97]] = np_of(token)[:T - 97]
    assert np.array_equal(np_of(column), back)

    # and in one call
    o2, lq2, lse2, dH2, dW2 = B.new_distill_out(dev), torch.empty_like(lq), torch.empty_like(lse), torch.empty_like(dH), torch.empty_like(dW)
    ctx.distill_update(h, Wd, ids, t, cu, o2, lq2, lse2, dH2, dW2, divergence=0, support=1, temperature=1.5)
    assert torch.equal(lq2, lq) and torch.equal(lse2, lse) and B.read_distill_out(o2) == B.read_distill_out(out)
    check_gradient(Hp, W, cand[rows], np_of(lse), np_of(g), dH2, dW2)


def test_preference_step(ctx):
    """token_logprob of the policy and of the reference -> preference_loss -> policy_loss_backward."""
    from paper_2507_01663_b200 import binding as B
    dev = device()
    rng = np.random.default_rng(41)
    T, d, V = 700, 128, 1000
    H, W, _ = model(42, T, d, V, 1)
    W0 = (W.float() + 0.05 * torch.as_tensor(rng.standard_normal((V, d)).astype(np.float32)) / d ** 0.5).to(torch.bfloat16)
    y = rng.integers(0, V, T).astype(np.int32)
    cu = cuts(rng, 10, T)
    Hd, Wd, yd = H.to(dev), W.to(dev), dev_of(y)
    logp, ref, lse, g = (torch.empty(T, device=dev) for _ in range(4))
    ctx.token_logprob(Hd, Wd, yd, logp, lse=lse)
    ctx.token_logprob(Hd, W0.to(dev), yd, ref)
    out, pair, score = B.new_preference_out(dev), torch.empty(5, device=dev), torch.empty(10, device=dev)
    how = dict(beta=0.5, nll_coef=0.2, length_norm=True, pair_layout=1)
    ctx.preference_loss(logp, ref, dev_of(cu), out, pair, score, g, **how)
    dH, dW = torch.empty(T, d, dtype=torch.bfloat16, device=dev), torch.empty(V, d, device=dev)
    ctx.policy_loss_backward(Hd, Wd, yd, lse, g, dH, dW)
    assert ctx.check_device_errors() == 0
    for got, weight in ((logp, W), (ref, W0)):
        assert np.abs(np_of(got) - O.token_logprob_ref(bits(H), bits(weight), y)[0]).max() <= LOGP_TOL
    check_preference(np_of(logp), np_of(ref), cu, (B.read_preference_out(out), np_of(pair).astype(np.float64),
                                                   np_of(score).astype(np.float64), np_of(g).astype(np.float64)), **how)
    dH_ref, dW_ref = O.policy_loss_backward_ref(bits(H), bits(W), y, np_of(lse), np_of(g))
    assert np.linalg.norm(np_of(dH.float()) - dH_ref) <= GRAD_RTOL * np.linalg.norm(dH_ref)
    assert np.linalg.norm(np_of(dW) - dW_ref) <= GRAD_RTOL * np.linalg.norm(dW_ref)


class Work:
    """Buffers of one batch of every call, and the calls on them."""

    def __init__(self, seed, T, d, V, K, dtype):
        from paper_2507_01663_b200 import binding as B
        dev = device()
        self.shape = T, d, V, K
        self.H, self.W, self.cand = (x.to(dev) if torch.is_tensor(x) else dev_of(x) for x in model(seed, T, d, V, K))
        rng = np.random.default_rng(seed)
        self.cu = dev_of(cuts(rng, 6, T))
        self.logp, self.ref = -2 * torch.rand(T, device=dev), -2 * torch.rand(T, device=dev)
        self.lt = torch.empty(T, K, device=dev)
        self.fill(seed)
        f = lambda *s, t=torch.float32: torch.zeros(*s, dtype=t, device=dev)   # noqa: E731
        self.o = {"lq": f(T, K), "ent": f(T), "lse": f(T), "token": f(T), "g": f(T, K), "dH": f(T, d, t=torch.bfloat16),
                  "dW": f(V, d, t=dtype), "few": f(min(T, 9), K), "lq2": f(T, K), "lse2": f(T), "dH2": f(T, d, t=torch.bfloat16),
                  "dW2": f(V, d, t=dtype), "out": B.new_distill_out(dev), "out2": B.new_distill_out(dev),
                  "pref": B.new_preference_out(dev), "pair": f(3), "score": f(6), "dlogp": f(T)}

    def fill(self, seed):
        T, d, V, K = self.shape
        rng = np.random.default_rng(seed + 5)
        self.H.copy_(torch.as_tensor(rng.standard_normal((T, d)).astype(np.float32)))
        self.lt.copy_(torch.as_tensor(teacher_lists(rng, T, K, short=False)[0].astype(np.float32)))
        self.logp.copy_(torch.as_tensor((-2 * rng.random(T)).astype(np.float32)))

    def reserve(self, ctx):
        T, d, V, K = self.shape
        ctx.reserve_candidates(T, K, d, V, with_backward=2, dW_type=ctx._dtype(self.o["dW"]))
        ctx.reserve_preference(T, 6)

    def calls(self, ctx, which=(0, 1, 2, 3), stream=None):
        o = self.o
        if 0 in which:
            ctx.candidate_logprob(self.H, self.W, self.cand, o["lq"], o["ent"], o["lse"], stream=stream)
            ctx.distill_loss(o["lq"], self.lt, self.cu, o["out"], o["token"], o["g"], stream=stream)
            ctx.candidate_logprob_backward(self.H, self.W, self.cand, o["lse"], o["g"], o["dH"], o["dW"], stream=stream)
        if 1 in which:
            ctx.distill_update(self.H, self.W, self.cand, self.lt, self.cu, o["out2"], o["lq2"], o["lse2"], o["dH2"], o["dW2"],
                               stream=stream)
        if 2 in which:
            ctx.preference_loss(self.logp, self.ref, self.cu, o["pref"], o["pair"], o["score"], o["dlogp"], stream=stream)
        if 3 in which:
            ctx.candidate_logprob(self.H, self.W, self.cand, o["few"], T=o["few"].shape[0], stream=stream)

    def poison(self):
        for v in self.o.values():
            v.fill_(3)

    def results(self):
        torch.cuda.synchronize()
        return {k: v.clone() for k, v in self.o.items()}


def same(a, b):
    for k in a:
        assert torch.equal(a[k].view(torch.uint8), b[k].view(torch.uint8)), k


@pytest.mark.parametrize("T,d,V,K,block,dtype", [(300, 128, 1000, 12, 128, torch.bfloat16), (70, 256, 4104, 20, 0, torch.float32),
                                                 (513, 64, 520, 33, 0, torch.bfloat16), (9, 64, 2048, 5, 0, torch.float32)])
def test_graphs_of_one_context_replayed_in_turn(ctx, T, d, V, K, block, dtype):
    """Each call's kernels recorded into a graph of their own right after the reserving calls, replayed in two orders
    and on new data: the bits of the plain calls, and nothing is allocated."""
    w = Work(51, T, d, V, K, dtype)
    ctx.set_tuning(0, block)
    w.reserve(ctx)
    reserved = ctx.workspace_bytes()
    graphs = []
    for part in range(4):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            w.calls(ctx, (part,))
    assert ctx.workspace_bytes() == reserved
    for seed, order in ((51, (0, 1, 2, 3)), (52, (3, 2, 1, 0)), (53, (1, 0, 3, 2, 0, 1))):
        w.fill(seed)
        w.poison()
        for part in order:
            graphs[part].replay()
        replayed = w.results()
        w.poison()
        w.calls(ctx)
        same(w.results(), replayed)
    assert ctx.workspace_bytes() == reserved and ctx.check_device_errors() == 0
    H, W, cand = w.H.cpu(), w.W.cpu(), np_of(w.cand)
    check_gradient(H, W, cand, np_of(w.o["lse"]), np_of(w.o["g"]), w.o["dH"], w.o["dW"], blocks=4)


def test_two_contexts_on_two_streams():
    """Nothing is shared between contexts: work on two streams at the same time gives the bits of work alone."""
    from paper_2507_01663_b200 import binding as B
    ctxs = [B.Context(0), B.Context(0)]
    try:
        works = [Work(61, 300, 128, 4104, 12, torch.float32), Work(62, 190, 256, 2048, 7, torch.bfloat16)]
        for c, w in zip(ctxs, works):
            w.reserve(c)
            w.calls(c)
        alone = [w.results() for w in works]
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        for w in works:
            w.poison()
        torch.cuda.synchronize()
        for _ in range(5):
            for c, w, s in zip(ctxs, works, streams):
                w.calls(c, stream=s)
        for w, a in zip(works, alone):
            same(a, w.results())
        assert all(c.check_device_errors() == 0 for c in ctxs)
    finally:
        for c in ctxs:
            c.close()


def test_calls_of_different_kinds_in_turn(ctx):
    """The kernels of a call may start while the one before drains: every pair of calls in a row, on data that the
    first leaves to the second in the shared workspace, against each call alone."""
    w = Work(71, 260, 128, 2048, 16, torch.float32)
    w.calls(ctx)
    want = w.results()
    for first in range(4):
        for second in range(4):
            w.poison()
            torch.cuda.synchronize()
            w.calls(ctx, (first,))
            w.calls(ctx, (second,))
            w.calls(ctx, [p for p in range(4) if p not in (first, second)])
            same(want, w.results())
    assert ctx.check_device_errors() == 0


@pytest.mark.parametrize("T,d,V,K,block", [(300, 128, 4104, 12, 0), (300, 128, 1000, 12, 128), (40, 64, 2048, 20, 0), (9, 256, 520, 3, 0)])
def test_two_batches_in_turn_through_the_same_buffers(ctx, T, d, V, K, block):
    """Call after call without a pause, two sets of inputs and one of outputs and workspace: every call reads what the
    kernel before it in the same call wrote, not what the other batch had left there."""
    a, b = Work(95, T, d, V, K, torch.bfloat16), Work(96, T, d, V, K, torch.bfloat16)
    b.o = a.o
    ctx.set_tuning(0, block)
    want = []
    for w in (a, b):
        w.calls(ctx)
        want.append(w.results())
    assert not torch.equal(want[0]["g"], want[1]["g"])
    for n in range(1, 41):
        for i in range(n % 7 + 1):
            last = (n + i) & 1
            (a, b)[last].calls(ctx, (0, 1, 2, 3) if n % 2 else (1, 3, 0, 2))
        same(want[last], a.results())
    ctx.set_tuning(0, 0)
    assert ctx.check_device_errors() == 0


def test_what_is_reserved_holds_every_smaller_batch(ctx):
    """No call within the reserved sizes allocates, whatever way of launching its shape leads to."""
    from paper_2507_01663_b200 import binding as B
    dev = device()
    rng = np.random.default_rng(77)
    T, K, d, V = 1500, 40, 512, 6000
    ctx.set_tuning(0, 256)
    ctx.reserve_candidates(T, K, d, V, with_backward=2, dW_type=B.BF16)
    ctx.reserve_preference(T, 100)
    reserved = ctx.workspace_bytes()
    H, W = torch.randn(T * d, device=dev).to(torch.bfloat16), (0.05 * torch.randn(V * d, device=dev)).to(torch.bfloat16)
    shapes = [(T, K, d, V), (1, 1, 8, 8), (16, K, d, V), (17, K, d, V), (128, K, d, V), (129, K, d, V), (257, 3, 64, 5992)]
    shapes += [(int(rng.integers(1, T + 1)), int(rng.integers(1, K + 1)), 8 * int(rng.integers(1, d // 8 + 1)),
                8 * int(rng.integers(1, V // 8 + 1))) for _ in range(25)]
    for t, k, e, v in shapes:
        h, w = H[:t * e].view(t, e), W[:v * e].view(v, e)
        cand = torch.randint(0, v, (t, k), dtype=torch.int32, device=dev)
        lt, lq, g = -5 * torch.rand(t, k, device=dev), torch.empty(t, k, device=dev), torch.empty(t, k, device=dev)
        lse, dH, dW = torch.empty(t, device=dev), torch.empty_like(h), torch.empty_like(w)
        cu = dev_of(cuts(rng, 4, t))
        ctx.candidate_logprob(h, w, cand, lq, lse=lse)
        first = lq.clone()
        ctx.distill_update(h, w, cand, lt, cu, B.new_distill_out(dev), lq, lse, dH, dW, dcand=g)
        ctx.candidate_logprob_backward(h, w, cand, lse, g, dH, dW)
        ctx.preference_loss(lse, None, cu, B.new_preference_out(dev), T=t)
        assert ctx.workspace_bytes() == reserved, (t, k, e, v)
        assert float((first - lq).abs().max()) <= 1e-4, (t, k, e, v)
    ctx.set_tuning(0, 0)
    assert ctx.check_device_errors() == 0


@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_dw_ready_event(ctx, dtype, fused):
    """Another stream that waits for the event sees the whole d_W, although d_hidden may still be under way."""
    w = Work(81, 900, 128, 2048, 8, dtype)
    ctx.set_tuning(0, 256)
    w.calls(ctx, (0, 1))
    want = w.results()["dW2" if fused else "dW"]
    event, side = torch.cuda.Event(), torch.cuda.Stream()
    event.record()                                   # an event exists on the device from its first record on
    ctx.set_dw_ready_event(event)
    try:
        w.poison()
        torch.cuda.synchronize()
        w.calls(ctx, (1 if fused else 0,))
        with torch.cuda.stream(side):
            side.wait_event(event)
            seen = w.o["dW2" if fused else "dW"].clone()
        torch.cuda.synchronize()
        assert torch.equal(seen, want)
    finally:
        ctx.set_dw_ready_event(None)
    assert ctx.check_device_errors() == 0


@pytest.mark.parametrize("T,d,V", [(20000, 256, 8200), (19000, 520, 8192)])
def test_gradient_whose_last_tiles_are_cut_along_the_vocabulary(ctx, T, d, V):
    """A few more tiles of d_hidden than there are pairs of SMs: the whole ones and the cut ones, on sampled rows
    (every 128-row boundary and rows of both kinds among them)."""
    dev = device()
    rng = np.random.default_rng(91)
    H, W, cand = model(92, T, d, V, 6)
    g = (rng.standard_normal((T, 6)) / T).astype(np.float32)
    lq, lse = torch.empty(T, 6, device=dev), torch.empty(T, device=dev)
    dH = torch.full((T, d), 7.0, dtype=torch.bfloat16, device=dev)
    Hd, Wd, cd = H.to(dev), W.to(dev), dev_of(cand)
    ctx.candidate_logprob(Hd, Wd, cd, lq, lse=lse)
    ctx.set_tuning(0, (T + 127) // 128 * 128)
    try:
        ctx.candidate_logprob_backward(Hd, Wd, cd, lse, dev_of(g), dH)
    finally:
        ctx.set_tuning(0, 0)
    assert ctx.check_device_errors() == 0
    rows = np.unique(np.concatenate([np.arange(0, T, 128), np.arange(127, T, 128), rng.integers(0, T, 200), [T - 1]]))
    r = torch.as_tensor(rows)
    check_gradient(H[r], W, cand[rows], np_of(lse)[rows], g[rows], dH[r.to(dev)], None)
