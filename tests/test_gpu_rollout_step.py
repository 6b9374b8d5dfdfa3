"""The rollout calls as a speculative decoding step uses them: a head's codes, logits of target and draft, the verdict, and rows for
what was emitted; eager, captured, on other streams, and in turn with batches of other sizes."""
import numpy as np
import pytest
import torch

from gpu_util import device
from oracle import rollout_oracle as O
from rollout_util import bf16, f64, i32, logits_tol, logp_tol, verify_case
from test_gpu_block_slots import case as blocks_case
from test_gpu_block_slots import check as check_blocks
from test_gpu_draft_verify import check as check_verify

pytestmark = pytest.mark.gpu


@pytest.fixture()
def ctx():
    from paper_2507_01663_b200 import binding as B
    c = B.Context(0)
    yield c
    c.close()


class Step:
    """R requests, D drafts, all buffers fixed."""

    def __init__(self, ctx, seed, R, D, V=1003, d=256, block_size=4, dtype=torch.float32):
        dev = device()
        self.ctx, self.R, self.D, self.V, self.d, self.bs = ctx, R, D, V, d, block_size
        rng = np.random.default_rng(seed)
        W = bf16(rng.standard_normal((V, d)) * 0.15)
        small = bf16(f64(W) + rng.standard_normal((V, d)) * 0.01)
        self.values = torch.empty(V, d, dtype=torch.bfloat16, device=dev)
        self.heads = []
        for w, group, values in ((W, 128, self.values), (small, 32, None)):
            codes = torch.empty(V, d // 8, dtype=torch.int32, device=dev)
            scale = torch.empty(V, -(-d // group), dtype=torch.bfloat16, device=dev)
            ctx.quantize_head(w.to(dev), codes, scale, group=group, values=values)
            self.heads.append((codes, scale, group))
        self.H = torch.empty(D + R, d, dtype=torch.bfloat16, device=dev)
        self.Hd = torch.empty(max(D, 1), d, dtype=torch.bfloat16, device=dev)
        self.target = torch.empty(D + R, V + 5, dtype=dtype, device=dev)[:, :V]          # rows apart
        self.draft = torch.empty(max(D, 1), V, dtype=torch.float32, device=dev)
        self.ids, self.cu = i32(np.zeros(D)), i32(np.zeros(R + 1))
        self.ua, self.us = torch.empty(D, device=dev), torch.empty(R, device=dev)
        self.token, self.n = i32(np.zeros(D + R)), i32(np.zeros(R))
        self.logp = torch.empty(D + R, device=dev)
        per = 64
        self.n_blocks = R * per
        self.length, self.held, self.count = i32(np.zeros(R)), i32(np.zeros(R)), i32([0])
        self.table, self.free = i32(np.zeros((R, per))), i32(np.zeros(self.n_blocks))
        self.held_out, self.count_out, self.granted = i32(np.zeros(R)), i32([0]), i32(np.zeros(R))
        self.cu_new, self.position = i32(np.zeros(R + 1)), i32(np.zeros(D + R))
        self.slot = torch.empty(D + R, dtype=torch.int64, device=dev)
        self.load(seed + 1)

    def load(self, seed):
        """New inputs in the same buffers."""
        rng = np.random.default_rng(seed)
        R, D, d = self.R, self.D, self.d
        cuts = np.sort(rng.integers(0, D + 1, R - 1))
        cu = np.concatenate([[0], cuts, [D]]).astype(np.int32)
        H = rng.standard_normal((D + R, d))
        rows = np.array([int(cu[r]) + r + i for r in range(R) for i in range(cu[r + 1] - cu[r])], dtype=int)
        self.H.copy_(bf16(H))
        self.cu.copy_(torch.as_tensor(cu))
        if D:
            self.Hd.copy_(bf16(H[rows]))
            z = f64(self.Hd.cpu()) @ f64(self.values).T
            self.ids.copy_(torch.as_tensor((z - np.log(-np.log(rng.random(z.shape)))).argmax(1).astype(np.int32)))
        self.ua.copy_(torch.as_tensor(rng.random(D).astype(np.float32)))
        self.us.copy_(torch.as_tensor(rng.random(R).astype(np.float32)))
        length = rng.integers(0, 100, R).astype(np.int32)
        held = (-(-length // self.bs)).astype(np.int32)
        ids = rng.permutation(self.n_blocks).astype(np.int32)
        table, at = np.full(tuple(self.table.shape), -5, np.int32), 0
        for r in range(R):
            table[r, :held[r]] = ids[at:at + held[r]]
            at += held[r]
        free = np.full(self.n_blocks, -9, np.int32)
        free[:self.n_blocks - at] = ids[at:]
        self.before = (length, held, table, free, self.n_blocks - at)
        self.length.copy_(torch.as_tensor(length))
        self.restore()
        for t in (self.token, self.n, self.cu_new, self.slot, self.position, self.held_out, self.count_out, self.granted):
            t.fill_(-7)
        self.logp.fill_(-7.0)
        self.target.fill_(7.0)
        self.draft.fill_(7.0)

    def restore(self):
        length, held, table, free, count = self.before
        self.held.copy_(torch.as_tensor(held))
        self.table.copy_(torch.as_tensor(table))
        self.free.copy_(torch.as_tensor(free))
        self.count.fill_(count)

    def run(self):
        ctx, D, R = self.ctx, self.D, self.R
        (codes, scale, group), (dcodes, dscale, dgroup) = self.heads
        ctx.quant_logits(self.H, codes, scale, self.target, group=group)
        ctx.quant_logits(self.Hd, dcodes, dscale, self.draft, group=dgroup, T=D)
        ctx.draft_verify(self.target, self.draft, self.ids, self.cu, self.ua, self.us, self.token, self.n, logp=self.logp)
        ctx.block_slots(self.length, self.n, self.held, self.table, self.free, self.count, self.held_out, self.count_out,
                        self.cu_new, self.slot, block_size=self.bs, position=self.position, granted=self.granted)

    def results(self):
        torch.cuda.synchronize()
        names = "target draft token logp n table free held_out count_out granted cu_new slot position".split()
        return {k: getattr(self, k).clone() for k in names}

    def check(self, got):
        token, logp, n = got["token"].cpu().numpy(), f64(got["logp"]), got["n"].cpu().numpy()
        z, zq = f64(got["target"]), f64(got["draft"][:self.D])
        cu = self.cu.cpu().numpy()
        H, W = f64(self.H), f64(self.values)
        mag = np.abs(H) @ np.abs(W).T
        off = logits_tol(self.d, mag, H @ W.T, got["target"].dtype is torch.bfloat16)
        assert (np.abs(z - H @ W.T) <= off).all()
        want = O.draft_verify_ref(z, zq, self.ids.cpu().numpy(), cu, self.ua.cpu().numpy(), self.us.cpu().numpy())
        assert want["margin"] > 1e-11 and want["flags"] == set() and want["written"].all()
        assert np.array_equal(token, want["token"]) and np.array_equal(n, want["n_emitted"])
        assert np.abs(logp - want["logp"]).max() <= logp_tol(self.V, z.max() - z.min())
        # the same log-probs by the scoring path over the values that the codes stand for.  Logits off by `off` at most move a
        # log-prob by twice that; the scoring path's own bound is 2e-3.
        some = torch.as_tensor(np.flatnonzero(token >= 0), device=device())
        scored = torch.empty(len(some), device=device())
        self.ctx.token_logprob(self.H[some].contiguous(), self.values, got["token"][some].contiguous(), scored)
        assert np.abs(f64(scored) - logp[token >= 0]).max() <= 2e-3 + 2 * off.max() + logp_tol(self.V, z.max() - z.min())
        length, held, table, free, count = self.before
        ref = O.block_slots_ref(length, n, held, table, free, count, self.bs, self.D + self.R)
        total = int(n.sum())
        for name, key in (("table", "table"), ("free", "free"), ("held_out", "held"), ("granted", "granted"), ("cu_new", "cu")):
            assert np.array_equal(got[name].cpu().numpy(), np.asarray(ref[key])), name
        assert int(got["count_out"]) == ref["free_count"]
        for name in ("slot", "position"):
            x = got[name].cpu().numpy()
            assert np.array_equal(x[:total], np.asarray(ref[name][:total])) and (x[total:] == -7).all(), name
        assert self.ctx.check_device_errors() == 0


def same(a, b):
    for k in a:
        assert torch.equal(a[k], b[k]), k


@pytest.mark.parametrize("R,D,dtype", [(1, 0, torch.float32), (1, 4, torch.float32), (7, 20, torch.bfloat16), (40, 60, torch.float32)])
def test_a_step(ctx, R, D, dtype):
    st = Step(ctx, R + D, R, D, dtype=dtype)
    for seed in (3, 4):
        st.load(seed)
        st.run()
        st.check(st.results())


def test_captured_steps_of_two_sizes_share_a_context(ctx):
    ctx.reserve_rollout(40, 60)
    small, large = Step(ctx, 1, 3, 9), Step(ctx, 2, 40, 60)
    graphs, plain = [], []
    for st in (small, large):
        st.run()
        plain.append(st.results())
    reserved = ctx.workspace_bytes()
    for st in (small, large):
        st.restore()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            st.run()
        graphs.append(g)
    assert ctx.workspace_bytes() == reserved       # nothing was grown while recording
    for turn in range(3):
        for st, g, want in zip((small, large), graphs, plain):
            st.restore()
            g.replay()
            got = st.results()
            if turn == 0:
                same(want, got)
            st.check(got)
            st.load(50 + turn)
    reserved = ctx.workspace_bytes()               # the scoring path's, used by the checks, among it
    ctx.reserve_rollout(40, 60)                    # asks for what is there: nothing moves
    assert ctx.workspace_bytes() == reserved
    small.restore()
    graphs[0].replay()
    small.check(small.results())


def test_first_call_recorded_after_a_reservation(ctx):
    st = Step(ctx, 5, 6, 14)
    ctx.reserve_rollout(6, 14)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        st.run()
    for seed in (8, 9):
        st.load(seed)
        g.replay()
        st.check(st.results())


def test_on_a_stream_of_its_own(ctx):
    st = Step(ctx, 11, 9, 30)
    st.run()
    want = st.results()
    st.load(12)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        x = torch.randn(4096, 4096, device=device())
        for _ in range(20):
            x = x @ x * 1e-2                       # the step waits behind it on this stream, and would not on another
        keep = st.before
        st.length.add_(0)
        st.run()
        first = {k: getattr(st, k).clone() for k in want}
    side.synchronize()
    st.before = keep
    st.check(first)


def soil(nbytes=64 << 20):
    """Leaves memory behind that holds no zeros."""
    x = torch.full((nbytes,), 0xff, dtype=torch.uint8, device=device())
    torch.cuda.synchronize()
    del x
    torch.cuda.empty_cache()


@pytest.mark.parametrize("mode", ["dense", "lookup"])
@pytest.mark.parametrize("on_side", [False, True])
def test_batches_of_growing_and_shrinking_size(ctx, mode, on_side):
    """Workspaces that grow come from memory that was used before."""
    side = torch.cuda.Stream()
    for turn, (R, most, V) in enumerate([(2, 3, 500), (40, 4, 500), (3, 9, 70000), (1, 1, 50), (90, 2, 300), (2, 3, 500)]):
        soil()
        c = verify_case(70 + turn, R, most, V, mode)
        torch.cuda.synchronize()
        with torch.cuda.stream(side if on_side else torch.cuda.current_stream()):
            check_verify(ctx, c)
            check_blocks(ctx, blocks_case(turn, 30 * R, 3, 5, 40 * R))


def test_after_a_reservation_any_smaller_batch(ctx):
    ctx.reserve_rollout(64, 7)
    reserved = ctx.workspace_bytes()
    for turn, (R, most, V) in enumerate([(64, 7, 300), (1, 7, 90000), (64, 1, 128), (5, 0, 77), (30, 5, 4001)]):
        check_verify(ctx, verify_case(90 + turn, R, most, V, "dense" if turn & 1 else "lookup"), max_draft=most)
        check_blocks(ctx, blocks_case(turn, R, 16, 4, 3 * R))
        assert ctx.workspace_bytes() == reserved


def test_vocabularies_past_2_30_are_refused(ctx):
    """Before anything is read: the pointers are of one small buffer."""
    from paper_2507_01663_b200 import binding as B
    p, V = torch.zeros(64, device=device()).data_ptr(), (1 << 30) + 1
    shape = next(k for k, name in B.STATUS_NAMES.items() if name == "AF_ERR_SHAPE")
    assert ctx.lib.af_quantize_head(ctx.handle, p, V, 32, 32, p, p, None, None) == shape
    assert ctx.lib.af_quant_logits(ctx.handle, p, p, p, 1, 32, V, 32, p, B.F32, V, None) == shape
    assert ctx.lib.af_draft_verify(ctx.handle, p, B.F32, V, None, B.F32, 0, p, p, p, p, 1, 1, V, 1, 1.0, p, p, p, None) == shape
