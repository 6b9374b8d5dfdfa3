"""af_block_slots against a stack worked block by block: every output, exactly."""
import numpy as np
import pytest
import torch

from gpu_util import device
from oracle import rollout_oracle as O
from rollout_util import i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2507_01663_b200 import binding as B
    c = B.Context(0)
    yield c
    c.close()


def case(seed, R, bs, per, spare, shrink=0.3, most=None):
    """Tables of disjoint blocks, a free list with `spare` blocks, and lengths of which some have shrunk."""
    rng = np.random.default_rng(seed)
    held = rng.integers(0, per + 1, R)
    length = np.maximum(held * bs - rng.integers(0, bs, R), 0) * (held > 0)
    length = np.where(rng.random(R) < shrink, (length * rng.random(R)).astype(int), length)
    most = 2 * bs + 3 if most is None else most
    grow = np.minimum(rng.integers(0, most + 1, R), per * bs - length)
    n = int(held.sum()) + spare
    ids = rng.permutation(n).astype(np.int32)
    table = np.full((R, per), -5, np.int32)
    at = 0
    for r in range(R):
        table[r, :held[r]] = ids[at:at + held[r]]
        at += held[r]
    free = np.full(n, -9, np.int32)
    free[:spare] = ids[at:]
    return dict(length=length, grow=grow, held=held, table=table, free=free, count=spare, bs=bs)


def run(ctx, c, capacity=None, in_place=False, pad=0, optional=True, spare=5):
    dev = device()
    R, per = c["table"].shape
    total = int(np.maximum(c["grow"], 0).sum())
    cap = total if capacity is None else capacity
    length, grow, held, count = i32(c["length"]), i32(c["grow"]), i32(c["held"]), i32([c["count"]])
    wide = torch.full((R, per + pad), -6, dtype=torch.int32, device=dev)
    table = wide[:, :per]
    table.copy_(torch.as_tensor(c["table"]))
    free = i32(c["free"])
    held_out, count_out = (held, count) if in_place else (torch.full((R + spare,), -7, dtype=torch.int32, device=dev), i32([-7]))
    granted = torch.full((R + spare,), -7, dtype=torch.int32, device=dev)
    cu = torch.full((R + 1 + spare,), -7, dtype=torch.int32, device=dev)
    buf = torch.full((cap + spare,), -7, dtype=torch.int64, device=dev)
    pos = torch.full((cap + spare,), -7, dtype=torch.int32, device=dev)
    ctx.block_slots(length, grow, held, table, free, count, held_out, count_out, cu, buf[:cap], block_size=c["bs"],
                    position=pos[:cap] if optional else None, granted=granted if optional else None, R=R)
    torch.cuda.synchronize()
    assert bool((buf[cap:] == -7).all()) and bool((pos[cap:] == -7).all()) and bool((granted[R:] == -7).all()) and bool((cu[R + 1:] == -7).all())
    assert bool((held_out[R:] == -7).all()) and bool((wide[:, per:] == -6).all())
    return dict(table=table.cpu().numpy(), free=free.cpu().numpy(), free_count=int(count_out), held=held_out[:R].cpu().numpy(),
                granted=granted[:R].cpu().numpy(), cu=cu[:R + 1].cpu().numpy(), slot=buf[:cap].cpu().numpy(), position=pos[:cap].cpu().numpy())


def check(ctx, c, capacity=None, optional=True, **how):
    from paper_2507_01663_b200 import binding as B
    got = run(ctx, c, capacity, optional=optional, **how)
    total = int(np.maximum(c["grow"], 0).sum())
    want = O.block_slots_ref(c["length"], c["grow"], c["held"], c["table"], c["free"], c["count"], c["bs"], total if capacity is None else capacity)
    for name in ("table", "free", "free_count", "held", "cu") + (("granted",) if optional else ()):
        assert np.array_equal(got[name], np.asarray(want[name])), name
    for name in ("slot",) + (("position",) if optional else ()):
        assert np.array_equal(got[name], np.array([-7 if x is None else x for x in want[name]], dtype=np.int64)), name
    bits = {"request": B.DEVERR_REQUEST, "blocks": B.DEVERR_BLOCKS}
    assert ctx.check_device_errors() == sum(bits[f] for f in want["flags"])
    return want


@pytest.mark.parametrize("bs", [1, 2, 3, 16, 24, 64, 128, 1000])
@pytest.mark.parametrize("R", [1, 2, 31, 33, 300, 1023, 1024, 1025, 2500])
def test_requests_and_blocks(ctx, R, bs):
    want = check(ctx, case(R + bs, R, bs, 7, 8 * R), in_place=bool(R & 1), pad=R % 3)
    assert "blocks" not in want["flags"]


@pytest.mark.parametrize("seed", range(12))
def test_too_few_blocks(ctx, seed):
    R = (1, 5, 60, 1100)[seed % 4]
    want = check(ctx, case(seed, R, 4, 9, (0, 1, R // 2)[seed % 3], shrink=0.1 * (seed % 5), most=20), in_place=bool(seed & 1))
    if R > 1 and seed % 3 == 0:
        assert "blocks" in want["flags"] or sum(want["granted"]) == R


def test_blocks_given_back_serve_the_same_call(ctx):
    c = case(1, 40, 8, 10, 0, shrink=0.0, most=0)
    c["length"][::2] = 0                                       # half of the responses have ended, the others grow
    c["length"][1::2] = np.minimum(c["length"][1::2], 40)
    c["grow"][1::2] = 40
    want = check(ctx, c)
    assert sum(want["granted"]) > 30 and want["free_count"] < int(c["held"][::2].sum())


def test_long_prompts_many_tokens(ctx):
    c = case(2, 50, 16, 1500, 50 * 1400, shrink=0.9, most=20000)
    want = check(ctx, c)
    assert want["cu"][-1] > 200000


def test_nothing_to_do(ctx):
    check(ctx, case(3, 5, 16, 4, 3, shrink=0.0, most=0))
    empty = dict(length=np.zeros(0, int), grow=np.zeros(0, int), held=np.zeros(0, int), table=np.zeros((0, 4), np.int32),
                 free=np.arange(6, dtype=np.int32), count=4, bs=16)
    got = run(ctx, empty)
    assert got["cu"].tolist() == [0] and got["free_count"] == 4 and got["free"].tolist() == list(range(6))
    no_table = dict(length=np.zeros(3, int), grow=np.array([0, 1, 0]), held=np.zeros(3, int), table=np.zeros((3, 0), np.int32),
                    free=np.zeros(0, np.int32), count=0, bs=16)
    check(ctx, no_table)
    assert ctx.check_device_errors() == 0


def test_optional_outputs(ctx):
    check(ctx, case(4, 70, 16, 5, 300), optional=False)


@pytest.mark.parametrize("capacity", [0, 1, 100])
def test_more_tokens_than_rows(ctx, capacity):
    want = check(ctx, case(5, 60, 4, 6, 400), capacity=capacity)
    assert "request" in want["flags"]


def test_more_rows_than_tokens(ctx):
    check(ctx, case(6, 60, 4, 6, 400), capacity=3000)


def test_impossible_numbers(ctx):
    c = case(7, 24, 8, 6, 100)
    c["length"][1], c["grow"][2], c["held"][3], c["held"][4] = -1, -5, -1, 7
    c["length"][5], c["grow"][5] = 6 * 8, 1                    # does not fit its table
    c["length"][6], c["grow"][6] = 2 ** 31 - 1, 1
    c["length"][7] = -2 ** 31
    want = check(ctx, c)
    assert sum(want["granted"]) == 24 - 7
    for count in (-4, 10 ** 6):
        check(ctx, dict(case(8, 9, 8, 6, 30), count=count))


def test_more_blocks_come_back_than_there_are(ctx):
    c = case(9, 20, 4, 5, 10)
    c["length"][:] = 0
    c["grow"][:] = 3
    c["free"] = c["free"][:30].copy()
    want = check(ctx, c)
    assert "request" in want["flags"]


def test_slots_past_32_bits(ctx):
    c = case(10, 6, 128, 5, 20)
    c["table"] = np.where(c["table"] >= 0, c["table"] + (2 ** 31 - 1000), c["table"]).astype(np.int32)
    c["free"] = np.where(c["free"] >= 0, c["free"] + (2 ** 31 - 1000), c["free"]).astype(np.int32)
    want = check(ctx, c)
    assert max(s for s in want["slot"] if s is not None) > 2 ** 37


def test_totals_past_31_bits_are_cut(ctx):
    """Prompts of 2^30 tokens: the running sums stop at 2^31 - 1."""
    from paper_2507_01663_b200 import binding as B
    c = dict(length=np.zeros(4, int), grow=np.full(4, 2 ** 30), held=np.zeros(4, int), table=np.full((4, 2), -1, np.int32),
             free=np.arange(8, dtype=np.int32), count=8, bs=2 ** 30)
    got = run(ctx, c, capacity=1000)
    assert got["cu"].tolist() == [0, 2 ** 30, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1] and got["held"].tolist() == [1] * 4
    assert got["slot"].tolist() == [7 * 2 ** 30 + i for i in range(1000)] and got["free_count"] == 4
    assert ctx.check_device_errors() == B.DEVERR_REQUEST


def test_refusals(ctx):
    dev = device()
    z = lambda n: torch.zeros(n, dtype=torch.int32, device=dev)
    length, grow, held, table, free, count, ho, co, cu, slot = z(3), z(3), z(3), z(12), z(5), z(1), z(3), z(1), z(4), z(20)
    p = lambda t: t.data_ptr()
    ok = dict(length=p(length), grow=p(grow), held=p(held), R=3, bs=16, table=p(table), pitch=4, per=4, free=p(free), n=5, count=p(count),
              ho=p(ho), co=p(co), granted=None, cu=p(cu), slot=p(slot), pos=None, cap=10)
    call = lambda **k: ctx.lib.af_block_slots(ctx.handle, *{**ok, **k}.values(), None)
    assert call() == 0
    for name in ("length", "grow", "held", "table", "free", "count", "ho", "co", "cu", "slot"):
        assert call(**{name: None}) == -1
    assert call(R=-1) == -1 and call(bs=0) == -1 and call(per=-1) == -1 and call(n=-1) == -1 and call(cap=-1) == -1
    assert call(pitch=3) == -2 and call(R=(1 << 20) + 1) == -2
    torch.cuda.synchronize()
    assert ctx.check_device_errors() == 0
    with pytest.raises(ValueError):
        ctx.block_slots(length, grow, held, table.view(3, 4).t(), free, count, ho, co, cu, slot.long(), block_size=16)
