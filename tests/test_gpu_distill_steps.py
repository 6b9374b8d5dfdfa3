"""af_distill_loss where a CTA works through many steps of its ring: every row against the same sums in 64 bits.

Sizes: 592 CTAs (four per SM) of 128 / G rows, G the lanes of a row; lists of up to 8 slots are taken in several batches of
rows per step.  Sequences are short and empty ones beside long ones, so that a lane's place in the list of sequences is
carried over, hops and is searched for again; the last step is ragged everywhere."""
import numpy as np
import pytest
import torch

from distill_util import U, dev_of
from gpu_util import device

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2507_01663_b200 import binding as B
    c = B.Context(0)
    yield c
    c.close()


def lists(seed, T, K):
    """Teacher's and student's float32 log-probs on the device; a tenth of the lists are short, some of them empty."""
    dev = device()
    g = torch.Generator(device=dev).manual_seed(seed)
    lt, lq = (torch.log_softmax(2.0 * torch.randn(T, K, generator=g, device=dev), dim=1)
              + torch.log(0.5 + 0.45 * torch.rand(T, 1, generator=g, device=dev)) for _ in range(2))
    kept = torch.where(torch.rand(T, 1, generator=g, device=dev) < 0.1,
                       torch.floor((K + 1) * torch.rand(T, 1, generator=g, device=dev)), torch.full((T, 1), float(K), device=dev))
    absent = torch.arange(K, device=dev) >= kept
    return lt.masked_fill(absent, -np.inf), lq


def sequences(seed, T):
    """Half of the tokens in three long sequences, the others in ones of 0 to 12."""
    rng = np.random.default_rng(seed)
    lengths, left = [], T - T // 2
    while left > 0:
        n = rng.integers(0, 13, max(left // 6, 1))
        n = n[:int(np.searchsorted(np.cumsum(n), left, side="right")) + 1]
        lengths.append(n)
        left -= int(n.sum())
    lengths = np.concatenate(lengths)
    lengths[-1] += left                            # the last one may have gone past
    long = np.array([T // 2 - 2 * (T // 7), T // 7, T // 7])
    at = np.sort(rng.integers(0, len(lengths), 3))
    lengths = np.insert(lengths, at, long)
    assert lengths.sum() == T and (lengths >= 0).all()
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)


def exact(lt, lq, how):
    """(loss [T], gradient [T, K], tolerance of either) in float64; the tolerances as in row_scales of the small tests."""
    direction, support, tau = how
    on = lt != -np.inf
    zero = torch.zeros((), dtype=torch.float64, device=lt.device)
    x, y = (torch.where(on, v.double() / tau, zero) for v in (lt, lq))
    some = on.any(1)
    size = x.abs().amax(1) + y.abs().amax(1) + 1
    c = (20 * U + size * 2 * U)[:, None]
    a, b = torch.where(on, x.exp(), zero), torch.where(on, y.exp(), zero)
    if support == 1:
        za, zb = (torch.where(some, v.sum(1), zero + 1)[:, None] for v in (a, b))
        a, b = a / za, b / zb
        d = torch.where(on, x - y - torch.log(za / zb), zero)
        scale = torch.where(on, d.abs() + 1 + x.abs() + y.abs(), zero)
        tl = 4 * c[:, 0] * tau * tau * ((a + b) * scale).sum(1)
        tg = 4 * c * tau * (a + b * (scale + (b * scale).sum(1, keepdim=True)))
        if direction == 0:
            return tau * tau * (a * d).sum(1), tau * (b - a), tl, tg
        r = -(b * d).sum(1, keepdim=True)
        return tau * tau * r[:, 0], tau * b * (-d - r), tl, tg
    d = torch.where(on, x - y, zero)
    scale = torch.where(on, d.abs() + 1, zero)
    tl, tg = 4 * c[:, 0] * ((a + b) * scale).sum(1), 4 * c * (a + b * scale)
    loss, grad = ((a * d).sum(1), -a) if direction == 0 else (-(b * d).sum(1), b * (1 - d))
    if support == 2:
        pr, qr = (torch.clamp(1 - v.sum(1, keepdim=True), min=2.0 ** -16) for v in (a, b))
        held = 1 - b.sum(1, keepdim=True) <= 2.0 ** -16
        ratio = torch.log(pr / qr)
        loss = loss + (pr * ratio if direction == 0 else -qr * ratio)[:, 0]
        grad = grad + torch.where(held, zero, b * (pr / qr if direction == 0 else ratio - 1))
        far = ratio.abs() + 1
        tl = tl + torch.where(some, (8 * c * (far + pr / qr + qr / pr + 1))[:, 0], zero)
        tg = tg + 8 * c * b * (far + 1 / qr + 1 / pr + pr / qr * (1 + 1 / qr))
    return loss, torch.where(on, grad, zero), tl, tg


CASES = [(1, 3_700_001, 0, (1, 2, 1.0)), (1, 3_700_003, 1, (0, 0, 1.0)), (3, 1_200_007, 0, (0, 1, 1.0)), (3, 1_200_007, 2, (1, 0, 1.0)),
         (8, 500_009, 0, (0, 2, 1.0)), (8, 500_009, 2, (1, 1, 2.0)), (8, 290, 0, (1, 1, 1.0)), (7, 500_011, 1, (0, 1, 0.5)),
         (7, 500_011, 0, (1, 2, 1.0)), (14, 300_017, 0, (1, 1, 1.0)), (50, 700_001, 0, (0, 1, 2.0)), (50, 350_003, 2, (1, 2, 1.0)),
         (50, 350_003, 1, (0, 0, 1.0)), (64, 700_003, 0, (1, 1, 1.0)), (64, 200_003, 1, (0, 2, 1.0)), (64, 200_003, 2, (1, 0, 1.0)),
         (129, 200_001, 0, (0, 1, 1.0)), (250, 150_001, 0, (1, 2, 1.0))]


@pytest.mark.parametrize("agg", [0, 1])
@pytest.mark.parametrize("K,T,offset,how", CASES)
def test_every_row_of_many_steps(ctx, K, T, offset, how, agg):
    from paper_2507_01663_b200 import binding as B
    dev = device()
    lt, lq = lists(K + T, T, K)
    cu = sequences(T, T)

    def place(x):                                  # `offset` floats past a 16-byte boundary
        buf = torch.full((T * K + 8,), 3.0, device=dev)
        view = buf[offset:offset + T * K].view(T, K)
        if x is not None:
            view.copy_(x)
        return buf, view

    a, b = place(lq)[1], place(lt)[1]
    gbuf, g = place(None)
    out, token = B.new_distill_out(dev), torch.full((T,), 3.0, device=dev)
    ctx.distill_loss(a, b, dev_of(cu), out, token_loss=token, dcand=g, divergence=how[0], support=how[1], temperature=how[2],
                     agg_mode=agg, loss_scale=1.0)
    assert ctx.check_device_errors() == 0
    res = B.read_distill_out(out)
    assert bool((gbuf[:offset] == 3.0).all()) and bool((gbuf[offset + T * K:] == 3.0).all())
    n = torch.as_tensor(np.diff(cu).astype(np.int64), device=dev)
    w = torch.full((T,), 1.0 / T, dtype=torch.float64, device=dev)
    if agg == 0:
        w = torch.repeat_interleave(1.0 / (n.clamp(min=1).double() * n.numel()), n)
    loss, grad, tl, tg = exact(lt, lq, how)
    assert bool(((token.double() - loss).abs() <= tl + 2 * U * loss.abs()).all())
    grad *= w[:, None]
    assert bool(((g.double() - grad).abs() <= w[:, None] * tg + 6 * U * grad.abs()).all())
    # a lane adds up to 256 rows in 32 bits, or 256 rows of 16 slots, before 64 bits take over
    want = float((w * loss).sum())
    assert abs(res["loss"] - want) <= float((w * tl).sum()) + 264 * U * float((w * loss.abs()).sum())
    for name, v in (("teacher_mass", lt), ("student_mass", lq)):
        p = torch.where(lt != -np.inf, v.double().exp(), torch.zeros((), dtype=torch.float64, device=dev))
        size = float(torch.where(lt != -np.inf, v.double().abs(), torch.zeros((), dtype=torch.float64, device=dev)).max())
        assert abs(res[name] - float(p.sum()) / T) <= (272 + 8 + 2 * size) * U * float(p.sum()) / T
    assert res["n_tokens"] == T
