"""af_quant_logits against 64 bits: token counts, odd vocabularies, group sizes, types, pitches, NaN."""
import numpy as np
import pytest
import torch

from gpu_util import device
from oracle import rollout_oracle as O
from rollout_util import bf16, f64, logits_tol

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2507_01663_b200 import binding as B
    c = B.Context(0)
    yield c
    c.close()


def head(seed, T, d, V, group, any_scale=False):
    rng = np.random.default_rng(seed)
    words = rng.integers(-2 ** 31, 2 ** 31, (V, d // 8)).astype(np.int32)
    scale = (1 + rng.integers(0, 128 if any_scale else 16, (V, -(-d // group))) / (128.0 if any_scale else 16.0)) * 2.0 ** rng.integers(-11, -6, (V, -(-d // group)))
    return bf16(rng.standard_normal((T, d))), torch.as_tensor(words), bf16(scale)


def run(ctx, H, words, scale, group, dtype=torch.float32, pad=0, offset=0, T=None):
    """logits in rows `pad` apart, from an address that is only aligned to the type."""
    dev = device()
    n, V = (H.shape[0] if T is None else T), words.shape[0]
    buf = torch.full(((n + 1) * (V + pad) + offset,), 3.0, dtype=dtype, device=dev)
    rows = buf[offset:offset + (n + 1) * (V + pad)].view(n + 1, V + pad)
    ctx.quant_logits(H.to(dev), words.to(dev), scale.to(dev), rows[:n, :V] if n else rows[:1, :V], group=group, T=n)
    assert bool((rows[:n, V:] == 3.0).all()) and bool((rows[n:] == 3.0).all()) and bool((buf[:offset] == 3.0).all())
    return f64(rows[:n, :V])


def check(ctx, T, d, V, group, dtype=torch.float32, seed=0, **how):
    H, words, scale = head(seed + T + d + V, T, d, V, group, any_scale=bool(seed & 1))
    got = run(ctx, H, words, scale, group, dtype, **how)
    want, mag = O.quant_logits_ref(f64(H), words.numpy(), f64(scale), group)
    off = np.abs(got - want)
    assert (off <= logits_tol(d, mag, want, dtype is torch.bfloat16)).all(), float((off / mag).max())


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 15, 16, 17, 31, 33, 64, 65])
def test_token_counts(ctx, T, group):
    check(ctx, T, 384, 517, group)


@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 224, 256, 288, 640, 992, 2080, 3584, 5120, 6144, 6176, 8192, 12320])
@pytest.mark.parametrize("T", [1, 5, 16, 40])
def test_widths(ctx, T, d):
    check(ctx, T, d, 131, (32, 64, 128)[d // 32 % 3], seed=d // 32)


@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 15, 16, 17, 31, 63, 127, 128, 129, 255, 1000, 4099, 20011])
@pytest.mark.parametrize("T", [1, 11, 48])
def test_vocabularies(ctx, T, V):
    check(ctx, T, 160, V, 64, dtype=(torch.float32, torch.bfloat16)[V % 2], seed=V)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,pad,offset", [(1, 0, 1), (3, 1, 0), (6, 5, 3), (16, 8, 8), (20, 13, 1), (64, 3, 5)])
def test_rows_apart_and_off_alignment(ctx, T, pad, offset, dtype):
    check(ctx, T, 256, 333, 128, dtype, pad=pad, offset=offset)


def test_no_tokens_and_more_rows_than_tokens(ctx):
    H, words, scale = head(1, 4, 64, 40, 32)
    assert run(ctx, H, words, scale, 32, T=0).shape == (0, 40)
    whole = run(ctx, H, words, scale, 32)
    assert np.array_equal(run(ctx, H, words, scale, 32, T=2), whole[:2])


@pytest.mark.parametrize("T", [1, 9, 24])
def test_nan_stays_where_it_is(ctx, T):
    H, words, scale = head(2, T, 256, 300, 64)
    clean = run(ctx, H, words, scale, 64)
    scale[17, 2] = float("nan")
    H[T - 1, 3] = float("nan")
    got = run(ctx, H, words, scale, 64)
    nan = np.zeros((T, 300), dtype=bool)
    nan[:, 17] = nan[T - 1] = True
    assert np.array_equal(np.isnan(got), nan) and np.array_equal(got[~nan], clean[~nan])


@pytest.mark.parametrize("T", [1, 12, 64])
def test_results_repeat_bit_for_bit(ctx, T):
    H, words, scale = head(4, T, 1024, 5000, 128)
    first = run(ctx, H, words, scale, 128)
    for _ in range(3):
        assert np.array_equal(first, run(ctx, H, words, scale, 128))


def test_a_tokens_logits_of_a_quantized_head_are_those_of_its_values(ctx):
    """codes and scales of af_quantize_head stand for exactly its values."""
    dev = device()
    rng = np.random.default_rng(8)
    W, H = bf16(rng.standard_normal((700, 416)) * 0.05).to(dev), bf16(rng.standard_normal((3, 416)))
    codes, scale, values = torch.empty(700, 52, dtype=torch.int32, device=dev), torch.empty(700, 4, dtype=torch.bfloat16, device=dev), torch.empty_like(W)
    ctx.quantize_head(W, codes, scale, group=128, values=values)
    got = run(ctx, H, codes.cpu(), scale.cpu(), 128)
    want, mag = f64(H) @ f64(values).T, np.abs(f64(H)) @ np.abs(f64(values)).T
    assert (np.abs(got - want) <= logits_tol(416, mag, want, False)).all()


def test_codes_past_2_31_weights(ctx):
    """Offsets past 32 bits in the head (2.3e9 weights) and in the logits' pitch."""
    dev = device()
    V, d, group, T = 4_500_000, 512, 64, 3
    codes = torch.empty(V, d // 8, dtype=torch.int32, device=dev).random_(-2 ** 31, 2 ** 31)
    scale = torch.full((V, d // group), 2.0 ** -8, dtype=torch.bfloat16, device=dev)
    H = bf16(np.random.default_rng(1).standard_normal((T, d))).to(dev)
    logits = torch.zeros(T * 1_500_000_000, dtype=torch.bfloat16, device=dev).view(T, -1)[:, :V]
    ctx.quant_logits(H, codes, scale, logits, group=group)
    rows = torch.tensor([0, 5, V // 2, V - 17, V - 1], device=dev)
    want, mag = O.quant_logits_ref(f64(H), codes[rows].cpu().numpy(), f64(scale[rows]), group)
    assert (np.abs(f64(logits[:, rows]) - want) <= logits_tol(d, mag, want, True)).all()
    del codes, scale, logits
    torch.cuda.empty_cache()


def test_refusals(ctx):
    dev = device()
    H, words, scale = (t.to(dev) for t in head(1, 4, 64, 40, 32))
    out = torch.zeros(4, 40, device=dev)
    p = lambda t: t.data_ptr()
    ok = dict(hidden=p(H), codes=p(words), scale=p(scale), T=4, d=64, V=40, group=32, logits=p(out), kind=0, pitch=40)
    call = lambda **k: ctx.lib.af_quant_logits(ctx.handle, *{**ok, **k}.values(), None)
    assert call() == 0 and call(T=0, hidden=None) == 0
    for name in ("hidden", "codes", "scale", "logits"):
        assert call(**{name: None}) == -1
    assert call(T=-1) == -1 and call(d=0) == -1 and call(V=0) == -1 and call(group=31) == -1 and call(kind=2) == -1
    assert call(d=40) == -3 and call(hidden=p(H) + 2) == -3 and call(codes=p(words) + 8) == -3 and call(scale=p(scale) + 2) == -3
    assert call(pitch=39) == -2 and call(T=65537) == -2
    assert call(logits=p(out) + 2) == -3 and call(kind=1, logits=p(out) + 1) == -3
    torch.cuda.synchronize()
    for bad in (out.t(), out[:, ::2], out[:, :39], out.double(), out.cpu()):
        with pytest.raises(ValueError):
            ctx.quant_logits(H, words, scale, bad, group=32)
