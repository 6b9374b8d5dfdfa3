"""af_quantize_head: bit for bit what the oracle says, in every output."""
import numpy as np
import pytest
import torch

from gpu_util import device
from oracle import rollout_oracle as O
from rollout_util import bf16, f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2507_01663_b200 import binding as B
    c = B.Context(0)
    yield c
    c.close()


def quantize(ctx, W, group, values=True, stream=None):
    V, d = W.shape
    dev = device()
    codes = torch.full((V, d // 8), 7, dtype=torch.int32, device=dev)
    scale = torch.full((V, -(-d // group)), 9.0, dtype=torch.bfloat16, device=dev)
    out = torch.full((V, d), 5.0, dtype=torch.bfloat16, device=dev) if values else None
    ctx.quantize_head(W.to(dev), codes, scale, group=group, values=out, stream=stream)
    torch.cuda.synchronize()
    return codes, scale, out


def same(a, b):
    return np.array_equal(a, b, equal_nan=True)


def check(ctx, W, group):
    codes, scale, values = quantize(ctx, W, group)
    with np.errstate(invalid="ignore"):
        q, s, v = O.quantize_head_ref(f64(W), group)
    assert np.array_equal(codes.cpu().numpy(), O.pack_digits(q))
    assert same(f64(scale), s) and same(f64(values), v)
    codes2, scale2, _ = quantize(ctx, W, group, values=False)
    assert torch.equal(codes, codes2) and same(f64(scale), f64(scale2))


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("V,d", [(1, 32), (1, 96), (3, 128), (5, 160), (129, 256), (33, 288), (2, 2080), (1000, 640)])
def test_sizes(ctx, V, d, group):
    rng = np.random.default_rng(V * d + group)
    check(ctx, bf16(rng.standard_normal((V, d)) * 0.02 * np.exp(rng.standard_normal((V, 1)))), group)


def test_every_ratio_of_a_weight_to_its_scale(ctx):
    """All bf16 significands against all of them as the largest weight: halves, and the neighbours of halves."""
    top = (128 + np.arange(128)) / 128.0
    W = np.zeros((128 * 16, 96), dtype=np.float64)
    for i in range(128):
        for k in range(16):
            row = W[i * 16 + k]
            row[0] = top[i]
            row[1:65] = (top[(k % 2) * 64:(k % 2) * 64 + 64]) / 2.0 ** (k // 2) * (1 if k % 3 else -1)
            row[1:65][np.abs(row[1:65]) > row[0]] = 0.0
    check(ctx, bf16(W), 128)


def test_zeros_tiny_huge_and_not_numbers(ctx):
    rng = np.random.default_rng(3)
    W = (rng.standard_normal((12, 64)) * 0.1).astype(np.float32)
    W[0] = 0.0
    W[1] = -0.0
    W[2] *= 2.0 ** -110
    W[3], W[3, 40] = 2.0 ** -101, -2.0 ** -100
    W[4, 5] = np.nan
    W[5, 40] = np.inf
    W[6, 63] = -np.inf
    W[7, 0] = 2.0 ** 120
    W[8, 0] = 1.5 * 2.0 ** 120
    W[9] = 1e-40
    W[10] = 3e38
    check(ctx, bf16(W), 32)
    check(ctx, bf16(W), 64)


def test_rows_behind_and_between_are_left(ctx):
    dev = device()
    W = bf16(np.random.default_rng(5).standard_normal((70, 96))).to(dev)
    codes, scale = torch.full((80, 12), 7, dtype=torch.int32, device=dev), torch.full((80, 2), 9.0, dtype=torch.bfloat16, device=dev)
    values = torch.full((80, 96), 5.0, dtype=torch.bfloat16, device=dev)
    ctx.quantize_head(W, codes, scale, group=64, values=values)
    assert bool((codes[70:] == 7).all()) and bool((scale[70:] == 9.0).all()) and bool((values[70:] == 5.0).all())


def test_a_head_of_more_than_2_31_weights(ctx):
    """Offsets past 32 bits: rows at both ends, of a whole-group and of a ragged row length."""
    dev = device()
    for V, d, group in ((4_500_000, 512, 128), (7_600_000, 288, 64)):
        W = torch.empty(V, d, dtype=torch.bfloat16, device=dev).normal_()
        codes, scale = torch.empty(V, d // 8, dtype=torch.int32, device=dev), torch.empty(V, -(-d // group), dtype=torch.bfloat16, device=dev)
        ctx.quantize_head(W, codes, scale, group=group)
        rows = torch.tensor([0, 1, V // 2, V - 2, V - 1], device=dev)
        q, s, _ = O.quantize_head_ref(f64(W[rows]), group)
        assert np.array_equal(codes[rows].cpu().numpy(), O.pack_digits(q)) and same(f64(scale[rows]), s)
        del W, codes, scale
        torch.cuda.empty_cache()


def test_refusals(ctx):
    from paper_2507_01663_b200 import binding as B
    dev = device()
    W = torch.zeros(4, 64, dtype=torch.bfloat16, device=dev)
    codes, scale = torch.zeros(4, 8, dtype=torch.int32, device=dev), torch.zeros(4, 2, dtype=torch.bfloat16, device=dev)
    lib, p = ctx.lib, lambda t: t.data_ptr()
    ok = lambda **k: {**dict(W=p(W), V=4, d=64, group=32, codes=p(codes), scale=p(scale), values=None), **k}
    call = lambda **k: lib.af_quantize_head(ctx.handle, *ok(**k).values(), None)
    assert call() == 0
    assert call(W=None) == -1 and call(codes=None) == -1 and call(scale=None) == -1
    assert call(V=0) == -1 and call(d=0) == -1 and call(group=16) == -1 and call(group=0) == -1
    assert call(d=48) == -3 and call(W=p(W) + 2) == -3 and call(codes=p(codes) + 4) == -3 and call(values=p(W) + 8) == -3
    torch.cuda.synchronize()
    assert ctx.check_device_errors() == 0
    with pytest.raises(ValueError):
        ctx.quantize_head(W, codes, scale, group=48)
    with pytest.raises(B.AfError):
        ctx.quantize_head(torch.zeros(4, 48, dtype=torch.bfloat16, device=dev), torch.zeros(4, 6, dtype=torch.int32, device=dev), scale, group=32)
