"""The gradients through the head are the same bits every time: no sum depends on the order in which CTAs finish."""
import numpy as np
import pytest
import torch

from gpu_util import device

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2507_01663_b200 import binding as B
    c = B.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, None], ids=["f32", "bf16", "frozen"])
@pytest.mark.parametrize("T,d,V,K,block", [(29, 512, 19000, 9, 0), (300, 256, 4104, 16, 128), (1195, 256, 4096, 16, 0), (4001, 1024, 32768, 50, 0)])
def test_gradient_and_update_repeat_themselves(ctx, T, d, V, K, block, dtype):
    from paper_2507_01663_b200 import binding as B
    dev = device()
    g = torch.Generator(device=dev).manual_seed(T)
    H = torch.randn(T, d, generator=g, device=dev).to(torch.bfloat16)
    W = (torch.randn(V, d, generator=g, device=dev) / d ** 0.5).to(torch.bfloat16)
    cand = torch.randint(-1, V, (T, K), generator=g, device=dev, dtype=torch.int32)
    lt = torch.log_softmax(torch.randn(T, K, generator=g, device=dev), dim=1) - 0.1
    lt = torch.where(cand < 0, torch.full_like(lt, -np.inf), lt)
    cu = torch.tensor([0, T // 3, T], dtype=torch.int32, device=dev)
    ctx.set_tuning(0, block)
    seen = []
    for turn in range(4):
        lq, lse, dH, dH2, dc = (torch.full(s, float(turn), dtype=t, device=dev) for s, t in
                                (((T, K), torch.float32), ((T,), torch.float32), ((T, d), torch.bfloat16), ((T, d), torch.bfloat16),
                                 ((T, K), torch.float32)))
        dW, dW2 = ((None, None) if dtype is None else
                   (torch.full((V, d), float(turn), dtype=dtype, device=dev), torch.full((V, d), float(turn), dtype=dtype, device=dev)))
        ctx.distill_update(H, W, cand, lt, cu, B.new_distill_out(dev), lq, lse, dH, dW, dcand=dc)
        ctx.candidate_logprob_backward(H, W, cand, lse, dc, dH2, dW2)
        seen.append([x for x in (lq, lse, dc, dH, dW, dH2, dW2) if x is not None])
    ctx.set_tuning(0, 0)
    assert ctx.check_device_errors() == 0
    for later in seen[1:]:
        assert all(torch.equal(a, b) for a, b in zip(seen[0], later))
