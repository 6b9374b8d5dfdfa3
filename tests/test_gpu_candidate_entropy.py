"""Entropy of the scoring call for a few tokens where the logits are large and the distribution is not."""
import numpy as np
import pytest
import torch

from distill_util import U, dev_of, np_of
from gpu_util import device

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2507_01663_b200 import binding as B
    c = B.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("T", [1, 3, 8, 9, 16])
@pytest.mark.parametrize("top", [0.0, 64.0, 4096.0])
def test_entropy_does_not_inherit_the_size_of_the_logits(ctx, T, top):
    """Logits that are bf16 values (one coordinate of the hidden row is 1), so they are exact.  With x = z - max the
    entropy is log s - sum e^x x / s, s = sum e^x: an exponential is off by (4 + 2 |x|) U relative, the sums by one U per
    addition, a rescaling when a larger logit comes along is one more exponential.  At most n = 64 additions and joins lie
    on the way of a term, each of them with an exponential of its own whose arguments add up to |x|."""
    dev = device()
    V, d = 20000, 8
    rng = np.random.default_rng(int(top) + T)
    W = torch.zeros(V, d, dtype=torch.bfloat16)
    W[:, 0] = torch.as_tensor((top + rng.choice([0.0, -16.0, -32.0], V, p=[0.3, 0.5, 0.2])).astype(np.float32))
    H = torch.zeros(T, d, dtype=torch.bfloat16)
    H[:, 0] = 1.0
    lq, ent, lse = torch.empty(T, 1, device=dev), torch.empty(T, device=dev), torch.empty(T, device=dev)
    ctx.candidate_logprob(H.to(dev), W.to(dev), dev_of(np.zeros((T, 1), np.int32)), lq, ent, lse)
    z = W[:, 0].double().numpy()
    x = z - z.max()
    s, m1 = np.exp(x).sum(), (np.exp(x) * x).sum()
    e = lambda v: 64 * (1 + 4) * U + (4 + 2 * np.abs(v)) * U   # noqa: E731
    es, em = (np.exp(x) * e(x)).sum() / s, (np.exp(x) * np.abs(x) * e(x)).sum() / s
    want = np.log(s) - m1 / s
    tol = es + em + abs(m1 / s) * es + 4 * U * (abs(np.log(s)) + abs(m1 / s) + 1)
    assert np.abs(np_of(ent).astype(np.float64) - want).max() <= tol
    assert np.abs(np_of(lse).astype(np.float64) - (z.max() + np.log(s))).max() <= es + 2 * U * (abs(z.max()) + np.log(s))
    assert ctx.check_device_errors() == 0
