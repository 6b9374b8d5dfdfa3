"""draft_verify without max_draft: any batch that the call takes, however many drafts it has in all."""
import types

import numpy as np
import pytest
import torch

from paper_2507_01663_b200 import binding as B


class Library:
    def af_draft_verify(self, handle, t, tt, tp, q, qt, qp, draft, cu, ua, us, R, D, V, max_draft, *rest):
        self.max_draft = max_draft
        return 0


@pytest.mark.parametrize("R,D,want", [(1, 0, 0), (1, 4, 4), (5, 20, 20), (1, 1023, 1023), (256, 1024, 1023), (300, 1200, 1023), (16384, 16384, 1023),
                                      (16385, 65540, 1022), (1 << 20, 1 << 20, 15), ((1 << 24) - 1, 0, 0), (1 << 24, 5, 0), ((1 << 24) + 1, 5, 0)])
def test_what_is_passed_on(R, D, want):
    """The limits of the call: max_draft <= 1023 and R * (max_draft + 1) <= 2^24."""
    c = object.__new__(B.Context)
    c.lib, c.handle, c.device = Library(), None, -1
    V, z = 1, lambda *shape, t=torch.float32: torch.zeros(*shape, dtype=t)
    kw = dict(target_logits=z(D + R, V), draft_logits=None, draft=z(D, t=torch.int32), cu_draft=z(R + 1, t=torch.int32), u_accept=z(D),
              u_sample=z(R), token=z(D + R, t=torch.int32), n_emitted=z(R, t=torch.int32), stream=types.SimpleNamespace(cuda_stream=0))
    c.draft_verify(**kw)
    assert c.lib.max_draft == want
    c.draft_verify(**kw, max_draft=3)
    assert c.lib.max_draft == 3
    c.handle = None


@pytest.mark.gpu
@pytest.mark.parametrize("R,each", [(256, 4), (300, 5), (17000, 1)])
def test_batches_of_more_drafts_than_one_request_may_have(R, each):
    from oracle import rollout_oracle as O
    from rollout_util import f32, f64, i32
    dev, V, D = torch.device("cuda", 0), 24, R * each
    rng = np.random.default_rng(R)
    target, draft = (torch.as_tensor(rng.standard_normal((n, V)).astype(np.float32)) for n in (D + R, D))
    ids, cu = rng.integers(0, V, D).astype(np.int32), (np.arange(R + 1) * each).astype(np.int32)
    ua, us = rng.random(D).astype(np.float32), rng.random(R).astype(np.float32)
    token, n = torch.empty(D + R, dtype=torch.int32, device=dev), torch.empty(R, dtype=torch.int32, device=dev)
    ctx = B.Context(0)
    ctx.draft_verify(target.to(dev), draft.to(dev), i32(ids), i32(cu), f32(ua), f32(us), token, n)
    want = O.draft_verify_ref(f64(target), f64(draft), ids, cu, ua, us)
    assert want["margin"] > 1e-11 and ctx.check_device_errors() == 0
    assert np.array_equal(token.cpu().numpy(), want["token"]) and np.array_equal(n.cpu().numpy(), want["n_emitted"])
    ctx.close()
