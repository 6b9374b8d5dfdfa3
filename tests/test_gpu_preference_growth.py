"""af_preference_loss while its workspace grows from call to call, over memory that held other things."""
import numpy as np
import pytest
import torch

from gpu_util import device
from test_gpu_preference import call, check, data

pytestmark = pytest.mark.gpu


def soil():
    """Leaves freed device memory behind with no zero in it."""
    blocks = [torch.full((n,), -1, dtype=torch.int32, device=device()) for n in (1 << 10, 1 << 17, 1 << 18, 1 << 20, 1 << 22)]
    torch.cuda.synchronize()
    del blocks
    torch.cuda.empty_cache()


def test_results_do_not_depend_on_what_the_workspace_held():
    from paper_2507_01663_b200 import binding as B
    ctx = B.Context(0)
    try:
        before = ctx.workspace_bytes()
        for n, (T, seqs) in enumerate([(40, 2), (300, 4), (2000, 200), (9000, 900), (9000, 900), (30000, 6000), (64, 2), (80000, 40000)]):
            soil()
            logp, ref, cu = data(T, T, seqs)
            how = dict(length_norm=bool(n & 1), pair_layout=n & 1)
            for _ in range(2):
                check(logp, ref, cu, call(ctx, logp, ref, cu, **how), **how)
        assert ctx.workspace_bytes() > before + 20 * 40000 and ctx.check_device_errors() == 0
    finally:
        ctx.close()


def test_growth_on_a_stream_of_its_own():
    """A stream that does not wait for the default stream sees the barriers at rest from the first call on."""
    from paper_2507_01663_b200 import binding as B
    logp, ref, cu = data(9, 5000, 500)
    first = None
    for _ in range(5):
        soil()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            ctx = B.Context(0)
            got = call(ctx, logp, ref, cu)
            big = call(ctx, *data(10, 60000, 30000))
            again = call(ctx, logp, ref, cu)
            assert ctx.check_device_errors() == 0
        ctx.close()
        check(logp, ref, cu, got)
        first = got if first is None else first
        assert got[0] == again[0] == first[0] and all(np.array_equal(a, b) and np.array_equal(a, c) for a, b, c in zip(got[1:], again[1:], first[1:]))
        assert big[0]["n_pairs"] == 15000
