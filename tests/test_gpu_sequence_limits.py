"""More sequences than 32-bit searches over cu_seqlens can take are refused before anything is launched or allocated."""
import ctypes

import pytest
import torch

from gpu_util import device

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B", [2 ** 30 + 2, 2 ** 31 - 2])
@pytest.mark.parametrize("T", [0, 40])
def test_too_many_sequences(B, T):
    from paper_2507_01663_b200 import binding
    ctx = binding.Context(0)
    try:
        before = ctx.workspace_bytes()
        x = torch.zeros(40 * 64, device=device())
        p, lib, h = x.data_ptr(), ctx.lib, ctx.handle
        pp = binding.PreferenceParams(0, 0, 0, 0.1, 0.0, 0.0, 0.0, 1.0)
        dp = binding.DistillParams(0, 1, 0, 1.0, 1.0)
        assert lib.af_preference_loss(h, p, None, p, B, T, ctypes.byref(pp), p, None, None, None, None) == -2
        assert lib.af_reserve_preference(h, T, B) == -2
        assert lib.af_distill_loss(h, p, p, p, B, T, 3, ctypes.byref(dp), p, None, None, None) == -2
        assert lib.af_distill_update(h, p, p, p, p, p, B, T, 3, 16, 24, ctypes.byref(dp), p, p, None, p, None, None, p, None, 0, 0,
                                     None) == -2
        assert ctx.workspace_bytes() == before and ctx.check_device_errors() == 0
    finally:
        ctx.close()
