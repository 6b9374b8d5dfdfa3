"""Widths of a 4-bit head that leave 32-bit arithmetic are refused, before anything is read: the pointers are of one small buffer."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [(1 << 30) + 32, 2 ** 31 - 128, 2 ** 31 - 32])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_widths_past_2_30_are_refused(d, group):
    from paper_2507_01663_b200 import binding as B
    ctx = B.Context(0)
    p = torch.zeros(64, device="cuda:0").data_ptr()
    shape = next(k for k, name in B.STATUS_NAMES.items() if name == "AF_ERR_SHAPE")
    assert ctx.lib.af_quantize_head(ctx.handle, p, 1, d, group, p, p, None, None) == shape
    assert ctx.lib.af_quant_logits(ctx.handle, p, p, p, 1, d, 1, group, p, B.F32, 1, None) == shape
    ctx.close()
