"""The bounded waits of the kernels, asking and sleeping: each lasts as long as its limit says, and ends."""
import time

import pytest

pytestmark = pytest.mark.gpu


def test_both_waits_last_their_limit_and_end():
    from paper_2507_01663_b200 import binding as B
    ctx = B.Context(0)
    ctx.selftest_bounded_wait()
    assert ctx.check_device_errors() == B.DEVERR_WATCHDOG
    for _ in range(5):
        start = time.monotonic()
        shorter = ctx.selftest_bounded_wait()          # microseconds, of two limits of 1000
        assert 1000 <= shorter < 20000 and 0.002 <= time.monotonic() - start < 0.2
        assert ctx.check_device_errors() == B.DEVERR_WATCHDOG
    assert ctx.check_device_errors() == 0
    ctx.close()
