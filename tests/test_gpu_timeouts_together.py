"""Error latches of several files set at once: one call reads and clears them all."""
import pytest
import torch

from paper_2209_05433_b200 import api

pytestmark = pytest.mark.gpu
LIMIT = 2_000_000           # SM clocks: about a millisecond


def test_one_read_clears_every_latch():
    torch.cuda.synchronize()
    assert api.fp8_async_status() == (0, 0)
    for first, second in ((api.WAIT_MBARRIER, api.WAIT_GRID_BARRIER), (api.WAIT_GRID_BARRIER, api.WAIT_MBARRIER)):
        api.fp8_self_test_expire_wait(first, LIMIT)
        api.fp8_self_test_expire_wait(second, LIMIT)
        status, detail = api.fp8_async_status()
        assert status == api.TIMEOUT and detail in (9, 16)
        assert api.fp8_async_status() == (0, 0)
