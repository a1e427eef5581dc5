"""Plans of very many tensors.  Runs without a GPU: plans are made on the host."""
import ctypes
import time

import pytest

from paper_2209_05433_b200 import api


def _sized(sizes, state=0):
    items = (api.AdamWItem * len(sizes))()
    for it, n in zip(items, sizes):
        it.g = it.p = it.m = it.v = it.m_scale = it.v_scale = 4096
        it.n, it.state = n, state
    plan = api.AdamWSizes()
    assert api.load().fp8_adamw_plan_size(items, len(sizes), ctypes.byref(plan)) == 0
    return plan


def test_a_plan_takes_time_in_proportion_to_its_tensors():
    """200000 small tensors: a few passes over the list, milliseconds each"""
    api.load()
    t0 = time.perf_counter()
    plan = _sized([300] * 200000, 1)
    assert time.perf_counter() - t0 < 3.0
    assert plan.chunks == 200000 and plan.chunk == 2048


@pytest.mark.parametrize("sizes", [[300] * 5000, [3000, 20000] * 700, [1 << 20] * 300 + [1] * 1000, [65537] * 1000, [1], [70000000]])
@pytest.mark.parametrize("state", [0, 1])
def test_the_chunk_is_the_smallest_that_needs_the_fewest_rounds(sizes, state):
    """148 SMs of three CTAs; chunks of 2048 to 8192 elements, or 65536 with 8-bit moments"""
    most, held = (65536 if state else 8192), 444
    chunks = lambda c: sum(-(-n // c) for n in sizes)  # noqa: E731
    fewest = -(-chunks(most) // held)
    least = max(2048, sum(-(-n // 256) * 256 for n in sizes) // (fewest * held) // 2048 * 2048)
    want = next(c for c in range(least, most + 1, 2048) if chunks(c) <= fewest * held)
    plan = _sized(sizes, state)
    assert (plan.chunk, plan.chunks) == (want, chunks(want))
