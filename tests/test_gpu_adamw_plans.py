"""Plans that name a tensor twice."""
import pytest
import torch

from paper_2209_05433_b200 import api

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_a_tensor_that_is_written_is_in_a_plan_once():
    """tied weights listed twice, one moment for two parameters, a copy in the place of its parameter, one amax for two copies"""
    new = lambda n=300: torch.zeros(n, device=DEV)  # noqa: E731
    u8 = lambda: torch.zeros(300, dtype=torch.uint8, device=DEV)  # noqa: E731
    p, g, m, v = new(), new(), new(), new()
    for bad in (([p, p], [g, new()], [m, new()], [v, new()]), ([p, new()], [g, new()], [m, m], [v, new()]), ([p], [g], [m], [m]), ([p], [g], [p], [v])):
        with pytest.raises(ValueError):
            api.AdamWPlan(*bad)
    half = torch.zeros(300, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(ValueError):
        api.AdamWPlan([half], [g], [m], [v], copies=[half])
    scale, amax = torch.ones(1, device=DEV), torch.zeros(1, device=DEV)
    lists = lambda: ([new(), new()], [g, g], [new(), new()], [new(), new()])  # noqa: E731
    with pytest.raises(ValueError):
        api.AdamWPlan(*lists(), copies=[u8(), u8()], fmt=api.E4M3, scales=[scale, scale], amax_outs=[amax, amax])
    # what is read may be shared, and empty tensors have no place
    api.AdamWPlan(*lists(), copies=[u8(), u8()], fmt=api.E4M3, scales=[scale, scale])
    e = torch.empty(0, device=DEV)
    api.fp8_adamw_step(api.AdamWPlan([e, e, p], [e, e, g], [e, e, m], [e, e, v]), 1e-3, 1)
    torch.cuda.synchronize()
    assert api.fp8_async_status()[0] == 0
