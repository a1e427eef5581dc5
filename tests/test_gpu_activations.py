"""The activations and their slopes by themselves, in binary32 against binary64: the value through a product without
contraction (z = bias), the slope through the backward pass of dy = 1.

Bounds, derived from the arithmetic (u = 2^-24; a hardware exponential is good to 2 ulp, a reciprocal to 1 ulp).
gelu: the tail Phi(-|z|) = bell * t q(t).  Exponent: two roundings of z^2/2, so z^2 u relative; exponential 4u; t: the
denominator's rounding and the Newton step's, 2u, counted 2.7 times; q: eight steps whose terms add up to 1.9 times the sum,
below 9u; two products 2u; the fit 14u at most (8e-7, beyond z = 6) and 1u below 2.5: all within (24 + 2 z^2) u.
Values below 1e-30 are of no consequence (results below the normal range become 0)."""
import math

import pytest
import torch

from paper_2209_05433_b200 import api
from tests.test_gpu_fused import ACTS, E4, K_, _ok, _scalar

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
RANGES = [(-12, -6), (-6, -4), (-4, -2), (-2, -1), (-1, 0), (0, 1), (1, 4), (4, 12)]


def _values(lo, hi, n=1 << 18):
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    return torch.rand(n, generator=g, device=DEV) * (hi - lo) + lo


def _gelu64(x):
    """(value, slope); Phi by erfc, which has no cancellation in the tail"""
    p = torch.erfc(-x / math.sqrt(2)) / 2
    return x * p, p + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)


def _value(z, act):
    n, one = z.numel(), _scalar(1.0)
    A, B = (torch.empty(r, 16, dtype=torch.uint8, device=DEV)[:, :0] for r in (1, n))
    D = torch.empty(1, n, device=DEV)
    api.fp8_gemm_epilogue(A, E4, K_, B, E4, K_, D, one, one, act=ACTS[act], bias=z)
    return D[0].double()


def _slope(z, act):
    out = torch.empty(1, z.numel(), device=DEV)
    api.fp8_epilogue_backward(torch.ones_like(out), z.view(1, -1), out, act=ACTS[act])
    return out[0].double()


@pytest.mark.parametrize("lo,hi", RANGES)
def test_gelu_and_its_slope(lo, hi):
    z = _values(lo, hi)
    x = z.double()
    tail = torch.erfc(x.abs() / math.sqrt(2)) / 2 * (24 + 2 * x * x) * U
    value, slope = _gelu64(x)
    got, got_slope = _value(z, "gelu"), _slope(z, "gelu")
    _ok()
    over = (got - value).abs() - (x.abs() * tail + 3 * U * value.abs() + 1e-30)
    assert float(over.max()) <= 0, float((over / value.abs()).max())
    bump = x.abs() * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi) * (10 + x * x) * U
    over = (got_slope - slope).abs() - (tail + bump + 3 * U * slope.abs() + 1e-30)
    assert float(over.max()) <= 0, float(over.max())


def test_gelu_slopes_do_not_add_up_an_error_of_one_sign():
    """the mean error over a range is what a column sum of gradients sees: below an eighth of a rounding of numbers of size 1"""
    for lo, hi in RANGES:
        z = _values(lo, hi)
        err = (_slope(z, "gelu") - _gelu64(z.double())[1]).mean()
        assert abs(float(err)) <= 2.0 ** -26, (lo, hi, float(err))
    _ok()
