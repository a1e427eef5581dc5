"""The activations and their slopes by themselves, in binary32 against binary64: the value through a product without
contraction (z = bias), the slope through the backward pass of dy = 1.

Bounds, derived from the arithmetic (u = 2^-24; a hardware exponential is good to 2 ulp, a reciprocal to 1 ulp).
gelu: the tail Phi(-|z|) = bell * t q(t).  Exponent: two roundings of z^2/2, so z^2 u relative; exponential 4u; t: the
denominator's rounding and the Newton step's, 2u, counted 2.7 times; q: eight steps whose terms add up to 1.9 times the sum,
below 9u; two products 2u; the fit 14u at most (8e-7, beyond z = 6) and 1u below 2.5: all within (24 + 2 z^2) u.
silu, gelu_tanh: w = 1/(1+e), e = 2^(-c log2 e) with c = z or 1.5958 (z + 0.044715 z^3).  The exponent is within A u of
itself: silu one rounding and the constant's 0.22u, A = 1.25; gelu_tanh z^2, two products of three and two constants, sum and
product, A = 7.  So e is within (A |c| + 5) u of itself (the exponential 4u, 1u to spare), w within w' (A |c| + 5) u + 4u with
w' = 1 - w; w' itself, which is computed as e w, within that and (A |c| + 6) u; the slope is w plus z w w' g with g = 1 or
c'(z), 8 roundings more.
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


@pytest.mark.parametrize("lo,hi", RANGES)
@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
def test_silu_and_gelu_tanh_and_their_slopes(act, lo, hi):
    z = _values(lo, hi)
    x = z.double()
    k = 2 * math.sqrt(2 / math.pi)
    c, g, A = (x, torch.ones_like(x), 1.25) if act == "silu" else (k * (x + 0.044715 * x ** 3), k * (1 + 3 * 0.044715 * x * x), 7)
    w, rest = torch.sigmoid(c), torch.sigmoid(-c)
    de = (A * c.abs() + 5) * U
    dw = rest * de + 4 * U
    value, bend = x * w, x * w * rest * g
    got, got_slope = _value(z, act), _slope(z, act)
    _ok()
    over = (got - value).abs() - (value.abs() * (dw + U) + 1e-30)
    assert float(over.max()) <= 0, float(over.max())
    over = (got_slope - w - bend).abs() - (w * dw + bend.abs() * (2 * dw + de + 9 * U) + U * (w + bend).abs() + 1e-30)
    assert float(over.max()) <= 0, float(over.max())
