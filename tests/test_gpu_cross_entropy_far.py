"""Softmax cross entropy where the logits are far from zero: of ten thousand and more, up to 1e18, and with a common offset.

What binary32 allows.  A logit and an lse are binary32 numbers: where one logit of a row stands alone, by more than 200 above all others, the
sum of exponentials is 1, the lse is that logit, and softmax is 1 there and 0 (below 1e-86) elsewhere, whatever the logit's size and
whatever rounding its sum has had.  With factors dloss of one power of two the gradient of the logits is then -dloss, 0 or dloss without any rounding."""
import pytest
import torch

from paper_2209_05433_b200 import api
from tests.test_gpu_cross_entropy import DEV, E4, F32, _ok, _operand
from tests.test_gpu_fused import _gen, _matrix, _scalar

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size", [1e4, 1e6, 1e9, 1e18])
@pytest.mark.parametrize("T,K,V", [(3, 256, 1000), (100, 512, 40000), (200, 256, 40000), (300, 1090, 25001), (5000, 1090, 20000)])
@pytest.mark.parametrize("fmt", [E4, None], ids=["fp8", "bf16"])
def test_a_logit_that_stands_alone(fmt, T, K, V, size):
    g = _gen(T + V)
    x = torch.randn(T, K, generator=g, device=DEV) * (1.0 if fmt is not None else size)
    w = torch.randn(V, K, generator=g, device=DEV) * K ** -0.5
    (x, x64), (w, w64) = _operand(x, fmt), _operand(w, fmt)
    sx, sw = (None, None) if fmt is None else (_scalar(size), _scalar(1.0))
    a = 1.0 if fmt is None else float(sx)
    z = x64 @ w64.T * a
    two, at = z.topk(2, dim=1)
    tol = 1e-5 * (x64.abs() @ w64.abs().T).max(1)[0] * a              # the products' own criterion
    alone = two[:, 0] - two[:, 1] > 200 + 2 * tol + 2.0 ** -22 * two[:, 0].abs()
    assert int(alone.sum()) >= T // 3
    rows = torch.arange(T, device=DEV)
    target = torch.where(rows % 2 == 0, at[:, 0], torch.randint(0, V, (T,), generator=g, device=DEV))
    target = torch.where(alone, target, torch.full_like(target, -100))
    dloss = torch.full((T,), 2.0 ** -8, device=DEV)
    loss, lse = torch.empty(T, device=DEV), torch.empty(T, device=DEV)
    (dx, _), (dw, _) = _matrix(T, K, F32), _matrix(V, K, F32)
    api.fp8_cross_entropy(x, fmt, w, fmt, target, loss, lse, scale_inv_x=sx, scale_inv_w=sw)
    api.fp8_cross_entropy_backward(x, fmt, w, fmt, target, lse, dloss, dx, dw, scale_inv_x=sx, scale_inv_w=sw)
    _ok()
    right = alone & (target == at[:, 0])
    assert bool(((lse.double() - two[:, 0]).abs() <= tol + 2.0 ** -22 * two[:, 0].abs())[alone].all())
    assert not loss[right].any() and not loss[~alone].any()
    assert not dx[right].any() and not dx[~alone].any()
    # the others: one logit too high, the target's too low
    dz = torch.zeros(T, V, dtype=torch.float64, device=DEV)
    wrong = alone & ~right
    dz[rows[wrong], at[wrong, 0]] = 2.0 ** -8
    dz[rows[wrong], target[wrong]] = -2.0 ** -8
    for got, want, most in ((dx, dz @ w64, dz.abs() @ w64.abs()), (dw, dz.T @ x64 * a, dz.abs().T @ x64.abs() * a)):
        assert bool(((got.double() - want).abs() <= 1e-5 * most).all())


@pytest.mark.parametrize("offset", [0, 32, 100, -100])
@pytest.mark.parametrize("fmt", [E4, None], ids=["fp8", "bf16"])
@pytest.mark.parametrize("T,V", [(5, 3000), (150, 777)])
def test_a_common_offset_leaves_the_loss_alone(T, V, fmt, offset):
    """Small whole operands, whose sums are exact, and an offset of up to 10000 in every logit.  lse is top + log(sum), one rounding of its
    size, the loss (top - logit) + log(sum) with an exact difference; the logarithm's argument carries 32 + 7 + 5 additions and 2 ulp of
    each exponential and of its argument, of up to 64 log2(e): 2^-17."""
    g = _gen(T + V + offset)
    x = torch.randint(-2, 3, (T, 64), generator=g, device=DEV).float()
    w = torch.randint(-1, 2, (V, 64), generator=g, device=DEV).float()
    x[:, 0], w[:, 0] = abs(offset), offset
    if fmt is not None and abs(offset) == 100:
        x[:, 0], w[:, 0] = 96, offset * 0.96                          # E4M3 holds 96
    (x, x64), (w, w64) = _operand(x, fmt), _operand(w, fmt)
    one = None if fmt is None else _scalar(1.0)
    target = torch.randint(0, V, (T,), generator=g, device=DEV)
    loss, lse = torch.empty(T, device=DEV), torch.empty(T, device=DEV)
    api.fp8_cross_entropy(x, fmt, w, fmt, target, loss, lse, scale_inv_x=one, scale_inv_w=one)
    _ok()
    z = x64 @ w64.T
    want = torch.logsumexp(z, 1)
    assert bool(((lse.double() - want).abs() <= 2.0 ** -24 * want.abs() + 2.0 ** -17).all())
    exact = want - z.gather(1, target[:, None]).squeeze(1)
    assert bool(((loss.double() - exact).abs() <= 2.0 ** -24 * exact + 2.0 ** -17).all())
