"""Fused products where a call is refused late, has no contraction, or is larger than one launch."""
import pytest
import torch

from paper_2209_05433_b200 import api
from tests.test_gpu_fused import BF, E4, E5, F32, K_, MN, _act64, _gen, _ok, _scalar

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _empty(rows):
    return torch.empty(rows, 16, dtype=torch.uint8, device=DEV)[:, :0]


@pytest.mark.parametrize("M", [64 * 65535, 64 * 65535 + 77])
def test_empty_sum_over_more_rows_than_one_launch(M):
    """K == 0: z = bias.  The binary32 values are exact, so there is one rounding, of what is stored."""
    N = 3
    bias = torch.tensor([0.5, -0.25, 1.75], device=DEV)
    D, pre = (torch.full((M + 1, 8), 9.0, dtype=BF, device=DEV) for _ in range(2))
    residual = torch.zeros(M, 8, dtype=BF, device=DEV)
    residual[:, 0] = torch.arange(M, device=DEV) % 200               # whole numbers below 256: bf16 holds them
    residual[M - 1, 2] = 100.0
    amax = _scalar(-1.0)
    api.fp8_gemm_epilogue(_empty(M), E4, K_, _empty(N), E4, K_, D[:M, :N], _scalar(1.0), _scalar(1.0), act=api.ACT_RELU, bias=bias,
                          residual=residual[:, :N], pre=pre[:M, :N], amax_out=amax)
    _ok()
    want = bias.clamp(min=0) + residual[:, :N].float()
    assert torch.equal(D[:M, :N], want.to(BF)) and bool((D[:M, N:] == 9).all()) and bool((D[M] == 9).all())
    assert bool((pre[:M, :N] == bias.to(BF)).all()) and bool((pre[:M, N:] == 9).all()) and bool((pre[M] == 9).all())
    assert float(amax) == float(want.to(BF).abs().max())


def test_empty_sum_of_the_gated_block_over_more_rows_than_one_launch():
    M, N = 32 * 65535 + 5, 16
    H = torch.full((M + 1, N), 0x5A, dtype=torch.uint8, device=DEV)
    gate, up = (torch.full((M + 1, N), 9.0, dtype=BF, device=DEV) for _ in range(2))
    amax, one = _scalar(-1.0), _scalar(1.0)
    api.fp8_gemm_gated(_empty(M), E4, K_, _empty(N), _empty(N), E4, K_, H[:M], one, one, one, gate=gate[:M], up=up[:M], fd=E4, scale_d=one, amax_out=amax)
    _ok()
    assert int(H[:M].max()) == 0 and bool((H[M] == 0x5A).all()) and float(amax) == 0
    for t in (gate, up):
        assert float(t[:M].abs().max()) == 0 and bool((t[M] == 9).all())


def test_empty_sum_of_the_gated_backward_over_more_rows_than_one_launch():
    M, N = 64 * 65535 + 1, 8
    gate = torch.ones(M, N, dtype=BF, device=DEV)
    out = torch.full((M + 1, 2 * N), 9.0, dtype=BF, device=DEV)
    amax, one = _scalar(-1.0), _scalar(1.0)
    api.fp8_gemm_gated_backward(_empty(M), E5, K_, _empty(N), E4, K_, gate, gate, out[:M, :N], out[:M, N:], one, one, amax_out=amax)
    _ok()
    assert float(out[:M].abs().max()) == 0 and bool((out[M] == 9).all()) and float(amax) == 0


@pytest.mark.parametrize("M", [1, 300])
def test_a_refused_call_leaves_nothing_behind(M):
    """a row pitch of 2^40 bytes cannot be described to the copy unit; the amax keeps its value and nothing is launched.  The
    rows of B exist once (N == 1), so the pitch is never walked."""
    A = torch.zeros(M, 64, dtype=torch.uint8, device=DEV)
    B = torch.zeros(64, dtype=torch.uint8, device=DEV).as_strided((1, 64), (1 << 40, 1))
    D = torch.zeros(M, 8, dtype=BF, device=DEV)[:, :1]
    amax, one = _scalar(7.0), _scalar(1.0)
    torch.cuda.synchronize()
    before = api.fp8_launch_count()
    with pytest.raises(api.Fp8Error):
        api.fp8_gemm_epilogue(A, E4, K_, B, E4, K_, D, one, one, amax_out=amax)
    _ok()
    assert api.fp8_launch_count() == before and float(amax) == 7.0


@pytest.mark.parametrize("M", [1, 20, 40, 64])
def test_few_rows_add_partial_sums_every_512_of_k(M):
    """The tensor core's additions truncate at 24 bits.  Behind one product of 448 * 448 come 15/1024 in every step of 32 of K:
    beside the large number (units of 2^-6) each may be lost, but only in the 16 steps of one partial sum.  Then two terms of
    the bound: 16 units, and one rounding by half a unit for each of at most 3 + 7 additions of partial sums that hold the
    large number (4 partial sums in a slice of 2048, 8 slices)."""
    K, N = 16384, 128
    a, b = torch.zeros(M, K, device=DEV), torch.zeros(N, K, device=DEV)
    a[:, ::32], b[:, ::32] = 0.5, 15.0 / 512
    a[:, 0], b[:, 0] = 448.0, 448.0
    A, B = (t.to(torch.float8_e4m3fn).view(torch.uint8) for t in (a, b))
    D = torch.empty(M, N, device=DEV)
    api.fp8_gemm_epilogue(A, E4, K_, B, E4, K_, D, _scalar(1.0), _scalar(1.0))
    _ok()
    want = 448.0 * 448 + (K // 32 - 1) * 15.0 / 1024
    assert bool(((D.double() - want).abs() <= (16 + 10 * 0.5) * 2.0 ** -6).all()), (float(D.min()) - want, float(D.max()) - want)
