"""Fused operators on more than 2^31 elements: addresses, tile coordinates and counts past 32 bits.  Sampled rows and the
corners against binary64; values that are whole numbers over powers of two keep sums and column sums exact."""
import pytest
import torch

from paper_2209_05433_b200 import api
from tests.test_gpu_fused import BF, E4, E5, K_, _gen, _ok, _scalar

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _few(g, rows, cols, dtype=torch.float8_e4m3fn):
    """multiples of 1/4 up to 2 in magnitude, exact in every format"""
    out = torch.empty(rows, cols, dtype=dtype, device=DEV)
    for lo in range(0, rows, 1 << 14):                        # block by block: the random numbers are 32-bit
        out[lo:lo + (1 << 14)] = (torch.randint(-8, 9, (min(1 << 14, rows - lo), cols), generator=g, device=DEV, dtype=torch.int8).float() / 4).to(dtype)
    return out


def test_products_with_more_than_2pow31_outputs():
    """M x N = 70003 x 32768: the epilogue product with the kept value and a residual in place, then the gated block"""
    M, N, K = 70003, 32768, 64
    g = _gen(1)
    A, B, B2 = (_few(g, r, K).view(torch.uint8) for r in (M, N, N))
    a, b, b2 = (t.view(torch.float8_e4m3fn).float() for t in (A, B, B2))
    D = torch.empty(M + 1, N, dtype=BF, device=DEV)
    for lo in range(0, M + 1, 8192):
        D[lo:lo + 8192] = (torch.arange(lo, min(lo + 8192, M + 1), device=DEV) % 128).to(BF)[:, None]      # the residual is its row's number
    amax, one = _scalar(-1.0), _scalar(1.0)
    api.fp8_gemm_epilogue(A, E4, K_, B, E4, K_, D[:M], one, one, act=api.ACT_RELU, residual=D[:M], amax_out=amax)
    _ok()
    rows = torch.cat([torch.arange(5), torch.randint(0, M, (40,)), torch.tensor([65535, 65536, 65537]), torch.arange(M - 5, M)]).to(DEV)
    z = (a[rows] @ b.T).clamp(min=0) + (rows % 128).float()[:, None]
    assert torch.equal(D[rows], z.to(BF)) and bool((D[M] == M % 128).all())
    assert float(amax) == max(float(D[lo:min(lo + 8192, M)].float().abs().max()) for lo in range(0, M, 8192))
    del D
    H = torch.full((M + 1, N), 0x5A, dtype=torch.uint8, device=DEV)
    gate = torch.empty(M, N, dtype=BF, device=DEV)
    up = torch.empty(M, N, dtype=BF, device=DEV)
    api.fp8_gemm_gated(A, E4, K_, B, B2, E4, K_, H[:M], one, one, one, act=api.ACT_RELU, gate=gate, up=up, fd=E4, scale_d=_scalar(0.25), amax_out=amax)
    _ok()
    G, U = a[rows] @ b.T, a[rows] @ b2.T
    h = G.clamp(min=0) * U
    assert torch.equal(gate[rows], G.to(BF)) and torch.equal(up[rows], U.to(BF))
    want = (h * 0.25).clamp(-448, 448).to(torch.float8_e4m3fn)
    assert torch.equal(H[:M][rows].view(torch.float8_e4m3fn).float(), want.float()) and bool((H[M] == 0x5A).all())
    del H
    # and its backward pass, into the two halves of one tensor of 2^32 and more codes
    out = torch.full((M + 1, 2 * N), 0x5A, dtype=torch.uint8, device=DEV)
    api.fp8_gemm_gated_backward(A, E4, K_, B, E4, K_, gate, up, out[:M, :N], out[:M, N:], one, one, act=api.ACT_NONE, fd=E5, scale_d=one, amax_out=amax)
    _ok()
    dh = a[rows] @ b.T
    for got, other in ((out[rows, :N], up[rows].float()), (out[rows, N:], gate[rows].float())):
        assert torch.equal(got.view(torch.float8_e5m2).float(), (dh * other).clamp(-57344, 57344).to(torch.float8_e5m2).float())
    assert bool((out[M] == 0x5A).all())


def test_epilogue_backward_on_more_than_2pow31_elements():
    M, N = 70003, 32768
    g = _gen(2)
    dy = _few(g, M, N, BF)
    out = torch.full((M + 1, N), 0x5A, dtype=torch.uint8, device=DEV)
    dbias, amax = torch.empty(N, device=DEV), _scalar(-1.0)
    dy[M - 1, N - 1] = 96.0                                  # decides the amax, in the last element
    pre = dy                                                 # relu of the gradient itself: dz = max(dy, 0), slope 0 or 1
    api.fp8_epilogue_backward(dy, pre, out[:M], act=api.ACT_RELU, fd=E5, scale_d=_scalar(4.0), dbias=dbias, amax_out=amax)
    _ok()
    total = torch.zeros(N, dtype=torch.float64, device=DEV)
    for lo in range(0, M, 8192):
        part = dy[lo:lo + 8192].float().clamp(min=0)
        total += part.double().sum(0)
        got = out[lo:min(lo + 8192, M)].view(torch.float8_e5m2).float()
        assert torch.equal(got, (part * 4).to(torch.float8_e5m2).float()), lo
    assert float(amax) == 96.0 and bool((out[M] == 0x5A).all())
    assert torch.equal(dbias.double(), total)                # sums below 2^24 quarters: exact


def test_clip_of_a_tensor_of_more_than_2pow31_elements():
    n = (1 << 31) + 70001
    x = torch.zeros(n, dtype=BF, device=DEV)
    x[5], x[(1 << 31) + 9], x[n - 1] = 3.0, 4.0, 12.0        # norm 13
    out = torch.full((n + 8,), 7.0, dtype=BF, device=DEV)
    norm = _scalar(-1.0)
    plan = api.ClipPlan([x], [out[:n]])
    api.fp8_grad_clip(plan, 6.5, norm)
    _ok()
    assert float(norm) == 13.0
    assert float(out[5]) == 1.5 and float(out[(1 << 31) + 9]) == 2.0 and float(out[n - 1]) == 6.0 and bool((out[n:] == 7).all())
    nonzero = sum(int((out[lo:min(lo + (1 << 28), n)] != 0).sum()) for lo in range(0, n, 1 << 28))
    assert nonzero == 3
