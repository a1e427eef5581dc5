"""Special values, overflow, operand formats and accumulation modes of the fused products at row counts that the kernel for
many rows takes (above 256, gated above 64), beside a count that the other kernel takes."""
import numpy as np
import pytest
import torch

import oracle
import tests.test_gpu_fused as base
from paper_2209_05433_b200 import api
from tests.test_gpu_fused import ACTS, ARITH, BF, E4, E5, F32, K_, MN, _act64, _check, _codes, _gen, _guards_kept, _matrix, _ok, _run_epilogue, _scalar

pytestmark = pytest.mark.gpu
DEV = "cuda"
MANY = 300
INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("overflow", [api.SATURATE, api.NOSAT])
@pytest.mark.parametrize("fmt", [E4, E5])
def test_epilogue_overflow_and_special_values(fmt, overflow):
    base.test_epilogue_overflow_and_special_values(MANY, fmt, overflow)


@pytest.mark.parametrize("fa,fb", [(E4, E4), (E4, E5), (E5, E4), (E5, E5)])
@pytest.mark.parametrize("acc", [api.ACC_FAST, api.ACC_SPLIT])
@pytest.mark.parametrize("K", [1040, 5000])
def test_epilogue_formats_and_accumulation(fa, fb, acc, K):
    _run_epilogue(MANY, 272, K, K_, MN, "silu", BF, BF, BF, BF, False, fa=fa, fb=fb, acc=acc)


@pytest.mark.parametrize("M", [MANY, 515])
@pytest.mark.parametrize("out", [BF, F32])
def test_epilogue_nan_code_in_an_operand_reaches_its_row_only(M, out):
    def edit(A, a, bias, residual):
        A[2, 5] = A[M - 1, 63] = 0x7F
        a[2, 5] = a[M - 1, 63] = NAN
    D, _, _ = _run_epilogue(M, 96, 64, K_, MN, "none", None, BF, None, out, False, edit=edit)
    assert torch.isnan(D[2]).all() and torch.isnan(D[M - 1]).all() and int(torch.isnan(D).sum()) == 2 * 96


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
def test_activation_at_infinity(act):
    def edit(A, a, bias, residual):
        bias[0], bias[1], bias[2], bias[3], bias[4] = INF, -INF, NAN, 1e30, -1e30
    D, _, _ = _run_epilogue(MANY, 64, 32, K_, K_, act, F32, None, None, F32, False, edit=edit)
    assert bool((D[:, 0] == INF).all()) and bool(torch.isnan(D[:, 2]).all())
    assert bool((D[:, 1] == (-INF if act == "none" else 0)).all())


def _as_codes(v, s, fmt, overflow):
    v = v.contiguous().cpu().numpy()
    return v, oracle.quantize(v.reshape(-1), s, fmt, overflow).reshape(v.shape)


def _same_codes(got, v, want):
    got, nan = got.cpu().numpy(), np.isnan(v)
    assert np.array_equal(got[~nan], want[~nan]) and bool(((got[nan] & 0x7F) == 0x7F).all())


@pytest.mark.parametrize("overflow", [api.SATURATE, api.NOSAT])
@pytest.mark.parametrize("fmt", [E4, E5])
@pytest.mark.parametrize("M", [20, MANY])
@pytest.mark.parametrize("gate_scale", [3e36, 4e37, 0.02])
def test_gated_overflow_and_special_values(gate_scale, M, fmt, overflow):
    """gates that overflow binary32 in some places, NaN operands, results past the format's maximum: the codes are the
    conversion of the fp32 form of the same call, code for code"""
    N, K = 160, 256
    g = _gen(M)
    A, a = _codes(g, M, K, E4, False)
    Bg, bg = _codes(g, N, K, E4, False)
    Bu, bu = _codes(g, N, K, E4, False)
    A[3, 7] = Bu[9, 1] = 0x7F
    a[3, 7] = bu[9, 1] = NAN
    H, whole = _matrix(M, N, torch.uint8)
    W, _ = _matrix(M, N, F32)
    sa, sg, su, s, amax = _scalar(1.0), _scalar(gate_scale), _scalar(0.01), (2e-36 if fmt == E4 else 4e-34) if gate_scale > 1 else (2e3 if fmt == E4 else 3e5), _scalar(0.0)
    api.fp8_gemm_gated(A, E4, K_, Bg, Bu, E4, K_, W, sa, sg, su, act=api.ACT_SILU)
    api.fp8_gemm_gated(A, E4, K_, Bg, Bu, E4, K_, H, sa, sg, su, act=api.ACT_SILU, fd=fmt, scale_d=_scalar(s), overflow=overflow, amax_out=amax)
    _ok()
    v, want = _as_codes(W, s, fmt, overflow)
    _same_codes(H, v, want)
    assert _guards_kept(H, whole) and bool(torch.isnan(amax).all())
    G, U = (a @ bg.T) * sg.double(), (a @ bu.T) * su.double()
    assert bool(torch.isnan(W[3]).all()) and bool(torch.isnan(W[:, 9]).all())
    rest = ~torch.isnan(G) & ~torch.isnan(U)
    sure = rest & (G > 3.5e38) & (U.abs() > 1e-3)                       # act(inf) * u
    assert bool((W[sure] == (INF * U[sure].sign()).float()).all())
    assert gate_scale < 1e37 or int(sure.sum()) > 100
    sure = rest & (G < -1e30)                                           # act is 0 there, whatever overflowed
    assert (gate_scale < 1 or int(sure.sum()) > 100) and bool((W[sure] == 0).all())
    top = oracle.quantize(np.array([1.0], np.float32), 1e9, fmt, overflow)[0]
    past = int(((want == top) & np.isfinite(v)).sum())                  # finite values past the format's range
    assert gate_scale > 1 or past >= 20


@pytest.mark.parametrize("overflow", [api.SATURATE, api.NOSAT])
@pytest.mark.parametrize("fmt", [E4, E5])
@pytest.mark.parametrize("gate_t", [BF, F32])
@pytest.mark.parametrize("M", [20, MANY])
def test_gated_backward_overflow_and_special_values(M, gate_t, fmt, overflow):
    N, K = 96, 128
    g = _gen(M)
    A, a = _codes(g, M, K, E5, False)
    B, bt = _codes(g, N, K, E4, False)
    gate, up = (_matrix(M, N, gate_t)[0] for _ in range(2))
    for t in (gate, up):
        t.copy_(2 * torch.randn(M, N, generator=g, device=DEV))
    gate[:, 0], gate[:, 1], gate[:, 2], gate[:, 3], gate[:, 4] = INF, -INF, NAN, 1e25, -1e25
    up[:, 40], up[M - 1, 41], up[M // 2, 42] = 0.0, INF, NAN
    outs = {dt: [torch.full((M, N), 3, dtype=dt, device=DEV) for _ in range(2)] for dt in (F32, torch.uint8)}
    one, s = _scalar(0.01), 30.0 if fmt == E4 else 4000.0
    for act in ("gelu", "gelu_tanh", "silu", "relu"):
        amax = _scalar(0.0)
        api.fp8_gemm_gated_backward(A, E5, K_, B, E4, K_, gate, up, *outs[F32], one, one, act=ACTS[act])
        api.fp8_gemm_gated_backward(A, E5, K_, B, E4, K_, gate, up, *outs[torch.uint8], one, one, act=ACTS[act], fd=fmt, scale_d=_scalar(s),
                                    overflow=overflow, amax_out=amax)
        _ok()
        for w, c in zip(outs[F32], outs[torch.uint8]):
            v, want = _as_codes(w, s, fmt, overflow)
            _same_codes(c, v, want)
        assert bool(torch.isnan(amax).all())
        dG, dU = outs[F32]
        dh = (a @ bt.T) * one.double() ** 2
        S = (a.abs() @ bt.abs().T) * one.double() ** 2
        keep = torch.ones(M, dtype=torch.bool, device=DEV)
        # up[:, 0..4] is finite: slopes of 1 and 0 far out
        for col, slope in ((0, 1.0), (1, 0.0), (3, 1.0), (4, 0.0)):
            want = dh[:, col] * up[:, col].double() * slope
            tol = (1e-5 * S[:, col] + ARITH * dh[:, col].abs()) * up[:, col].double().abs() + ARITH * want.abs()
            assert bool(((dG[:, col].double() - want).abs()[keep] <= tol[keep]).all()), (act, col)
        assert bool((dU[:, 1] == 0).all()) and bool((dU[:, 4] == 0).all())
        if act != "relu":                                               # relu's slope at NaN is that of z > 0, false
            assert bool(torch.isnan(dG[:, 2]).all())
        assert bool(torch.isnan(dU[:, 2]).all())
        assert bool(torch.isnan(dG[M // 2, 42])) and not bool(torch.isnan(dU[M // 2, 42])) and bool((dG[:, 40] == 0).all())


@pytest.mark.parametrize("acc", [api.ACC_FAST, api.ACC_SPLIT])
@pytest.mark.parametrize("M", [40, 70, MANY])
def test_gated_accumulation(M, acc):
    N, K = 150, 5000
    g = _gen(M)
    A, a = _codes(g, M, K, E4, False)
    Bg, bg = _codes(g, N, K, E4, True)
    Bu, bu = _codes(g, N, K, E4, True)
    H, whole = _matrix(M, N, F32)
    sa, sg, su, amax = _scalar(0.011), _scalar(0.02), _scalar(0.017), _scalar(-1.0)
    api.fp8_gemm_gated(A, E4, K_, Bg, Bu, E4, MN, H, sa, sg, su, act=api.ACT_SILU, amax_out=amax, acc=acc)
    _ok()
    ag, au = sa.double() * sg.double(), sa.double() * su.double()
    G, U = (a @ bg.T) * ag, (a @ bu.T) * au
    tg = 1e-5 * (a.abs() @ bg.abs().T) * ag + ARITH * G.abs()
    tu = 1e-5 * (a.abs() @ bu.abs().T) * au + ARITH * U.abs()
    value, _ = _act64(G, "silu")
    ta = 1.13 * tg + ARITH * (G.abs() + 1e-3)
    _check(H, value * U, ta * (U.abs() + tu) + value.abs() * tu + ARITH * (value * U).abs(), what="H")
    assert _guards_kept(H, whole) and float(amax) == float(H.abs().max())


@pytest.mark.parametrize("acc", [api.ACC_FAST, api.ACC_SPLIT])
@pytest.mark.parametrize("M", [40, MANY])
def test_gated_backward_accumulation(M, acc):
    """act none: dG = dh * up, dU = dh * gate"""
    N, K = 150, 5000
    g = _gen(M)
    A, a = _codes(g, M, K, E5, False)
    B, bt = _codes(g, N, K, E4, False)
    gate, up = (_matrix(M, N, F32)[0] for _ in range(2))
    for t in (gate, up):
        t.copy_(2 * torch.randn(M, N, generator=g, device=DEV))
    dG, dU = torch.empty(M, N + 2, device=DEV)[:, :N], torch.empty(M, N + 2, device=DEV)[:, :N]
    sa, sb = _scalar(0.013), _scalar(0.019)
    api.fp8_gemm_gated_backward(A, E5, K_, B, E4, K_, gate, up, dG, dU, sa, sb, act=api.ACT_NONE, acc=acc)
    _ok()
    alpha = sa.double() * sb.double()
    dh, th = (a @ bt.T) * alpha, 1e-5 * (a.abs() @ bt.abs().T) * alpha
    for got, other, name in ((dG, up, "dG"), (dU, gate, "dU")):
        o = other.double()
        _check(got, dh * o, th * o.abs() + ARITH * (dh * o).abs(), what=name)
