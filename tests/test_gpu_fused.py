"""GPU parity of the products with fused epilogues (bias, activation, residual; the gated feed-forward block and its
backward pass) against their definitions in binary64 on the decoded codes.

Tolerances, derived: the dot products are within 1e-5 * S of the exact ones, S = sum|a.b| * scales (the product's own
criterion); every activation here has |act'| <= 1.13, and the binary32 arithmetic of activation, bias, residual and
products adds a few roundings, bounded by 2^-19 of the magnitudes involved (the erf form of gelu subtracts numbers of
size 1, so its absolute error is 2^-22 * |z|; the exponential's argument carries |z| * 2^-23 relative).  Storing adds half
an ulp: 2^-9 relative for bf16 (2^-8 here, next to a power of two), 2^-23 for fp32; codes must lie between the conversions
of the two ends of the interval.  NaN and infinities must match."""
import math

import numpy as np
import pytest
import torch

import oracle
from paper_2209_05433_b200 import api
from tests._util import check_gemm_fp8out

pytestmark = pytest.mark.gpu
DEV = "cuda"
E4, E5 = api.E4M3, api.E5M2
FMAX = {E4: 448.0, E5: 57344.0}
F8 = {E4: torch.float8_e4m3fn, E5: torch.float8_e5m2}
ACTS = {"none": api.ACT_NONE, "relu": api.ACT_RELU, "gelu": api.ACT_GELU, "gelu_tanh": api.ACT_GELU_TANH, "silu": api.ACT_SILU}
ARITH = 2.0 ** -19
GUARD = 771.0


def _scalar(v):
    return torch.tensor([v], dtype=torch.float32, device=DEV)


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _matrix(rows, cols, dtype, fill=GUARD, extra_rows=1):
    """([rows, cols] view, whole buffer): rows start on 16 bytes, padding and a guard row hold `fill`"""
    size = torch.empty(0, dtype=dtype).element_size()
    unit = 16 // size
    pitch = -(-max(cols, 1) // unit) * unit + unit
    whole = torch.full((rows + extra_rows, pitch), 0x5A if dtype == torch.uint8 else fill, dtype=dtype, device=DEV)
    return whole[:rows, :cols], whole


def _guards_kept(view, whole):
    rows, cols = view.shape
    fill = 0x5A if whole.dtype == torch.uint8 else torch.tensor(GUARD, dtype=whole.dtype, device=DEV)
    return bool((whole[rows:] == fill).all()) and bool((whole[:, cols:] == fill).all())


def _codes(g, rows, cols, fmt, mn):
    """(codes stored [rows, cols], or [cols, rows] when mn; their values as [rows, cols] in binary64); padding holds NaN codes"""
    x = torch.randn(rows, cols, generator=g, device=DEV) * torch.exp2(torch.rand(rows, cols, generator=g, device=DEV) * 6 - 4)
    q = x.clamp(-FMAX[fmt], FMAX[fmt]).to(F8[fmt])
    stored = (q.view(torch.uint8).t() if mn else q.view(torch.uint8)).contiguous()
    view, whole = _matrix(stored.shape[0], stored.shape[1], torch.uint8)
    whole.fill_(0x7F)
    view.copy_(stored)
    return view, q.double()


def _act64(z, kind):
    if kind == "none":
        return z, torch.ones_like(z)
    if kind == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z), (z > 0).double()
    if kind == "gelu":
        p = torch.special.ndtr(z)
        return z * p, p + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if kind == "gelu_tanh":
        t = math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
        p = torch.sigmoid(2 * t)
        return z * p, p + z * p * (1 - p) * 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
    p = torch.sigmoid(z)
    return z * p, p + z * p * (1 - p)


def _encode(fmt):
    return lambda a: oracle.quantize(np.ascontiguousarray(a, dtype=np.float32).reshape(-1), 1.0, fmt).reshape(a.shape)


def _check(got, want, tol, fd=None, scale_d=1.0, what=""):
    """one stored matrix against its exact values and their tolerance"""
    if got.dtype == torch.uint8:
        ok, _ = check_gemm_fp8out(got.cpu().numpy(), want.cpu().numpy(), tol.cpu().numpy(), scale_d, _encode(fd), rel=1.0)
        assert ok.all(), "%s: %d of %d codes outside the interval" % (what, (~ok).sum(), ok.size)
        return
    v = got.double()
    tol = tol + want.abs() * (2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -23)
    finite = torch.isfinite(want)
    assert torch.equal(torch.isnan(v), torch.isnan(want)), what + ": NaN places differ"
    assert torch.equal(v[~finite & ~torch.isnan(want)], want[~finite & ~torch.isnan(want)]), what + ": infinities differ"
    worst = ((v - want).abs() - tol)[finite]
    assert worst.numel() == 0 or float(worst.max()) <= 0.0, "%s: %d outside, worst excess %g" % (what, int((worst > 0).sum()), float(worst.max()))


def _check_amax(amax, stored, want, tol, codes):
    if codes:                                              # of the value before scaling and conversion
        a = float(want.abs().max()) if want.numel() else 0.0
        t = float(tol.max()) if want.numel() else 0.0
        assert abs(float(amax) - a) <= t, (float(amax), a, t)
    else:                                                  # of what was stored, bit for bit
        assert float(amax) == (float(stored.float().abs().max()) if stored.numel() else 0.0)


def _ok():
    torch.cuda.synchronize()
    st, detail = api.fp8_async_status()
    assert st == 0, "device-side wait expired, code %d" % detail


# (M, N, K, ma, mb, act, bias, residual, pre, out, channel)
K_, MN = api.MAJOR_K, api.MAJOR_MN
BF, F32 = torch.bfloat16, torch.float32
EPILOGUES = [
    (1, 256, 512, K_, MN, "none", None, BF, None, BF, False),
    (1, 1, 1, K_, K_, "silu", F32, None, F32, F32, False),
    (1, 4096, 4096, K_, K_, "gelu", BF, None, None, E4, True),
    (3, 130, 2500, K_, MN, "gelu_tanh", F32, F32, BF, F32, False),
    (16, 1000, 8192, K_, K_, "relu", BF, BF, F32, E5, True),
    (17, 129, 640, K_, MN, "silu", None, F32, None, BF, False),
    (33, 515, 300, K_, K_, "gelu", F32, BF, BF, E4, False),
    (64, 256, 16400, K_, MN, "none", BF, F32, None, F32, True),
    (65, 384, 1100, K_, K_, "gelu_tanh", None, None, F32, E5, False),
    (100, 77, 144, MN, MN, "silu", BF, F32, BF, BF, False),
    (129, 513, 4500, K_, MN, "gelu_tanh", BF, None, BF, E4, False),
    (257, 300, 2049, MN, K_, "relu", F32, BF, F32, F32, True),
    (300, 1030, 1536, K_, K_, "gelu", BF, BF, None, BF, False),
    (512, 768, 4096, K_, MN, "none", None, BF, None, BF, False),
    (1000, 1111, 520, K_, MN, "silu", F32, F32, F32, E4, True),
    (700, 2048, 6144, K_, K_, "gelu_tanh", BF, F32, BF, F32, False),
    (260, 515, 0, K_, K_, "gelu", BF, F32, F32, BF, False),
    (5, 64, 0, K_, MN, "silu", None, None, None, E4, False),
]


def _run_epilogue(M, N, K, ma, mb, act, bias_t, res_t, pre_t, out, channel, fa=E4, fb=E4, acc=api.ACC_SPLIT, overflow=api.SATURATE, seed=7, edit=None):
    g = _gen(seed + M * 31 + N * 17 + K)
    A, a = _codes(g, M, K, fa, ma == MN)
    B, bt = _codes(g, N, K, fb, mb == MN)
    sa = _scalar(0.0137)
    sb = torch.rand(N, generator=g, device=DEV) * 0.02 + 0.01 if channel else _scalar(0.021)
    bias = torch.randn(N, generator=g, device=DEV).to(bias_t) if bias_t is not None else None
    residual = None
    if res_t is not None:
        residual, _ = _matrix(M, N, res_t)
        residual.copy_(torch.randn(M, N, generator=g, device=DEV))
    pre, pre_whole = _matrix(M, N, pre_t) if pre_t is not None else (None, None)
    codes = out in (E4, E5) and not isinstance(out, torch.dtype)
    D, D_whole = _matrix(M, N, torch.uint8 if codes else out)
    if edit:
        edit(A, a, bias, residual)
    amax, scale_d = _scalar(-1.0), 3.7
    api.fp8_gemm_epilogue(A, fa, ma, B, fb, mb, D, sa, sb, act=ACTS[act], bias=bias, residual=residual, pre=pre,
                          fd=out if codes else None, scale_d=_scalar(scale_d) if codes else None, amax_out=amax, acc=acc, overflow=overflow)
    _ok()
    alpha = sa.double() * sb.double()
    z, S = (a @ bt.T) * alpha, (a.abs() @ bt.abs().T) * alpha
    tol = 1e-5 * S
    if bias is not None:
        z = z + bias.double()
    tol = tol + ARITH * z.abs()
    if pre is not None:
        _check(pre, z, tol, what="pre")
        assert _guards_kept(pre, pre_whole)
    v, _ = _act64(z, act)
    v = torch.where(torch.isneginf(z) & torch.tensor(act not in ("none", "relu"), device=DEV), torch.zeros_like(v), v)
    tol = 1.13 * tol + ARITH * (z.abs() + 1e-3)
    if residual is not None:
        v, tol = v + residual.double(), tol + ARITH * (v.abs() + residual.double().abs())
    tol = torch.nan_to_num(tol, nan=0.0, posinf=0.0)
    _check(D, v, tol, out if codes else None, scale_d, "D")
    assert _guards_kept(D, D_whole)
    if torch.isfinite(v).all():
        _check_amax(amax, D, v, tol, codes)
    return D, v, amax


@pytest.mark.parametrize("case", EPILOGUES, ids=lambda c: "%dx%dx%d_%s" % (c[0], c[1], c[2], c[5]))
def test_epilogue(case):
    _run_epilogue(*case)


@pytest.mark.parametrize("fa,fb", [(E4, E5), (E5, E4), (E5, E5)])
@pytest.mark.parametrize("M", [9, 200])
@pytest.mark.parametrize("acc", [api.ACC_FAST, api.ACC_SPLIT])
def test_epilogue_formats_and_accumulation(fa, fb, M, acc):
    _run_epilogue(M, 272, 1040, K_, MN, "silu", BF, BF, BF, BF, False, fa=fa, fb=fb, acc=acc)


@pytest.mark.parametrize("overflow", [api.SATURATE, api.NOSAT])
@pytest.mark.parametrize("fmt", [E4, E5])
@pytest.mark.parametrize("M", [4, 150])
def test_epilogue_overflow_and_special_values(M, fmt, overflow):
    """codes of results past the format's maximum, infinities and NaN from bias and residual"""
    N, K = 160, 256
    g = _gen(M)
    A, a = _codes(g, M, K, E4, False)
    B, bt = _codes(g, N, K, E4, False)
    bias = torch.randn(N, generator=g, device=DEV)
    bias[3], bias[50], bias[77] = float("inf"), float("-inf"), float("nan")
    residual, _ = _matrix(M, N, F32)
    residual.copy_(torch.randn(M, N, generator=g, device=DEV) * 30)
    residual[0, 8], residual[M - 1, 9], residual[M // 2, 50] = float("nan"), float("-inf"), float("inf")
    D, whole = _matrix(M, N, torch.uint8)
    amax, s = _scalar(0), 40.0 if fmt == E4 else 5000.0
    api.fp8_gemm_epilogue(A, E4, K_, B, E4, K_, D, _scalar(0.02), _scalar(0.02), act=api.ACT_RELU, bias=bias, residual=residual,
                          fd=fmt, scale_d=_scalar(s), overflow=overflow, amax_out=amax)
    W, _ = _matrix(M, N, F32)
    api.fp8_gemm_epilogue(A, E4, K_, B, E4, K_, W, _scalar(0.02), _scalar(0.02), act=api.ACT_RELU, bias=bias, residual=residual)
    _ok()
    # the fp32 form of the same call holds v; its conversion is the oracle's, code for code
    v = W.contiguous().cpu().numpy()
    want = oracle.quantize(v.reshape(-1), s, fmt, overflow).reshape(v.shape)
    got = D.cpu().numpy()
    nan = np.isnan(v)
    assert np.array_equal(got[~nan], want[~nan]) and bool(((got[nan] & 0x7F) == 0x7F).all())
    assert math.isnan(float(amax)) and _guards_kept(D, whole)
    z = (a @ bt.T) * 0.0004 + bias.double()
    z = torch.where(z < 0, torch.zeros_like(z), z) + residual.double()
    assert torch.equal(torch.isnan(z), torch.isnan(W)) and torch.equal(torch.isinf(z), torch.isinf(W))


def test_epilogue_nan_code_in_an_operand_reaches_its_row_only():
    def edit(A, a, bias, residual):
        A[2, 5] = 0x7F
        a[2, 5] = float("nan")
    for M in (6, 140):
        D, v, _ = _run_epilogue(M, 96, 64, K_, MN, "none", None, BF, None, BF, False, edit=edit)
        assert torch.isnan(D[2]).all() and not torch.isnan(D[3:]).any()


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu", "relu"])
def test_activation_at_infinity(act):
    for M in (2, 140):
        def edit(A, a, bias, residual):
            bias[0], bias[1], bias[2] = float("inf"), float("-inf"), float("nan")
            bias[3], bias[4] = 1e30, -1e30
        D, v, _ = _run_epilogue(M, 64, 32, K_, K_, act, F32, None, None, F32, False, edit=edit)
        assert bool((D[:, 0] == float("inf")).all()) and bool((D[:, 1] == 0).all()) and bool(torch.isnan(D[:, 2]).all())


@pytest.mark.parametrize("M", [1, 20, 200, 515])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_residual_in_place(M, dtype):
    """D and the residual may be one matrix"""
    N, K = 520, 700
    g = _gen(M)
    A, a = _codes(g, M, K, E4, False)
    B, bt = _codes(g, N, K, E4, True)
    D, whole = _matrix(M, N, dtype)
    D.copy_(torch.randn(M, N, generator=g, device=DEV))
    other, _ = _matrix(M, N, dtype)
    r = D.clone()
    sa, sb = _scalar(0.01), _scalar(0.02)
    api.fp8_gemm_epilogue(A, E4, K_, B, E4, MN, other, sa, sb, residual=D)
    api.fp8_gemm_epilogue(A, E4, K_, B, E4, MN, D, sa, sb, residual=D)
    _ok()
    assert torch.equal(D, other) and _guards_kept(D, whole)
    v, S = (a @ bt.T) * 0.0002 + r.double(), (a.abs() @ bt.abs().T) * 0.0002
    _check(D, v, 1e-5 * S + ARITH * (v.abs() + r.double().abs()), what="D")


# (M, N, K, ma, mb, act, save, out)
GATED = [
    (1, 256, 512, K_, MN, "silu", None, E4),
    (1, 3, 17, K_, K_, "gelu", F32, F32),
    (2, 1000, 4096, K_, K_, "gelu_tanh", BF, BF),
    (16, 384, 9000, K_, MN, "silu", BF, E4),
    (31, 129, 1234, K_, K_, "relu", F32, E5),
    (50, 640, 2048, K_, MN, "none", BF, F32),
    (64, 777, 100, MN, K_, "silu", None, BF),
    (129, 300, 2200, K_, MN, "silu", BF, E4),
    (300, 515, 4100, MN, MN, "gelu", F32, F32),
    (513, 1024, 1024, K_, K_, "gelu_tanh", BF, E4),
    (700, 130, 5000, K_, MN, "silu", None, E5),
    (260, 2100, 640, K_, K_, "silu", BF, BF),
    (4, 40, 0, K_, K_, "silu", BF, BF),
    (300, 40, 0, K_, MN, "gelu", None, E4),
]


@pytest.mark.parametrize("case", GATED, ids=lambda c: "%dx%dx%d_%s" % (c[0], c[1], c[2], c[5]))
@pytest.mark.parametrize("packed", [False, True])
def test_gated(case, packed):
    M, N, K, ma, mb, act, save, out = case
    g = _gen(M + N + K)
    A, a = _codes(g, M, K, E4, ma == MN)
    Bg, bg = _codes(g, N, K, E4, mb == MN)
    Bu, bu = _codes(g, N, K, E4, mb == MN)
    if packed:                                               # the two operands as halves of one matrix
        if mb == MN:
            half = -(-N // 16) * 16
            both = torch.full((max(K, 1), 2 * half), 0x7F, dtype=torch.uint8, device=DEV)[:K]
            both[:, :N].copy_(Bg)
            both[:, half:half + N].copy_(Bu)
            Bg, Bu = both[:, :N], both[:, half:half + N]
        else:
            pitch = -(-max(K, 1) // 16) * 16
            both = torch.full((2 * N, pitch), 0x7F, dtype=torch.uint8, device=DEV)
            both[:N, :K].copy_(Bg)
            both[N:, :K].copy_(Bu)
            Bg, Bu = both[:N, :K], both[N:, :K]
    codes = not isinstance(out, torch.dtype)
    H, H_whole = _matrix(M, N, torch.uint8 if codes else out)
    gate, gate_whole = _matrix(M, N, save) if save is not None else (None, None)
    up, up_whole = _matrix(M, N, save) if save is not None else (None, None)
    sa, sg, su, amax, scale_d = _scalar(0.011), _scalar(0.02), _scalar(0.017), _scalar(-1.0), 2.3
    api.fp8_gemm_gated(A, E4, ma, Bg, Bu, E4, mb, H, sa, sg, su, act=ACTS[act], gate=gate, up=up, fd=out if codes else None,
                       scale_d=_scalar(scale_d) if codes else None, amax_out=amax)
    _ok()
    ag, au = sa.double() * sg.double(), sa.double() * su.double()
    G, U = (a @ bg.T) * ag, (a @ bu.T) * au
    tg = 1e-5 * (a.abs() @ bg.abs().T) * ag + ARITH * G.abs()
    tu = 1e-5 * (a.abs() @ bu.abs().T) * au + ARITH * U.abs()
    if save is not None:
        _check(gate, G, tg, what="gate")
        _check(up, U, tu, what="up")
        assert _guards_kept(gate, gate_whole) and _guards_kept(up, up_whole)
    value, _ = _act64(G, act)
    ta = 1.13 * tg + ARITH * (G.abs() + 1e-3)
    h = value * U
    tol = ta * (U.abs() + tu) + value.abs() * tu + ARITH * h.abs()
    _check(H, h, tol, out if codes else None, scale_d, "H")
    assert _guards_kept(H, H_whole)
    _check_amax(amax, H, h, tol, codes)


# (M, N, K, ma, mb, act, gate type, out)
GATED_BWD = [
    (1, 256, 512, K_, K_, "silu", BF, E5),
    (3, 17, 33, K_, MN, "gelu", F32, F32),
    (40, 1000, 2049, K_, K_, "gelu_tanh", BF, BF),
    (64, 130, 4500, K_, MN, "relu", F32, E4),
    (128, 515, 256, MN, K_, "silu", BF, E5),
    (130, 260, 3000, K_, K_, "silu", F32, F32),
    (333, 1028, 1024, K_, K_, "gelu_tanh", BF, E5),
    (600, 2048, 2304, K_, MN, "gelu", BF, BF),
    (515, 77, 128, MN, MN, "none", F32, E5),
    (6, 48, 0, K_, K_, "silu", BF, BF),
]


@pytest.mark.parametrize("case", GATED_BWD, ids=lambda c: "%dx%dx%d_%s" % (c[0], c[1], c[2], c[5]))
def test_gated_backward(case):
    M, N, K, ma, mb, act, gate_t, out = case
    g = _gen(M * 3 + N + K)
    A, a = _codes(g, M, K, E5, ma == MN)
    B, bt = _codes(g, N, K, E4, mb == MN)
    gate, _ = _matrix(M, N, gate_t)
    up, _ = _matrix(M, N, gate_t)
    gate.copy_(2 * torch.randn(M, N, generator=g, device=DEV))
    up.copy_(2 * torch.randn(M, N, generator=g, device=DEV))
    codes = not isinstance(out, torch.dtype)
    dt = torch.uint8 if codes else out
    half = -(-N // 16) * 16
    whole = torch.full((M + 1, 2 * half), 0x5A if codes else GUARD, dtype=dt, device=DEV)      # [dG | dU] as one tensor
    dG, dU = whole[:M, :N], whole[:M, half:half + N]
    sa, sb, amax, scale_d = _scalar(0.013), _scalar(0.019), _scalar(-1.0), 1.9
    api.fp8_gemm_gated_backward(A, E5, ma, B, E4, mb, gate, up, dG, dU, sa, sb, act=ACTS[act], fd=out if codes else None,
                                scale_d=_scalar(scale_d) if codes else None, amax_out=amax)
    _ok()
    alpha = sa.double() * sb.double()
    dh, S = (a @ bt.T) * alpha, (a.abs() @ bt.abs().T) * alpha
    th = 1e-5 * S + ARITH * dh.abs()
    G, U = gate.double(), up.double()
    value, slope = _act64(G, act)
    # the slope is a sum of terms of size up to 1.13 + |z| phi(z): a few roundings of numbers of size 1 to 2
    ts, tv = ARITH * (1.0 + slope.abs()), ARITH * (G.abs() + 1e-3)
    wg, wu = dh * U * slope, dh * value
    tg = (th * (slope.abs() + ts) + dh.abs() * ts) * U.abs() + ARITH * wg.abs()
    tu = th * (value.abs() + tv) + dh.abs() * tv + ARITH * wu.abs()
    _check(dG, wg, tg, out if codes else None, scale_d, "dG")
    _check(dU, wu, tu, out if codes else None, scale_d, "dU")
    fill = 0x5A if codes else GUARD
    assert bool((whole[M:] == fill).all()) and bool((whole[:, N:half] == fill).all()) and bool((whole[:, half + N:] == fill).all())
    both, tol = torch.cat([wg, wu], 1), torch.cat([tg, tu], 1)
    _check_amax(amax, torch.cat([dG, dU], 1) if not codes else dG, both, tol, codes)


@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
def test_gated_backward_against_differences(act):
    """dG and dU are the derivatives of sum(dh * act(g) * u): compared with central differences in binary64.
    Step 1e-4: truncation h^2/6 |f'''| <= 1e-8, rounding 1e-12; the binary32 side is within 2^-18 of the magnitudes."""
    M, N, K = 5, 96, 64
    g = _gen(3)
    A, a = _codes(g, M, K, E5, False)
    B, bt = _codes(g, N, K, E4, False)
    gate = torch.randn(M, N, generator=g, device=DEV)
    gate = torch.where(gate.abs() < 1e-2, gate.sign() * 1e-2, gate)              # relu has no derivative at 0
    up = torch.randn(M, N, generator=g, device=DEV)
    dG, dU = torch.empty(M, N, device=DEV), torch.empty(M, N, device=DEV)
    sa, sb = _scalar(0.02), _scalar(0.03)
    api.fp8_gemm_gated_backward(A, E5, K_, B, E4, K_, gate, up, dG, dU, sa, sb, act=ACTS[act])
    _ok()
    dh = (a @ bt.T) * (sa.double() * sb.double())
    S = (a.abs() @ bt.abs().T) * (sa.double() * sb.double())
    f = lambda x, y: dh * _act64(x, act)[0] * y  # noqa: E731
    x, y, e = gate.double(), up.double(), 1e-4
    ng, nu = (f(x + e, y) - f(x - e, y)) / (2 * e), (f(x, y + e) - f(x, y - e)) / (2 * e)
    bound = (1e-5 * S + 2.0 ** -18 * dh.abs() + 1e-7) * 2.0
    assert bool(((dG.double() - ng).abs() <= bound * (1 + y.abs())).all())
    assert bool(((dU.double() - nu).abs() <= bound * (1 + x.abs())).all())


def test_gate_infinities_do_not_make_nan_slopes():
    """far out the derivative is 0 or 1, not 0 * inf"""
    for act in ("gelu", "gelu_tanh", "silu"):
        for M in (2, 150):
            A, a = _codes(_gen(1), M, 32, E5, False)
            B, bt = _codes(_gen(2), 32, 32, E4, False)
            gate = torch.zeros(M, 32, device=DEV)
            gate[:, 0], gate[:, 1], gate[:, 2], gate[:, 3], gate[:, 4] = float("inf"), float("-inf"), 1e25, -1e25, float("nan")
            up = torch.ones(M, 32, device=DEV)
            dG, dU = torch.empty(M, 32, device=DEV), torch.empty(M, 32, device=DEV)
            api.fp8_gemm_gated_backward(A, E5, K_, B, E4, K_, gate, up, dG, dU, _scalar(1.0), _scalar(1.0), act=ACTS[act])
            _ok()
            dh = (a @ bt.T)
            for col, slope in ((0, 1.0), (1, 0.0), (2, 1.0), (3, 0.0)):
                assert torch.allclose(dG[:, col].double(), dh[:, col] * slope, rtol=1e-4, atol=1e-3)
            assert bool((dU[:, 1] == 0).all()) and bool((dU[:, 3] == 0).all()) and bool(torch.isnan(dG[:, 4]).all())


def test_empty_products():
    one = _scalar(1.0)
    A = torch.zeros(0, 64, dtype=torch.uint8, device=DEV)
    B = torch.zeros(32, 64, dtype=torch.uint8, device=DEV)
    D = torch.zeros(0, 32, dtype=BF, device=DEV)
    amax = _scalar(5.0)
    api.fp8_gemm_epilogue(A, E4, K_, B, E4, K_, D, one, one, amax_out=amax)
    assert float(amax) == 0.0
    amax.fill_(5.0)
    api.fp8_gemm_gated(A, E4, K_, B, B, E4, K_, D, one, one, one, amax_out=amax)
    assert float(amax) == 0.0
    _ok()


@pytest.mark.parametrize("M", [1, 40, 300])
def test_repeated_calls_and_other_streams_are_bit_identical(M):
    N, K = 1040, 3000
    g = _gen(M)
    A, _ = _codes(g, M, K, E4, False)
    Bg, _ = _codes(g, N, K, E4, True)
    Bu, _ = _codes(g, N, K, E4, True)
    s = _scalar(0.01)
    outs = [torch.empty(M, N, dtype=F32, device=DEV) for _ in range(8)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        with torch.cuda.stream(streams[i % 2]):
            api.fp8_gemm_gated(A, E4, K_, Bg, Bu, E4, MN, o, s, s, s)
    _ok()
    assert all(torch.equal(outs[0], o) for o in outs[1:])


def test_seeded_shapes():
    """random shapes, layouts and parts through the epilogue product"""
    import random
    r = random.Random(11)
    for i in range(24):
        M, N, K = (int(2 ** r.uniform(0, 9.5)) for _ in range(3))
        out = r.choice([BF, F32, E4, E5])
        pick = lambda: r.choice([None, BF, F32])  # noqa: E731
        _run_epilogue(M, N, K, r.choice([K_, MN]), r.choice([K_, MN]), r.choice(list(ACTS)), pick(), pick(), pick(), out, r.random() < 0.3, seed=i)


def test_refusals():
    one = _scalar(1.0)
    z = lambda *s, dtype=torch.uint8: torch.zeros(*s, dtype=dtype, device=DEV)  # noqa: E731
    A, B, D = z(32, 64), z(48, 64), z(32, 48, dtype=BF)
    ok = dict(act=api.ACT_SILU)
    call = lambda **k: api.fp8_gemm_epilogue(A, E4, K_, B, E4, K_, D, one, one, **{**ok, **k})  # noqa: E731
    call()
    with pytest.raises(ValueError):
        call(bias=z(47, dtype=BF))
    with pytest.raises(ValueError):
        call(residual=z(32, 47, dtype=BF))
    with pytest.raises(TypeError):
        call(residual=z(32, 48, dtype=torch.float16))
    with pytest.raises(ValueError):
        call(pre=z(48, 32, dtype=BF).t())
    with pytest.raises(TypeError):
        call(fd=E4)                                          # a wide output takes no format
    with pytest.raises(TypeError):
        api.fp8_gemm_epilogue(A, E4, K_, B, E4, K_, z(32, 48), one, one)            # codes need fd and scale_d
    with pytest.raises(api.Fp8Error):
        call(act=9)
    with pytest.raises(api.Fp8Error):
        call(residual=z(32, 49, dtype=BF)[:, :48])           # rows do not start on 16 bytes
    with pytest.raises(api.Fp8Error):
        api.fp8_gemm_epilogue(A, 3, K_, B, E4, K_, D, one, one)
    with pytest.raises(TypeError):
        api.fp8_gemm_epilogue(A, E4, K_, B, E4, K_, D, one, z(47, dtype=F32))        # scales: one, or one per column
    with pytest.raises(ValueError):
        api.fp8_gemm_gated(A, E4, K_, B, z(48, 80)[:, :64], E4, K_, D, one, one, one)     # another row pitch
    with pytest.raises(ValueError):
        api.fp8_gemm_gated(A, E4, K_, B, B, E4, K_, D, one, one, one, gate=z(32, 48, dtype=BF))
    with pytest.raises(ValueError):
        api.fp8_gemm_gated_backward(A, E4, K_, B, E4, K_, z(32, 48, dtype=BF), z(32, 48, dtype=F32), D, z(32, 48, dtype=BF), one, one)
    with pytest.raises(ValueError):
        api.fp8_gemm_gated_backward(A, E4, K_, B, E4, K_, None, None, D, z(32, 48, dtype=BF), one, one)
    _ok()


@pytest.mark.parametrize("M", [3, 300])
def test_amax_with_and_without_a_workspace(M):
    """the C entry with a workspace, left zeroed by every call, and without one"""
    import ctypes
    N, K = 384, 256
    g = _gen(M)
    A, a = _codes(g, M, K, E4, False)
    B, bt = _codes(g, N, K, E4, False)
    D = torch.empty(M, N, dtype=F32, device=DEV)
    d = api.GemmDesc(M, N, K, E4, E4, K_, K_, A.stride(0), B.stride(0), N, api.F32, api.ACC_SPLIT)
    e = api.Epilogue(api.ACT_NONE, api.STORE_F32, api.SATURATE, 0, 0, 0)
    one = _scalar(1.0)
    ws = torch.zeros(16, dtype=torch.uint8, device=DEV)
    for use in (None, ws, ws, None, ws):
        amax = _scalar(-3.0)
        st = api.load().fp8_gemm_epilogue(ctypes.byref(d), ctypes.byref(e), A.data_ptr(), B.data_ptr(), D.data_ptr(), one.data_ptr(), one.data_ptr(), None,
                                          amax.data_ptr(), None if use is None else use.data_ptr(), torch.cuda.current_stream().cuda_stream)
        _ok()
        assert st == 0 and float(amax) == float(D.abs().max()) and int(ws.sum()) == 0
