"""GPU parity of the epilogue's backward pass and of the gradient norm with clipping against their definitions in
binary64.

Tolerances, derived: dz is one binary32 product of dy and the slope, the slope a sum of terms of size at most 1.13 (erf
form: absolute error 2^-22 of numbers of size 1; exponential: |z| * 2^-23 relative, and the terms vanish beyond |z| = 16),
so |error| <= 2^-19 (1 + |slope|) |dy|.  A column sum of M terms in binary32, added in chunks: every partial sum is
rounded once per addition, at most (rows of a warp + warps + chunks) <= M/8 + 8 + M/16 + 1 additions of numbers
below sum|dz|.  The norm: squares with 2^-24 relative error, sums of 64 in binary32 (64 * 2^-24 = 2^-18 relative, all
terms positive), the rest in binary64: 2^-18 on the sum, 2^-19 on its root.  Clipped values: 2^-18 from the norm, then one product and one
rounding."""
import math

import pytest
import torch

from paper_2209_05433_b200 import api
from tests.test_gpu_fused import ACTS, ARITH, BF, E4, E5, F32, _act64, _check, _check_amax, _gen, _guards_kept, _matrix, _scalar

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _ok():
    torch.cuda.synchronize()
    assert api.fp8_async_status()[0] == 0


BACKWARD = [
    # M, N, act, dy type, pre type, out, bias
    (1, 1, "silu", BF, BF, BF, True),
    (1, 4096, "gelu_tanh", BF, BF, E5, True),
    (7, 300, "gelu", F32, BF, E4, True),
    (16, 256, "relu", BF, F32, F32, True),
    (17, 257, "silu", F32, F32, E5, True),
    (100, 8, "gelu_tanh", BF, BF, BF, True),
    (333, 1031, "gelu", BF, BF, E5, True),
    (1000, 2000, "none", BF, None, E5, True),
    (2049, 515, "silu", F32, BF, F32, True),
    (5000, 70, "gelu", BF, BF, E4, False),
    (4096, 1024, "gelu_tanh", BF, BF, E5, True),
    (3, 100003, "silu", BF, BF, E5, True),
]


@pytest.mark.parametrize("case", BACKWARD, ids=lambda c: "%dx%d_%s" % c[:3])
def test_epilogue_backward(case):
    M, N, act, dy_t, pre_t, out, bias = case
    g = _gen(M + N)
    dy, _ = _matrix(M, N, dy_t)
    dy.copy_(torch.randn(M, N, generator=g, device=DEV))
    pre = None
    if pre_t is not None:
        pre, _ = _matrix(M, N, pre_t)
        pre.copy_(2.5 * torch.randn(M, N, generator=g, device=DEV))
    codes = not isinstance(out, torch.dtype)
    dz, whole = _matrix(M, N, torch.uint8 if codes else out)
    dbias = torch.full((N,), 9.0, device=DEV) if bias else None
    amax, s = _scalar(-1.0), 5.3
    api.fp8_epilogue_backward(dy, pre, dz, act=ACTS[act], fd=out if codes else None, scale_d=_scalar(s) if codes else None, dbias=dbias, amax_out=amax)
    _ok()
    y = dy.double()
    slope = torch.ones_like(y) if pre is None else _act64(pre.double(), act)[1]
    want, tol = y * slope, ARITH * (1 + slope.abs()) * y.abs()
    _check(dz, want, tol, out if codes else None, s, "dz")
    assert _guards_kept(dz, whole)
    _check_amax(amax, dz, want, tol, codes)
    if bias:
        adds = M / 8 + M / 16 + 9
        bound = tol.sum(0) + adds * 2.0 ** -24 * want.abs().sum(0) * 1.01
        assert bool(((dbias.double() - want.sum(0)).abs() <= bound).all())


@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
def test_epilogue_backward_against_differences(act):
    """dz and dbias are the derivatives of sum(dy * act(z + b)): central differences in binary64, step 1e-4 (truncation
    below 1e-8 of |dy|, rounding below 1e-11)."""
    M, N = 6, 40
    g = _gen(5)
    dy = torch.randn(M, N, generator=g, device=DEV)
    z = torch.randn(M, N, generator=g, device=DEV)
    z = torch.where(z.abs() < 1e-2, z.sign() * 1e-2, z)
    dz, db = torch.empty_like(z), torch.empty(N, device=DEV)
    api.fp8_epilogue_backward(dy, z, dz, act=ACTS[act], dbias=db)
    _ok()
    x, y, e = z.double(), dy.double(), 1e-4
    num = y * (_act64(x + e, act)[0] - _act64(x - e, act)[0]) / (2 * e)
    bound = (2 * ARITH * 2.2 + 1e-7) * y.abs()
    assert bool(((dz.double() - num).abs() <= bound).all())
    assert bool(((db.double() - num.sum(0)).abs() <= bound.sum(0) + 2.0 ** -20 * y.abs().sum(0)).all())


def test_epilogue_backward_in_place_special_values_and_repeats():
    M, N = 300, 520
    for dt in (BF, F32):
        dy, whole = _matrix(M, N, dt)
        dy.copy_(torch.randn(M, N, generator=_gen(1), device=DEV))
        z, _ = _matrix(M, N, dt)
        z.copy_(torch.randn(M, N, generator=_gen(2), device=DEV))
        z[0, 0], z[1, 1], z[2, 2], z[3, 3] = float("inf"), float("-inf"), float("nan"), 1e30
        dy[4, 4], dy[5, 5] = float("inf"), float("nan")
        other, _ = _matrix(M, N, dt)
        d1, d2 = torch.empty(N, device=DEV), torch.empty(N, device=DEV)
        src = dy.clone()
        api.fp8_epilogue_backward(dy, z, other, act=api.ACT_SILU, dbias=d1)
        api.fp8_epilogue_backward(dy, z, dy, act=api.ACT_SILU, dbias=d2)
        _ok()
        assert torch.equal(dy.nan_to_num(nan=7.0), other.nan_to_num(nan=7.0)) and _guards_kept(dy, whole)
        assert torch.equal(d1.nan_to_num(nan=7.0), d2.nan_to_num(nan=7.0))
        assert float(dy[0, 0]) == float(src[0, 0]) and float(dy[1, 1]) == 0 and math.isnan(float(dy[2, 2])) and float(dy[3, 3]) == float(src[3, 3])
        assert math.isnan(float(dy[5, 5])) and math.isinf(float(dy[4, 4])) and int(torch.isnan(dy).sum()) == 2
        assert int(torch.isnan(d1).sum()) == 2 and int(torch.isinf(d1).sum()) == 1


def test_epilogue_backward_one_workspace_serves_shapes_in_any_order():
    """the partial sums of one shape do not lie where another shape's counters are"""
    ws = torch.zeros(int(api.load().fp8_epilogue_backward_workspace_bytes(4096, 4096)), dtype=torch.uint8, device=DEV)
    for M, N in ((4096, 304), (40, 70000), (4096, 4096), (64, 104), (300, 20000), (1, 8), (4096, 304)):
        need = int(api.load().fp8_epilogue_backward_workspace_bytes(M, N))
        if need > ws.numel():
            continue
        dy = torch.randn(M, N, generator=_gen(N), device=DEV).to(BF)
        out, db = torch.empty_like(dy), torch.empty(N, device=DEV)
        api.fp8_epilogue_backward(dy, None, out, dbias=db, workspace=ws)
        _ok()
        assert torch.equal(out, dy)
        want = dy.double().sum(0)
        assert bool(((db.double() - want).abs() <= (M / 8 + M / 16 + 9) * 2.0 ** -23 * dy.double().abs().sum(0)).all())


def test_epilogue_backward_empty_and_refusals():
    dy, out = torch.zeros(0, 24, dtype=BF, device=DEV), torch.zeros(0, 24, dtype=BF, device=DEV)
    db, amax = torch.full((24,), 3.0, device=DEV), _scalar(4.0)
    api.fp8_epilogue_backward(dy, None, out, dbias=db, amax_out=amax)
    _ok()
    assert float(db.abs().max()) == 0 and float(amax) == 0
    dy, z = torch.zeros(8, 24, dtype=BF, device=DEV), torch.zeros(8, 24, dtype=BF, device=DEV)
    with pytest.raises(api.Fp8Error):
        api.fp8_epilogue_backward(dy, None, torch.empty_like(dy), act=api.ACT_SILU)
    with pytest.raises(ValueError):
        api.fp8_epilogue_backward(dy, z[:, :16], torch.empty_like(dy), act=api.ACT_SILU)
    with pytest.raises(TypeError):
        api.fp8_epilogue_backward(dy, z, torch.empty_like(dy), dbias=torch.zeros(23, device=DEV))
    with pytest.raises(api.Fp8Error):
        api.fp8_epilogue_backward(dy, z, torch.empty_like(dy), act=17)
    with pytest.raises(api.Fp8Error):
        api.fp8_epilogue_backward(torch.zeros(8, 25, dtype=BF, device=DEV)[:, :24], z, torch.empty_like(dy))
    with pytest.raises(api.Fp8Error):
        api.fp8_epilogue_backward(dy, z, torch.empty_like(dy), dbias=torch.zeros(24, device=DEV), workspace=torch.zeros(16, dtype=torch.uint8, device=DEV))
    _ok()


CLIPS = [
    # sizes, input type, output type (None: in place)
    ([1], BF, None),
    ([1], F32, BF),
    ([5, 0, 17, 1000], BF, BF),
    ([32768, 32769, 32767, 1], F32, F32),
    ([65536 * 3 + 11], BF, F32),
    ([100] * 300, F32, BF),
    ([4096, 3, 16384, 5, 1 << 20, 7], BF, None),
    ([(1 << 24) + 5, 9, 12345], BF, BF),
    ([(1 << 23) + 1], F32, None),
]


@pytest.mark.parametrize("case", CLIPS, ids=lambda c: "%dx%d_%s" % (len(c[0]), max(c[0]), "inplace" if c[2] is None else "out"))
@pytest.mark.parametrize("factor", [0.5, 2.0])
@pytest.mark.parametrize("shift", [0, 1])
def test_clip(case, factor, shift):
    """clipped (max below the norm) and not; tensors that start on 16 bytes and one element off"""
    sizes, x_t, out_t = case
    g = _gen(len(sizes))
    whole = [torch.full((n + 9,), 55.0, dtype=x_t, device=DEV) for n in sizes]
    grads = [w[shift:shift + n] for w, n in zip(whole, sizes)]
    for i, t in enumerate(grads):
        t.copy_(torch.randn(t.numel(), generator=g, device=DEV) * 1e-3 * (1 + i % 3))
    before = [t.double() for t in grads]
    outs_whole = whole if out_t is None else [torch.full((n + 9,), 55.0, dtype=out_t, device=DEV) for n in sizes]
    outs = [w[shift:shift + n] for w, n in zip(outs_whole, sizes)]
    plan = api.ClipPlan(grads, None if out_t is None else outs)
    want = math.sqrt(sum(float((t * t).sum()) for t in before))
    limit = float(torch.tensor(want * factor, dtype=torch.float32))
    norm = _scalar(-1.0)
    api.fp8_grad_norm(plan, norm)
    _ok()
    assert abs(float(norm) - want) <= 2.0 ** -19 * want + 2.0 ** -24 * want
    norm.fill_(-1.0)
    api.fp8_grad_clip(plan, limit, norm)
    _ok()
    assert abs(float(norm) - want) <= (2.0 ** -19 + 2.0 ** -24) * want
    coef = min(1.0, limit / want)
    for x, o, w in zip(before, outs, outs_whole):
        rounding = 2.0 ** -8 if o.dtype == BF else 2.0 ** -23
        assert bool(((o.double() - x * coef).abs() <= x.abs() * coef * (rounding + 2.0 ** -18)).all())
        if coef == 1.0 and o.dtype == x_t:
            assert torch.equal(o.double(), x)
        assert bool((w[:shift] == 55.0).all()) and bool((w[shift + o.numel():] == 55.0).all())
    if out_t is not None:
        again = [o.clone() for o in outs]
        api.fp8_grad_clip(plan, limit, norm)
        _ok()
        assert all(torch.equal(a, o) for a, o in zip(again, outs))


def test_clip_special_values():
    x = torch.randn(100000, generator=_gen(1), device=DEV)
    for bad, finite in ((float("nan"), None), (float("inf"), 0.0)):
        y = x.clone()
        y[77777] = bad
        out, norm = torch.empty_like(y), _scalar(0.0)
        api.fp8_grad_clip(api.ClipPlan([y, x], [out, torch.empty_like(x)]), 1.0, norm)
        _ok()
        if finite is None:
            assert math.isnan(float(norm)) and bool(torch.isnan(out).all())
        else:
            assert math.isinf(float(norm)) and math.isnan(float(out[77777])) and int(torch.isnan(out).sum()) == 1 and float(out.nan_to_num().abs().max()) == 0
    zero, norm = torch.zeros(1000, device=DEV), _scalar(5.0)
    api.fp8_grad_clip(api.ClipPlan([zero]), 0.0, norm)
    _ok()
    assert float(norm) == 0 and float(zero.abs().max()) == 0


def test_clip_empty_list_and_refusals():
    norm = _scalar(5.0)
    api.fp8_grad_clip(api.ClipPlan([]), 1.0, norm)
    _ok()
    assert float(norm) == 0
    x = torch.ones(10, device=DEV)
    plan = api.ClipPlan([x])
    for bad in (-1.0, float("nan")):
        with pytest.raises(api.Fp8Error):
            api.fp8_grad_clip(plan, bad, norm)
    with pytest.raises(ValueError):
        api.ClipPlan([x], [torch.ones(9, device=DEV)])
    with pytest.raises(ValueError):
        api.ClipPlan([x], [])
    with pytest.raises(TypeError):
        api.ClipPlan([x.half()])
    with pytest.raises(ValueError):
        api.ClipPlan([torch.ones(4, 6, device=DEV).t()])
    with pytest.raises(TypeError):
        api.fp8_grad_norm(plan, torch.zeros(2, device=DEV))
    _ok()
    assert float(x.min()) == 1.0


def test_clip_two_streams():
    """plans of their own on streams of their own"""
    xs = [torch.randn(1 << 20, generator=_gen(i), device=DEV) for i in range(2)]
    outs = [[torch.empty_like(x) for _ in range(4)] for x in xs]
    norms = [[_scalar(0.0) for _ in range(4)] for _ in xs]
    plans = [[api.ClipPlan([x], [o]) for o in row] for x, row in zip(xs, outs)]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    for k in range(4):
        for s, row, nrow in zip(streams, plans, norms):
            with torch.cuda.stream(s):
                api.fp8_grad_clip(row[k], 3.0, nrow[k])
    _ok()
    for x, row, nrow in zip(xs, outs, norms):
        n = float(x.double().norm())
        assert all(abs(float(v) - n) <= 2.0 ** -19 * n * 1.1 for v in nrow) and all(torch.equal(row[0], o) for o in row[1:])
