"""GPU parity of the AdamW step against its definition in binary64.

Tolerances, derived, in units of the terms' magnitudes.  g' = g * coef carries the division's and the product's rounding
(2^-23); m = b1 m + (1 - b1) g' adds at most three more of its terms: 2^-21 (|b1 m| + |(1 - b1) g'|).  v squares g': 2^-20 of its
terms, all positive.  8-bit moments are read as code * scale (2^-24) and r squared (2^-22 more): 2^-20 covers both.  r = sqrt(v):
half of v's relative error and 1 ulp, 2^-20.  The divisor r / sqrt(1 - b2^t) + eps and the factor lr / (1 - b1^t) carry a few
roundings each, the reciprocal 1 ulp: 2^-18 of the update, plus m's own error through it.  p: the factor 1 - lr wd and the product
are rounded, 2^-22 |p|; storing adds half a step (2^-8 bf16, 2^-24 binary32).
8-bit m: the code lies between the conversions of the ends of its interval.  8-bit r: floor(y / step + u) with the u that its
place, the seed and t give, where y / step (at most 16) carries 2^-19 relative: the code of either end of that interval."""
import math

import numpy as np
import pytest
import torch

from paper_2209_05433_b200 import api
from tests.test_gpu_fused import _gen, _scalar

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32, U8 = torch.bfloat16, torch.float32, torch.uint8
E4, E5 = api.E4M3, api.E5M2
F8 = {E4: torch.float8_e4m3fn, E5: torch.float8_e5m2}
FMAX = {E4: 448.0, E5: 57344.0}
HALF = {BF: 2.0 ** -8, F32: 2.0 ** -24}
GUARD = 5.0


def _ok():
    torch.cuda.synchronize()
    assert api.fp8_async_status()[0] == 0


def _mix(x):
    x = ((x ^ (x >> np.uint32(16))) * np.uint32(0x7FEB352D)).astype(np.uint32)
    x = ((x ^ (x >> np.uint32(15))) * np.uint32(0x846CA68B)).astype(np.uint32)
    return x ^ (x >> np.uint32(16))


def chances(number, n, seed, t):
    """the random numbers of elements number .. number + n - 1 (number even)"""
    one = lambda v: np.array([v & 0xFFFFFFFF], dtype=np.uint32)  # noqa: E731
    key = _mix(one(seed) ^ _mix(one(seed >> 32) ^ _mix(one(t))))
    pairs = (np.arange(number // 2, number // 2 + (n + 1) // 2, dtype=np.uint64) & np.uint64(0xFFFFFFFF)).astype(np.uint32)
    with np.errstate(over="ignore"):
        word = _mix(pairs * np.uint32(0x9E3779B1) + key)
    u = np.stack([word & np.uint32(0xFFFF), word >> np.uint32(16)], axis=1).reshape(-1)[:n]
    return torch.from_numpy(u.astype(np.float64) / 65536.0).to(DEV)


class Tensors:
    """One parameter with everything that belongs to it, each inside a buffer with guards, `shift` elements from its start."""

    def __init__(self, n, p_t, g_t, codes, copy, g, shift=0, decay=0.1, start=True):
        self.n, self.p_t, self.g_t, self.codes, self.copy_t, self.decay = n, p_t, g_t, codes, copy, decay
        self.whole = []

        def put(values, dtype):
            w = torch.full((n + 64,), GUARD, device=DEV).to(dtype)
            w[32 + shift:32 + shift + n] = values
            self.whole.append((w, 32 + shift, n))
            return w[32 + shift:32 + shift + n]

        self.p = put((torch.randn(n, generator=g, device=DEV) * 0.05).to(p_t), p_t)
        grad = torch.randn(n, generator=g, device=DEV) * torch.exp2(torch.rand(n, generator=g, device=DEV) * 12 - 16)
        self.g = put(grad.to(g_t), g_t)
        blocks = -(-n // 256)
        if codes:
            some = 1 if start else 0
            self.m = put(torch.randint(0, 256, (n,), generator=g, device=DEV).where(torch.rand(n, generator=g, device=DEV) < 0.9, torch.zeros(n, device=DEV)).mul(some).to(U8), U8)
            self.m[(self.m & 0x7F) == 0x7F] = 0x7E * some                 # NaN codes
            self.v = put(torch.randint(0, 0x7F, (n,), generator=g, device=DEV).mul(some).to(U8), U8)
            self.ms = torch.rand(blocks, generator=g, device=DEV) * 1e-5 * some
            self.vs = torch.rand(blocks, generator=g, device=DEV) * 1e-5 * some
        else:
            self.m = put(torch.randn(n, generator=g, device=DEV) * 1e-3, F32)
            self.v = put(torch.rand(n, generator=g, device=DEV).square() * 1e-5, F32)
            self.ms = self.vs = None
        self.copy = self.scale = self.amax = None
        if copy is not None:
            self.copy = put(torch.zeros(n, device=DEV), BF if copy == "bf16" else U8)
            if copy != "bf16":
                self.scale, self.amax = _scalar(FMAX[copy] / 0.2), _scalar(-1.0)
        self.old = {k: getattr(self, k).clone() for k in ("p", "g", "m", "v") if getattr(self, k) is not None}
        self.old_scales = (None, None) if not codes else (self.ms.clone(), self.vs.clone())

    def guards_kept(self):
        return all(bool((w[:a] == w[0]).all()) and bool((w[a + n:] == w[-1]).all()) for w, a, n in self.whole)

    def moments(self):
        """the moments before the step in binary64: m, and r or v"""
        if not self.codes:
            return self.old["m"].double(), self.old["v"].double()
        spread = lambda s: s.double().repeat_interleave(256)[:self.n]  # noqa: E731
        m = self.old["m"].view(F8[E4]).double() * spread(self.old_scales[0])
        r = self.old["v"].view(F8[E4]).double() * spread(self.old_scales[1])
        return m, r * r


def _plan(ts):
    by = lambda k: [getattr(t, k) for t in ts]  # noqa: E731
    fmts = {t.copy_t for t in ts} & {E4, E5}
    return api.AdamWPlan(by("p"), by("g"), by("m"), by("v"), weight_decay=by("decay"), exp_avg_scales=by("ms"), exp_avg_sq_scales=by("vs"), copies=by("copy"),
                         fmt=fmts.pop() if fmts else None, scales=by("scale"), amax_outs=by("amax"))


def _grid(y):
    return torch.exp2((torch.frexp(y)[1] - 1).clamp(min=-6).double() - 3)


def _check_tensor(t, number, lr, step, b1, b2, eps, coef, seed):
    m, v = t.moments()
    g = t.old["g"].double() * coef
    tol_m = 2.0 ** -21 * ((b1 * m).abs() + ((1 - b1) * g).abs())
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    tol_v = 2.0 ** -20 * v + 1e-44
    r = v.sqrt()
    tol_r = 2.0 ** -20 * r + 1e-22
    rate, div = lr / (1 - b1 ** step), r / math.sqrt(1 - b2 ** step) + eps
    p0 = t.old["p"].double()
    p = p0 * (1 - lr * t.decay) - rate * m / div
    tol_p = 2.0 ** -22 * p0.abs() + rate * (tol_m + 2.0 ** -18 * m.abs()) / div
    tol_p = tol_p + HALF[t.p_t] * (p.abs() + tol_p)
    assert bool(((t.p.double() - p).abs() <= tol_p).all())
    if t.codes:
        n, blocks = t.n, -(-t.n // 256)
        pad = lambda a: torch.nn.functional.pad(a, (0, blocks * 256 - n)).view(blocks, 256)  # noqa: E731
        for got, scale, exact, tol in ((t.m, t.ms, m, tol_m), (t.v, t.vs, r, tol_r)):
            top, off = pad(exact).abs().amax(1), pad(tol).amax(1)
            assert bool(((scale.double() * 448 - top).abs() <= off + 2.0 ** -22 * top).all())
        spread = lambda s: s.double().repeat_interleave(256)[:n]  # noqa: E731
        ms, vs = spread(t.ms), spread(t.vs)
        y, off = m / ms.clamp(min=1e-300), tol_m / ms.clamp(min=1e-300) + 2.0 ** -21 * (m / ms.clamp(min=1e-300)).abs()
        enc = lambda a: a.clamp(-448.0, 448.0).float().to(F8[E4]).double()  # noqa: E731
        got = t.m.view(F8[E4]).double()
        assert bool(((got >= enc(y - off)) & (got <= enc(y + off)))[ms > 0].all()) and bool((got[ms == 0] == 0).all())
        y = (r / vs.clamp(min=1e-300)).clamp(max=448.0)
        u = chances(number, n, seed, step)
        got = t.v.view(F8[E4]).double()
        ends = []
        for way in (1 - 2.0 ** -19, 1 + 2.0 ** -19):
            a = (y * way).clamp(max=448.0)
            ends.append(torch.maximum(torch.floor(a / _grid(a) + u) * _grid(a), (r > 0).double() * 2.0 ** -9).clamp(max=448.0))
        # beside the two ends, the value of a sum that rounds up to a whole number of steps
        up = torch.floor(y / _grid(y) + u + 2.0 ** -18) * _grid(y)
        assert bool(((got >= torch.minimum(*ends)) & (got <= torch.maximum(torch.maximum(*ends), up.clamp(max=448.0)))).all())
    else:
        assert bool(((t.m.double() - m).abs() <= tol_m + 1e-44).all())
        assert bool(((t.v.double() - v).abs() <= tol_v).all())
    _check_copy(t)


def _check_copy(t):
    """the copy is that of the parameters as stored, bit for bit"""
    if t.copy is not None and t.copy_t == "bf16":
        assert torch.equal(t.copy.view(torch.int16), t.p.to(BF).view(torch.int16))
    elif t.copy is not None:
        want = torch.empty(t.n, dtype=U8, device=DEV)
        amax = _scalar(0.0)
        api.fp8_quantize(t.p.contiguous().clone(), t.copy_t, t.scale, want, amax_out=amax)
        assert torch.equal(t.copy, want)
        assert float(t.amax) == float(amax)
    assert torch.equal(t.g, t.old["g"]) and t.guards_kept()


SIZES = [1, 7, 8, 255, 256, 257, 1000, 2048, 2049, 4096, 33333, 100001]
KINDS = [(p, g, codes, copy) for p in (F32, BF) for g in (F32, BF) for codes, copy in ((False, None), (False, E4), (True, None), (True, E5), (True, "bf16"))]


@pytest.mark.parametrize("kind", KINDS, ids=lambda k: "%s-%s-%s-%s" % (str(k[0])[6:], str(k[1])[6:], "8bit" if k[2] else "32bit", k[3]))
def test_step(kind):
    g = _gen(3)
    ts = [Tensors(n, *kind, g, shift=i % 3 if i % 2 else 0, decay=0.1 * (i % 3)) for i, n in enumerate(SIZES)]
    plan = _plan(ts)
    lr, step, b1, b2, eps, norm, most, seed = 2e-3, 7, 0.9, 0.98, 1e-8, 3.0, 1.25, 0x123456789ABC
    api.fp8_adamw_step(plan, lr, step, beta1=b1, beta2=b2, eps=eps, seed=seed, norm=_scalar(norm), max_norm=most)
    _ok()
    number = 0
    for t in ts:
        _check_tensor(t, number, lr, step, b1, b2, eps, most / norm, seed)
        number += -(-t.n // 256) * 256
    assert int(plan.workspace.max()) == 0                          # left zeroed


@pytest.mark.parametrize("step,b1,b2", [(1, 0.9, 0.999), (2, 0.0, 0.0), (100000, 0.95, 0.9999)])
def test_bias_correction(step, b1, b2):
    g = _gen(4)
    ts = [Tensors(n, F32, F32, codes, None, g, start=step > 1) for n in (300, 5000) for codes in (False, True)]
    api.fp8_adamw_step(_plan(ts), 1e-3, step, beta1=b1, beta2=b2)
    _ok()
    number = 0
    for t in ts:
        _check_tensor(t, number, 1e-3, step, b1, b2, 1e-8, 1.0, 0)
        number += -(-t.n // 256) * 256


def test_state_from_zeros_and_zero_gradients():
    """zeros stay zeros: no scale, no code, no NaN, with and without eps"""
    n = 777
    z = lambda dt, k=n: torch.zeros(k, dtype=dt, device=DEV)  # noqa: E731
    p = torch.randn(n, device=DEV)
    was, m, v, ms, vs = p.clone(), z(U8), z(U8), z(F32, 4), z(F32, 4)
    api.fp8_adamw_step(api.AdamWPlan([p], [z(BF)], [m], [v], weight_decay=0.5, exp_avg_scales=[ms], exp_avg_sq_scales=[vs]), 1e-2, 1)
    _ok()
    assert not m.any() and not v.any() and not ms.any() and not vs.any()
    assert bool(((p.double() - was.double() * (1 - 0.5e-2)).abs() <= 2.0 ** -22 * was.abs()).all())
    # eps 0: 0 / 0 where nothing has happened yet, and an amax of the elements that are there alone
    p, copy, amax = torch.ones(3, device=DEV), z(U8, 3), _scalar(0.0)
    api.fp8_adamw_step(api.AdamWPlan([p], [torch.ones(3, device=DEV)], [z(F32, 3)], [z(F32, 3)], copies=[copy], fmt=E4, scales=[_scalar(1.0)], amax_outs=[amax]), 0.5, 1, eps=0.0)
    _ok()
    assert bool(((p - 0.5).abs() < 1e-5).all()) and float(amax) == float(p.abs().max())


def test_a_norm_that_is_not_finite_skips_the_step():
    g = _gen(6)
    for bad in (float("nan"), float("inf")):
        ts = [Tensors(n, F32, BF, codes, E4, g, shift=s) for n, s in ((5000, 0), (777, 1)) for codes in (False, True)]
        count = torch.tensor([4], device=DEV)
        api.fp8_adamw_step(_plan(ts), 1e-2, count, norm=_scalar(bad), max_norm=1.0)
        _ok()
        assert int(count) == 4
        for t in ts:
            assert all(torch.equal(getattr(t, k), t.old[k]) for k in ("p", "m", "v"))
            assert not t.codes or (torch.equal(t.ms, t.old_scales[0]) and torch.equal(t.vs, t.old_scales[1]))
            _check_copy(t)


def test_gradients_that_are_not_finite_without_a_norm():
    """32-bit moments: their element alone; 8-bit: their block's moments; the rest of the tensor as if nothing had been"""
    n = 1000
    for codes in (False, True):
        a, b = (Tensors(n, F32, F32, codes, None, _gen(8)) for _ in range(2))
        a.g[300], a.g[700] = float("nan"), float("inf")
        api.fp8_adamw_step(_plan([a]), 1e-2, 3, seed=5)
        api.fp8_adamw_step(_plan([b]), 1e-2, 3, seed=5)
        _ok()
        hit = torch.zeros(n, dtype=torch.bool, device=DEV)
        hit[300] = hit[700] = True
        assert bool(torch.isnan(a.p[hit]).all()) and torch.equal(a.p[~hit], b.p[~hit])
        if codes:
            assert bool((~torch.isfinite(a.ms[1:3])).all()) and torch.equal(a.ms[[0, 3]], b.ms[[0, 3]]) and torch.equal(a.v[:256], b.v[:256])
        else:
            assert torch.equal(a.m[~hit], b.m[~hit]) and torch.equal(a.v[~hit], b.v[~hit])


@pytest.mark.parametrize("codes", [False, True], ids=["32bit", "8bit"])
def test_second_moments_that_overflow_stop_their_elements(codes):
    a = Tensors(600, F32, F32, codes, None, _gen(9), decay=0.0)
    a.g[40] = 1e25
    api.fp8_adamw_step(_plan([a]), 1e-2, 3, beta2=0.9)
    _ok()
    assert bool(torch.isfinite(a.p).all()) and float(a.p[40]) == float(a.old["p"][40])


def test_captured_steps_go_on_with_the_counter_and_the_rate():
    """a replayed step reads its rate and counts for itself: the same bits as plain steps (at rates that binary32 holds)"""
    make = lambda: [Tensors(n, F32, BF, codes, E4, _gen(20 + n), start=False) for n in (3000, 70000) for codes in (False, True)]  # noqa: E731
    plain, played = make(), make()
    plan = _plan(plain)
    lrs = [2.0 ** -10, 2.0 ** -9, 3 * 2.0 ** -12, 2.0 ** -10]
    for i, lr in enumerate(lrs):
        api.fp8_adamw_step(plan, lr, i + 1, seed=77, norm=_scalar(2.0), max_norm=1.0)
    plan, lr, count, norm = _plan(played), _scalar(0.0), torch.tensor([0], device=DEV), _scalar(2.0)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        api.fp8_adamw_step(plan, lr, count, seed=77, norm=norm, max_norm=1.0)
    for v in lrs:
        lr.fill_(v)
        g.replay()
    _ok()
    assert int(count) == len(lrs)
    for a, b in zip(plain, played):
        for k in ("p", "m", "v", "copy", "amax"):
            assert torch.equal(getattr(a, k), getattr(b, k)), k
        assert not a.codes or (torch.equal(a.ms, b.ms) and torch.equal(a.vs, b.vs))


def test_plans_on_two_streams_at_once():
    sets = [[Tensors(n, F32, BF, True, E4, _gen(30 + n + 7 * i)) for n in (100000, 5000)] for i in range(2)]
    want = [[Tensors(n, F32, BF, True, E4, _gen(30 + n + 7 * i)) for n in (100000, 5000)] for i in range(2)]
    for ts in want:
        plan = _plan(ts)
        for i in range(6):
            api.fp8_adamw_step(plan, 1e-3, i + 1, seed=3)
    torch.cuda.synchronize()
    plans, streams = [_plan(ts) for ts in sets], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for i in range(6):
        for plan, s in zip(plans, streams):
            with torch.cuda.stream(s):
                api.fp8_adamw_step(plan, 1e-3, i + 1, seed=3)
    _ok()
    for a, b in zip(sum(sets, []), sum(want, [])):
        assert all(torch.equal(getattr(a, k), getattr(b, k)) for k in ("p", "m", "v", "ms", "vs", "copy", "amax"))


def test_eight_bit_second_moments_follow_their_mean():
    """With a gradient of constant magnitude r goes to that magnitude, from below and from above, although a step moves it by far
    less than the distance of two codes.  Rounding by chance leaves the mean of r alone and adds at most step^2 / 4 to the mean
    of r^2, step <= r / 8, in each step; v forgets (1 - b2) of itself meanwhile, so the mean square is between v and
    v (1 + b2 / (1 - b2) / 256) = 1.19 v for b2 = 0.98.  The mean over 65536 elements, whose squares scatter by less than v,
    is within 5 standard deviations, 0.02 v, of its own.  (600 steps: what is left of the start is below 2e-3.)"""
    n, b2, mag = 65536, 0.98, 3e-4
    for r0 in (0.0, 4e-3):
        p, g = torch.zeros(n, device=DEV), torch.full((n,), mag, device=DEV)
        m, v, ms, vs = torch.zeros(n, dtype=U8, device=DEV), torch.zeros(n, dtype=U8, device=DEV), torch.zeros(256, device=DEV), torch.zeros(256, device=DEV)
        if r0:
            v.fill_(0x7E)
            vs.fill_(r0 / 448)
        plan = api.AdamWPlan([p], [g], [m], [v], exp_avg_scales=[ms], exp_avg_sq_scales=[vs])
        for i in range(600):
            api.fp8_adamw_step(plan, 0.0, i + 1, beta2=b2, seed=11)
        _ok()
        r = v.view(F8[E4]).double().view(256, 256) * vs.double()[:, None]
        want = mag ** 2 + (r0 ** 2 - mag ** 2) * b2 ** 600
        assert -0.02 <= float(r.square().mean()) / want - 1 <= 0.21


def test_more_than_2_to_the_31_parameters():
    n = 2 ** 31 + 1000
    z = lambda dt: torch.zeros(n, dtype=dt, device=DEV)  # noqa: E731
    p, g, m, v = z(BF), z(BF), z(U8), z(U8)
    blocks = -(-n // 256)
    ms, vs = torch.zeros(blocks, device=DEV), torch.zeros(blocks, device=DEV)
    at = [0, 2 ** 31 - 300, 2 ** 31 + 5, n - 1]
    for i in at:
        g[i] = 1.0 + i % 7
    copy, amax = z(U8), _scalar(0.0)
    api.fp8_adamw_step(api.AdamWPlan([p], [g], [m], [v], exp_avg_scales=[ms], exp_avg_sq_scales=[vs], copies=[copy], fmt=E4, scales=[_scalar(1.0)], amax_outs=[amax]), 0.5, 1)
    _ok()
    for i in at:
        assert abs(float(p[i]) + 0.5) < 0.01 and float(amax) == abs(float(p[i])) and int(copy[i]) == 0xB0 and int(m[i]) == 0x7E and int(v[i]) == 0x7E
    for t in (p, m, v, copy):
        assert int(torch.count_nonzero(t)) == len(at)


def test_refusals_of_the_binding():
    f, u = torch.zeros(300, device=DEV), torch.zeros(300, dtype=U8, device=DEV)
    s = torch.zeros(2, device=DEV)
    for bad in (dict(exp_avg_scales=[s], exp_avg_sq_scales=[s]), dict(copies=[u]), dict(copies=[u], fmt=7, scales=[_scalar(1.0)]), dict(copies=[f]),
                dict(copies=[f.to(BF)], scales=[_scalar(1.0)]), dict(scales=[_scalar(1.0)]), dict(copies=[u[:200]], fmt=E4, scales=[_scalar(1.0)])):
        with pytest.raises((TypeError, ValueError)):
            api.AdamWPlan([f], [f], [f], [f], **bad)
    with pytest.raises((TypeError, ValueError)):
        api.AdamWPlan([f], [f], [u], [u])
    with pytest.raises((TypeError, ValueError)):
        api.AdamWPlan([f], [f], [u], [u], exp_avg_scales=[s[:1]], exp_avg_sq_scales=[s])
    with pytest.raises(ValueError):
        api.AdamWPlan([f[::2]], [f[::2]], [f[::2]], [f[::2]])
    plan = api.AdamWPlan([f], [f.clone()], [f.clone()], [f.clone()])
    for bad in (dict(step=0), dict(step=1, beta1=1.0), dict(step=1, eps=-1.0)):
        with pytest.raises(api.Fp8Error):
            api.fp8_adamw_step(plan, 1e-3, **bad)
    with pytest.raises(ValueError):
        api.fp8_adamw_step(plan, 1e-3, 1, norm=_scalar(1.0))
    with pytest.raises(TypeError):
        api.fp8_adamw_step(plan, 1e-3, torch.zeros(1, device=DEV))
    _ok()


def test_empty_tensors_and_empty_plans():
    e, amax, count = torch.empty(0, device=DEV), _scalar(5.0), torch.tensor([8], device=DEV)
    api.fp8_adamw_step(api.AdamWPlan([], [], [], []), 1e-3, count)
    assert int(count) == 9
    api.fp8_adamw_step(api.AdamWPlan([], [], [], []), 1e-3, 1)
    p = torch.ones(10, device=DEV)
    z = torch.zeros(10, device=DEV)
    plan = api.AdamWPlan([e, p, e], [e, z, e], [e, z.clone(), e], [e, z.clone(), e], copies=[torch.empty(0, dtype=U8, device=DEV), None, None], fmt=E4,
                         scales=[_scalar(1.0), None, None], amax_outs=[amax, None, None])
    api.fp8_adamw_step(plan, 1e-3, count)
    _ok()
    assert float(amax) == 0.0 and int(count) == 10 and bool((p == 1).all())
