"""The AdamW step against its documented sequence of operations in binary32, bit for bit.

`follow` evaluates the sequence of include/fp8_b200.h on the host in numpy's binary32, one rounded operation at a time.  Moments, scales, codes and
copies have to be equal to the bit; so have parameters, but for what the kernel's quotients may leave: where the numerator is not zero
and below 2^-100, its residual is not a binary32 number, and the quotient may be off by 2 units of its own last place, which adds half a unit of p's."""
import math

import numpy as np
import pytest
import torch

from paper_2209_05433_b200 import api
from tests.test_gpu_adamw import BF, DEV, E4, F32, F8, FMAX, U8, Tensors, _check_copy, _ok, _plan, chances
from tests.test_gpu_fused import _gen, _scalar

pytestmark = pytest.mark.gpu
f32 = np.float32


def _np(t):
    return t.detach().float().cpu().numpy()


def _decode(codes, scale):
    """values of a flat 8-bit state: one product each"""
    return _np(codes.view(F8[E4])) * np.repeat(_np(scale), 256)[:codes.numel()]


def _tops(x):
    n = len(x)
    return np.abs(np.pad(x, (0, -n % 256))).reshape(-1, 256).max(axis=1)


def _spread(s, n):
    return np.repeat(s, 256)[:n]


def _encode(y, fmt):
    return torch.from_numpy(np.clip(y, -FMAX[fmt], FMAX[fmt])).to(F8[fmt]).view(U8).numpy()


def _up(top):
    """448 / top as the kernel takes it: the reciprocal, then the product"""
    return np.where(top == 0, f32(0), f32(1) / np.where(top == 0, f32(1), top) * f32(448))


def _times_448_over(x, top, scale):
    """what is rounded to codes; where the largest magnitude is below 2^-119, x over the scale, or 0 where that is 0"""
    n = len(x)
    small, at_all = _spread(top < 2.0 ** -119, n), _spread(scale > 0, n)
    over = (x * f32(2.0 ** 100)) * np.where(at_all, f32(1) / (_spread(scale, n) * f32(2.0 ** 100)), f32(0))
    return np.where(small, over, x * _spread(_up(top), n))


def follow(t, number, lr, step, b1, b2, eps, seed=0, norm=None, max_norm=None):
    """what the step leaves: p, m, v, scales, and the numerator of p's quotient"""
    with np.errstate(all="ignore"):
        coef = f32(1) if norm is None or norm <= max_norm else f32(max_norm) / f32(norm)
        g, p = _np(t.old["g"]) * coef, _np(t.old["p"])
        if t.codes:
            m, r = _decode(t.old["m"], t.old_scales[0]), _decode(t.old["v"], t.old_scales[1])
            v = r * r
        else:
            m, v = _np(t.old["m"]), _np(t.old["v"])
        m = f32(b1) * m + f32(1.0 - b1) * g
        v = f32(b2) * v + f32(1.0 - b2) * g * g
        r = np.sqrt(v)
        up = -f32(lr / (1.0 - b1 ** step)) * m
        change = up / (r * f32(1.0 / math.sqrt(1.0 - b2 ** step)) + f32(eps))
        p = p * (f32(1) - f32(lr) * f32(t.decay)) + change
        out = dict(up=up, change=change)
        if t.codes:
            n, top = t.n, _tops(m)
            out["ms"] = top * f32(1.0 / 448.0)
            out["m"] = _encode(_times_448_over(m, top, out["ms"]), E4)
            top = _tops(r)
            out["vs"] = top * f32(1.0 / 448.0)
            y = np.minimum(r * _spread(_up(top), n), f32(448))
            grid = np.exp2(np.maximum(np.frexp(y)[1] - 1, -6).astype(np.float64) - 3).astype(np.float32)
            q = np.floor(y / grid + chances(number, n, seed, step).cpu().numpy().astype(np.float32)) * grid
            out["v"] = _encode(np.where(r > 0, np.maximum(q, f32(2.0 ** -9)), f32(0)), E4)
        else:
            out["m"], out["v"] = m, v
        out["p"] = torch.from_numpy(p).to(t.p_t)
        return out


def same(got, want):
    """equal bits; NaN of any kind is NaN"""
    if isinstance(want, np.ndarray):
        want = torch.from_numpy(want)
    got = got.cpu()
    assert got.dtype == want.dtype
    nan = lambda x: (x & 0x7F) == 0x7F if x.dtype == U8 else x != x  # noqa: E731
    differ = (got != want) & ~(nan(got) & nan(want))
    assert not bool(differ.any()), "%d of %d differ, the first at %d: %r for %r" % (
        int(differ.sum()), differ.numel(), int(differ.nonzero()[0]), got[differ][0].item(), want[differ][0].item())


def check(t, number, **how):
    want = follow(t, number, **how)
    same(t.m, want["m"])
    same(t.v, want["v"])
    if t.codes:
        same(t.ms, want["ms"])
        same(t.vs, want["vs"])
    got, p = t.p.cpu(), want["p"]
    ends = torch.from_numpy((np.abs(want["up"]) < 2.0 ** -100) & (want["up"] != 0))
    same(got[~ends], p[~ends])
    if bool(ends.any()):
        change = torch.from_numpy(np.abs(want["change"]).astype(np.float64))[ends]
        allowed = 2 * 2.0 ** -23 * change + torch.finfo(t.p_t).eps * p[ends].double().abs() + 1e-45
        assert bool(((got[ends].double() - p[ends].double()).abs() <= allowed).all())
    assert t.guards_kept()


def run(ts, **how):
    more = dict(how)
    more["beta1"], more["beta2"] = more.pop("b1"), more.pop("b2")
    if "norm" in more:
        more["norm"] = _scalar(more["norm"])
    plan = _plan(ts)
    api.fp8_adamw_step(plan, more.pop("lr"), more.pop("step"), **more)
    _ok()
    number = 0
    for t in ts:
        check(t, number, **how)
        number += -(-t.n // 256) * 256


def _small(n, g, least, most, **kind):
    """a tensor whose gradients have magnitudes of 10^least to 10^most, a magnitude for each block of 256; half of its parameters start at zero"""
    t = Tensors(n, kind.get("p_t", F32), kind.get("g_t", F32), kind["codes"], None, g, shift=kind.get("shift", 0), start=False)
    size = torch.pow(10.0, least + (most - least) * torch.rand(-(-n // 256), generator=g, device=DEV, dtype=torch.float64)).repeat_interleave(256)[:n]
    t.g.copy_(torch.randn(n, generator=g, device=DEV).double() * size)
    t.p[::2] = 0.0
    if not t.codes:
        t.m.zero_()
        t.v.zero_()
    t.old = {k: getattr(t, k).clone() for k in t.old}
    return t


@pytest.mark.parametrize("eps", [1e-18, 1e-12, 1e-8])
@pytest.mark.parametrize("codes", [False, True], ids=["32bit", "8bit"])
def test_second_moments_at_the_bottom_of_the_range(codes, eps):
    """gradients whose squares are subnormal or near it, from zero states and once more on what that left"""
    g = _gen(51)
    for g_t in (F32, BF):
        ts = [_small(n, g, -23, -15, codes=codes, g_t=g_t, shift=s) for n, s in ((40000, 0), (2049, 0), (300, 1), (7, 0))]
        run(ts, lr=1.0, step=1, b1=0.9, b2=0.999, eps=eps, seed=5)
        for t in ts:
            t.old = {k: getattr(t, k).clone() for k in t.old}
            t.old_scales = (None, None) if not codes else (t.ms.clone(), t.vs.clone())
        run(ts, lr=1.0, step=2, b1=0.9, b2=0.999, eps=eps, seed=5)


@pytest.mark.parametrize("eps", [1e-18, 1e-8])
def test_first_moments_at_the_bottom_of_the_range(eps):
    """8-bit first moments whose scales are subnormal, or too small to be there at all; besides the bits, that they are worth what they
    should be: within half a step of a code, 2^-4, and half a step of the scale, 2^-150, 448 times"""
    g = _gen(52)
    ts = [_small(n, g, -45, -33, codes=True, shift=s) for n, s in ((60000, 0), (2049, 0), (300, 1), (7, 0))]
    run(ts, lr=1.0, step=1, b1=0.9, b2=0.999, eps=eps)
    for t in ts:
        exact = t.g.double() * 0.1
        worth = t.m.view(F8[E4]).double() * t.ms.double().repeat_interleave(256)[:t.n]
        top = torch.nn.functional.pad(exact, (0, -t.n % 256)).view(-1, 256).abs().amax(1).repeat_interleave(256)[:t.n]
        assert bool(((worth - exact).abs() <= 2.0 ** -4 * 1.001 * exact.abs() + top * 2.0 ** -18 + 448 * 2.0 ** -150 * 1.01 + 2.0 ** -149).all())


@pytest.mark.parametrize("eps", [1e-18, 1e-8, 1e15, 1e25, 1e38])
def test_first_moments_that_do_not_fit_their_second_ones(eps):
    """states that were not grown together, infinities among them: quotients that overflow, or have a divisor whose reciprocal is subnormal"""
    for n, shift in ((3000, 0), (100, 1)):
        t = Tensors(n, F32, F32, False, None, _gen(53), shift=shift)
        at = torch.arange(n, device=DEV)
        for k, value in enumerate((float("inf"), -float("inf"), 1e30, -3e38, 1e20, 0.0)):
            t.m[at % 97 == 2 * k] = value
        t.v[at % 2 == 0] = 0.0
        t.g[at % 3 == 0] = 0.0
        t.old = {k: getattr(t, k).clone() for k in t.old}
        run([t], lr=1e-2, step=3, b1=0.9, b2=0.99, eps=eps)
        t = Tensors(n, F32, BF, True, None, _gen(54), shift=shift)
        values = torch.tensor([1e30, float("inf"), 1e12, 3.4e38, 1e-5, 1e18], device=DEV)
        t.ms.copy_(values[torch.arange(t.ms.numel(), device=DEV) % 6])
        t.vs[::4] = 0.0
        t.g[torch.arange(n, device=DEV) % 3 == 0] = 0.0
        t.old = {k: getattr(t, k).clone() for k in t.old}
        t.old_scales = t.ms.clone(), t.vs.clone()
        run([t], lr=1e-2, step=3, b1=0.9, b2=0.99, eps=eps, seed=9)


@pytest.mark.parametrize("lr", [1e-3, 1e6, 1e20])
def test_rates_and_gradients_of_any_size(lr):
    g = _gen(55)
    for codes in (False, True):
        ts = [_small(n, g, -10, 19, codes=codes, shift=s) for n, s in ((40000, 0), (300, 1))]
        run(ts, lr=lr, step=1, b1=0.9, b2=0.999, eps=1e-8, seed=6)


KINDS = [(p, g, codes) for p in (F32, BF) for g in (F32, BF) for codes in (False, True)]


@pytest.mark.parametrize("kind", KINDS, ids=lambda k: "%s-%s-%s" % (str(k[0])[6:], str(k[1])[6:], "8bit" if k[2] else "32bit"))
@pytest.mark.parametrize("numbers", [dict(lr=2e-3, step=7, b1=0.9, b2=0.98, eps=1e-8, seed=0x123456789ABC, norm=3.0, max_norm=1.25),
                                     dict(lr=0.3, step=1, b1=0.0, b2=0.0, eps=1e-12), dict(lr=1e-4, step=100000, b1=0.95, b2=0.9999, eps=1e-6, seed=3)],
                         ids=["clipped", "no memory", "long run"])
def test_every_operation_is_rounded_as_documented(kind, numbers):
    g = _gen(56)
    sizes = [1, 7, 8, 255, 256, 257, 1000, 2048, 2049, 33333, 100001]
    copies = [None, "bf16", E4]
    ts = [Tensors(n, *kind, copies[i % 3], g, shift=i % 3 if i % 2 else 0, decay=0.1 * (i % 3)) for i, n in enumerate(sizes)]
    run(ts, **numbers)
    for t in ts:
        _check_copy(t)


@pytest.mark.parametrize("codes", [False, True], ids=["32bit", "8bit"])
def test_roots_and_quotients_of_many_numbers(codes):
    """8 million roots and quotients of ordinary size beside the host's.  (A root's correction is exact arithmetic; a quotient's reciprocal is
    only near, which leaves about one in 10^9 an ulp off: none is to be expected here.)"""
    t = _small(1 << 23, _gen(57), -9, 0, codes=codes)
    run([t], lr=1e-2, step=1, b1=0.9, b2=0.999, eps=1e-8, seed=8)
