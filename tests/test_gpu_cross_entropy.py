"""GPU parity of the softmax cross entropy of a vocabulary projection and of its gradients against their definition in
binary64 on the operands' values.

Tolerances, derived.  A logit is a dot product within 1e-5 * S, S = sum|x w| * scales (the products' own criterion), and is
scaled, shifted and exponentiated in binary32: four roundings of numbers up to |z| log2(e) and |lse| log2(e), and 2 ulp of the
exponential: dz = 1e-5 S + 2^-21 (|z| + |lse| + 1).  lse: the weighted mean of the logits' errors, below their largest; the
sum has 32 + 7 + 5 additions in a row at most (a thread's quarter, the pairs of a thread of the joining kernel for up to 8192
columns a warp, the tree), each with an exponential's error in the joins: 2^-17 for vocabularies up to 2^18.
The logits' gradient p - 1 or p, times a factor: p's relative error is the logit's and lse's together, plus 2^-21 of the
operands of the difference and the product.  It is then rounded: the value the kernel holds is one of those between the
conversions of the two ends of that interval, so the definition's own conversion is off by at most the farther end.  dx and dw
sum these over the vocabulary or the tokens: the intervals' widths times |w| or |x|, 1e-5 of the sum of magnitudes, and one
rounding of the result (2^-8 bf16, 2^-24 binary32)."""
import pytest
import torch

from paper_2209_05433_b200 import api
from tests.test_gpu_fused import _gen, _guards_kept, _matrix, _scalar

pytestmark = pytest.mark.gpu
DEV = "cuda"
E4, E5, BF, F32 = api.E4M3, api.E5M2, torch.bfloat16, torch.float32
F8 = {E4: torch.float8_e4m3fn, E5: torch.float8_e5m2}
HALF = {BF: 2.0 ** -8, F32: 2.0 ** -24}


def _ok():
    torch.cuda.synchronize()
    assert api.fp8_async_status()[0] == 0


def _operand(values, fmt):
    """(stored matrix with guards, its buffer, its values in binary64 without the scale)"""
    q = values.to(BF) if fmt is None else values.to(F8[fmt])
    view, whole = _matrix(values.shape[0], values.shape[1], BF if fmt is None else torch.uint8)
    whole.fill_(float("nan") if fmt is None else 0x7F)           # padding is not read
    view.copy_(q if fmt is None else q.view(torch.uint8))
    return view, q.double()


class Problem:
    def __init__(self, T, K, V, fx, fw, seed=0, ignored=0.2, weighted=True, sx=0.37, sw=0.11):
        g = _gen(1000 * T + 10 * K + V + seed)
        self.T, self.K, self.V, self.fx, self.fw = T, K, V, fx, fw
        bf = fx is None
        self.sx, self.sw = (None, None) if bf else (_scalar(sx), _scalar(sw))
        a = 1.0 if bf else float(self.sx) * float(self.sw)
        self.a, self.ax, self.aw = a, 1.0 if bf else float(self.sx), 1.0 if bf else float(self.sw)
        x = torch.randn(T, K, generator=g, device=DEV)
        w = torch.randn(V, K, generator=g, device=DEV) * (2.0 / (a * K ** 0.5))
        self.x, self.x64 = _operand(x, fx)
        self.w, self.w64 = _operand(w, fw)
        target = torch.randint(0, V, (T,), generator=g, device=DEV)
        drop = torch.rand(T, generator=g, device=DEV) < ignored
        away = torch.tensor([-100, -1, V, V + 5, -2 ** 40, 2 ** 40], device=DEV)[torch.randint(0, 6, (T,), generator=g, device=DEV)]
        self.target = torch.where(drop, away, target)
        self.dloss = (0.5 + torch.rand(T, generator=g, device=DEV) if weighted else torch.ones(T, device=DEV)) / T
        self.dloss = torch.where(drop, torch.full_like(self.dloss, float("nan")), self.dloss)      # not looked at
        self.loss, self.lse = torch.full((T,), 7.0, device=DEV), torch.full((T,), 7.0, device=DEV)

    def forward(self, **more):
        api.fp8_cross_entropy(self.x, self.fx, self.w, self.fw, self.target, self.loss, self.lse, scale_inv_x=self.sx, scale_inv_w=self.sw, **more)

    def backward(self, dx, dw, **more):
        api.fp8_cross_entropy_backward(self.x, self.fx, self.w, self.fw, self.target, self.lse, self.dloss, dx, dw, scale_inv_x=self.sx,
                                       scale_inv_w=self.sw, **more)

    def exact(self):
        z = self.x64 @ self.w64.T * self.a
        self.z = z
        self.tol_z = 1e-5 * (self.x64.abs() @ self.w64.abs().T) * self.a
        self.lse64 = torch.logsumexp(z, 1)
        self.tol_z += 2.0 ** -21 * (z.abs() + self.lse64.abs()[:, None] + 1)
        self.tol_lse = self.tol_z.max(1)[0] + 2.0 ** -17
        self.rows = torch.nonzero((self.target >= 0) & (self.target < self.V)).squeeze(1)
        return self

    def check_forward(self):
        self.exact()
        rows = self.rows
        loss, tol = torch.zeros_like(self.lse64), torch.zeros_like(self.lse64)
        loss[rows] = self.lse64[rows] - self.z[rows, self.target[rows]]
        tol[rows] = self.tol_lse[rows] + self.tol_z[rows, self.target[rows]]
        assert bool(((self.lse.double() - self.lse64).abs() <= self.tol_lse).all())
        assert bool(((self.loss.double() - loss).abs() <= tol).all())

    def check_backward(self, dx, dw):
        self.exact()
        rows, T, V = self.rows, self.T, self.V
        lse = self.lse.double()                                   # what the backward pass is given
        p = torch.exp(self.z - lse[:, None])
        hot = torch.zeros(T, V, dtype=torch.float64, device=DEV)
        hot[rows, self.target[rows]] = 1.0
        g = torch.zeros(T, 1, dtype=torch.float64, device=DEV)
        g[rows] = self.dloss[rows].double()[:, None]
        dz = (p - hot) * g
        off = ((torch.expm1(self.tol_z) + 2.0 ** -20) * p + 2.0 ** -22 * hot) * g.abs()
        if self.fx is None:
            scale, store = 1.0, lambda t: t.to(torch.float32).to(BF).double()
        else:
            most = float(g.abs().max())
            scale = 57344.0 / most if most > 0 else 1.0
            store = lambda t: (t * scale).clamp(-57344.0, 57344.0).to(torch.float32).to(F8[E5]).double() / scale  # noqa: E731
        mid = store(dz)
        wide = torch.maximum((store(dz + off) - mid).abs(), (store(dz - off) - mid).abs()) + off * 2.0 ** -10
        for name, got, other, a, left, width in (("dx", dx, self.w64, self.aw, mid, wide), ("dw", dw, self.x64, self.ax, mid.T, wide.T)):
            if got is None:
                continue
            want = left @ other * a
            tol = (width @ other.abs() + 1e-5 * (left.abs() @ other.abs())) * a
            tol = tol + HALF[got.dtype] * (want.abs() + tol) + 1e-38
            bad = ~((got.double() - want).abs() <= tol)
            assert not bool(bad.any()), "%s: %d of %d values outside, worst %.3g of the tolerance" % (
                name, int(bad.sum()), bad.numel(), float(((got.double() - want).abs() / tol).max()))


FORWARD = [
    # tokens, width, vocabulary, formats of x and w
    (1, 1, 1, E4, E4), (1, 64, 1000, E4, E4), (1, 4096, 20011, E4, E5), (1, 96, 300, None, None),
    (2, 17, 255, E5, E4), (31, 128, 256, E4, E4), (37, 256, 257, None, None), (33, 2049, 513, E4, E4),
    (128, 1000, 777, E4, E4), (129, 333, 1001, E4, E4), (127, 72, 40000, None, None), (200, 4100, 130, E5, E5),
    (257, 64, 5000, None, None), (300, 6150, 2000, E4, E4), (513, 3000, 999, None, None), (1024, 512, 3001, E4, E4),
]


@pytest.mark.parametrize("case", FORWARD, ids=lambda c: "%dx%dx%d" % c[:3])
def test_forward(case):
    p = Problem(*case)
    p.forward()
    _ok()
    p.check_forward()
    first = p.loss.clone(), p.lse.clone()
    p.loss.fill_(1.0), p.lse.fill_(1.0)
    p.forward()
    assert torch.equal(p.loss, first[0]) and torch.equal(p.lse, first[1])


BACKWARD = [
    # tokens, width, vocabulary, formats, types of dx and dw
    (1, 1, 1, E4, E4, BF, BF), (1, 64, 1000, E4, E4, F32, BF), (1, 96, 300, None, None, BF, F32), (2, 17, 255, E5, E4, BF, F32),
    (37, 256, 1000, E4, E4, BF, BF), (37, 512, 20000, E4, E4, BF, BF), (33, 260, 9001, None, None, F32, BF), (31, 1001, 513, E4, E5, BF, BF),
    (128, 300, 4000, None, None, BF, BF), (129, 333, 1001, E4, E4, F32, F32), (200, 4100, 130, E5, E5, BF, BF), (257, 72, 5003, None, None, BF, F32),
    (300, 515, 20000, E4, E4, F32, BF), (1000, 1030, 2000, E4, E4, BF, BF), (513, 3000, 999, None, None, BF, BF),
    (2500, 200, 300, E4, E4, F32, F32), (4500, 130, 257, None, None, F32, F32),
    # more than one piece of the vocabulary
    (8200, 70, 9001, E4, E4, BF, BF), (5000, 136, 20000, None, None, F32, BF), (5000, 33, 8193, None, None, BF, F32),
]


@pytest.mark.parametrize("case", BACKWARD, ids=lambda c: "%dx%dx%d" % c[:3])
def test_backward(case):
    T, K, V, fx, fw, dx_t, dw_t = case
    p = Problem(T, K, V, fx, fw)
    (dx, all_dx), (dw, all_dw) = _matrix(T, K, dx_t), _matrix(V, K, dw_t)
    p.forward()
    p.backward(dx, dw)
    _ok()
    p.check_backward(dx, dw)
    assert _guards_kept(dx, all_dx) and _guards_kept(dw, all_dw)
    ignored = torch.ones(T, dtype=torch.bool, device=DEV)
    ignored[p.rows] = False
    assert bool((dx[ignored] == 0).all())
    first = dx.clone(), dw.clone()
    p.backward(dx, None)
    p.backward(None, dw)                                          # one at a time: the same bits
    assert torch.equal(dx, first[0]) and torch.equal(dw, first[1])


@pytest.mark.parametrize("shape", [(5, 24, 37), (130, 16, 300)])
def test_gradients_are_the_derivatives_of_the_loss(shape):
    """dx and dw against central differences of sum(dloss * loss) in binary64 (step 1e-4: truncation below 1e-8 of the
    magnitudes): off by the rounding of dz to bf16, 2^-8 of each, and by the bounds above."""
    T, K, V = shape
    p = Problem(T, K, V, None, None, ignored=0.0)
    dx, dw = torch.empty(T, K, device=DEV), torch.empty(V, K, device=DEV)
    p.forward()
    p.backward(dx, dw)
    _ok()
    x, w, g = p.x64, p.w64, p.dloss.double()
    z = x @ w.T
    pr = torch.softmax(z, 1)
    dz = (pr - torch.nn.functional.one_hot(p.target, V)) * g[:, None]

    def total(x, w):
        z = x @ w.T
        return ((torch.logsumexp(z, 1) - z.gather(1, p.target[:, None]).squeeze(1)) * g).sum()

    h, gen = 1e-4, _gen(9)
    for name, got, a, tol in (("dx", dx, x, dz.abs() @ w.abs()), ("dw", dw, w, dz.abs().T @ x.abs())):
        for _ in range(20):
            way = torch.randn(a.shape, generator=gen, device=DEV, dtype=torch.float64)
            diff = (total(a + h * way, w) - total(a - h * way, w) if name == "dx" else total(x, a + h * way) - total(x, a - h * way)) / (2 * h)
            bound = 1.05 * 2.0 ** -8 * (tol * way.abs()).sum() + 1e-6
            assert abs(float((got.double() * way).sum() - diff)) <= float(bound), name


@pytest.mark.parametrize("T", [3, 200])
def test_special_values(T):
    """NaN and infinities stay in the rows of the tokens that have them, and out of what does not count"""
    K, V = 32, 700
    p = Problem(T, K, V, None, None, ignored=0.0)
    p.x[0, 3] = float("nan")
    p.x[1, 0] = float("inf")                                     # logits of both signs, infinite
    p.target[2] = -100
    p.forward()
    assert bool(torch.isnan(p.loss[:2]).all()) and bool(torch.isnan(p.lse[:2]).all())
    assert float(p.loss[2]) == 0.0 and bool(torch.isfinite(p.lse[2]))
    assert bool(torch.isfinite(p.loss[2:]).all())
    p.target[0] = V                                              # the NaN token does not count any more: its loss and its gradient are zero
    p.forward()
    assert float(p.loss[0]) == 0.0 and bool(torch.isnan(p.lse[0]))
    dx = torch.empty(T, K, device=DEV)
    p.backward(dx, None)
    _ok()
    assert not dx[0].any() and bool(torch.isnan(dx[1]).all()) and not dx[2].any()
    assert bool(torch.isfinite(dx[3:]).all()) and (T == 3 or bool(dx[3:].any()))
    # a row of logits that are all minus infinity, and one whose logits are as large as they get
    x, w = torch.zeros(2, 16, device=DEV, dtype=BF), torch.zeros(300, 16, device=DEV, dtype=BF)
    x[0, 0], x[1, 0] = float("-inf"), 1e18
    w[:, 0] = 1.0
    w[7, 0] = 2.0
    t, loss, lse = torch.tensor([5, 7], device=DEV), torch.empty(2, device=DEV), torch.empty(2, device=DEV)
    api.fp8_cross_entropy(x, None, w, None, t, loss, lse)
    _ok()
    assert float(lse[0]) == float("-inf") and bool(torch.isnan(loss[0]))
    assert float(loss[1]) == 0.0 and abs(float(lse[1]) / 2e18 - 1) < 0.01


def test_nothing_counts_and_nothing_is_there():
    p = Problem(40, 64, 500, E4, E4, ignored=1.1)
    (dx, all_dx), (dw, all_dw) = _matrix(40, 64, BF), _matrix(500, 64, BF)
    p.forward()
    p.backward(dx, dw)
    _ok()
    assert not p.loss.any() and not dx.any() and not dw.any() and bool(torch.isfinite(p.lse).all())
    none = torch.empty(0, device=DEV)
    api.fp8_cross_entropy(p.x[:0], E4, p.w, E4, torch.empty(0, dtype=torch.int64, device=DEV), none, none, scale_inv_x=p.sx, scale_inv_w=p.sw)
    dw.fill_(3.0)
    api.fp8_cross_entropy_backward(p.x[:0], E4, p.w, E4, torch.empty(0, dtype=torch.int64, device=DEV), none, none, dx[:0], dw, scale_inv_x=p.sx, scale_inv_w=p.sw)
    _ok()
    assert not dw.any() and _guards_kept(dw, all_dw)


def test_gradient_factors_of_every_size():
    """dloss of zero, of 1e-30 and of 1e30: the codes' scale follows the largest; not finite: the scale is 1 and the rows say so"""
    for factor in (1e-30, 1.0, 1e30):
        p = Problem(64, 96, 300, E4, E4, ignored=0.0)
        p.dloss.mul_(factor)
        p.dloss[5] = 0.0
        dx, dw = torch.empty(64, 96, device=DEV), torch.empty(300, 96, device=DEV)
        p.forward()
        p.backward(dx, dw)
        _ok()
        p.check_backward(dx, dw)
        assert not dx[5].any()
    p.dloss.zero_()
    p.backward(dx, dw)
    assert not dx.any() and not dw.any()
    p.dloss[3] = float("nan")
    p.backward(dx, None)
    _ok()
    assert bool(torch.isnan(dx[3]).all()) and not dx[4:].any()


def test_captured_calls_replay_on_new_inputs():
    """two graphs of the same call, replayed on the inputs of two problems: the bits of plain calls"""
    problems = [Problem(200, 130, 3000, E4, E4, seed=s) for s in (0, 7)]
    shape = lambda: (torch.empty(200, 136, dtype=BF, device=DEV)[:, :130], torch.empty(3000, 136, dtype=BF, device=DEV)[:, :130])  # noqa: E731
    want = []
    for r in problems:
        dx, dw = shape()
        r.forward()
        r.backward(dx, dw)
        want.append((r.loss.clone(), dx, dw))
    p, (dx, dw) = Problem(200, 130, 3000, E4, E4, seed=1), shape()
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    _ok()
    for g in graphs:
        with torch.cuda.graph(g):
            p.forward()
            p.backward(dx, dw)
    for r, (loss, wx, ww) in zip(problems, want):
        for to, of in ((p.x, r.x), (p.w, r.w), (p.target, r.target), (p.dloss, r.dloss)):
            to.copy_(of)
        for g in graphs:
            dx.fill_(9.0), dw.fill_(9.0), p.loss.fill_(9.0)
            g.replay()
            _ok()
            assert torch.equal(p.loss, loss) and torch.equal(dx, wx) and torch.equal(dw, ww)


def test_two_streams_at_once():
    a, b = Problem(300, 256, 4000, None, None), Problem(37, 512, 9000, E4, E4)
    streams, out = (torch.cuda.Stream(), torch.cuda.Stream()), []
    for r in (a, b):
        dx, dw = torch.empty(r.T, r.K, dtype=BF, device=DEV), torch.empty(r.V, r.K, dtype=BF, device=DEV)
        r.forward()
        r.backward(dx, dw)
        out.append((r.loss.clone(), dx.clone(), dw.clone()))
    torch.cuda.synchronize()
    got = [(torch.empty_like(o[1]), torch.empty_like(o[2])) for o in out]
    for _ in range(5):
        for r, s, (dx, dw) in zip((a, b), streams, got):
            with torch.cuda.stream(s):
                r.forward()
                r.backward(dx, dw)
    _ok()
    for r, o, (dx, dw) in zip((a, b), out, got):
        assert torch.equal(r.loss, o[0]) and torch.equal(dx, o[1]) and torch.equal(dw, o[2])


def test_rows_that_are_slices_of_wider_ones():
    """operands and gradients with pitches above their width; single rows and columns of any stride"""
    T, K, V = 70, 48, 600
    p = Problem(T, K, V, E4, E4)
    wide = torch.full((T, 256), 0x7F, dtype=torch.uint8, device=DEV)
    wide[:, 64:64 + K] = p.x
    dx_all = torch.full((T, 128), 5.0, device=DEV, dtype=BF)
    dx, dw, flat = dx_all[:, 16:16 + K], torch.empty(V, K, device=DEV), torch.empty(T, K, device=DEV, dtype=BF)
    p.forward()
    p.backward(flat, None)
    loss = p.loss.clone()
    p.x = wide[:, 64:64 + K]
    p.forward()
    p.backward(dx, dw)
    _ok()
    assert torch.equal(p.loss, loss) and torch.equal(dx, flat) and bool((dx_all[:, :16] == 5).all()) and bool((dx_all[:, 16 + K:] == 5).all())
    p.check_backward(dx, dw)
    for bad in (p.x[:, 1:], p.x[::1, ::2], wide.t()):
        with pytest.raises((ValueError, TypeError, api.Fp8Error)):
            api.fp8_cross_entropy(bad, E4, p.w[:, :bad.shape[1]], E4, p.target, p.loss, p.lse, scale_inv_x=p.sx, scale_inv_w=p.sw)


def test_more_than_2_to_the_31_weights():
    """offsets that pass 32 bits: a projection of 2.3e9 codes; the last rows of the vocabulary are the ones that matter"""
    T, K, V = 3, 16384, 140000
    g = _gen(1)
    x = torch.randn(T, K, generator=g, device=DEV).to(F8[E4]).view(torch.uint8)
    w = torch.randint(0, 0x38, (V, K), generator=g, device=DEV, dtype=torch.uint8)          # 0 .. 0.94
    w[1::2] |= 0x80
    target = torch.tensor([V - 1, 7, V - 77], device=DEV)
    loss, lse, one = torch.empty(T, device=DEV), torch.empty(T, device=DEV), _scalar(2.0 ** -6)
    api.fp8_cross_entropy(x, E4, w, E4, target, loss, lse, scale_inv_x=one, scale_inv_w=_scalar(1.0))
    dx, dw = torch.empty(T, K, dtype=BF, device=DEV), torch.empty(V, K, dtype=BF, device=DEV)
    dloss = torch.full((T,), 1.0 / T, device=DEV)
    api.fp8_cross_entropy_backward(x, E4, w, E4, target, lse, dloss, dx, dw, scale_inv_x=one, scale_inv_w=_scalar(1.0))
    _ok()
    x64 = x.view(F8[E4]).double()
    z = torch.cat([x64 @ part.view(F8[E4]).double().T for part in w.split(20000)], 1) * 2.0 ** -6
    s = torch.cat([x64.abs() @ part.view(F8[E4]).double().abs().T for part in w.split(20000)], 1) * 2.0 ** -6
    want = torch.logsumexp(z, 1)
    tol = 1e-5 * s.max(1)[0] + 2.0 ** -16 + 2.0 ** -20 * want.abs()
    assert bool(((lse.double() - want).abs() <= tol).all())
    rows = torch.arange(T, device=DEV)
    assert bool(((loss.double() - (want - z[rows, target])).abs() <= 2 * tol).all())
    dz = torch.exp(z - want[:, None])
    dz[rows, target] -= 1
    dz /= T
    back = torch.zeros(T, K, dtype=torch.float64, device=DEV)
    mags = torch.zeros_like(back)
    for i, part in enumerate(w.split(20000)):
        v = part.view(F8[E4]).double()
        back += dz[:, i * 20000:i * 20000 + v.shape[0]] @ v
        mags += dz.abs()[:, i * 20000:i * 20000 + v.shape[0]] @ v.abs()
    assert bool(((dx.double() - back).abs() <= 0.135 * mags).all())                          # every term to 2^-3 and the logit's error
    for lo, hi in ((0, 300), (V - 300, V)):
        v = dz[:, lo:hi].T @ (x64 * 2.0 ** -6)
        assert bool(((dw[lo:hi].double() - v).abs() <= 0.135 * (dz[:, lo:hi].abs().T @ (x64.abs() * 2.0 ** -6)) + 1e-12).all())


@pytest.mark.parametrize("fx", [E4, None])
def test_the_smallest_vocabularies_and_widths(fx):
    """more rows than a tile has, on one, two and nine columns, widths of one and of a few bytes"""
    for T, K, V in ((200, 16, 1), (300, 1, 2), (129, 3, 9), (1, 5, 3)):
        p = Problem(T, K, V, fx, fx)
        (dx, all_dx), (dw, all_dw) = _matrix(T, K, F32), _matrix(V, K, BF)
        p.forward()
        p.backward(dx, dw)
        _ok()
        p.check_forward()
        p.check_backward(dx, dw)
        assert _guards_kept(dx, all_dx) and _guards_kept(dw, all_dw)


def test_workspaces_of_the_caller():
    p = Problem(150, 64, 2000, E4, E4)
    forward, backward = api.cross_entropy_workspace_bytes(150, 64, 2000)
    dx, dw = torch.empty(150, 64, device=DEV), torch.empty(2000, 64, device=DEV)
    p.forward()
    p.backward(dx, dw)
    want = p.loss.clone(), dx.clone(), dw.clone()
    ws = torch.full((max(forward, backward) + 64,), 0xFF, dtype=torch.uint8, device=DEV)     # its contents mean nothing
    p.forward(workspace=ws[:forward])
    p.backward(dx, dw, workspace=ws[:backward])
    _ok()
    assert torch.equal(p.loss, want[0]) and torch.equal(dx, want[1]) and torch.equal(dw, want[2])
    assert bool((ws[max(forward, backward):] == 0xFF).all())
    with pytest.raises(api.Fp8Error):
        p.forward(workspace=ws[:forward - 1])
    with pytest.raises(api.Fp8Error):
        p.backward(dx, dw, workspace=ws[:backward - 1])
    with pytest.raises(ValueError):
        p.forward(workspace=ws.cpu())
