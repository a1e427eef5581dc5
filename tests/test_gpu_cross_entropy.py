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
