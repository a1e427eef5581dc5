"""Training steps of a small feed-forward stack on the fused FP8 operators.

    P = gelu(X W1 + b1)            fp8_gemm_epilogue, codes out, the value before the activation kept
    H = silu(P Wg) * (P Wu)        fp8_gemm_gated, codes out, both products kept
    Y = H Wd + X                   fp8_gemm_epilogue with the residual

and back: fp8_gemm_gated_backward, fp8_epilogue_backward, the remaining products with fp8_gemm, then the global norm and
clipping of all weight gradients (fp8_grad_clip) and a plain SGD update of the bf16 weights.  Weights, inputs and output
gradients are converted with their current amax (fp8_quantize_current); tensors that leave a kernel as codes use the scale
chosen from the amax of the step before, a first pass without an update providing the starting values.

Run:  python examples/gated_ffn_step.py [steps]
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2209_05433_b200 import api

E4, E5, K, MN = api.E4M3, api.E5M2, api.MAJOR_K, api.MAJOR_MN


class Quantized:
    """Codes of a wide tensor with its current scale."""

    def __init__(self, like: torch.Tensor, fmt: int):
        self.fmt = fmt
        self.codes = torch.empty(like.shape, dtype=torch.uint8, device=like.device)
        self.s = torch.zeros(3, device=like.device)                      # amax, scale, 1 / scale
        self.inv = self.s[2:3]

    def __call__(self, x: torch.Tensor) -> "Quantized":
        api.fp8_quantize_current(x, self.fmt, self.codes, self.s[0:1], self.s[1:2], self.inv)
        return self


class Delayed:
    """Codes that a kernel writes itself, with the scale of the step before."""

    def __init__(self, shape, fmt: int, device):
        self.fmt = fmt
        self.codes = torch.empty(shape, dtype=torch.uint8, device=device)
        self.amax = torch.ones(1, device=device)
        self.scale, self.inv = torch.ones(1, device=device), torch.ones(1, device=device)

    def next_scale(self) -> None:
        api.fp8_scale_from_amax(self.amax, self.fmt, self.scale, self.inv)


class FeedForward:
    def __init__(self, tokens: int, d: int, inner: int, device="cuda", seed: int = 0):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        rand = lambda *s, std: (torch.randn(*s, generator=g, device=device) * std).to(torch.bfloat16)  # noqa: E731
        self.d, self.inner = d, inner
        self.w1, self.wgu, self.wd = rand(d, d, std=d ** -0.5), rand(d, 2 * inner, std=d ** -0.5), rand(inner, d, std=inner ** -0.5)
        self.b1 = torch.zeros(d, device=device)
        self.q = {n: Quantized(t, E4) for n, t in (("w1", self.w1), ("wgu", self.wgu), ("wd", self.wd))}
        wide = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device=device)  # noqa: E731
        self.qx, self.qdy = Quantized(wide(tokens, d), E4), Quantized(wide(tokens, d), E5)
        self.p, self.h = Delayed((tokens, d), E4, device), Delayed((tokens, inner), E4, device)
        self.dgu, self.dz = Delayed((tokens, 2 * inner), E5, device), Delayed((tokens, d), E5, device)
        self.pre, self.y, self.dp = wide(tokens, d), wide(tokens, d), wide(tokens, d)
        self.gate, self.up = wide(tokens, inner), wide(tokens, inner)
        self.grads = {"w1": wide(d, d), "wgu": wide(d, 2 * inner), "wd": wide(inner, d), "b1": torch.empty(d, device=device)}
        self.plan = api.ClipPlan(list(self.grads.values()))              # clips in place
        self.norm = torch.zeros(1, device=device)

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        q, n = {k: self.q[k](getattr(self, k)) for k in self.q}, self.inner
        self.qx(x)
        api.fp8_gemm_epilogue(self.qx.codes, E4, K, q["w1"].codes, E4, MN, self.p.codes, self.qx.inv, q["w1"].inv, act=api.ACT_GELU,
                              bias=self.b1, pre=self.pre, fd=E4, scale_d=self.p.scale, amax_out=self.p.amax)
        wg, wu = q["wgu"].codes[:, :n], q["wgu"].codes[:, n:]
        api.fp8_gemm_gated(self.p.codes, E4, K, wg, wu, E4, MN, self.h.codes, self.p.inv, q["wgu"].inv, q["wgu"].inv, act=api.ACT_SILU,
                           gate=self.gate, up=self.up, fd=E4, scale_d=self.h.scale, amax_out=self.h.amax)
        api.fp8_gemm_epilogue(self.h.codes, E4, K, q["wd"].codes, E4, MN, self.y, self.h.inv, q["wd"].inv, residual=x)
        return self.y

    def backward(self, dy: torch.Tensor) -> dict:
        q, n = self.q, self.inner
        self.qdy(dy)
        dg, du = self.dgu.codes[:, :n], self.dgu.codes[:, n:]
        api.fp8_gemm_gated_backward(self.qdy.codes, E5, K, q["wd"].codes, E4, K, self.gate, self.up, dg, du, self.qdy.inv, q["wd"].inv,
                                    act=api.ACT_SILU, fd=E5, scale_d=self.dgu.scale, amax_out=self.dgu.amax)
        api.fp8_gemm(self.h.codes, E4, MN, self.qdy.codes, E5, MN, self.grads["wd"], self.h.inv, self.qdy.inv)
        api.fp8_gemm(self.dgu.codes, E5, K, q["wgu"].codes, E4, K, self.dp, self.dgu.inv, q["wgu"].inv)
        api.fp8_gemm(self.p.codes, E4, MN, self.dgu.codes, E5, MN, self.grads["wgu"], self.p.inv, self.dgu.inv)
        api.fp8_epilogue_backward(self.dp, self.pre, self.dz.codes, act=api.ACT_GELU, fd=E5, scale_d=self.dz.scale,
                                  dbias=self.grads["b1"], amax_out=self.dz.amax)
        api.fp8_gemm(self.qx.codes, E4, MN, self.dz.codes, E5, MN, self.grads["w1"], self.qx.inv, self.dz.inv)
        return self.grads

    def new_scales(self) -> None:
        for t in (self.p, self.h, self.dgu, self.dz):
            t.next_scale()

    def step(self, x, target, lr: float, max_norm: float, update: bool = True):
        """One step on the squared error per token; returns the loss and the gradients' global norm (device scalars)."""
        y = self.forward(x)
        err = y.float() - target.float()
        grads = self.backward((err * (2.0 / err.shape[0])).to(torch.bfloat16))
        api.fp8_grad_clip(self.plan, max_norm, self.norm)
        if update:
            for name, g in grads.items():
                getattr(self, name).sub_(g, alpha=lr)
        self.new_scales()
        return err.square().sum() / err.shape[0], self.norm.clone()


def train(steps: int = 20, tokens: int = 512, d: int = 256, inner: int = 512, lr: float = 0.3, max_norm: float = 1.0, seed: int = 0):
    net = FeedForward(tokens, d, inner, seed=seed)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 1)
    x = torch.randn(tokens, d, generator=g, device="cuda").to(torch.bfloat16)
    target = x + torch.tanh(x.roll(1, dims=1).float()).to(torch.bfloat16)
    for _ in range(2):                                                    # scales settle: forward tensors first, then gradients
        net.step(x, target, lr, max_norm, update=False)
    losses = [net.step(x, target, lr, max_norm) for _ in range(steps)]
    return [(float(a), float(b)) for a, b in losses]


if __name__ == "__main__":
    for i, (loss, norm) in enumerate(train(int(sys.argv[1]) if len(sys.argv) > 1 else 20)):
        print("step %3d  loss %.5f  gradient norm %.5f" % (i, loss, norm))
