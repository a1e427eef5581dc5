"""Training steps of a small language model on the FP8 operators, from token indices to updated weights:

    X = embedding[tokens]                                  (fixed)
    Y = feed-forward stack of gated_ffn_step               fp8_gemm_epilogue, fp8_gemm_gated
    loss = mean cross entropy of (Y . head^T)              fp8_cross_entropy, logits never stored
    dY, dhead                                              fp8_cross_entropy_backward
    weight gradients of the stack                          as in gated_ffn_step
    one norm over all gradients, one AdamW step            fp8_grad_norm, fp8_adamw_step

Master weights are float32, the moments of the matrices 8-bit.  The optimiser writes what the next step reads: bf16 copies of
the stack's weights, and the head's E4M3 codes, made with the scale that its amax of the step before gave.  Rate and step count
live on the device, so that a captured step can be replayed.

Run:  python examples/language_model_step.py [steps]
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import torch

from gated_ffn_step import E4, FeedForward, Quantized
from paper_2209_05433_b200 import api


class LanguageModel:
    def __init__(self, tokens: int, d: int, inner: int, vocab: int, device="cuda", seed: int = 0, decay: float = 0.01):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.stack = s = FeedForward(tokens, d, inner, device=device, seed=seed)
        self.embedding = torch.randn(vocab, d, generator=g, device=device).to(torch.bfloat16)
        self.masters = {n: getattr(s, n).float() for n in ("w1", "wgu", "wd")}
        self.masters["b1"] = s.b1                                        # float32 already
        self.masters["head"] = torch.randn(vocab, d, generator=g, device=device) * d ** -0.5
        # the head's codes: `scale` is for the codes to come, `inv` its inverse, `used` the inverse that goes with the codes that are there
        self.head = torch.empty(vocab, d, dtype=torch.uint8, device=device)
        self.amax, self.scale, self.inv = (torch.zeros(1, device=device) for _ in range(3))
        api.fp8_quantize_current(self.masters["head"], E4, self.head, self.amax, self.scale, self.inv)
        self.used = self.inv.clone()
        self.qy = Quantized(s.y, E4)
        self.loss, self.lse, self.dloss = (torch.zeros(tokens, device=device) for _ in range(3))
        self.dy, self.dhead = torch.empty_like(s.y), torch.empty(vocab, d, dtype=torch.bfloat16, device=device)
        self.grads = {**s.grads, "head": self.dhead}
        names = list(self.masters)
        grads = [self.grads[n] for n in names]
        self.norms, self.norm = api.ClipPlan(grads), torch.zeros(1, device=device)
        state = lambda n: torch.zeros(self.masters[n].shape, dtype=torch.float32 if n == "b1" else torch.uint8, device=device)  # noqa: E731
        scales = lambda n: None if n == "b1" else torch.zeros(-(-self.masters[n].numel() // api.STATE_BLOCK), device=device)  # noqa: E731
        only_head = lambda t: [t if n == "head" else None for n in names]  # noqa: E731
        self.plan = api.AdamWPlan([self.masters[n] for n in names], grads, [state(n) for n in names], [state(n) for n in names],
                                  weight_decay=[0.0 if n == "b1" else decay for n in names], exp_avg_scales=[scales(n) for n in names],
                                  exp_avg_sq_scales=[scales(n) for n in names], copies=[s.w1, s.wgu, s.wd, None, self.head], fmt=E4,
                                  scales=only_head(self.scale), amax_outs=only_head(self.amax))
        self.lr, self.count = torch.zeros(1, device=device), torch.zeros(1, dtype=torch.int64, device=device)

    def gradients(self, tokens: torch.Tensor, target: torch.Tensor) -> dict:
        """Loss per token and all gradients; a target outside the vocabulary does not count."""
        vocab = self.head.shape[0]
        y = self.stack.forward(self.embedding.index_select(0, tokens))
        q = self.qy(y)
        counted = (target >= 0) & (target < vocab)
        torch.div(counted, counted.sum().clamp(min=1), out=self.dloss)
        api.fp8_cross_entropy(q.codes, E4, self.head, E4, target, self.loss, self.lse, scale_inv_x=q.inv, scale_inv_w=self.used)
        api.fp8_cross_entropy_backward(q.codes, E4, self.head, E4, target, self.lse, self.dloss, self.dy, self.dhead, scale_inv_x=q.inv,
                                       scale_inv_w=self.used)
        self.stack.backward(self.dy)
        return self.grads

    def step(self, tokens: torch.Tensor, target: torch.Tensor, max_norm: float = 1.0, seed: int = 0) -> torch.Tensor:
        """One step at the rate in self.lr; returns the mean loss (a device scalar)."""
        self.gradients(tokens, target)
        api.fp8_grad_norm(self.norms, self.norm)
        api.fp8_adamw_step(self.plan, self.lr, self.count, beta2=0.95, seed=seed, norm=self.norm, max_norm=max_norm)
        self.used.copy_(self.inv)                                        # the head's codes have just been made with `scale`
        api.fp8_scale_from_amax(self.amax, E4, self.scale, self.inv)
        self.stack.new_scales()
        return torch.dot(self.loss, self.dloss)


def data(tokens: int, vocab: int, seed: int = 1, device="cuda"):
    """Tokens with a rule to learn: the target is a fixed permutation of the token; every tenth is padding."""
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    rule = torch.randperm(vocab, generator=g, device=device)
    t = torch.randint(0, vocab, (tokens,), generator=g, device=device)
    target = rule[t]
    target[::10] = -100
    return t, target


def train(steps: int = 20, tokens: int = 512, d: int = 256, inner: int = 512, vocab: int = 1000, lr: float = 3e-3, seed: int = 0):
    net = LanguageModel(tokens, d, inner, vocab, seed=seed)
    t, target = data(tokens, vocab, seed + 1)
    for _ in range(2):                                                    # scales settle at a rate of zero
        net.step(t, target)
    net.count.zero_()
    net.lr.fill_(lr)
    losses = [net.step(t, target) for _ in range(steps)]
    return [float(v) for v in losses]


if __name__ == "__main__":
    for i, loss in enumerate(train(int(sys.argv[1]) if len(sys.argv) > 1 else 20)):
        print("step %3d  loss %.5f" % (i, loss))
