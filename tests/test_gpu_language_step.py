"""The operators of a whole training step together: from token indices through the feed-forward stack, the loss of the
vocabulary projection and its gradients to the clipped AdamW step, plain and captured."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

from paper_2209_05433_b200 import api

pytestmark = pytest.mark.gpu
SHAPE = dict(tokens=200, d=128, inner=176, vocab=515)


def _model(seed=3):
    import language_model_step as ex
    net = ex.LanguageModel(**SHAPE, seed=seed)
    return (net, *ex.data(SHAPE["tokens"], SHAPE["vocab"], seed=4))


def _ok():
    torch.cuda.synchronize()
    assert api.fp8_async_status()[0] == 0


def test_gradients_of_the_model():
    """Against autograd in binary64 on the unquantized weights.  Every E4M3 operand carries a relative rounding error of up to
    2^-4, every E5M2 one of up to 2^-3, uniform within a step: root mean square 2^-4 / sqrt(3) and 2^-3 / sqrt(3) at most.  A
    gradient passes through at most three E5M2 conversions (the logits' gradient among them) and six E4M3 ones on its path:
    sqrt(3) * 2^-3 / sqrt(3) + sqrt(6) * 2^-4 / sqrt(3) < 0.22 of its 2-norm; 0.3 is asserted."""
    net, t, target = _model()
    for _ in range(3):                                            # the delayed scales settle; at a rate of zero nothing else changes
        net.step(t, target)
    grads = net.gradients(t, target)
    w = {n: m.double().requires_grad_() for n, m in net.masters.items()}
    X = net.embedding[t].double()
    P = torch.nn.functional.gelu(X @ w["w1"] + w["b1"])
    G, U = (P @ w["wgu"]).chunk(2, dim=1)
    Y = (torch.nn.functional.silu(G) * U) @ w["wd"] + X
    want = torch.nn.functional.cross_entropy(Y @ w["head"].T, target, ignore_index=-100)
    want.backward()
    got = float(torch.dot(net.loss, net.dloss))
    assert abs(got - float(want.detach())) <= 0.05 * float(want.detach())
    for n, g in grads.items():
        ref = w[n].grad
        assert float((g.double() - ref).norm() / ref.norm()) < 0.3, n
    _ok()


def test_a_step_changes_what_it_should():
    net, t, target = _model()
    net.step(t, target)
    net.lr.fill_(1e-3)
    before = {n: m.clone() for n, m in net.masters.items()}
    made_with, old_scale = net.inv.clone(), net.scale.clone()
    loss = net.step(t, target)
    _ok()
    assert bool(torch.isfinite(loss)) and int(net.count) == 2
    for n, m in net.masters.items():
        moved = (m - before[n]).abs()
        assert float(moved.max()) > 0 and float(moved.max()) < 1.2e-2, n      # a few times the rate at most
    # the copies are those of the new masters
    for n, c in (("w1", net.stack.w1), ("wgu", net.stack.wgu), ("wd", net.stack.wd)):
        assert torch.equal(c, net.masters[n].to(torch.bfloat16))
    codes = torch.empty_like(net.head)
    api.fp8_quantize(net.masters["head"], api.E4M3, old_scale, codes)
    assert torch.equal(codes, net.head) and torch.equal(net.used, made_with)
    assert float(net.amax) == float(net.masters["head"].abs().max())


def test_captured_steps_are_the_plain_ones():
    a, t, target = _model()
    b, _, _ = _model()
    for net in (a, b):
        net.step(t, target)                                       # plans, workspaces
        net.lr.fill_(2e-3)
    losses = [float(a.step(t, target)) for _ in range(4)]
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = b.step(t, target)
    replayed = []
    for _ in range(4):
        g.replay()
        replayed.append(float(out))
    _ok()
    assert replayed == losses and int(a.count) == int(b.count) == 5
    for n in a.masters:
        assert torch.equal(a.masters[n], b.masters[n]), n
    assert torch.equal(a.head, b.head)


def test_the_example_runs():
    import language_model_step as ex
    losses = ex.train(steps=5, tokens=128, d=64, inner=96, vocab=300)
    assert len(losses) == 5 and all(v == v and v > 0 for v in losses)
