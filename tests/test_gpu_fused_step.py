"""The fused operators together: gradients of the example's feed-forward stack against binary64 autograd, its training run,
and capture of the whole step in a CUDA graph."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

from paper_2209_05433_b200 import api

pytestmark = pytest.mark.gpu


def _net(tokens=200, d=128, inner=176):
    import gated_ffn_step as ex
    net = ex.FeedForward(tokens, d, inner, seed=3)
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    x = torch.randn(tokens, d, generator=g, device="cuda").to(torch.bfloat16)
    target = torch.randn(tokens, d, generator=g, device="cuda").to(torch.bfloat16)
    return net, x, target


def test_gradients_of_the_stack():
    """Against autograd in binary64 on the unquantized weights.  Every E4M3 operand carries a relative rounding error of up
    to 2^-4, every E5M2 one of up to 2^-3, uniform within a step: root mean square 2^-4/sqrt(3) and 2^-3/sqrt(3) at most.  A
    weight gradient passes through at most two E5M2 and four E4M3 conversions on its path, so its relative error (2-norm) is
    below sqrt(2) * 2^-3/sqrt(3) + 2 * 2^-4/sqrt(3) < 0.18; 0.25 is asserted."""
    net, x, target = _net()
    for _ in range(2):
        net.step(x, target, 0.0, 1e9, update=False)
    loss, norm = net.step(x, target, 0.0, 1e9, update=False)
    w = {n: getattr(net, n).double().requires_grad_() for n in ("w1", "wgu", "wd", "b1")}
    X = x.double()
    P = torch.nn.functional.gelu(X @ w["w1"] + w["b1"])
    G, U = (P @ w["wgu"]).chunk(2, dim=1)
    Y = (torch.nn.functional.silu(G) * U) @ w["wd"] + X
    want = (Y - target.double()).square().sum() / x.shape[0]
    want.backward()
    assert abs(float(loss) - float(want.detach())) <= 0.05 * float(want.detach())
    for n, g in net.grads.items():
        ref = w[n].grad
        assert float((g.double() - ref).norm() / ref.norm()) < 0.25, n
    total = sum(float(g.double().square().sum()) for g in net.grads.values()) ** 0.5
    assert abs(float(norm) - total) <= 2.0 ** -18 * total
    torch.cuda.synchronize()
    assert api.fp8_async_status()[0] == 0


def test_training_lowers_the_loss_and_clips():
    """descent along clipped gradients: the loss falls, and the gradients in place have the norm that clipping leaves them
    (bf16 values: each within 2^-8 of the exact product, so their norm is too)"""
    import gated_ffn_step as ex
    got = ex.train(steps=30)
    losses = [a for a, _ in got]
    assert losses[-1] < losses[10] < losses[0], losses
    net, x, target = _net()
    for max_norm in (0.25, 1e9):
        net.step(x, target, 0.0, max_norm, update=False)
        _, norm = net.step(x, target, 0.0, max_norm, update=False)
        after = sum(float(g.double().square().sum()) for g in net.grads.values()) ** 0.5
        assert float(norm) > 0.25
        assert abs(after - min(float(norm), max_norm)) <= 2.0 ** -8 * after


def test_the_step_in_a_cuda_graph():
    """capture, replay and the plain calls give the same bits"""
    net, x, target = _net(tokens=70)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            net.step(x, target, 0.0, 0.01, update=False)
    side.synchronize()
    scales = {n: getattr(net, n).scale.clone() for n in ("p", "h", "dgu", "dz")}
    with torch.cuda.stream(side):
        net.forward(x)
        net.backward(target)
        api.fp8_grad_clip(net.plan, 0.01, net.norm)
        side.synchronize()
        want = {n: g.clone() for n, g in net.grads.items()}
        wy, wn = net.y.clone(), net.norm.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            net.forward(x)
            net.backward(target)
            api.fp8_grad_clip(net.plan, 0.01, net.norm)
        for _ in range(3):
            for g in net.grads.values():
                g.zero_()
            net.y.zero_()
            graph.replay()
        side.synchronize()
    assert all(torch.equal(scales[n], getattr(net, n).scale) for n in scales)
    assert torch.equal(net.y, wy) and torch.equal(net.norm, wn) and all(torch.equal(net.grads[n], want[n]) for n in want)
    assert api.fp8_async_status()[0] == 0


def test_first_calls_of_a_stream_inside_a_capture():
    """workspaces first needed while a graph is captured: the replays and later plain calls on that stream are both right"""
    M, N, K = 64, 256, 128
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    A, B = ((torch.randn(r, K, generator=g, device="cuda")).to(torch.float8_e4m3fn).view(torch.uint8) for r in (M, N))
    dy = torch.randn(300, N, generator=g, device="cuda").to(torch.bfloat16)
    one = torch.ones(1, device="cuda")
    D, dz = torch.empty(M, N, dtype=torch.uint8, device="cuda"), torch.empty(300, N, dtype=torch.uint8, device="cuda")
    amax, amax2, db = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda"), torch.zeros(N, device="cuda")

    def calls():
        api.fp8_gemm_epilogue(A, api.E4M3, api.MAJOR_K, B, api.E4M3, api.MAJOR_K, D, one, one, fd=api.E4M3, scale_d=one, amax_out=amax)
        api.fp8_epilogue_backward(dy, None, dz, fd=api.E5M2, scale_d=one, dbias=db, amax_out=amax2)

    calls()
    torch.cuda.synchronize()
    want = [t.clone() for t in (D, dz, amax, amax2, db)]
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        calls()

    def check():
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (D, dz, amax, amax2, db)))
        for t in (D, dz, amax, amax2, db):
            t.zero_()

    for t in (D, dz, amax, amax2, db):
        t.zero_()
    with torch.cuda.stream(side):
        calls()                                              # before any replay
    check()
    for _ in range(2):
        graph.replay()
        check()
    with torch.cuda.stream(side):
        calls()
    check()
