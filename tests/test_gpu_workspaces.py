"""Workspaces of the fused operators on the GPU: graphs that outlive a stream's workspace, and calls that overlap."""
import pytest
import torch

from paper_2209_05433_b200 import api
from tests.test_gpu_fused import BF, E4, E5, K_, _gen, _ok, _scalar

pytestmark = pytest.mark.gpu
DEV = "cuda"


class Calls:
    """A product with an amax and a backward pass with column sums and an amax, and their outputs.  Values are multiples of
    1/8 with few bits, so every sum is exact and the outputs do not depend on its order."""

    def __init__(self, M, N, seed):
        g = _gen(seed)
        few = lambda *s: torch.randint(-8, 9, s, generator=g, device=DEV).float() / 8      # noqa: E731
        self.A, self.B = ((few(r, 64)).to(torch.float8_e4m3fn).view(torch.uint8) for r in (M, N))
        self.dy = few(M, N).to(BF)
        self.one = _scalar(1.0)
        self.D, self.dz = torch.empty(M, N, dtype=BF, device=DEV), torch.empty(M, N, dtype=torch.uint8, device=DEV)
        self.outs = [_scalar(0.0), _scalar(0.0), torch.zeros(N, device=DEV)]
        a, b = (t.view(torch.float8_e4m3fn).double() for t in (self.A, self.B))
        self.want = [(a @ b.T).to(BF).float().abs().max().reshape(1), self.dy.float().abs().max().reshape(1), self.dy.double().sum(0).float()]

    def __call__(self):
        amax, amax_z, dbias = self.outs
        api.fp8_gemm_epilogue(self.A, E4, K_, self.B, E4, K_, self.D, self.one, self.one, amax_out=amax)
        api.fp8_epilogue_backward(self.dy, None, self.dz, fd=E5, scale_d=self.one, dbias=dbias, amax_out=amax_z)

    def clear(self):
        for t in self.outs:
            t.fill_(-5.0)

    def check(self):
        assert all(torch.equal(a, b) for a, b in zip(self.outs, self.want))


def test_a_graph_outlives_the_workspace_of_its_stream():
    """warm up, capture, warm up a larger shape (the stream's workspace grows), capture that, replay the first"""
    small, large = Calls(300, 256, 1), Calls(4096, 2048, 2)
    side = torch.cuda.Stream()
    graphs = []
    torch.cuda.synchronize()
    for c in (small, large):
        with torch.cuda.stream(side):
            c()
        side.synchronize()
        c.check()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            c()
    with torch.cuda.stream(side):
        others = [torch.full((n,), 17, dtype=torch.uint8, device=DEV) for n in (1 << 14, 1 << 16, 1 << 18, 1 << 20, 1 << 22) for _ in range(8)]
    torch.cuda.synchronize()
    for _ in range(3):
        for graph, c in zip(graphs, (small, large)):
            c.clear()
            graph.replay()
            torch.cuda.synchronize()
            c.check()
    assert all(bool((t == 17).all()) for t in others)
    _ok()


def test_graphs_of_one_stream_replayed_beside_its_plain_calls():
    """two graphs captured on one stream, replayed on two others, beside plain calls on the first"""
    calls = [Calls(70 + 30 * i, 384, 10 + i) for i in range(3)]
    home, others = torch.cuda.Stream(), [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    with torch.cuda.stream(home):
        for c in calls:
            c()
    home.synchronize()
    graphs = []
    for c in calls[1:]:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=home):
            for _ in range(4):
                c()
    for _ in range(40):
        for c in calls:
            c.clear()
        torch.cuda.synchronize()
        for s, graph in zip(others, graphs):
            with torch.cuda.stream(s):
                graph.replay()
        with torch.cuda.stream(home):
            for _ in range(4):
                calls[0]()
        torch.cuda.synchronize()
        for c in calls:
            c.check()
    _ok()


def test_a_clip_plan_is_ready_for_any_stream():
    """a plan made behind other work of its stream, used at once on another one"""
    xs = [torch.randint(-3, 4, (100000 + i,), generator=_gen(i), device=DEV).float() for i in range(3)]
    want = torch.stack([x.double().square().sum() for x in xs]).sum().sqrt().float().reshape(1)      # sums of whole numbers: exact
    junk = [torch.full((n,), 0xAB, dtype=torch.uint8, device=DEV) for n in (16, 128, 512, 1024, 4096) for _ in range(8)]
    first, second = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    del junk                                                 # what the allocator hands out next is not zero
    for _ in range(5):
        with torch.cuda.stream(first):
            torch.cuda._sleep(20_000_000)                    # some 10 ms
            plan = api.ClipPlan(xs, [torch.empty_like(x) for x in xs])
        norm = _scalar(0.0)
        torch.cuda.current_stream().synchronize()
        with torch.cuda.stream(second):
            api.fp8_grad_clip(plan, 1.0, norm)
        second.synchronize()
        assert torch.equal(norm, want)
    _ok()
