"""Products right behind the kernels that write their operands: the few-row kernel fetches weights into L2 ahead of the stream
dependency, while the kernel before it may still be writing them, and must read what was written."""
import pytest
import torch

from paper_2209_05433_b200 import api
from tests.test_gpu_fused import BF, E4, K_, MN, _gen, _ok, _scalar

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("shape", [(512, 256), (4096, 4096), (16384, 4096)], ids=str)
@pytest.mark.parametrize("writer", ["quantize", "current", "copy"])
@pytest.mark.parametrize("layout", [K_, MN])
def test_weights_written_by_the_kernel_before(shape, writer, layout):
    """each round converts other weights into the same buffer and multiplies at once; all values are small whole numbers, so
    the products are exact and each differs from the one of the round before"""
    K, N = shape
    g = _gen(K)
    rounds = 24
    wides = [torch.randint(-3, 4, (N, K) if layout == K_ else (K, N), generator=g, device=DEV, dtype=torch.int8).to(BF) for _ in range(4)]
    for w in wides:
        w[0, 0] = 7.0                                        # one amax, and so one current scale
    one = _scalar(1.0)
    s = torch.zeros(3, device=DEV)
    W = torch.zeros(wides[0].shape, dtype=torch.uint8, device=DEV)
    ready = [w.to(torch.float8_e4m3fn).view(torch.uint8) for w in wides]
    x = torch.randint(-2, 3, (3, K), generator=g, device=DEV).float()
    A = x.to(torch.float8_e4m3fn).view(torch.uint8)
    outs = [torch.full((3, N), 0.5, device=DEV) for _ in range(rounds)]
    torch.cuda.synchronize()
    for i, out in enumerate(outs):
        w = wides[i % 4]
        inv = one
        if writer == "quantize":
            api.fp8_quantize(w, E4, one, W)
        elif writer == "current":
            api.fp8_quantize_current(w, E4, W, s[0:1], s[1:2], s[2:3])      # scale 64: exact
            inv = s[2:3]
        else:
            W.copy_(ready[i % 4])
        api.fp8_gemm_epilogue(A, E4, K_, W, E4, layout, out, one, inv)
    _ok()
    for i, out in enumerate(outs):
        w = wides[i % 4].double()
        assert torch.equal(out.double(), x.double() @ (w.T if layout == K_ else w)), i


def test_tokens_and_weights_of_a_chain_of_products():
    """every product's output is the next one's operand"""
    g = _gen(4)
    N = 1024
    W = [torch.randint(0, 2, (N, N), generator=g, device=DEV).float() for _ in range(3)]
    codes = [w.to(torch.float8_e4m3fn).view(torch.uint8) for w in W]
    x = torch.randint(0, 2, (2, N), generator=g, device=DEV).float()
    bufs = [torch.zeros(2, N, dtype=torch.uint8, device=DEV) for _ in range(3)]
    one, scale = _scalar(1.0), _scalar(2.0 ** -7)
    bufs[0].copy_(x.to(torch.float8_e4m3fn).view(torch.uint8))
    finals = []
    for _ in range(30):                                      # values stay positive and in range: about 256 before each scale
        src = bufs[0]
        for w, dst in zip(codes, (bufs[1], bufs[2], bufs[1])):
            api.fp8_gemm_epilogue(src, E4, K_, w, E4, K_, dst, one, one, fd=E4, scale_d=scale)
            src = dst
        finals.append(src.clone())
    _ok()
    assert all(torch.equal(f, finals[0]) for f in finals)
    v = x
    for w in W:
        v = ((v @ w.T) * 2.0 ** -7).clamp(-448, 448).to(torch.float8_e4m3fn).float()
    assert torch.equal(finals[0].view(torch.float8_e4m3fn).float(), v)
