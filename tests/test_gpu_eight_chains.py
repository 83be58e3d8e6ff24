"""Chains of 8-bit calls whose operands are written again and again in place, with nothing waited for in between: every kernel begins while the one in front,
which writes its codes and scales, still runs."""
import pytest
import torch

from tests import eight_util as E
from tests import layer_util as L

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def S():
    from paper_2509_11628_b200 import binding
    binding._lib()
    return binding


def raw(m):
    return m.codes.view(torch.uint8), m.scales.view(torch.uint8)


# few rows in tiles of 16 and of 64, tiles of one SM, tiles of a pair
@pytest.mark.parametrize("m,n,k", [(3, 640, 2048), (200, 1000, 1152), (1100, 1504, 520), (2304, 4096, 384)])
def test_operands_rewritten_in_place(S, m, n, k):
    g = torch.Generator(device=DEV).manual_seed(m)
    # sizes from 2^-12 to 2^12, so that a scale of another step is far off
    xs = [torch.randn(m, k, generator=g, device=DEV).bfloat16() * 2.0 ** (8 * i - 12) for i in range(4)]
    ws = [torch.randn(n, k, generator=g, device=DEV).bfloat16() * 2.0 ** (6 - 5 * i) for i in range(3)]
    layer = S.SpecaLayer([0, m], S.SPECA_BF16, device=DEV)
    a, w, up = S.Matrix8.empty(m, k, DEV), S.Matrix8.empty(n, k, DEV), S.Matrix8.empty(m, n, DEV)
    square = S.quantize8(torch.randn(64, n, generator=g, device=DEV).bfloat16())

    def step(i, outs):
        S.quantize8(ws[i % 3], w)
        if i % 2:
            layer.norm8(xs[i % 4], a)
        else:
            layer.quantize8(xs[i % 4], a)
        layer.matmul8(a, w, outs[0])
        layer.matmul8(a, w, up, activation=S.SPECA_ACT_SILU)
        layer.matmul8(up, square, outs[1])

    def blank():
        return torch.zeros(m, n, dtype=torch.bfloat16, device=DEV), torch.zeros(m, 64, dtype=torch.bfloat16, device=DEV)

    want = []
    for i in range(12):
        want.append(blank())
        S.quantize8(ws[i % 3], w)
        torch.cuda.synchronize()
        (layer.norm8 if i % 2 else layer.quantize8)(xs[i % 4], a)
        torch.cuda.synchronize()
        layer.matmul8(a, w, want[-1][0])
        torch.cuda.synchronize()
        layer.matmul8(a, w, up, activation=S.SPECA_ACT_SILU)
        torch.cuda.synchronize()
        layer.matmul8(up, square, want[-1][1])
        torch.cuda.synchronize()
    got = [blank() for _ in range(12)]
    off = torch.zeros((), dtype=torch.int64, device=DEV)
    for _ in range(25):
        for i in range(12):
            step(i, got[i])
        for i in range(12):
            for x, y in zip(got[i], want[i]):
                off += (x != y).any()
                x.zero_()
    layer.check()
    assert int(off) == 0


@pytest.mark.parametrize("m,n,k", [(3, 640, 2048), (1100, 1504, 520), (2304, 4096, 384)])
def test_in_a_graph_behind_copies(S, m, n, k):
    # nodes in front that are no kernels: a copy from the host, a copy on the device, a fill
    g = torch.Generator(device=DEV).manual_seed(1)
    layer = S.SpecaLayer([0, m], S.SPECA_BF16, device=DEV)
    host = torch.empty(m, k, dtype=torch.bfloat16, pin_memory=True)
    x, y = (torch.zeros(m, k, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    w = S.quantize8(torch.randn(n, k, generator=g, device=DEV).bfloat16())
    a, out = S.Matrix8.empty(m, k, DEV), torch.zeros(m, n, dtype=torch.bfloat16, device=DEV)

    def run():
        x.copy_(host, non_blocking=True)
        layer.quantize8(x, a)
        y.copy_(x)
        layer.norm8(y, a)
        raw(a)[1][:, :m // 2].fill_(120)
        layer.matmul8(a, w, out)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for seed in range(8):
        host.copy_(torch.randn(m, k, generator=torch.Generator().manual_seed(seed)).bfloat16() * 2.0 ** seed)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        b, want = S.Matrix8.empty(m, k, DEV), torch.zeros_like(out)
        layer.norm8(host.to(DEV), b)
        torch.cuda.synchronize()
        raw(b)[1][:, :m // 2].fill_(120)
        torch.cuda.synchronize()
        layer.matmul8(b, w, want)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    layer.check()
