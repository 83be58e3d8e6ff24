"""speca_quantize8 on a stream that is not the current one."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("address", [False, True])
def test_a_new_matrix_belongs_to_the_stream_of_the_call(address):
    from paper_2509_11628_b200 import binding as S
    x = torch.randn(300, 1000, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).bfloat16()
    want = S.quantize8(x)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        torch.cuda._sleep(20_000_000)   # some 10 ms: what the current stream is given now comes late
        got = S.quantize8(x, stream=side.cuda_stream if address else side)
        torch.cuda.synchronize()
        assert torch.equal(got.codes.view(torch.uint8), want.codes.view(torch.uint8))
        assert torch.equal(got.scales.view(torch.uint8), want.scales.view(torch.uint8))


def test_the_default_stream_by_its_address():
    from paper_2509_11628_b200 import binding as S
    x = torch.randn(30, 100, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)
    want = S.quantize8(x)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got = S.quantize8(x, stream=0)
    torch.cuda.synchronize()
    assert torch.equal(got.codes.view(torch.uint8), want.codes.view(torch.uint8))
