"""How much the sums of the 8-bit products lose: the tensor cores cut what they add to a sum, so that k is summed in shares where that would be seen."""
import pytest
import torch

from tests import eight_util as E

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def S():
    from paper_2509_11628_b200 import binding
    binding._lib()
    return binding


def operand(S, g, rows, k, positive):
    m = S.Matrix8.empty(rows, k, DEV)
    for r in range(0, rows, 256):
        part = slice(r, min(r + 256, rows))
        n = part.stop - part.start
        x = torch.rand(n, k, generator=g, device=DEV) if positive else torch.randn(n, k, generator=g, device=DEV)
        S.quantize8(x, S.Matrix8(m.codes[part], m.scales[:, part]))
    return m


# of fp32 outputs. A single sum of normal values is 5.0e-7 off at 8192 elements, one of 4096 2.2e-7, in proportion to the length; of uniform positive values 2.7e-6
# and 9.4e-7. Shares are of 4096 elements at 16384, of k / 8 beyond 32768. Rows with one value 20 times the others' are up to twice as far off. The limits
# lie between what a share and what a single sum loses
@pytest.mark.parametrize("m,n", [(4, 512), (300, 512), (2304, 1024)])
@pytest.mark.parametrize("k,normal,positive", [(8192, 1.35e-6, 4.1e-6), (16384, 5.6e-7, 1.4e-6), (65536, 1.4e-6, 4.1e-6), (262144, 5.6e-6, 2.7e-5)])
def test_fp32_outputs_lose_no_more_than_a_share_does(S, m, n, k, normal, positive):
    if m * k > 300 * 262144:
        m = 300 * 262144 // k
    g = torch.Generator(device=DEV).manual_seed(k)
    for limit, sign in ((normal, False), (positive, True)):
        a, w = operand(S, g, m, k, sign), operand(S, g, n, k, sign)
        layer = S.SpecaLayer([0, m], S.SPECA_F32, device=DEV)
        out = torch.zeros(m, n, device=DEV)
        layer.matmul8(a, w, out)
        layer.check()
        want = torch.zeros(m, n, dtype=torch.float64, device=DEV)
        for c in range(0, k, 16384):
            part = lambda x: E.values(S.Matrix8(x.codes[:, c:c + 16384], x.scales[c // 512:(c + 16384) // 512][:-(-min(16384, k - c) // 512)]))
            want += part(a) @ part(w).T
        assert float((out.double() - want).norm() / want.norm()) < limit


# the few rows' kernel with shares of its own accord and without, tiles of one SM, of a pair
@pytest.mark.parametrize("m,n", [(4, 512), (4, 10000), (300, 2048), (2304, 2048)])
@pytest.mark.parametrize("k", [32768, 65536, 262144])
def test_a_large_term_and_many_small_ones_of_its_sign(S, m, n, k):
    # 1 and k - 128 terms of 1.875 * 2^-25, which a sum of 1 cuts. Of s of them summed at once next to the 1 up to 2^-25 each may be lost: with s at most 32768 that is
    # 2^-10, beside a bf16 rounding of 2^-8 at most (half a step of the binade of 1) of a result up to 1.015; shares without the 1 lose nothing of that
    # size (terms alike: 2^-14 of their sum, as above)
    codes = lambda rows, byte: torch.full((rows, k), byte, dtype=torch.uint8, device=DEV)

    def matrix(rows, byte, exponent):
        c = codes(rows, byte)
        c[:, 0], c[:, 1:128] = 0x38, 0
        s = torch.full((k // 512, rows, 4), exponent, dtype=torch.uint8, device=DEV)
        s[0, :, 0] = 127
        return S.Matrix8(c.view(torch.float8_e4m3fn), s.view(torch.float8_e8m0fnu))

    a, w = matrix(m, 0x38, 127 - 12), matrix(n, 0x3f, 127 - 13)
    layer = S.SpecaLayer([0, m], S.SPECA_BF16, device=DEV)
    out = torch.zeros(m, n, dtype=torch.bfloat16, device=DEV)
    layer.matmul8(a, w, out)
    layer.check()
    want = 1 + (k - 128) * 1.875 * 2.0 ** -25
    low = want - 2.0 ** -10 - 2.0 ** -14 * (want - 1)
    assert bool((out.double() >= low - 2.0 ** -8).all() and (out.double() <= want + 2.0 ** -8).all())
    # in fp32, which is shared out sooner, without that rounding
    exact = S.SpecaLayer([0, m], S.SPECA_F32, device=DEV)
    out32 = torch.zeros(m, n, device=DEV)
    exact.matmul8(a, w, out32)
    exact.check()
    assert bool((out32.double() >= low).all() and (out32.double() <= want * (1 + 2.0 ** -22)).all())
