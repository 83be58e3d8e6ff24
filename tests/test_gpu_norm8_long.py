"""speca_layer_norm8 over rows of millions of elements, whose sums are not exact in 32 bits."""
import pytest
import torch

from tests import eight_util as E

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def S():
    from paper_2509_11628_b200 import binding
    binding._lib()
    return binding


@pytest.mark.parametrize("dt", list(DT))
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("dim", [16385, 1 << 20, (1 << 24) + 77])
def test_sums_of_long_rows(S, dt, kind, dim):
    # +-0.3: every square is the same and no sum of them exact, which is where adding one after another loses most. A mean of 1/16 beside them for the layer norm
    g = torch.Generator(device=DEV).manual_seed(dim)
    x = ((torch.randint(0, 2, (2, dim), generator=g, device=DEV) * 2 - 1) * 0.3 + (0.0625 if kind == "layer" else 0.0)).to(DT[dt])
    layer = S.SpecaLayer([0, 1, 2], S.SPECA_BF16 if dt == "bf16" else S.SPECA_F32, device=DEV)
    m, xo = S.Matrix8.empty(2, dim, DEV), torch.zeros_like(x)
    layer.norm8(x, m, S.SPECA_NORM_RMS if kind == "rms" else S.SPECA_NORM_LAYER, x_out=xo)
    layer.check()
    assert torch.equal(xo, x)
    for r in range(2):
        z = x[r].double()
        mean = z.mean() if kind == "layer" else 0.0
        y = (z - mean) / torch.sqrt(((z - mean) ** 2).mean() + 1e-6)
        # 16 terms in 32 bits (15 roundings each way, and the square's), the rest in 64; the mean rounded once and taken off with a rounding: relative to what is
        # left, sqrt(mean^2 / var + 1) of each; then rstd (half the sum's 17 roundings, the division, the root and the addition of eps: 4), difference and product
        bound = (17 / 2 + 4 + 2 + 16 * (1 + abs(float(mean)) / 0.3)) * E.U32 * y.abs()
        E.check8(S.Matrix8(m.codes[r:r + 1], m.scales[:, r:r + 1]), y[None], bound[None], "row %d" % r)


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_codes_next_to_a_border_tell_sums_apart(S, kind):
    # those of 0.7 rstd change when rstd is 1.1e-4 off, as adding up 16384 squares
    # a thread in 32 bits leaves it, since the weight puts them 2e-5 before or behind the border between them
    dim = 1 << 24
    g = torch.Generator(device=DEV).manual_seed(1)
    signs = (torch.randint(0, 2, (1, dim), generator=g, device=DEV) * 2 - 1).float()
    x = signs * torch.tensor(0.7, device=DEV)
    z = x.double()
    mean = z.mean() if kind == "layer" else 0.0
    unit = ((z - mean) / torch.sqrt(((z - mean) ** 2).mean() + 1e-6)).abs().mean()
    # codes of 1 and 1.125: their border is 1.0625. Weights on either side of it, and a 1.7 in every block, so that its scale is the one of values up to 1.75
    weight = torch.full((dim,), 1.0625, dtype=torch.float64, device=DEV)
    weight[0::2] *= 1 + 2e-5
    weight[1::2] *= 1 - 2e-5
    weight /= unit
    weight[::128] = 1.7 / unit
    layer = S.SpecaLayer([0, 1], S.SPECA_F32, device=DEV)
    m = S.Matrix8.empty(1, dim, DEV)
    layer.norm8(x, m, S.SPECA_NORM_RMS if kind == "rms" else S.SPECA_NORM_LAYER, weight=weight.float())
    layer.check()
    v = E.values(m).abs().float()[0]
    keep = torch.ones(dim, dtype=torch.bool, device=DEV)
    keep[::128] = False
    if kind == "layer":   # the mean, some 1e-4 of 0.7, moves the two signs apart by more than the weights do
        assert bool(((v == 1) | (v == 1.125))[keep].all())
        want = ((z - mean) / torch.sqrt(((z - mean) ** 2).mean() + 1e-6) * weight.float().double()).abs()[0]
        keep &= (want - 1.0625).abs() > 1e-5
        assert bool(((v == 1.125) == (want > 1.0625))[keep].all())
    else:
        assert bool((v[0::2] == 1.125)[keep[0::2]].all()) and bool((v[1::2] == 1).all())
