"""Activations of the 8-bit products where their arguments are far off or not finite: a column with such values next to ordinary ones, which two kernels put
through one reciprocal in pairs."""
import pytest
import torch

from tests import eight_util as E

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF, NAN = float("inf"), float("nan")
FAR = [-1e20, 1e20, -1e38, -INF, INF, NAN, -44.0, -50.0, -90.0, -1000.0, -8.0, -1e4, 60.0, 1e4]


@pytest.fixture(scope="module")
def S():
    from paper_2509_11628_b200 import binding
    binding._lib()
    return binding


def limit(t, kind):
    """x / (1 + exp(-s)) in 64 bits, as it is written: an infinite exponential makes zero of all that is finite, and a NaN of -inf."""
    t = t.double()
    return t / (1 + torch.exp(-t if kind == "silu" else -1.5957691216057308 * (t + 0.044715 * t ** 3)))


# few rows, tiles of one SM, tiles of a pair
@pytest.mark.parametrize("m,n,k", [(9, 512, 256), (1100, 1504, 128), (2304, 4096, 128)])
@pytest.mark.parametrize("kind", ["gelu", "silu"])
def test_far_and_not_finite_arguments(S, m, n, k, kind):
    g = torch.Generator(device=DEV).manual_seed(m)
    a = S.quantize8(torch.randn(m, k, generator=g, device=DEV))
    w = S.quantize8(torch.randn(n, k, generator=g, device=DEV) * k ** -0.5)
    bias = torch.randn(n, generator=g, device=DEV)
    act = S.SPECA_ACT_GELU if kind == "gelu" else S.SPECA_ACT_SILU
    layer = S.SpecaLayer([0, m], S.SPECA_F32, device=DEV)
    out, out8, far, far8 = torch.zeros(m, n, device=DEV), S.Matrix8.empty(m, n, DEV), torch.zeros(m, n, device=DEV), S.Matrix8.empty(m, n, DEV)
    layer.matmul8(a, w, out, bias=bias, activation=act)
    layer.matmul8(a, w, out8, bias=bias, activation=act)
    # at both places of a pair, in the columns of a block of 128, the other blocks left alone
    cols = [128 + 3 * i for i in range(len(FAR))]
    rows_cols = torch.tensor(cols, device=DEV)
    bias[rows_cols] = torch.tensor(FAR, device=DEV)
    layer.matmul8(a, w, far, bias=bias, activation=act)
    layer.matmul8(a, w, far8, bias=bias, activation=act)
    layer.check()
    # the other element of a pair has its factor from one reciprocal of both, 1 / a = b / (a b): the product's rounding, the reciprocal's (2^-23), two more
    # and the output's are five roundings in either evaluation, so they differ by ten at most; elements of other pairs are the same
    others = torch.ones(n, dtype=torch.bool, device=DEV)
    others[rows_cols] = False
    assert bool(((far - out).double().abs() <= 10 * E.U32 * out.double().abs())[:, others].all())
    others[rows_cols ^ 1] = False
    assert torch.equal(far[:, others], out[:, others])
    t, bound = E.product(a, w, bias.nan_to_num(0, 0, 0))
    for c, f in zip(cols, FAR):
        want = limit(t[:, c] if abs(f) < INF else t[:, c] + f, kind)
        got = far[:, c].double()
        if f != f or f == -INF:
            assert bool(want.isnan().all() and got.isnan().all()), f
        elif f == INF:
            assert bool((want == INF).all() and (got == INF).all()), f
        else:
            # a factor below 2^-63 may be zero: the argument is then some -8 (GELU) or -44 (SILU). Else the sum's bound (slope at most 1.13) and 64 roundings
            # of the argument, as in the other tests of the activations, and the output's rounding
            allow = 1.13 * bound[:, c] + 65 * E.U32 * t[:, c].abs() * (t[:, c] > -100) + 64 * 2.0 ** -63
            assert bool(((got - want).abs() <= allow).all()), (f, float((got - want).abs().max()))
    # in 8 bits: what is not finite is NaN; other blocks as before
    codes = far8.codes.float()
    for c, f in zip(cols, FAR):
        assert bool(codes[:, c].isnan().all()) == (not abs(f) < INF), f
    rest = torch.cat([torch.arange(128, device=DEV), torch.arange(256, n, device=DEV)])
    assert torch.equal(far8.codes.view(torch.uint8)[:, rest], out8.codes.view(torch.uint8)[:, rest])
    # far arguments that come to nothing leave a block's scale to the others
    bias[128:256] = torch.randn(128, generator=g, device=DEV)
    bias[130], bias[133] = -1e20, -1e30
    layer.matmul8(a, w, far, bias=bias, activation=act)
    layer.matmul8(a, w, far8, bias=bias, activation=act)
    layer.check()
    assert bool((far[:, [130, 133]] == 0).all() and (far8.codes.float()[:, [130, 133]] == 0).all())
    assert torch.equal(E.bytes_of(far8).long(), E.eight(far.double())[1])
