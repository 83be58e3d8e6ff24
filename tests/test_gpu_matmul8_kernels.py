"""Every kernel of the 8-bit products, in every tile and with k shared out in every way, through the checks against 64 bits. Which kernel a size goes to is
asserted where the lists are."""
import pytest
import torch

from tests import eight_plan as P
from tests import eight_util as E
from tests import test_gpu_matmul8 as T

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SIZES = list(P.FEW.values()) + P.ONE + P.PAIR + [P.MASKED_TO_PAIR, P.MASKED_TO_ONE]


@pytest.fixture(scope="module")
def S():
    from paper_2509_11628_b200 import binding
    binding._lib()
    return binding


def check8(m, y, bound, what="", live=None):
    """E.check8, and blocks all of whose values may be zero within their bounds may be zeros, with the scale of a block of zeros. E.check8 holds the scale of a block that is
    not zero for certain to a byte of at most that of |y| + bound, which 127 is not where that is below 2^-1: GELU of -30 is 0 (its exponential's argument is -1975),
    alone in a block of one column it makes zeros with 127, and the bound, which goes by the argument, is 4e-3."""
    rows = slice(None) if live is None else live
    got, byte = E.values(m)[rows], E.bytes_of(m)[rows].long()
    zeros = (E.blocks((y[rows].abs() - bound[rows]).clamp_min(0)).amax(2) == 0) & (E.blocks(got).abs().amax(2) == 0) & (byte == 127)
    wide = torch.zeros(y.shape, dtype=torch.bool, device=y.device)
    wide[rows] = zeros.repeat_interleave(128, 1)[:, :y.shape[1]]
    ORIGINAL(m, torch.where(wide, 0.0, y), torch.where(wide, 0.0, bound), what, live)


ORIGINAL = E.check8


@pytest.mark.parametrize("m,n,k", SIZES)
def test_whole_numbers(S, m, n, k):
    T.test_whole_numbers_are_exact(S, m, n, k)


@pytest.mark.parametrize("dt,kind", [("bf16", "gelu"), ("f32", "silu"), ("bf16", "none")])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_epilogues(S, monkeypatch, dt, kind, m, n, k):
    monkeypatch.setattr(E, "check8", check8)
    T.test_epilogues(S, dt, kind, m, n, k)


@pytest.mark.parametrize("m,n,k", SIZES)
def test_masks(S, m, n, k):
    T.test_masked_samples_are_left_alone_and_others_do_not_see_it(S, m, n, k)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_strides(S, dt, m, n, k):
    T.test_strides_offsets_and_in_place(S, dt, m, n, k)


@pytest.mark.parametrize("m,n,k", SIZES)
def test_nan(S, m, n, k):
    T.test_nan_stays_in_its_row_and_column(S, m, n, k)


@pytest.mark.parametrize("m,n,k", SIZES)
def test_the_same_bits_every_time(S, m, n, k):
    g = T.gen(m)
    a, w = T.real(g, m, k), T.real(g, n, k, k ** -0.5)
    layer = S.SpecaLayer([0, m], S.SPECA_BF16, device=DEV)
    first, again = T.blank(S, m, n), T.blank(S, m, n)
    layer.matmul8(a, w, first, activation=S.SPECA_ACT_GELU)
    for _ in range(10):
        layer.matmul8(a, w, again, activation=S.SPECA_ACT_GELU)
        assert all(torch.equal(x, y) for x, y in zip(T.raw(first), T.raw(again)))
