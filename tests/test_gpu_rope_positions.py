"""speca_layer_rope at positions far from the origin."""
import pytest
import torch

from tests import layer_util as L

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("far", [2.0 ** 15, 2.0 ** 20, 2.0 ** 26])
def test_far_positions_cost_no_accuracy(far, halves):
    from paper_2509_11628_b200 import binding as S
    rows, h, hd = 96, 3, 64
    g = torch.Generator(device=DEV).manual_seed(2)
    layer = S.SpecaLayer([0, rows], S.SPECA_F32, n_heads=h, n_kv_heads=h, head_dim=hd, axis_dims=(48, 16),
                         pairing=S.SPECA_ROPE_HALVES if halves else S.SPECA_ROPE_INTERLEAVED, device=DEV)
    q = torch.randn(rows, h, hd, generator=g, device=DEV)
    pos = ((torch.rand(rows, 2, generator=g, device=DEV) * 2 - 1) * far).round()
    pos[0], pos[1] = far, -far
    out = torch.zeros_like(q)
    layer.rope(q, out, None, None, pos)
    want, bound = L.rope(q, None, pos, (48, 16), 10000.0, halves, 1e-6)
    # the angle in fp64: 4 roundings of position x frequency here, 2 in the definition: 6 * 2^26 * 2^-53 = 0.8 * 2^-24 more than
    # the 8 * 2^-24 that the turn itself is allowed
    L.check(out, want, bound * (1 + 1 / 8))
