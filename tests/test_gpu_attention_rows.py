"""speca_layer_attention: a row's result depends on its own query and keys, on nothing that shares a launch with it."""
import pytest
import torch

from tests import layer_util as L
from tests.test_gpu_attention import DEV, DT, code, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    from paper_2509_11628_b200 import binding
    binding._lib()
    return binding


def call(layer, q, k, v, **kw):
    o = torch.full(q.shape, 3.0, device=DEV).to(q.dtype)
    lse = torch.full((q.shape[1], q.shape[0]), 3.0, device=DEV)
    layer.attention(q, k, v, o, lse=lse, **kw)
    return o, lse


def stir(S, hd):
    """Another call that leaves other rows in shared and tensor memory."""
    q, k, v = make(77, "bf16", 400, 400, 2, 2, hd, 30.0)
    other = S.SpecaLayer([0, 400], S.SPECA_BF16, n_heads=2, n_kv_heads=2, head_dim=hd, device=DEV)
    call(other, q, k, v)
    return other


def growing(k, off):
    """Keys whose lengths grow along each sequence, so that running maxima rise in many tiles, by little."""
    k = k.clone()
    for a, b in zip(off, off[1:]):
        if b > a:
            k[a:b] = (k[a:b].float() * torch.linspace(0.7, 1.5, b - a, device=DEV)[:, None, None]).to(k.dtype)
    return k


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("group", [1, 3, 7, 100])
@pytest.mark.parametrize("q_len,kv", [(1, 1500), (2, 900), (45, 1100)])
def test_neighbours_and_earlier_calls_do_not_show(S, dt, group, causal, q_len, kv):
    off, koff = L.offsets([q_len] * 3), L.offsets([kv] * 3)
    q, k, v = make(group, dt, off[-1], koff[-1], 2 * group, 2, 64)
    k = growing(k, koff)
    layer = S.SpecaLayer(off, code(S, dt), kv_start=koff, n_heads=2 * group, n_kv_heads=2, head_dim=64, causal=causal, device=DEV)
    want, want_lse = call(layer, q, k, v)
    keep = stir(S, 64)
    loud = q.clone()
    loud[off[0]:off[1]] *= 40          # the sequences around the middle one
    loud[off[2]:off[3]] *= -40
    for active in (None, torch.tensor([0, 1, 0], dtype=torch.uint8, device=DEV)):
        got, lse = call(layer, loud, k, v, active=active)
        rows = slice(off[1], off[2])
        assert torch.equal(got[rows], want[rows]) and torch.equal(lse[:, rows], want_lse[:, rows])
    layer.check()
    keep.check()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("group", [1, 4, 7])
def test_rows_of_one_sequence_do_not_show_in_each_other(S, dt, group):
    n = 500
    q, k, v = make(5, dt, n, n, 2 * group, 2, 64)
    k = growing(k, [0, n])
    layer = S.SpecaLayer([0, n], code(S, dt), n_heads=2 * group, n_kv_heads=2, head_dim=64, device=DEV)
    want, want_lse = call(layer, q, k, v)
    loud = q.clone()
    loud[1::2] *= 25
    got, lse = call(layer, loud, k, v)
    assert torch.equal(got[::2], want[::2]) and torch.equal(lse[:, ::2], want_lse[:, ::2])
    assert not torch.equal(got[1::2], want[1::2])
    layer.check()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("q_len,kv,split", [(200, 40, False), (64, 10, False), (140, 130, False), (6, 3000, True)])
def test_rows_that_see_nothing_are_zero_whatever_is_hidden_from_them(S, dt, q_len, kv, split):
    # causal, more queries than keys that hold data: the first rows see nothing, while other rows of their block read the tile
    fill = 4 if split else kv
    q, k, v = make(9, dt, q_len, kv, 4, 2, 64)
    v[:fill, 0, :] = float("inf")
    v[1, 1, 3] = float("nan")
    k[2, 1, 5] = float("nan")
    layer = S.SpecaLayer([0, q_len], code(S, dt), kv_start=[0, kv], n_heads=4, n_kv_heads=2, head_dim=64, causal=True, device=DEV)
    o, lse = call(layer, q, k, v, kv_len=torch.tensor([fill], dtype=torch.int32, device=DEV))
    n = q_len - fill
    assert n > 0 and bool((o[:n] == 0).all()) and bool((lse[:, :n] == -float("inf")).all())
    layer.check()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("group", [1, 3])
def test_keys_and_values_expanded_over_heads(S, dt, group):
    q, k, v = make(11, dt, 90, 300, 4 * group, 4, 64)
    layer = S.SpecaLayer([0, 40, 90], code(S, dt), kv_start=[0, 150, 300], n_heads=4 * group, n_kv_heads=4, head_dim=64, device=DEV)
    for wide_k, wide_v in ((True, True), (True, False), (False, True)):
        kk = k[:, 1:2].expand(-1, 4, -1) if wide_k else k
        vv = v[:, 2:3].expand(-1, 4, -1) if wide_v else v
        got, want = call(layer, q, kk, vv), call(layer, q, kk.contiguous(), vv.contiguous())
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    layer.check()
