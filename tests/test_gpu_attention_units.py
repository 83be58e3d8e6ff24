"""speca_layer_attention with more units of work than the device has SMs, and keys shared out over many units."""
import pytest
import torch

from tests import layer_util as L
from tests.test_gpu_attention import DEV, code, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    from paper_2509_11628_b200 import binding
    binding._lib()
    return binding


def verify(S, dt, q_lens, kv_lens, h, kv, hd, causal, masks, kv_len=None, seed=0):
    """One handle under several active masks in turn (None: all), directly and from a graph, against 64 bits."""
    off, koff = L.offsets(q_lens), L.offsets(kv_lens)
    q, k, v = make(seed, dt, off[-1], koff[-1], h, kv, hd, 1.5)
    layer = S.SpecaLayer(off, code(S, dt), kv_start=koff, n_heads=h, n_kv_heads=kv, head_dim=hd, causal=causal, device=DEV)
    lens = None if kv_len is None else torch.tensor(kv_len, dtype=torch.int32, device=DEV)
    want, bound, wl, bl = L.attention(off, koff, q, k, v, causal, hd ** -0.5, kv_len)
    seq = torch.repeat_interleave(torch.arange(len(q_lens), device=DEV), torch.tensor(q_lens, device=DEV))
    active = torch.ones(len(q_lens), dtype=torch.uint8, device=DEV)
    o, lse = torch.zeros_like(q), torch.zeros(h, off[-1], device=DEV)
    graph, first = None, None
    for mask in masks:
        active.copy_(torch.tensor([1] * len(q_lens) if mask is None else mask, dtype=torch.uint8))
        on = active.bool()[seq]
        got = []
        for way in range(3):
            o.fill_(7.0)
            lse.fill_(7.0)
            if way < 2:
                layer.attention(q, k, v, o, lse=lse, kv_len=lens, active=active)
            else:
                if graph is None:
                    graph = torch.cuda.CUDAGraph()
                    with torch.cuda.graph(graph):
                        layer.attention(q, k, v, o, lse=lse, kv_len=lens, active=active)
                graph.replay()
            got.append((o.clone(), lse.clone()))
        for a, b in got[1:]:
            assert torch.equal(a, got[0][0]) and torch.equal(b, got[0][1])
        a, b = got[0]
        assert bool((a[~on] == 7.0).all()) and bool((b[:, ~on] == 7.0).all())
        L.check(a[on], want[on], bound[on], "o")
        L.check(b[:, on], wl[:, on], bl[:, on], "lse")
        if mask is None:
            first = got[0]
        elif first is not None:     # who else is recomputed does not show
            assert torch.equal(a[on], first[0][on]) and torch.equal(b[:, on], first[1][:, on])
    layer.check()


def masks_of(n):
    g = torch.Generator().manual_seed(n)
    some = (torch.rand(n, generator=g) < 0.6).int().tolist()
    return [None, some, [1 - x for x in some], [int(i == n // 2) for i in range(n)], [0] * n]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("hd", [16, 64, 72, 128])
def test_units_of_two_blocks_follow_one_another(S, causal, hd):
    # 45 samples of 1 to 300 rows x 8 heads: over 400 units on 148 SMs, of one row block and of two, with one tile and with three
    lens = [1 + (i * 67) % 300 for i in range(45)]
    verify(S, "bf16", lens, lens, 8, 8, hd, causal, masks_of(45), seed=hd)


@pytest.mark.parametrize("group", [3, 4])
def test_units_of_shared_heads_follow_one_another(S, group):
    lens = [97, 0, 310, 12, 128, 129, 64, 1, 255, 200] * 3
    verify(S, "bf16", lens, lens, 4 * group, 4, 64, True, masks_of(30), seed=group)


def test_one_long_sequence_of_many_heads(S):
    verify(S, "bf16", [2100], [2100], 24, 24, 64, False, [None, [1]], seed=3)
    verify(S, "bf16", [1500, 900], [1500, 900], 24, 24, 64, True, [None, [0, 1], [1, 0]], seed=4)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_many_single_tokens(S, dt):
    # 200 sequences x 2 key heads: over 148 units that take two shares of their keys at once, next to short ones
    n = 200
    kv = [40 + (i * 331) % 1500 for i in range(n)]
    fill = [max(0, x - (i * 17) % 60) for i, x in enumerate(kv)]
    verify(S, dt, [1] * n, kv, 8, 2, 64, True, masks_of(n), kv_len=fill, seed=5)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("q_lens,kv_lens,fill", [([1], [40000], [39991]), ([3, 1], [30000, 9000], [1, 8999]), ([2], [70000], [4000])])
def test_keys_shared_out_over_more_units_than_a_warp_has_lanes(S, dt, q_lens, kv_lens, fill):
    # the join takes 32 shares at a time: these have 40 and more, most of them empty where the cache is hardly filled
    verify(S, dt, q_lens, kv_lens, 4, 1, 64, True, [None, [1] * len(q_lens), [0] * len(q_lens)], kv_len=fill, seed=6)


def test_a_wait_that_ran_out_is_reported_once(S):
    # the word that a kernel sets when it gives up on a wait, set from the host: behind the row map of a layer without heads
    layer = S.SpecaLayer([0, 100], S.SPECA_BF16, device=DEV)
    word = layer.workspace[-256:].view(torch.int32)[:1]
    assert int(word) == 0
    layer.check()
    word.fill_(1)
    with pytest.raises(S.SpecaError) as e:
        layer.check()
    assert e.value.status == S.SPECA_ERR_CUDA and "gave up" in str(e.value)
    layer.check()                      # cleared
    assert int(word) == 0
    word.fill_(1)
    with pytest.raises(S.SpecaError) as e:
        layer.close()
    assert e.value.status == S.SPECA_ERR_CUDA
    assert layer.handle is None
