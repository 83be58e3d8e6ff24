"""speca_layer_attention against its definition in 64 bits."""
import math

import pytest
import torch

from tests import layer_util as L

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def S():
    from paper_2509_11628_b200 import binding
    binding._lib()
    return binding


def code(S, dt):
    return S.SPECA_BF16 if dt == "bf16" else S.SPECA_F32


def make(seed, dt, rows, kv_rows, h, kv, hd, sharp=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    q = (sharp * torch.randn(rows, h, hd, generator=g, device=DEV)).to(DT[dt])
    k = (torch.randn(kv_rows, kv, hd, generator=g, device=DEV) + 0.5).to(DT[dt])
    v = (torch.randn(kv_rows, kv, hd, generator=g, device=DEV) + 0.25).to(DT[dt])
    return q, k, v


def run(S, dt, q_lens, kv_lens, h, kv, hd, causal, kv_len=None, sharp=1.0, seed=0, scale=0.0, qkv=None):
    off, koff = L.offsets(q_lens), L.offsets(kv_lens)
    q, k, v = qkv if qkv is not None else make(seed, dt, off[-1], koff[-1], h, kv, hd, sharp)
    layer = S.SpecaLayer(off, code(S, dt), kv_start=koff, n_heads=h, n_kv_heads=kv, head_dim=hd, causal=causal, scale=scale,
                         device=DEV)
    o = torch.full((off[-1], h, hd), 5.0, device=DEV).to(DT[dt])
    lse = torch.full((h, off[-1]), 5.0, device=DEV)
    lens = None if kv_len is None else torch.tensor(kv_len, dtype=torch.int32, device=DEV)
    layer.attention(q, k, v, o, lse=lse, kv_len=lens)
    layer.check()
    want, bound, wl, bl = L.attention(off, koff, q, k, v, causal, scale if scale > 0 else hd ** -0.5, kv_len)
    L.check(o, want, bound, "o")
    L.check(lse, wl, bl, "lse")
    # once more, bit for bit: the counters of shared rows are ready again and no order of arrival shows
    o2, lse2 = torch.zeros_like(o), torch.zeros_like(lse)
    layer.attention(q, k, v, o2, lse=lse2, kv_len=lens)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    return o


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [8, 16, 24, 32, 40, 64, 72, 80, 96, 104, 120, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_head_dims(S, dt, hd, causal):
    run(S, dt, [150, 33], [150, 33], 2, 2, hd, causal, seed=hd)


@pytest.mark.parametrize("hd", [1, 2, 7, 36, 65, 127])
def test_f32_odd_head_dims(S, hd):
    run(S, "f32", [70], [70], 3, 3, hd, True, seed=hd)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 63, 64, 65, 127, 128, 129, 143, 255, 256, 257, 383, 385, 512, 700])
def test_lengths(S, dt, causal, n):
    run(S, dt, [n], [n], 2, 2, 64, causal, seed=n, sharp=2.0)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True])
def test_ragged_packed_with_empty_sequences(S, dt, causal):
    lens = [1, 0, 77, 300, 16, 0, 129, 5, 0]
    run(S, dt, lens, lens, 4, 2, 72, causal)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("group", [1, 2, 3, 4, 5, 7, 8, 12, 64, 100, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_shared_heads(S, dt, group, causal):
    run(S, dt, [37, 4], [37, 4], 2 * group, 2, 32, causal, seed=group)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True])
def test_queries_and_keys_of_different_length(S, dt, causal):
    # more queries than keys: with the causal rule the first rows see nothing
    run(S, dt, [200, 3, 130, 9, 4, 1], [40, 300, 130, 0, 600, 1], 4, 4, 64, causal)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True])
def test_valid_keys_and_whatever_lies_behind_them(S, dt, causal):
    q_lens, kv_lens = [3, 60, 1, 2, 140, 8, 5], [500, 200, 130, 64, 260, 33, 40]
    kv_len = [499, 129, 1, 0, 257, 33, -4]
    koff = L.offsets(kv_lens)
    q, k, v = make(1, dt, sum(q_lens), sum(kv_lens), 4, 2, 64)
    for s, n in enumerate(kv_len):   # what a cache holds behind its fill: anything
        k[koff[s] + max(0, n):koff[s + 1]] = float("nan")
        v[koff[s] + max(0, n):koff[s + 1]] = float("inf") if s % 2 else float("nan")
    run(S, dt, q_lens, kv_lens, 4, 2, 64, causal, kv_len=kv_len, qkv=(q, k, v))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("hd,kv,group", [(128, 1, 1), (64, 2, 4), (72, 1, 7), (128, 8, 4)])
@pytest.mark.parametrize("q_len", [1, 2, 5])
def test_few_queries_long_keys(S, dt, hd, kv, group, q_len):
    run(S, dt, [q_len, q_len, q_len], [5000, 1, 2111], kv * group, kv, hd, True, kv_len=[4999, 1, 1500], sharp=2.0)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_sharp_scores_and_growing_maxima(S, dt):
    # keys of growing length: every tile raises the running maximum, by a lot
    n = 700
    q, k, v = make(4, dt, n, n, 2, 2, 64)
    k = (k.float() * torch.linspace(0.01, 6, n, device=DEV)[:, None, None]).to(DT[dt])
    run(S, dt, [n], [n], 2, 2, 64, False, qkv=(q * 2, k, v))
    run(S, dt, [n], [n], 2, 2, 64, True, qkv=(q * 2, -k, v))
    run(S, dt, [n], [n], 2, 2, 64, False, qkv=(q * 2, k.flip(0), v))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_scale_is_used_and_equal_keys_average(S, dt):
    run(S, dt, [100], [100], 2, 2, 64, False, scale=0.7)
    q, k, v = make(4, dt, 90, 90, 1, 1, 64)
    o = run(S, dt, [90], [90], 1, 1, 64, False, qkv=(q, k[:1].expand_as(k).contiguous(), v))
    torch.testing.assert_close(o.double()[:, 0], v.double()[:, 0].mean(0).expand(90, -1), rtol=2.0 ** -6, atol=2.0 ** -7)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_layouts(S, dt):
    off = L.offsets([40, 150])
    rows, h, kv, hd = off[-1], 4, 4, 64
    layer = S.SpecaLayer(off, code(S, dt), n_heads=h, n_kv_heads=kv, head_dim=hd, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(8)
    qkv = torch.randn(rows, 3, h, hd, generator=g, device=DEV).to(DT[dt])
    q, k, v = qkv.unbind(1)
    want, bound, _, _ = L.attention(off, off, q, k, v, False, hd ** -0.5)
    o = torch.zeros(rows, h, hd, device=DEV).to(DT[dt])
    layer.attention(q, k, v, o)                                  # parts of one projection
    L.check(o, want, bound)
    heads_first = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v)]
    oh = torch.zeros(h, rows, hd, device=DEV).to(DT[dt]).transpose(0, 1)
    layer.attention(*heads_first, oh)                            # [heads, rows, hd] in memory, in and out
    assert torch.equal(o, oh)
    padded = torch.full((rows, h, hd + 24), 3.0, device=DEV).to(DT[dt])
    layer.attention(q, k, v, padded[..., 8:8 + hd])              # an output inside a wider tensor
    assert torch.equal(padded[..., 8:8 + hd], o)
    assert bool((padded[..., :8] == 3.0).all()) and bool((padded[..., 8 + hd:] == 3.0).all())


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_inactive_sequences_are_not_written(S, dt):
    lens = [70, 300, 1, 0, 140]
    off = L.offsets(lens)
    q, k, v = make(2, dt, off[-1], off[-1], 2, 2, 64)
    active = torch.tensor([1, 0, 1, 1, 0], dtype=torch.uint8, device=DEV)
    layer = S.SpecaLayer(off, code(S, dt), n_heads=2, n_kv_heads=2, head_dim=64, causal=True, device=DEV)
    o = torch.full_like(q, 9.0)
    lse = torch.full((2, off[-1]), 9.0, device=DEV)
    layer.attention(q, k, v, o, lse=lse, active=active)
    want, bound, wl, bl = L.attention(off, off, q, k, v, True, 0.125)
    for s, on in enumerate([1, 0, 1, 1, 0]):
        r = slice(off[s], off[s + 1])
        if on:
            L.check(o[r], want[r], bound[r])
            L.check(lse[:, r], wl[:, r], bl[:, r])
        else:
            assert bool((o[r] == 9.0).all()) and bool((lse[:, r] == 9.0).all())
    # few rows against long keys, shared out over units: the inactive ones stay out there too
    few = S.SpecaLayer([0, 1, 2, 3], code(S, dt), kv_start=[0, 900, 1800, 2700], n_heads=2, n_kv_heads=2, head_dim=64, device=DEV)
    q, k, v = make(3, dt, 3, 2700, 2, 2, 64)
    o = torch.full_like(q, 9.0)
    for _ in range(2):
        few.attention(q, k, v, o, active=active[:3])
    want, bound, _, _ = L.attention([0, 1, 2, 3], [0, 900, 1800, 2700], q, k, v, False, 0.125)
    L.check(o[[0, 2]], want[[0, 2]], bound[[0, 2]])
    assert bool((o[1] == 9.0).all())


def test_nan_query_stays_in_its_row_and_infinite_keys_in_hidden_places(S):
    for dt in ("bf16", "f32"):
        off = [0, 200]
        q, k, v = make(6, dt, 200, 200, 2, 1, 64)
        q[17, 1, 3] = float("nan")
        k[150, 0, 5] = float("nan")   # seen by the rows from 150 on
        layer = S.SpecaLayer(off, code(S, dt), n_heads=2, n_kv_heads=1, head_dim=64, causal=True, device=DEV)
        o = torch.zeros_like(q)
        layer.attention(q, k, v, o)
        bad = o.isnan().all(-1)
        want = torch.zeros(200, 2, dtype=torch.bool, device=DEV)
        want[17, 1] = True
        want[150:] = True
        assert torch.equal(bad, want) and torch.equal(o.isnan().any(-1), want)


def test_kv_len_is_read_on_the_device(S):
    layer = S.SpecaLayer([0, 1], S.SPECA_BF16, kv_start=[0, 4000], n_heads=8, n_kv_heads=2, head_dim=128, causal=True, device=DEV)
    q, k, v = make(7, "bf16", 1, 4000, 8, 2, 128)
    o = torch.zeros_like(q)
    n = torch.tensor([100], dtype=torch.int32, device=DEV)
    layer.attention(q, k, v, o, kv_len=n)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.attention(q, k, v, o, kv_len=n)
    for fill in (1, 129, 2048, 4000):
        n.fill_(fill)
        graph.replay()
        want, bound, _, _ = L.attention([0, 1], [0, 4000], q, k, v, True, 128 ** -0.5, [fill])
        L.check(o, want, bound, "fill %d" % fill)


def test_offsets_beyond_32_bits(S):
    # the last sequence of a cache of 2.2e9 elements; only its own rows are written
    hd, kv, rows = 128, 4, 4_300_000
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("not enough memory")
    k = torch.empty(rows, kv, hd, dtype=torch.bfloat16, device=DEV)
    v = torch.empty(rows, kv, hd, dtype=torch.bfloat16, device=DEV)
    n = 1000
    q, kt, vt = make(12, "bf16", 2, n, kv, kv, hd)
    k[-n:], v[-n:] = kt, vt
    assert (rows - n) * kv * hd > 1 << 31
    layer = S.SpecaLayer([0, 0, 2], S.SPECA_BF16, kv_start=[0, rows - n, rows], n_heads=kv, n_kv_heads=kv, head_dim=hd, device=DEV)
    o = torch.zeros_like(q)
    layer.attention(q, k, v, o)
    want, bound, _, _ = L.attention([0, 2], [0, n], q, kt, vt, False, hd ** -0.5)
    L.check(o, want, bound)


def test_shards_join_by_lse(S):
    # keys split over two layers (a sequence-parallel cache) and joined by their lse
    q, k, v = make(13, "bf16", 64, 500, 4, 4, 64)
    whole = run(S, "bf16", [64], [500], 4, 4, 64, False, qkv=(q, k, v))
    outs, ls = [], []
    for a, b in ((0, 200), (200, 500)):
        layer = S.SpecaLayer([0, 64], S.SPECA_BF16, kv_start=[0, b - a], n_heads=4, n_kv_heads=4, head_dim=64, device=DEV)
        o, lse = torch.zeros_like(q), torch.zeros(4, 64, device=DEV)
        layer.attention(q, k[a:b], v[a:b], o, lse=lse)
        outs.append(o.double())
        ls.append(lse.double())
    w = torch.softmax(torch.stack(ls), 0).transpose(1, 2)[..., None]
    torch.testing.assert_close((w[0] * outs[0] + w[1] * outs[1]), whole.double(), rtol=2.0 ** -6, atol=2.0 ** -6)


def test_refusals(S):
    layer = S.SpecaLayer([0, 8], S.SPECA_BF16, n_heads=4, n_kv_heads=2, head_dim=64, device=DEV)
    q, k, v = make(0, "bf16", 8, 8, 4, 2, 64)
    o = torch.zeros_like(q)
    none = S.SpecaLayer([0, 8], S.SPECA_BF16, device=DEV)
    with pytest.raises(S.SpecaError) as e:
        S.speca_layer_attention(none.handle, (q.data_ptr(), 256, 64), (k.data_ptr(), 128, 64), (v.data_ptr(), 128, 64),
                                (o.data_ptr(), 256, 64), None, None, None)
    assert e.value.status == S.SPECA_ERR_STATE
    odd = torch.zeros(8, 2, 68, device=DEV).bfloat16()
    with pytest.raises(S.SpecaError) as e:     # rows that the copy engine cannot address
        layer.attention(q, odd[..., :64], v, o)
    assert e.value.status == S.SPECA_ERR_ALIGNMENT and "16 bytes" in str(e.value)
    with pytest.raises(S.SpecaError) as e:
        layer.attention(q, k, v, o.as_strided(o.shape, (256, 32, 1)))
    assert e.value.status == S.SPECA_ERR_SHAPE
    eighths = S.SpecaLayer([0, 8], S.SPECA_BF16, n_heads=1, n_kv_heads=1, head_dim=36, device=DEV)
    wide = torch.zeros(8, 1, 40, device=DEV).bfloat16()
    with pytest.raises(S.SpecaError) as e:     # bf16 heads come in multiples of 8 elements
        eighths.attention(*[wide[..., :36]] * 4)
    assert e.value.status == S.SPECA_ERR_SHAPE
    with pytest.raises(ValueError):
        layer.attention(q, k[:7], v, o)
    with pytest.raises(TypeError):
        layer.attention(q, k.float(), v, o)
    with pytest.raises(TypeError):
        layer.attention(q, k, v, o, kv_len=torch.tensor([8], device=DEV))
    with pytest.raises(ValueError):
        layer.attention(q, k, v, o, active=torch.ones(2, dtype=torch.uint8, device=DEV))
    with pytest.raises(S.SpecaError) as e:
        S.speca_layer_attention(layer.handle, (None, 256, 64), (k.data_ptr(), 128, 64), (v.data_ptr(), 128, 64),
                                (o.data_ptr(), 256, 64), None, None, None)
    assert e.value.status == S.SPECA_ERR_INVALID_ARG
    layer.check()


def test_workspace_guards(S):
    kw = dict(n_heads=2, n_kv_heads=2, head_dim=64)
    need = S.speca_layer_workspace_bytes([0, 4], S.SPECA_BF16, **kw)
    ws = torch.empty(need + 256, dtype=torch.uint8, device=DEV)
    for bad, status in ((dict(workspace=ws, workspace_bytes=need - 1), S.SPECA_ERR_NOMEM),
                        (dict(workspace=ws[8:]), S.SPECA_ERR_ALIGNMENT), (dict(workspace=None), S.SPECA_ERR_INVALID_ARG),
                        (dict(workspace=ws, device=99), S.SPECA_ERR_INVALID_ARG)):
        with pytest.raises(S.SpecaError) as e:
            S.speca_layer_create([0, 4], S.SPECA_BF16, **bad, **kw)
        assert e.value.status == status
    assert math.isfinite(need)
