"""speca_layer_modulate and speca_layer_rope against their definitions in 64 bits."""
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


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


# ---- adaptive layer norm ---------------------------------------------------------------------------

@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [1, 2, 7, 64, 255, 384, 511, 513, 1152, 1537, 2049, 3072, 4097, 8192, 16384, 33000])
def test_modulate_dims(S, dt, dim):
    g = gen(dim)
    lens = [3, 0, 1, 9]
    off = L.offsets(lens)
    x, br = normal(g, off[-1], dim).to(DT[dt]), normal(g, off[-1], dim).to(DT[dt])
    x[:, dim // 2] *= 50
    mod = (0.3 * normal(g, len(lens), 3, dim)).to(DT[dt])
    layer = S.SpecaLayer(off, code(S, dt), norm_eps=1e-6, device=DEV)
    y, xo = torch.zeros_like(x), torch.zeros_like(x)
    layer.modulate(x, y, branch=br, gate=mod[:, 0], scale=mod[:, 1], shift=mod[:, 2], x_out=xo)
    wy, wx, by, bx = L.modulate(off, x, br, mod[:, 0], mod[:, 1], mod[:, 2], 1e-6)
    L.check(xo, wx, bx, "x'")
    L.check(y, wy, by, "y")


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("have", ["", "s", "t", "b", "bg", "bgst", "bst", "st"])
def test_modulate_optional_parts(S, dt, have):
    g = gen(11)
    off = L.offsets([5, 2])
    x, br = normal(g, 7, 384).to(DT[dt]), normal(g, 7, 384).to(DT[dt])
    mod = (0.3 * normal(g, 2, 3, 384)).to(DT[dt])
    layer = S.SpecaLayer(off, code(S, dt), device=DEV)
    y = torch.zeros_like(x)
    b = br if "b" in have else None
    ga, sc, sh = (mod[:, i] if c in have else None for i, c in enumerate("gst"))
    layer.modulate(x, y, branch=b, gate=ga, scale=sc, shift=sh)
    wy, _, by, _ = L.modulate(off, x, b, ga, sc, sh, 1e-6)
    L.check(y, wy, by)
    # x' alone, without a branch, is a copy
    if b is None:
        xo = torch.zeros_like(x)
        layer.modulate(x, y, x_out=xo)
        assert torch.equal(xo, x)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [384, 1155])
def test_modulate_strides_offsets_and_in_place(S, dt, dim):
    g = gen(3)
    off = L.offsets([4, 6])
    wide = normal(g, 10, dim + 5).to(DT[dt])
    x = wide[:, 3:3 + dim]                       # rows that start on no 16-byte boundary
    br = normal(g, 10, 2 * dim).to(DT[dt])[:, dim:]
    mod = (0.3 * normal(g, 2, 6 * dim)).to(DT[dt])
    ga, sc, sh = mod[:, :dim], mod[:, dim:2 * dim], mod[:, 5 * dim:]
    layer = S.SpecaLayer(off, code(S, dt), device=DEV)
    y = torch.zeros(10, dim + 1, dtype=DT[dt], device=DEV)[:, :dim]
    wy, wx, by, bx = L.modulate(off, x, br, ga, sc, sh, 1e-6)
    keep = wide.clone()
    layer.modulate(x, y, branch=br, gate=ga, scale=sc, shift=sh, x_out=x)   # x' over x
    L.check(y, wy, by)
    L.check(x, wx, bx)
    assert torch.equal(wide[:, :3], keep[:, :3]) and torch.equal(wide[:, 3 + dim:], keep[:, 3 + dim:])
    x2 = keep[:, 3:3 + dim].contiguous()
    b2 = br.contiguous()
    layer.modulate(x2, b2, branch=b2, gate=ga, scale=sc, shift=sh, x_out=x2)  # y over the branch, x' over x
    L.check(b2, wy, by)
    L.check(x2, wx, bx)


def test_modulate_leaves_inactive_rows_alone_and_nan_in_its_row(S):
    g = gen(5)
    lens = [3, 1, 0, 40, 2]
    off = L.offsets(lens)
    x = normal(g, off[-1], 256).bfloat16()
    x[1, 7] = float("nan")
    x[off[3]:off[4]] = float("inf")
    active = torch.tensor([1, 0, 1, 0, 1], dtype=torch.uint8, device=DEV)
    layer = S.SpecaLayer(off, S.SPECA_BF16, device=DEV)
    y = torch.full_like(x, 7.0)
    layer.modulate(x, y, active=active)
    wy, _, by, _ = L.modulate(off, x, None, None, None, None, 1e-6)
    for r in [0, 2] + list(range(off[4], off[5])):
        L.check(y[r], wy[r], by[r], "row %d" % r)
    assert bool(y[1].isnan().all())
    for s in (1, 3):
        assert bool((y[off[s]:off[s + 1]] == 7.0).all())


def test_modulate_constant_rows_give_the_shift(S):
    off = L.offsets([2])
    x = torch.full((2, 1152), 3.0, device=DEV)
    sh = torch.randn(1, 1152, device=DEV)
    layer = S.SpecaLayer(off, S.SPECA_F32, device=DEV)
    y = torch.zeros_like(x)
    layer.modulate(x, y, shift=sh)
    assert torch.equal(y, sh.expand(2, -1))


# ---- rotary positions ------------------------------------------------------------------------------

CASES = [  # heads, kv heads, head_dim, axes
    (24, 24, 128, (16, 56, 56)), (32, 8, 128, (128,)), (6, 6, 64, (16, 24, 24)), (16, 16, 72, (24, 24, 24)),
    (3, 1, 72, (36, 36)), (2, 2, 34, (10, 6)), (1, 1, 2, (2,)), (5, 5, 30, (30,)), (1, 1, 128, (32,)), (40, 2, 96, (48,)),
    (70, 7, 8, (4,)), (4, 4, 126, (42, 40, 20, 24)),
]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("case", CASES)
def test_rope(S, dt, halves, norm, case):
    h, kv, hd, axes = case
    g = gen(h * 1000 + hd)
    off = L.offsets([1, 0, 13, 5])
    qkv = normal(g, off[-1], h + 2 * kv, hd).to(DT[dt])
    q, k = qkv[:, :h], qkv[:, h:h + kv]
    pos = torch.randint(0, 5000, (off[-1], len(axes)), generator=g, device=DEV).float()
    pos[2] = 0.0
    pos[3] = 0.37
    wq = (1 + 0.3 * normal(g, hd)).to(DT[dt]) if norm else None
    wk = (1 + 0.3 * normal(g, hd)).to(DT[dt]) if norm else None
    layer = S.SpecaLayer(off, code(S, dt), n_heads=h, n_kv_heads=kv, head_dim=hd, axis_dims=axes, theta=10000.0,
                         pairing=S.SPECA_ROPE_HALVES if halves else S.SPECA_ROPE_INTERLEAVED, device=DEV)
    qo, ko = torch.zeros(off[-1], h, hd, dtype=DT[dt], device=DEV), torch.zeros(off[-1], kv, hd, dtype=DT[dt], device=DEV)
    layer.rope(q, qo, k, ko, pos, q_weight=wq, k_weight=wk)
    for x, w, out in ((q, wq, qo), (k, wk, ko)):
        want, bound = L.rope(x, w, pos, axes, 10000.0, halves, 1e-6)
        L.check(out, want, bound)
    before = qkv.clone()
    layer.rope(q, q, k, k, pos, q_weight=wq, k_weight=wk)   # in place: the same bits, the values untouched
    assert torch.equal(q, qo) and torch.equal(k, ko) and torch.equal(qkv[:, h + kv:], before[:, h + kv:])


def test_rope_layouts_masks_and_queries_alone(S):
    g = gen(9)
    off = L.offsets([4, 3, 8])
    q = normal(g, 4, 15, 64).bfloat16().transpose(0, 1)          # [heads, rows, hd] in memory
    k = normal(g, 15, 4, 65).bfloat16()[..., 1:]                 # starts on no 16-byte boundary
    pos = torch.arange(15, device=DEV).float()[:, None].contiguous()
    layer = S.SpecaLayer(off, S.SPECA_BF16, n_heads=4, n_kv_heads=4, head_dim=64, axis_dims=(64,), device=DEV)
    active = torch.tensor([1, 0, 1], dtype=torch.uint8, device=DEV)
    qo = torch.full((4, 15, 64), 9.0, device=DEV).bfloat16().transpose(0, 1)
    ko = torch.full((15, 4, 64), 9.0, device=DEV).bfloat16()
    layer.rope(q, qo, k, ko, pos, active=active)
    for x, out in ((q, qo), (k, ko)):
        want, bound = L.rope(x, None, pos, (64,), 10000.0, False, 1e-6)
        L.check(out[:4], want[:4], bound[:4])
        L.check(out[7:], want[7:], bound[7:])
        assert bool((out[4:7] == 9.0).all())
    only = torch.zeros_like(qo)
    layer.rope(q, only, None, None, pos)
    assert torch.equal(only[:4], qo[:4])


def test_rope_keeps_length_and_far_positions_and_nonfinite_neighbours(S):
    off = L.offsets([3])
    layer = S.SpecaLayer(off, S.SPECA_F32, n_heads=1, n_kv_heads=1, head_dim=16, axis_dims=(4, 4), device=DEV)
    q = torch.randn(3, 1, 16, device=DEV)
    q[0, 0, 9] = float("inf")    # kept element: stays, alone
    q[1, 0, 0] = float("nan")    # rotated pair 0
    pos = torch.tensor([[16777215.0, -3.0], [1.0, 2.0], [1e6, 0.5]], device=DEV)
    out = torch.zeros_like(q)
    layer.rope(q, out, None, None, pos)
    want, bound = L.rope(q, None, pos, (4, 4), 10000.0, False, 1e-6)
    assert torch.equal(out[0, 0, 8:], q[0, 0, 8:])
    assert bool(out[1, 0, :2].isnan().all()) and bool(out[1, 0, 2:].isfinite().all())
    for r in (0, 2):
        L.check(out[r, :, :8], want[r, :, :8], bound[r, :, :8])


# ---- refusals --------------------------------------------------------------------------------------

def test_refusals(S):
    layer = S.SpecaLayer([0, 4], S.SPECA_BF16, n_heads=2, n_kv_heads=1, head_dim=64, device=DEV)   # no axes
    x = torch.zeros(4, 128, device=DEV).bfloat16()
    y = torch.zeros_like(x)
    q, k = torch.zeros(4, 2, 64, device=DEV).bfloat16(), torch.zeros(4, 1, 64, device=DEV).bfloat16()
    pos = torch.zeros(4, 0, device=DEV)
    with pytest.raises(S.SpecaError) as e:
        layer.rope(q, q, k, k, pos)
    assert e.value.status == S.SPECA_ERR_STATE
    with pytest.raises(S.SpecaError) as e:
        layer.modulate(x, y, gate=x[:1])
    assert e.value.status == S.SPECA_ERR_INVALID_ARG and "gate" in str(e.value)
    with pytest.raises(TypeError):
        layer.modulate(x.float(), y)
    with pytest.raises(ValueError):
        layer.modulate(x[:3], y)
    with pytest.raises(TypeError):
        layer.modulate(x.cpu(), y)
    with pytest.raises(TypeError):
        layer.modulate(x.t().contiguous().t(), y)
    with pytest.raises(S.SpecaError) as e:   # rows of the output overlap
        layer.modulate(x, y.as_strided((4, 128), (64, 1)))
    assert e.value.status == S.SPECA_ERR_SHAPE
    with pytest.raises(S.SpecaError) as e:
        S.speca_layer_modulate(layer.handle, 128, None, 128, None, 0, None, None, None, 0, None, None, 0, y.data_ptr(), 128)
    assert e.value.status == S.SPECA_ERR_INVALID_ARG
    with pytest.raises(S.SpecaError) as e:
        S.speca_layer_modulate(layer.handle, 128, x.data_ptr() + 1, 128, None, 0, None, None, None, 0, None, None, 0, y.data_ptr(), 128)
    assert e.value.status == S.SPECA_ERR_ALIGNMENT
    turning = S.SpecaLayer([0, 4], S.SPECA_BF16, n_heads=2, n_kv_heads=1, head_dim=64, axis_dims=(32, 32), device=DEV)
    pos = torch.zeros(4, 2, device=DEV)
    with pytest.raises(S.SpecaError) as e:
        turning.rope(q, q, k, None, pos)
    assert e.value.status == S.SPECA_ERR_INVALID_ARG
    with pytest.raises(ValueError):
        turning.rope(q, q, k, k, torch.zeros(4, 3, device=DEV))
    turning.check()
    torch.cuda.synchronize()


def test_other_stream_and_graph(S):
    g = gen(21)
    off = L.offsets([64, 64])
    x = normal(g, 128, 384)
    layer = S.SpecaLayer(off, S.SPECA_F32, device=DEV)
    y, z = torch.zeros_like(x), torch.zeros_like(x)
    layer.modulate(x, y)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.modulate(x, z)
    side.synchronize()
    assert torch.equal(y, z)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.modulate(x, z)
    x.copy_(normal(g, 128, 384))
    graph.replay()
    layer.modulate(x, y)
    torch.cuda.synchronize()
    assert torch.equal(y, z)
