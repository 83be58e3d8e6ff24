"""speca_layer_norm8, speca_layer_quantize8 and speca_quantize8 against their definitions in 64 bits."""
import pytest
import torch

from tests import eight_util as E
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


def fresh(S, rows, dim, fill=0x55):
    m = S.Matrix8.empty(rows, dim, DEV)
    m.codes.view(torch.uint8).fill_(fill)
    m.scales.view(torch.uint8).fill_(fill)
    return m


def same(m, x):
    """m is x in 8 bits, to the bit."""
    want, byte = E.eight(x.double())
    assert torch.equal(E.bytes_of(m).long(), byte)
    got = m.codes.double()
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan) and torch.equal(got[~nan], want[~nan])


# ---- rows as they are ------------------------------------------------------------------------------

@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [1, 2, 7, 16, 127, 128, 129, 511, 512, 513, 1152, 1155, 2048, 4104, 8192, 16384, 16385, 33000])
def test_quantize_dims(S, dt, dim):
    g = gen(dim)
    x = normal(g, 5, dim) * torch.exp2(torch.randint(-20, 20, (5, 1), generator=g, device=DEV).float())
    x[:, dim // 2] *= 50
    x[1] = 0
    x = x.to(DT[dt])
    m = fresh(S, 5, dim)
    assert S.quantize8(x, m) is m
    same(m, x)
    # bytes behind the last block are left as they were
    blocks = -(-dim // 128)
    rest = m.scales.view(torch.uint8).transpose(0, 1).reshape(5, -1)[:, blocks:]
    assert bool((rest == 0x55).all())
    layer = S.SpecaLayer([0, 2, 2, 5], code(S, dt), device=DEV)
    n = fresh(S, 5, dim)
    layer.quantize8(x, n)
    assert torch.equal(n.codes.view(torch.uint8), m.codes.view(torch.uint8)) and torch.equal(n.scales.view(torch.uint8), m.scales.view(torch.uint8))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_quantize_range_borders_and_what_is_not_finite(S, dt):
    x = torch.zeros(24, 256, device=DEV)
    tiny = torch.finfo(DT[dt]).tiny
    # largest magnitudes on and next to the border between two scales, over the whole range of exponents
    for i, e in enumerate((-126, -125, -100, -1, 0, 1, 60, 119)):
        x[i, 0] = 1.75 * 2.0 ** e
        x[i, 1] = 2.0 ** e * 1e-3
        x[8 + i, 0] = (1.75 + 2.0 ** -7) * 2.0 ** e
    x[16, 3], x[16, 200] = tiny / 4, -tiny              # below the smallest scale's reach: subnormal codes, or zero
    x[17] = torch.linspace(-448, 448, 256, device=DEV)  # every binade of the codes, ties among them
    x[18, :128] = torch.arange(128, device=DEV) * 2.0 ** -10   # around the codes' subnormals when the block's scale is 1
    x[18, 0] = 448
    x[19, 5], x[19, 6] = float("inf"), 3.0
    x[20, 5], x[20, 130] = float("-inf"), float("inf")
    x[21, 7], x[21, 8] = float("nan"), -1.0
    x[22] = float("inf")
    x[23] = torch.finfo(DT[dt]).max
    x = x.to(DT[dt])
    m = fresh(S, 24, 256)
    S.quantize8(x, m)
    same(m, x)
    assert int(E.bytes_of(m)[22, 0]) == 127 and bool(m.codes[22].double().isnan().all())


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_quantize_strides_offsets_mask_and_no_rows(S, dt):
    g = gen(2)
    lens = [3, 0, 4, 5]
    off = L.offsets(lens)
    wide = normal(g, 12, 400).to(DT[dt])
    x = wide[:, 3:3 + 257]                                   # rows that start on no 16-byte boundary
    buf = torch.full((12, 300), 0x33, dtype=torch.uint8, device=DEV)
    scales = torch.full((3, 40, 4), 0x33, dtype=torch.uint8, device=DEV)
    m = S.Matrix8(buf[:, 5:262].view(torch.float8_e4m3fn), scales[:1, 7:19].view(torch.float8_e8m0fnu))
    layer = S.SpecaLayer(off, code(S, dt), device=DEV)
    layer.quantize8(x, m, active=torch.tensor([1, 1, 0, 1], dtype=torch.uint8, device=DEV))
    want = S.quantize8(x.contiguous())
    for a, b in ((0, 3), (7, 12)):
        assert torch.equal(buf[a:b, 5:262], want.codes.view(torch.uint8)[a:b])
        assert torch.equal(scales[0, 7 + a:7 + b, :3], want.scales.view(torch.uint8)[0, a:b, :3])
    assert bool((buf[3:7] == 0x33).all() and (buf[:, :5] == 0x33).all() and (buf[:, 262:] == 0x33).all())
    assert bool((scales[0, 10:14] == 0x33).all() and (scales[0, :7] == 0x33).all() and (scales[0, 19:] == 0x33).all() and (scales[1:] == 0x33).all())
    empty = S.SpecaLayer([0, 0], code(S, dt), device=DEV)
    empty.quantize8(torch.empty(0, 64, dtype=DT[dt], device=DEV), S.Matrix8.empty(0, 64, DEV))
    assert S.quantize8(torch.empty(0, 64, dtype=DT[dt], device=DEV)).shape == (0, 64)


# ---- norms -----------------------------------------------------------------------------------------

@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("dim", [1, 2, 7, 64, 255, 384, 513, 1152, 2049, 4096, 5121, 16384, 33000])
def test_norm_dims(S, dt, kind, dim):
    g = gen(dim)
    lens = [3, 0, 1, 9]
    off = L.offsets(lens)
    x, br = normal(g, off[-1], dim).to(DT[dt]), normal(g, off[-1], dim).to(DT[dt])
    x[:, dim // 2] *= 50
    mod = (0.3 * normal(g, len(lens), 3, dim)).to(DT[dt])
    w = (1 + 0.2 * normal(g, dim)).to(DT[dt])
    layer = S.SpecaLayer(off, code(S, dt), norm_eps=1e-6, device=DEV)
    m, xo = fresh(S, off[-1], dim), torch.zeros_like(x)
    layer.norm8(x, m, S.SPECA_NORM_RMS if kind == "rms" else S.SPECA_NORM_LAYER, branch=br, gate=mod[:, 0], scale=mod[:, 1], shift=mod[:, 2], weight=w,
                x_out=xo)
    y, z, by, bz = E.norm(off, x, br, mod[:, 0], mod[:, 1], mod[:, 2], w, kind == "layer", 1e-6)
    L.check(xo, z, bz, "x'")
    E.check8(m, y, by, "y")


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("have", ["", "s", "t", "w", "b", "bg", "bgstw", "bsw", "stw"])
def test_norm_optional_parts(S, dt, have):
    g = gen(11)
    off = L.offsets([5, 2])
    x, br = normal(g, 7, 384).to(DT[dt]), normal(g, 7, 384).to(DT[dt])
    mod = (0.3 * normal(g, 2, 3, 384)).to(DT[dt])
    w = (1 + 0.2 * normal(g, 384)).to(DT[dt]) if "w" in have else None
    layer = S.SpecaLayer(off, code(S, dt), device=DEV)
    b = br if "b" in have else None
    ga, sc, sh = (mod[:, i] if c in have else None for i, c in enumerate("gst"))
    for centre in (False, True):
        m = fresh(S, 7, 384)
        layer.norm8(x, m, S.SPECA_NORM_LAYER if centre else S.SPECA_NORM_RMS, branch=b, gate=ga, scale=sc, shift=sh, weight=w)
        y, _, by, _ = E.norm(off, x, b, ga, sc, sh, w, centre, 1e-6)
        E.check8(m, y, by, "centre" if centre else "rms")
    if b is None:   # x' alone, without a branch, is a copy
        xo = torch.zeros_like(x)
        layer.norm8(x, m, x_out=xo)
        assert torch.equal(xo, x)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [384, 1155, 16400])
def test_norm_strides_offsets_and_in_place(S, dt, dim):
    g = gen(3)
    off = L.offsets([4, 6])
    wide = normal(g, 10, dim + 5).to(DT[dt])
    x = wide[:, 3:3 + dim]
    br = normal(g, 10, 2 * dim).to(DT[dt])[:, dim:]
    mod = (0.3 * normal(g, 2, 6 * dim)).to(DT[dt])
    ga, sc, sh = mod[:, :dim], mod[:, dim:2 * dim], mod[:, 5 * dim:]
    layer = S.SpecaLayer(off, code(S, dt), device=DEV)
    y, z, by, bz = E.norm(off, x, br, ga, sc, sh, None, True, 1e-6)
    keep = wide.clone()
    m = fresh(S, 10, dim)
    layer.norm8(x, m, S.SPECA_NORM_LAYER, branch=br, gate=ga, scale=sc, shift=sh, x_out=x)   # x' over x
    E.check8(m, y, by)
    L.check(x, z, bz)
    assert torch.equal(wide[:, :3], keep[:, :3]) and torch.equal(wide[:, 3 + dim:], keep[:, 3 + dim:])
    x2, b2 = keep[:, 3:3 + dim].contiguous(), br.contiguous()
    layer.norm8(x2, m, S.SPECA_NORM_LAYER, branch=b2, gate=ga, scale=sc, shift=sh, x_out=b2)  # x' over the branch
    E.check8(m, y, by)
    L.check(b2, z, bz)


def test_norm_leaves_inactive_rows_alone_and_nan_in_its_row(S):
    g = gen(5)
    lens = [3, 1, 0, 40, 2]
    off = L.offsets(lens)
    x = normal(g, off[-1], 256).bfloat16()
    x[1, 7] = float("nan")
    x[2, 7] = float("inf")
    x[off[3]:off[4]] = float("inf")
    layer = S.SpecaLayer(off, S.SPECA_BF16, device=DEV)
    m, xo = fresh(S, off[-1], 256, 0x11), torch.full_like(x, 7.0)
    layer.norm8(x, m, x_out=xo, active=torch.tensor([1, 0, 1, 0, 1], dtype=torch.uint8, device=DEV))
    y, _, by, _ = E.norm(off, x, None, None, None, None, None, False, 1e-6)
    live = [0, off[4], off[4] + 1]
    E.check8(m, y, by, live=live)
    # a row with a NaN, or whose sum of squares is infinite next to an infinity, is NaN in every such element
    assert bool(m.codes[1].double().isnan().all()) and bool(m.codes[2, 7].double().isnan()) and int(E.bytes_of(m)[1, 0]) == 127
    for s in (1, 3):
        rows = slice(off[s], off[s + 1])
        assert bool((m.codes.view(torch.uint8)[rows] == 0x11).all() and (m.scales.view(torch.uint8)[:, rows] == 0x11).all() and (xo[rows] == 7.0).all())


def test_norm_of_zeros_and_of_constants(S):
    layer = S.SpecaLayer([0, 2], S.SPECA_F32, device=DEV)
    m = fresh(S, 2, 640)
    layer.norm8(torch.zeros(2, 640, device=DEV), m)
    assert bool((m.codes.double() == 0).all()) and bool((E.bytes_of(m) == 127).all())
    layer.norm8(torch.full((2, 640), 3.0, device=DEV), m, S.SPECA_NORM_LAYER)
    assert bool((m.codes.double() == 0).all())
    layer.norm8(torch.full((2, 640), 3.0, device=DEV), m)
    assert bool((E.values(m) == 1.0).all())


def test_replayed_graph_follows_new_inputs_and_mask(S):
    g = gen(8)
    off = L.offsets([40, 30])
    x = normal(g, 70, 1152).bfloat16()
    mask = torch.ones(2, dtype=torch.uint8, device=DEV)
    layer = S.SpecaLayer(off, S.SPECA_BF16, device=DEV)
    m = fresh(S, 70, 1152)
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        layer.norm8(x, m, active=mask)
    for seed, live in ((1, [1, 0]), (2, [1, 1])):
        x.copy_(normal(gen(seed), 70, 1152).bfloat16())
        mask.copy_(torch.tensor(live, dtype=torch.uint8))
        m.codes.view(torch.uint8).fill_(0x21)
        graph.replay()
        torch.cuda.synchronize()
        want = fresh(S, 70, 1152, 0x21)
        want.scales.view(torch.uint8).copy_(m.scales.view(torch.uint8))
        layer.norm8(x, want, active=mask)
        assert torch.equal(m.codes.view(torch.uint8), want.codes.view(torch.uint8)) and torch.equal(m.scales.view(torch.uint8), want.scales.view(torch.uint8))


def test_rows_behind_32_bits(S):
    # 300 000 rows of 16384 codes: 4.9 GB; the last rows of x repeat the first
    rows, dim = 300000, 16384
    x = torch.zeros(rows, dim, dtype=torch.bfloat16, device=DEV)
    x[:4] = normal(gen(1), 4, dim).bfloat16()
    x[-4:] = x[:4]
    m = S.quantize8(x)
    first = S.quantize8(x[:4].contiguous())
    for part in (slice(0, 4), slice(rows - 4, rows)):
        assert torch.equal(m.codes.view(torch.uint8)[part], first.codes.view(torch.uint8))
        assert torch.equal(m.scales.view(torch.uint8)[:, part], first.scales.view(torch.uint8))
    assert int(m.codes.view(torch.uint8)[rows // 2].max()) == 0 and int(E.bytes_of(m)[rows // 2, 0]) == 127


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_the_longest_row(S, kind):
    # ones with a two at either end. RMS norm: of mean square 1 + 6 / dim, that is 1 off by 3e-6 with eps: codes of 1 and 2 (a step of e4m3 there is 2^-3
    # of the value or 2^-4). Layer norm: mean 1 + 2 / dim (rounded to 1: 2^-24 of it, 6e-8, is more), so zeros, and of the two 1 / sqrt(2 / dim + eps)
    dim = S.SPECA_MAX_ROWS
    x = torch.ones(1, dim, dtype=torch.bfloat16, device=DEV)
    x[0, 0], x[0, -1] = 2, 2
    layer = S.SpecaLayer([0, 1], S.SPECA_BF16, device=DEV)
    m = S.Matrix8.empty(1, dim, DEV)
    layer.norm8(x, m, S.SPECA_NORM_RMS if kind == "rms" else S.SPECA_NORM_LAYER)
    layer.check()
    got, byte = m.codes.view(torch.uint8)[0], m.scales.view(torch.uint8).view(-1)
    # e4m3: 256 is 0x78, 128 is 0x70
    inner, want = (0x78, 119) if kind == "rms" else (0x00, 127)
    assert bool((byte[1:-1] == want).all())
    assert bool((got[128:-128] == inner).all())
    top = 2.0 if kind == "rms" else 1 / (2 / dim + 1e-6) ** 0.5
    for edge, at in ((slice(0, 128), 0), (slice(dim - 128, dim), -1)):
        values = got[edge].view(torch.float8_e4m3fn).float() * 2.0 ** (int(byte[at]) - 127)
        want = torch.full((128,), 1.0 if kind == "rms" else 0.0, device=DEV)
        want[at] = top
        assert bool(((values - want).abs() <= want * (0 if kind == "rms" else 2.0 ** -4)).all())
