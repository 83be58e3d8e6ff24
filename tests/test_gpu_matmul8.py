"""speca_layer_matmul8 against its definition in 64 bits. Three kernels share the sizes out by a model of their times: few rows (transposed tiles,
shares of k over a cluster), tiles of one SM (128 x 128), tiles of a pair (256 x 256); the sizes below go to all of them."""
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


def whole(g, rows, k, lo=-1, hi=1):
    """Small whole numbers times powers of two: every order of their sums is exact in fp32."""
    codes = torch.randint(-4, 5, (rows, k), generator=g, device=DEV)
    return E.put(codes, torch.randint(127 + lo, 127 + hi + 1, (rows, -(-k // 128)), generator=g, device=DEV).to(torch.uint8))


def real(g, rows, k, size=1.0):
    x = size * torch.randn(rows, k, generator=g, device=DEV)
    x[:, k // 2] *= 20
    codes, byte = E.eight(x.double())
    return E.put(codes, byte.to(torch.uint8))


def raw(m):
    return m.codes.view(torch.uint8), m.scales.view(torch.uint8)


def blank(S, rows, n, fill=0x55):
    m = S.Matrix8.empty(rows, n, DEV)
    for t in raw(m):
        t.fill_(fill)
    return m


# rows, features, k
FEW = [(1, 1, 1), (1, 33, 16), (3, 77, 130), (8, 256, 512), (16, 128, 1152), (17, 1000, 1155), (32, 513, 4608), (64, 640, 2000), (5, 4000, 700),
       (100, 300, 8200), (4, 300, 16384)]
ONE = [(65, 129, 128), (128, 128, 64), (257, 513, 1000), (300, 1000, 1155), (1000, 77, 31), (640, 640, 640), (1100, 1500, 520), (1100, 1501, 1000), (1150, 1733, 31),
       (1025, 1280, 640)]
PAIR = [(2100, 4100, 300), (4099, 2048, 1152), (1025, 14336, 520), (2500, 4000, 17)]


@pytest.mark.parametrize("m,n,k", FEW + ONE + PAIR)
def test_whole_numbers_are_exact(S, m, n, k):
    g = gen(m + n + k)
    a, w = whole(g, m, k), whole(g, n, k)
    want = E.values(a) @ E.values(w).T
    layer = S.SpecaLayer([0, m], S.SPECA_F32, device=DEV)
    out = torch.full((m, n), float("nan"), device=DEV)
    layer.matmul8(a, w, out)
    layer.check()
    assert torch.equal(out.double(), want)
    m8 = blank(S, m, n)
    layer.matmul8(a, w, m8)
    layer.check()
    codes, byte = E.eight(want)
    assert torch.equal(m8.codes.double(), codes) and torch.equal(E.bytes_of(m8).long(), byte)
    half = S.SpecaLayer([0, m], S.SPECA_BF16, device=DEV)
    out16 = torch.zeros(m, n, dtype=torch.bfloat16, device=DEV)
    half.matmul8(a, w, out16)
    half.check()
    assert torch.equal(out16, want.float().bfloat16())


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["none", "gelu", "silu"])
@pytest.mark.parametrize("m,n,k", [(7, 300, 1155), (400, 333, 520), (1100, 1501, 520), (1100, 1504, 520), (2100, 4096, 384)])
def test_epilogues(S, dt, kind, m, n, k):
    g = gen(m)
    lens = [m // 3, 0, m - m // 3 - 2, 2]
    off = L.offsets(lens)
    seq = torch.repeat_interleave(torch.arange(4, device=DEV), torch.tensor(lens, device=DEV))
    a, w = real(g, m, k), real(g, n, k, 2 * k ** -0.5)
    bias = torch.randn(n, generator=g, device=DEV).to(DT[dt])
    res = torch.randn(m, n, generator=g, device=DEV).to(DT[dt])
    gate = torch.randn(4, n, generator=g, device=DEV).to(DT[dt])
    layer = S.SpecaLayer(off, code(S, dt), device=DEV)
    acts = {"none": S.SPECA_ACT_NONE, "gelu": S.SPECA_ACT_GELU, "silu": S.SPECA_ACT_SILU}
    t, bt = E.product(a, w, bias, kind)
    plain, pb = E.product(a, w, None, kind)
    out = torch.zeros(m, n, dtype=DT[dt], device=DEV)

    def call(**kw):
        out.fill_(9.0)
        layer.matmul8(a, w, out, activation=acts[kind], **kw)
        layer.check()

    call()
    L.check(out, plain, pb, "plain")
    call(bias=bias)
    L.check(out, t, bt, "bias")
    G, R = gate.double()[seq], res.double()
    call(bias=bias, residual=res)
    L.check(out, t + R, bt + L.U32 * (t.abs() + R.abs()), "residual")
    call(residual=res, gate=gate)
    L.check(out, plain * G + R, pb * G.abs() + 3 * L.U32 * ((plain * G).abs() + R.abs()), "residual, gate")
    call(bias=bias, gate=gate)
    L.check(out, t * G, bt * G.abs() + 2 * L.U32 * (t * G).abs(), "gate")
    m8 = blank(S, m, n)
    layer.matmul8(a, w, m8, bias=bias, activation=acts[kind])
    layer.check()
    E.check8(m8, t, bt, "8 bits")


# the third goes to tiles of one SM without a mask and to a pair's with one
@pytest.mark.parametrize("m,n,k", [(12, 200, 300), (500, 300, 256), (4096, 1152, 4608), (4608, 2304, 256), (100, 300, 8200), (1100, 1501, 520),
                                   (1100, 1504, 520)])
def test_masked_samples_are_left_alone_and_others_do_not_see_it(S, m, n, k):
    g = gen(1)
    lens = [m // 4, 0, 1, m // 2, m - m // 4 - 1 - m // 2]
    off = L.offsets(lens)
    a, w = real(g, m, k), real(g, n, k, k ** -0.5)
    bias = torch.randn(n, generator=g, device=DEV).bfloat16()
    res, gate = torch.randn(m, n, generator=g, device=DEV).bfloat16(), torch.randn(5, n, generator=g, device=DEV).bfloat16()
    layer = S.SpecaLayer(off, S.SPECA_BF16, device=DEV)
    full, full8, fullr = torch.zeros(m, n, dtype=torch.bfloat16, device=DEV), blank(S, m, n), torch.zeros(m, n, dtype=torch.bfloat16, device=DEV)
    layer.matmul8(a, w, full, bias=bias)
    layer.matmul8(a, w, full8, bias=bias)
    layer.matmul8(a, w, fullr, residual=res, gate=gate)
    for live in ([1, 1, 0, 1, 0], [0, 0, 1, 0, 0], [0, 1, 0, 0, 1], [0, 0, 0, 0, 0], [1, 1, 1, 1, 1]):
        mask = torch.tensor(live, dtype=torch.uint8, device=DEV)
        # what inactive rows hold is not even a number
        b = E.put(a.codes.view(torch.uint8).clone(), E.bytes_of(a).clone())
        for s in range(5):
            if not live[s]:
                b.codes.view(torch.uint8)[off[s]:off[s + 1]] = 0x7f
                b.scales.view(torch.uint8)[:, off[s]:off[s + 1]] = 255
        part, part8, partr = torch.full_like(full, 7.0), blank(S, m, n), torch.full_like(full, 7.0)
        layer.matmul8(b, w, part, bias=bias, active=mask)
        layer.matmul8(b, w, part8, bias=bias, active=mask)
        layer.matmul8(b, w, partr, residual=res, gate=gate, active=mask)
        layer.check()
        for s in range(5):
            rows = slice(off[s], off[s + 1])
            if live[s]:
                assert torch.equal(part[rows], full[rows]) and torch.equal(partr[rows], fullr[rows])
                assert torch.equal(raw(part8)[0][rows], raw(full8)[0][rows]) and torch.equal(raw(part8)[1][:, rows], raw(full8)[1][:, rows])
            else:
                assert bool((part[rows] == 7.0).all() and (partr[rows] == 7.0).all())
                assert bool((raw(part8)[0][rows] == 0x55).all() and (raw(part8)[1][:, rows] == 0x55).all())


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", [(9, 130, 200), (300, 264, 200), (1100, 1501, 200), (1100, 1504, 200), (2304, 4099, 130)])
def test_strides_offsets_and_in_place(S, dt, m, n, k):
    g = gen(4)
    a, w = real(g, m, k), real(g, 2 * n + 3, k, k ** -0.5)
    # the weights are rows of a larger matrix, from no multiple of 4 on
    part = S.Matrix8(w.codes[3:3 + n], w.scales[:, 3:3 + n])
    t, bt = E.product(a, part)
    layer = S.SpecaLayer([0, m], code(S, dt), device=DEV)
    wide = torch.full((m, n + 11), 5.0, dtype=DT[dt], device=DEV)
    out = wide[:, 3:3 + n]                                   # no 16-byte boundary
    layer.matmul8(a, part, out)
    layer.check()
    L.check(out, t, bt)
    assert bool((wide[:, :3] == 5.0).all() and (wide[:, 3 + n:] == 5.0).all())
    even = torch.full((m, n // 8 * 8 + 24), 5.0, dtype=DT[dt], device=DEV)   # 16-byte rows that the copy engine takes, ending inside a box
    out2 = even[:, 8:8 + n]
    layer.matmul8(a, part, out2)
    assert torch.equal(out2, out) and bool((even[:, :8] == 5.0).all() and (even[:, 8 + n:] == 5.0).all())
    # the residual's own place; a residual of one row for all
    res = torch.randn(m, n, generator=g, device=DEV).to(DT[dt])
    want = torch.zeros_like(res)
    layer.matmul8(a, part, want, residual=res)
    wide.fill_(5.0)
    out.copy_(res)
    layer.matmul8(a, part, out, residual=out)
    assert torch.equal(out, want) and bool((wide[:, :3] == 5.0).all())
    layer.matmul8(a, part, res, residual=res)
    assert torch.equal(res, want)
    one = torch.randn(1, n, generator=g, device=DEV).to(DT[dt])
    layer.matmul8(a, part, out2, residual=one.expand(m, n))
    L.check(out2, t + one.double(), bt + L.U32 * (t.abs() + one.double().abs()))
    # 8 bits into a part of a larger matrix
    buf = torch.full((m, n + 40), 0x44, dtype=torch.uint8, device=DEV)
    sc = torch.full((-(-n // 512), m + 9, 4), 0x44, dtype=torch.uint8, device=DEV)
    m8 = S.Matrix8(buf[:, 5:5 + n].view(torch.float8_e4m3fn), sc[:, 5:5 + m].view(torch.float8_e8m0fnu))
    layer.matmul8(a, part, m8)
    layer.check()
    E.check8(m8, t, bt)
    assert bool((buf[:, :5] == 0x44).all() and (buf[:, 5 + n:] == 0x44).all() and (sc[:, :5] == 0x44).all() and (sc[:, 5 + m:] == 0x44).all())


@pytest.mark.parametrize("m,n,k", [(6, 140, 300), (300, 264, 300), (1100, 1504, 300), (2304, 4100, 300)])
def test_nan_stays_in_its_row_and_column(S, m, n, k):
    g = gen(6)
    a, w = whole(g, m, k), whole(g, n, k)
    want = E.values(a) @ E.values(w).T
    a.codes.view(torch.uint8)[2, 5] = 0x7f
    a.scales.view(torch.uint8)[0, 4, 1] = 255
    w.codes.view(torch.uint8)[7, k - 1] = 0xff
    w.scales.view(torch.uint8)[0, 130, 2] = 255
    layer = S.SpecaLayer([0, m], S.SPECA_F32, device=DEV)
    out, m8 = torch.zeros(m, n, device=DEV), blank(S, m, n)
    layer.matmul8(a, w, out)
    layer.matmul8(a, w, m8)
    layer.check()
    nan = torch.zeros(m, n, dtype=torch.bool, device=DEV)
    nan[[2, 4]] = True
    nan[:, [7, 130]] = True
    assert torch.equal(out.isnan(), nan) and torch.equal(out.double()[~nan], want[~nan])
    assert torch.equal(m8.codes.double().isnan(), nan)
    codes, byte = E.eight(torch.where(nan, torch.full_like(want, float("nan")), want))
    assert torch.equal(m8.codes.double()[~nan], codes[~nan]) and torch.equal(E.bytes_of(m8).long(), byte)


@pytest.mark.parametrize("m,n", [(5, 140), (300, 264), (1100, 1504), (2304, 4100)])
@pytest.mark.parametrize("ea,ew", [(27, 227), (227, 27), (77, 177), (67, 67), (187, 180)])
def test_scales_far_from_one(S, m, n, ea, ew):
    # products of scales from 2^-120 to 2^113, of factors up to 2^100
    g = gen(9)
    k = 384
    a = E.put(torch.randint(-4, 5, (m, k), generator=g, device=DEV), torch.full((m, 3), ea, dtype=torch.uint8, device=DEV))
    w = E.put(torch.randint(-4, 5, (n, k), generator=g, device=DEV), torch.full((n, 3), ew, dtype=torch.uint8, device=DEV))
    layer = S.SpecaLayer([0, m], S.SPECA_F32, device=DEV)
    out = torch.zeros(m, n, device=DEV)
    layer.matmul8(a, w, out)
    layer.check()
    assert torch.equal(out.double(), E.values(a) @ E.values(w).T)


@pytest.mark.parametrize("m,n,k", [(8, 512, 16384), (300, 512, 8192), (2304, 2048, 4096), (2304, 2048, 8200), (2304, 2048, 16384)])
def test_fp32_sums_over_long_k(S, m, n, k):
    # a share of s elements is off by (1.04 s + 73) roundings of its magnitudes at most (eight_util.product has the count for s = k), and shares are at
    # most 4096 elements from k = 8193 on
    g = gen(k)
    a, w = real(g, m, k), real(g, n, k, k ** -0.5)
    layer = S.SpecaLayer([0, m], S.SPECA_F32, device=DEV)
    out = torch.zeros(m, n, device=DEV)
    layer.matmul8(a, w, out)
    layer.check()
    t, bt = E.product(a, w)
    share = (1.04 * (4096 if k > 8192 else k) + 73) / (1.04 * k + 73)
    L.check(out, t, share * bt)
    # a bias, an activation, a gate and a residual go with it, and a mask
    bias, res = torch.randn(n, generator=g, device=DEV), torch.randn(m, n, generator=g, device=DEV)
    gate = torch.randn(1, n, generator=g, device=DEV)
    t, bt = E.product(a, w, bias, "silu")
    want, bound = res.double() + gate.double() * t, gate.double().abs() * (bt + 2 * E.U32 * t.abs())
    layer.matmul8(a, w, res, bias=bias, activation=S.SPECA_ACT_SILU, residual=res, gate=gate, active=torch.ones(1, dtype=torch.uint8, device=DEV))
    layer.check()
    L.check(res, want, bound)


def test_the_same_bits_every_time(S):
    g = gen(12)
    for m, n, k in ((4, 512, 8192), (300, 1000, 1152), (2304, 4096, 1152)):
        a, w = real(g, m, k), real(g, n, k, k ** -0.5)
        layer = S.SpecaLayer([0, m], S.SPECA_F32, device=DEV)
        out, again = torch.zeros(m, n, device=DEV), torch.zeros(m, n, device=DEV)
        layer.matmul8(a, w, out, activation=S.SPECA_ACT_GELU)
        for _ in range(5):
            again.zero_()
            layer.matmul8(a, w, again, activation=S.SPECA_ACT_GELU)
            assert torch.equal(out, again)


@pytest.mark.parametrize("m,n,k", [(600000, 72, 100), (600000, 256, 100)])
def test_more_tiles_of_rows_than_one_launch_lists(S, m, n, k):
    g = gen(13)
    a, w = whole(g, m, k), whole(g, n, k)
    lens = [200000, 100001, 299999]
    layer = S.SpecaLayer(L.offsets(lens), S.SPECA_F32, device=DEV)
    want = (a.codes.float() * torch.exp2(E.bytes_of(a).float() - 127)) @ (w.codes.float() * torch.exp2(E.bytes_of(w).float() - 127)).T   # exact
    out = torch.full((m, n), -1.0, device=DEV)
    layer.matmul8(a, w, out)
    layer.check()
    assert torch.equal(out, want)
    out.fill_(0.5)
    layer.matmul8(a, w, out, active=torch.tensor([1, 0, 1], dtype=torch.uint8, device=DEV))
    layer.check()
    assert torch.equal(out[:200000], want[:200000]) and torch.equal(out[300001:], want[300001:]) and bool((out[200000:300001] == 0.5).all())


@pytest.mark.parametrize("m", [4, 300])
def test_weights_behind_32_bits(S, m):
    # 280 000 features of 16384: 4.6 GB of codes; the last features repeat the first
    n, k = 280000, 16384
    g = gen(14)
    codes = torch.randint(0, 0x38, (n, k), generator=g, device=DEV, dtype=torch.uint8)
    codes[-300:] = codes[:300]
    scales = torch.full((k // 512, n, 4), 121, dtype=torch.uint8, device=DEV)
    w = S.Matrix8(codes.view(torch.float8_e4m3fn), scales.view(torch.float8_e8m0fnu))
    a = whole(g, m, k)
    layer = S.SpecaLayer([0, m], S.SPECA_F32, device=DEV)
    out = torch.zeros(m, n, device=DEV)
    layer.matmul8(a, w, out)
    layer.check()
    t, bt = E.product(a, S.Matrix8(w.codes[:300], w.scales[:, :300]))
    L.check(out[:, :300].contiguous(), t, bt)
    L.check(out[:, -300:].contiguous(), t, bt)


def test_output_behind_32_bits(S):
    m, n, k = 36000, 62000, 64     # 2.2e9 elements
    g = gen(15)
    a, w = whole(g, m, k), whole(g, n, k)
    layer = S.SpecaLayer([0, m], S.SPECA_BF16, device=DEV)
    out = torch.zeros(m, n, dtype=torch.bfloat16, device=DEV)
    layer.matmul8(a, w, out)
    layer.check()
    av, wv = E.values(a), E.values(w)
    for rows in (slice(0, 300), slice(m - 300, m)):
        assert torch.equal(out[rows], (av[rows] @ wv.T).float().bfloat16())


def test_two_handles_on_two_streams_and_replayed_graphs(S):
    g = gen(16)
    sizes = [(4, 2048, 2048), (500, 1024, 1152), (2304, 4096, 512)]
    work = []
    for m, n, k in sizes:
        a, w = real(g, m, k), real(g, n, k, k ** -0.5)
        layer = S.SpecaLayer([0, m], S.SPECA_BF16, device=DEV)
        want = torch.zeros(m, n, dtype=torch.bfloat16, device=DEV)
        layer.matmul8(a, w, want)
        work.append((layer, a, w, want, torch.zeros_like(want), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(5):
        for layer, a, w, _, out, stream in work:
            with torch.cuda.stream(stream):
                out.zero_()
                layer.matmul8(a, w, out)
    torch.cuda.synchronize()
    for layer, _, _, want, out, stream in work:
        layer.check(stream.cuda_stream)
        assert torch.equal(out, want)
    graphs = []
    for layer, a, w, _, out, _ in work:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            layer.matmul8(a, w, out)
        graphs.append(graph)
    for layer, a, w, want, out, _ in work:
        # new operands in the same places
        a.codes.view(torch.uint8).copy_(a.codes.view(torch.uint8).flip(0))
        a.scales.view(torch.uint8).copy_(a.scales.view(torch.uint8).flip(1))
        out.zero_()
    for graph in graphs:
        graph.replay()
    torch.cuda.synchronize()
    for layer, _, _, want, out, _ in work:
        layer.check()
        assert torch.equal(out, want.flip(0))


@pytest.mark.parametrize("dt", list(DT))
@pytest.mark.parametrize("m,n", [(1, 1), (5, 200), (300, 700), (2400, 2100)])
def test_the_longest_k(S, dt, m, n):
    # ones: below 2^24 their sums are exact
    k = S.SPECA_MAX_K8
    a, w = S.Matrix8.empty(m, k, DEV), S.Matrix8.empty(n, k, DEV)
    for x in (a, w):
        raw(x)[0].fill_(0x38)
        raw(x)[1].fill_(127)
    out = torch.zeros(m, n, dtype=DT[dt], device=DEV)
    layer = S.SpecaLayer([0, m], code(S, dt), device=DEV)
    layer.matmul8(a, w, out)
    layer.check()
    assert bool((out == k).all())


def test_one_handle_on_two_streams_and_in_a_graph_with_branches(S):
    # kernels may start before the one in front has ended; they wait for it, whichever stream or branch it is on
    g = gen(17)
    m, k, n = 700, 1152, 640
    layer = S.SpecaLayer(L.offsets([300, 0, 400]), S.SPECA_BF16, device=DEV)
    x = torch.randn(m, k, generator=g, device=DEV).bfloat16()
    w = real(g, n, k, k ** -0.5)
    a, b = (S.Matrix8.empty(m, k, DEV) for _ in range(2))
    one, two, three = (torch.zeros(m, n, dtype=torch.bfloat16, device=DEV) for _ in range(3))
    side = torch.cuda.Stream()

    def run():
        main = torch.cuda.current_stream()
        x.mul_(1)
        side.wait_stream(main)
        layer.norm8(x, a)
        layer.matmul8(a, w, one)
        with torch.cuda.stream(side):
            layer.quantize8(x, b)
            layer.matmul8(b, w, two, activation=S.SPECA_ACT_SILU)
        main.wait_stream(side)
        layer.matmul8(a, w, three, residual=two)
        x.copy_(x.flip(0))
        layer.quantize8(x, a)

    def alone():
        y, c = x.clone(), S.Matrix8.empty(m, k, DEV)
        outs = [torch.zeros_like(one) for _ in range(3)]
        for step in (lambda: layer.norm8(y, c), lambda: layer.matmul8(c, w, outs[0]), lambda: layer.quantize8(y, c),
                     lambda: layer.matmul8(c, w, outs[1], activation=S.SPECA_ACT_SILU), lambda: layer.norm8(y, c),
                     lambda: layer.matmul8(c, w, outs[2], residual=outs[1]), lambda: layer.quantize8(y.flip(0).contiguous(), c)):
            step()
            torch.cuda.synchronize()
        return outs, c

    def check(outs, c):
        torch.cuda.synchronize()
        layer.check()
        for got, want in zip((one, two, three), outs):
            assert torch.equal(got, want)
        assert all(torch.equal(p, q) for p, q in zip(raw(a), raw(c)))

    want = alone()
    run()
    check(*want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for seed in (1, 2, 3):
        x.copy_(torch.randn(m, k, generator=gen(seed), device=DEV))
        want = alone()
        graph.replay()
        check(*want)


def test_no_rows(S):
    layer = S.SpecaLayer([0, 0, 0], S.SPECA_BF16, device=DEV)
    layer.matmul8(S.Matrix8.empty(0, 64, DEV), S.Matrix8.empty(32, 64, DEV), torch.zeros(0, 32, dtype=torch.bfloat16, device=DEV))
    layer.check()
