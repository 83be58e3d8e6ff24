"""The layer calls together: a transformer block against plain torch, and a stack of blocks as the sampler's model."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def M():
    from paper_2509_11628_b200 import binding, block
    binding._lib()
    return block


def plain(block, x, cond, pos):
    """The block in 64 bits, on the same (rounded) weights."""
    d = lambda t: t.double()
    b, n, h, hd, dim = block.batch, block.tokens, block.heads, block.head_dim, block.dim
    mod = (torch.nn.functional.silu(d(cond)) @ d(block.w_mod)).view(b, 1, 6, dim)
    sa, ca, ga, sm, cm, gm = (mod[:, :, i] for i in range(6))
    norm = lambda t: torch.nn.functional.layer_norm(t, (dim,), eps=1e-6)
    rms = lambda t, w: t / torch.sqrt((t * t).mean(-1, keepdim=True) + 1e-6) * d(w)
    x = d(x).view(b, n, dim)
    q, k, v = ((norm(x) * (1 + ca) + sa) @ d(block.w_qkv)).view(b, n, 3, h, hd).unbind(2)
    angle = torch.cat([d(pos).view(b, n, -1)[..., a:a + 1] * torch.tensor([10000.0 ** (-2.0 * i / e) for i in range(e // 2)], device=DEV,
                                                                          dtype=torch.float64) for a, e in enumerate(block.axes)], -1)
    turn = torch.polar(torch.ones_like(angle), angle)[:, :, None]
    rope = lambda t: torch.view_as_real(torch.view_as_complex(t.reshape(b, n, h, hd // 2, 2)) * turn).flatten(-2)
    q, k = rope(rms(q, block.q_norm)), rope(rms(k, block.k_norm))
    p = torch.softmax(torch.einsum("bnhd,bmhd->bhnm", q, k) * hd ** -0.5, -1)
    x = x + ga * (torch.einsum("bhnm,bmhd->bnhd", p, v).reshape(b, n, dim) @ d(block.w_out))
    up = torch.nn.functional.gelu((norm(x) * (1 + cm) + sm) @ d(block.w_up), approximate="tanh")
    return (x + gm * (up @ d(block.w_down))).view(b * n, dim)


@pytest.mark.parametrize("dtype,rel", [("bf16", 1.5e-2), ("f32", 2e-5)])
@pytest.mark.parametrize("heads,hd,axes,grid", [(6, 64, (16, 24, 24), (1, 8, 8)), (4, 72, (24, 24, 24), (2, 5, 7)), (2, 128, (16, 56, 56), (3, 6, 9))])
def test_block_against_plain_torch(M, dtype, rel, heads, hd, axes, grid):
    # rel: a dozen roundings to the storage type on the way, each at most 2^-8 (2^-24) of what passes through, averaged over
    # a row; fp32 adds the products' own sums over up to 4 dim terms
    code = M.S.SPECA_BF16 if dtype == "bf16" else M.S.SPECA_F32
    pos = M.grid_positions(9, *grid, DEV)
    block = M.TransformerBlock(2, pos.shape[0], heads, hd, axes, code, DEV, seed=3)
    block.axes = axes
    g = torch.Generator(device=DEV).manual_seed(1)
    tdt = M.S._TORCH_DTYPES[code]
    x = torch.randn(2 * pos.shape[0], heads * hd, generator=g, device=DEV).to(tdt)
    cond = torch.randn(2, heads * hd, generator=g, device=DEV).to(tdt)
    pos = pos.repeat(2, 1).contiguous()
    out = torch.zeros_like(x)
    block(x, cond, pos, out)
    block.layer.check()
    want = plain(block, x, cond, pos)
    err = (out.double() - want).norm(dim=1) / want.norm(dim=1)
    assert float(err.max()) < rel
    # one sample alone: the same bits for it, nothing written for the other
    part = torch.full_like(x, 7.0)
    block(x, cond, pos, part, active=torch.tensor([0, 1], dtype=torch.uint8, device=DEV))
    n = x.shape[0] // 2
    assert torch.equal(part[n:], out[n:]) and bool((part[:n] == 7.0).all())


def test_stack_as_the_samplers_model(M):
    from paper_2509_11628_b200.scheduler import ACCEPTED, FULL, SpecaCacheBackend, run_sampler
    pos = M.grid_positions(4, 1, 6, 6, DEV)
    stack = M.BlockStack(4, 2, pos.shape[0], 4, 64, (16, 24, 24), pos, device=DEV)
    cache = M.S.SpecaCache(stack.entries, 2, 1, M.S.SPECA_BF16, DEV)
    stack.backend = SpecaCacheBackend(cache)
    times = [1.0 - 0.01 * i for i in range(16)]
    trace = run_sampler(stack.backend, stack, times, tau0=0.5, beta=1.0, period=3, warm_refs=2, gamma=0.25)
    assert [row for row in trace.steps[:2]] == [[FULL] * 2] * 2
    assert any(ACCEPTED in row for row in trace.steps)
    errs = [e for row in trace.err for e in row if e == e]
    assert errs and all(0 < e < 0.5 for e in errs)      # smooth in time: small, but the block is really computed
    # a threshold nothing passes: every sample recomputes every step
    trace = run_sampler(stack.backend, stack, times, tau0=1e-6, beta=1.0, period=3, warm_refs=2, gamma=0.25)
    assert not any(ACCEPTED in row for row in trace.steps)
    for block in stack.blocks:
        block.layer.check()
    cache.close()
