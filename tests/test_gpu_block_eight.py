"""The 8-bit calls together: a transformer block against its definition in 64 bits, and a stack of blocks as the sampler's model."""
import pytest
import torch

from tests import eight_util as E

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def M():
    from paper_2509_11628_b200 import binding, block
    binding._lib()
    return block


def plain(block, x, cond, pos, axes):
    """The block in 64 bits, with the 8-bit roundings where the block has them."""
    b, n, h, hd, dim = block.batch, block.tokens, block.heads, block.head_dim, block.dim
    mod = (torch.nn.functional.silu(cond.double()) @ block.w_mod.double()).view(b, 1, 6, dim)
    sa, ca, ga, sm, cm, gm = (mod[:, :, i] for i in range(6))
    norm = lambda t: torch.nn.functional.layer_norm(t, (dim,), eps=1e-6)
    rms = lambda t, w: t / torch.sqrt((t * t).mean(-1, keepdim=True) + 1e-6) * w.double()
    product = lambda t, w: (E.rounded(t.reshape(b * n, -1)) @ E.values(w).T).view(b, n, -1)
    x = x.double().view(b, n, dim)
    q, k, v = product(norm(x) * (1 + ca) + sa, block.w_qkv).view(b, n, 3, h, hd).unbind(2)
    angle = torch.cat([pos.double().view(b, n, -1)[..., a:a + 1] * torch.tensor([10000.0 ** (-2.0 * i / e) for i in range(e // 2)], device=DEV,
                                                                                dtype=torch.float64) for a, e in enumerate(axes)], -1)
    turn = torch.polar(torch.ones_like(angle), angle)[:, :, None]
    rope = lambda t: torch.view_as_real(torch.view_as_complex(t.reshape(b, n, h, hd // 2, 2)) * turn).flatten(-2)
    q, k = rope(rms(q, block.q_norm)), rope(rms(k, block.k_norm))
    p = torch.softmax(torch.einsum("bnhd,bmhd->bhnm", q, k) * hd ** -0.5, -1)
    x = x + ga * product(torch.einsum("bhnm,bmhd->bnhd", p, v), block.w_out)
    up = torch.nn.functional.gelu(product(norm(x) * (1 + cm) + sm, block.w_up), approximate="tanh")
    return (x + gm * product(up, block.w_down)).view(b * n, dim)


@pytest.mark.parametrize("dtype,rel", [("bf16", 3e-2), ("f32", 5e-3)])
@pytest.mark.parametrize("heads,hd,axes,grid", [(6, 64, (16, 24, 24), (1, 8, 8)), (4, 72, (24, 24, 24), (2, 5, 7)), (2, 128, (16, 56, 56), (3, 6, 9))])
def test_block_against_its_definition(M, dtype, rel, heads, hd, axes, grid):
    # rel: bf16 as the block without 8 bits (1.5e-2: a dozen roundings to the type), and codes that round the other way: a value that is 2^-9 off
    # crosses one of the codes' borders (2^-4 apart at most, relative) once in 16 to 32 and is then a step of 2^-3 to 2^-4 off, so a rounding that
    # precedes adds sqrt(1/16) * 2^-4 = 1.6e-2 at most, of independent sign. fp32: values off by some 2^-18 cross once in 2^12, 1/64 * 2^-4 < 1e-3 of each of
    # the four roundings
    code = M.S.SPECA_BF16 if dtype == "bf16" else M.S.SPECA_F32
    pos = M.grid_positions(9, *grid, DEV)
    block = M.TransformerBlock(2, pos.shape[0], heads, hd, axes, code, DEV, seed=3, eight=True)
    g = torch.Generator(device=DEV).manual_seed(1)
    tdt = M.S._TORCH_DTYPES[code]
    x = torch.randn(2 * pos.shape[0], heads * hd, generator=g, device=DEV).to(tdt)
    cond = torch.randn(2, heads * hd, generator=g, device=DEV).to(tdt)
    pos = pos.repeat(2, 1).contiguous()
    out = torch.zeros_like(x)
    block(x, cond, pos, out)
    block.layer.check()
    want = plain(block, x, cond, pos, axes)
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
    stack = M.BlockStack(4, 2, pos.shape[0], 4, 64, (16, 24, 24), pos, device=DEV, eight=True)
    cache = M.S.SpecaCache(stack.entries, 2, 1, M.S.SPECA_BF16, DEV)
    stack.backend = SpecaCacheBackend(cache)
    times = [1.0 - 0.01 * i for i in range(16)]
    trace = run_sampler(stack.backend, stack, times, tau0=0.5, beta=1.0, period=3, warm_refs=2, gamma=0.25)
    assert [row for row in trace.steps[:2]] == [[FULL] * 2] * 2
    assert any(ACCEPTED in row for row in trace.steps)
    errs = [e for row in trace.err for e in row if e == e]
    assert errs and all(0 < e < 0.5 for e in errs)
    for block in stack.blocks:
        block.layer.check()
    cache.close()
