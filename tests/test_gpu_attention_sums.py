"""speca_layer_attention in bf16: the sums of the softmax, to much less than a rounding to bf16."""
import math

import pytest
import torch

from tests.test_gpu_attention import DEV

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -24
POLY = 7.6e-5  # relative error of an exponential formed by the polynomial (7.5e-5) with its roundings
FAR = -60.0    # log2 of a weight that no sum notices


@pytest.fixture(scope="module")
def S():
    from paper_2509_11628_b200 import binding
    binding._lib()
    return binding


def scores(g, at, n, rows, heads, one_v=None, seed=0):
    """q, k, v whose scores (in log2 units, scale = ln 2) are 0 for key 0, g[row] for the keys in `at`, FAR for the rest. g is
    carried by three bf16 terms, so that its values fall everywhere between bf16's own. Returns g as the terms add up."""
    q = torch.zeros(rows, heads, 64, device=DEV)
    left, got = g.double().clone(), torch.zeros_like(g, dtype=torch.float64)
    for i in range(3):
        part = left.to(torch.bfloat16)
        q[:, :, i] = part.float()[:, None]
        left, got = left - part.double(), got + part.double()
    q[:, :, 3] = 1.0
    k = torch.zeros(n, heads, 64, device=DEV)
    k[:, :, 3] = FAR
    k[0, :, 3] = 0.0
    k[at] = 0.0
    k[at, :, :3] = 1.0
    gen = torch.Generator(device=DEV).manual_seed(seed)
    if one_v:   # the same value behind every key
        v = torch.randn(1, heads, 64, generator=gen, device=DEV).expand(n, heads, 64)
    else:
        v = torch.randn(n, heads, 64, generator=gen, device=DEV)
    return q.bfloat16(), k.bfloat16(), v.bfloat16().contiguous(), got


def attend(S, q, k, v, kv_len=None):
    heads = q.shape[1]
    layer = S.SpecaLayer([0, q.shape[0]], S.SPECA_BF16, kv_start=[0, k.shape[0]], n_heads=heads, n_kv_heads=heads, head_dim=64,
                         scale=math.log(2.0), device=DEV)
    o, lse = torch.zeros_like(q), torch.zeros(heads, q.shape[0], device=DEV)
    layer.attention(q, k, v, o, lse=lse, kv_len=kv_len)
    layer.check()
    return o, lse.double()


# one key in a later tile outweighs the first tile's maximum by less than 2^8, so the reference stays behind and its
# weight is no power of two; keys 6 and 7 of eight are the polynomial's. 2048 rows: one tile range; 3 rows: shared out.
CASES = [(256 + 1, 700, 2048), (256 + 6, 700, 2048), (128 + 7, 700, 2048), (640 + 6, 20000, 3), (9000 + 7, 20000, 3), (9000 + 4, 20000, 3)]


@pytest.mark.parametrize("at,n,rows", CASES)
def test_lse_is_that_of_the_exact_weights(S, at, n, rows):
    g = torch.linspace(0.3, 7.9, rows, device=DEV)
    q, k, v, g = scores(g, [at], n, rows, 2)
    _, lse = attend(S, q, k, v)
    want = torch.log1p(torch.exp2(g)).expand(2, -1)
    # an exponential by polynomial; x = score * scale_log2 - reference * scale_log2 with three roundings of at most 8, and
    # scale_log2 itself rounded; sums of two weights; the logarithm
    bound = POLY + math.log(2) * 4 * 8 * U32 + 8 * U32 * (1 + want.abs())
    assert float(((lse - want).abs() - bound).max()) <= 0, float((lse - want).abs().max())


@pytest.mark.parametrize("at,n,rows", CASES)
def test_the_rounding_of_a_dominating_weight_divides_out(S, at, n, rows):
    # one value behind all keys: o is it, times the weights' sum as multiplied over the sum as divided by. They may differ by
    # the polynomial's error and the first key's, both far below half a unit of bf16 (2^-9), so the bits are v's.
    for seed in range(8 if rows < 100 else 1):
        g = torch.rand(rows, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV) * 7.6 + 0.3
        q, k, v, _ = scores(g, [at], n, rows, 2, one_v=True, seed=seed)
        o, _ = attend(S, q, k, v)
        want = v[:1].expand_as(o)
        off = (o != want).any(-1)
        assert not bool(off.any()), "%d of %d rows" % (int(off.sum()), off.numel())


def test_exponentials_of_every_key_of_eight(S):
    # the weights of the tile's keys of one residue mod 8 against key 0: an exponential off by more than the polynomial's
    # error shows in the sum, for arguments from 2^-8 to just below 2^8
    for r in range(8):
        at = [128 * t + 8 * i + r for t in range(1, 4) for i in range(16)]
        q, k, v, g = scores(torch.linspace(-8.0, 7.9, 1024, device=DEV), at, 512, 1024, 1)
        _, lse = attend(S, q, k, v)
        want = torch.log1p(len(at) * torch.exp2(g))[None]
        bound = POLY + math.log(2) * 4 * 8 * U32 + (len(at) + 8) * U32 * (1 + want.abs())
        assert float(((lse - want).abs() - bound).max()) <= 0, (r, float((lse - want).abs().max()))
