"""Definitions in 64 bits of the 8-bit operators, and checks of what they give. Plain torch, no code of the library."""
import torch

from tests import layer_util as L

U32 = L.U32


def put(codes, scales, pad=16):
    """A Matrix8 of codes (values of e4m3, or its bytes as uint8) [rows, dim] and scale bytes [rows, blocks]."""
    from paper_2509_11628_b200 import binding as S
    rows, dim = codes.shape
    raw = codes if codes.dtype is torch.uint8 else codes.float().to(torch.float8_e4m3fn).view(torch.uint8)
    wide = torch.full((rows, -(-dim // pad) * pad), 0x7f, dtype=torch.uint8, device=codes.device)   # NaN behind the end
    wide[:, :dim] = raw
    groups = -(-dim // 512)
    full = torch.full((rows, 4 * groups), 255, dtype=torch.uint8, device=codes.device)
    full[:, :scales.shape[1]] = scales
    return S.Matrix8(wide[:, :dim].view(torch.float8_e4m3fn), full.view(rows, groups, 4).transpose(0, 1).contiguous().view(torch.float8_e8m0fnu))


def bytes_of(m):
    """Scale bytes [rows, blocks] of a Matrix8."""
    rows, dim = m.codes.shape
    return m.scales.view(torch.uint8).transpose(0, 1).reshape(rows, -1)[:, :-(-dim // 128)]


def values(m):
    """What a Matrix8 stands for, in 64 bits."""
    scale = torch.exp2(bytes_of(m).double() - 127.0)
    return m.codes.double() * scale.repeat_interleave(128, 1)[:, :m.codes.shape[1]]


def blocks(y):
    """[rows, blocks, 128], zeros behind the end."""
    rows, dim = y.shape
    return torch.nn.functional.pad(y, (0, -dim % 128)).view(rows, -1, 128)


def byte_of(top):
    """The scale byte of blocks with these largest magnitudes: the smallest e with top <= 448 2^(e - 127), 1 <= e <= 254, by trying."""
    e = torch.full(top.shape, 254, dtype=torch.int64, device=top.device)
    for b in range(253, 0, -1):
        e = torch.where(top <= 448.0 * 2.0 ** (b - 127), torch.full_like(e, b), e)
    return torch.where(top == 0, torch.full_like(e, 127), e)


def half_step(y, scale):
    """Half of e4m3's step at y / scale, in y's units: 2^-4 of the binade, of 2^-6 below it."""
    q = (y.abs() / scale).clamp_min(2.0 ** -6)
    return torch.exp2(torch.floor(torch.log2(q)) - 4) * scale


def eight(y):
    """(codes as values, scale bytes) of y in 64 bits, from the definition."""
    rows, dim = y.shape
    b = blocks(torch.where(torch.isfinite(y), y, torch.zeros_like(y)))
    e = byte_of(b.abs().amax(2))
    scale = torch.exp2(e.double() - 127.0)[..., None]
    step = 2 * half_step(b, scale)
    q = (torch.round(b / step) * step / scale).reshape(rows, -1)[:, :dim]
    return torch.where(torch.isfinite(y), q, torch.full_like(y, float("nan"))), e


def rounded(y):
    """y in 64 bits through the 8-bit format."""
    codes, e = eight(y)
    return codes * torch.exp2(e.double() - 127.0).repeat_interleave(128, 1)[:, :y.shape[1]]


def check8(m, y, bound, what="", live=None):
    """Every block's scale is that of a largest magnitude within `bound` of the 64-bit one, every value within the bound and half a step."""
    rows = slice(None) if live is None else live
    got, byte, y, bound = values(m)[rows], bytes_of(m)[rows].long(), y[rows], bound[rows]
    lo = byte_of(blocks((y.abs() - bound).clamp_min(0)).amax(2))
    hi = byte_of(blocks(y.abs() + bound).amax(2))
    zero = blocks(y.abs() + bound).amax(2) == 0
    assert bool(((byte >= torch.where(lo == 127, byte.clamp_max(127), lo)) & (byte <= torch.maximum(hi, torch.where(zero, 127, 1)))).all()), what + ": scale"
    scale = torch.exp2(byte.double() - 127.0).repeat_interleave(128, 1)[:, :y.shape[1]]
    allow = bound + half_step(y.abs() + bound, scale)
    bad = ~((got - y).abs() <= allow)
    if bool(bad.any()):
        i = tuple(bad.nonzero()[0].tolist())
        raise AssertionError("%s: %d of %d elements off, first at %s: got %r, want %r, allowed %.3g" % (
            what, int(bad.sum()), bad.numel(), i, float(got[i]), float(y[i]), float(allow[i])))


def norm(off, x, branch, gate, scale, shift, weight, centre, eps):
    """(y, x', bound of y before its rounding, bound of x' before its rounding) in 64 bits."""
    seq = torch.repeat_interleave(torch.arange(len(off) - 1, device=x.device), torch.tensor([b - a for a, b in zip(off, off[1:])], device=x.device))
    z = x.double()
    mag = z.abs()
    if branch is not None:
        t = branch.double() * (gate.double()[seq] if gate is not None else 1.0)
        z, mag = z + t, mag + t.abs()
    n = z.shape[1]
    mean = z.mean(1, keepdim=True) if centre else torch.zeros_like(z[:, :1])
    var = ((z - mean) ** 2).mean(1, keepdim=True)
    r = 1.0 / torch.sqrt(var + eps)
    f = torch.ones_like(z)
    if weight is not None:
        f = f * weight.double()
    if scale is not None:
        f = f * (1.0 + scale.double()[seq])
    t = shift.double()[seq] if shift is not None else torch.zeros_like(z)
    y = (z - mean) * r * f + t
    # as for the adaptive layer norm: x' two roundings, a sum over n terms log2(n) and the 40 terms that a thread adds one after another; rstd half
    # the variance's relative error; then five more roundings (difference, rstd, weight, scale, the last sum)
    depth = torch.log2(torch.tensor(float(max(n, 2)))).item() + 72
    dz = 2 * U32 * mag + (depth * U32 * mag.mean(1, keepdim=True) if centre else 0.0)
    dvar = (depth + 4) * U32 + 2 * (dz * (z - mean).abs()).mean(1, keepdim=True) / (var + eps)
    bound = (dz * r + (z - mean).abs() * r * (dvar + 8 * U32)) * f.abs() + 4 * U32 * (y.abs() + t.abs())
    return y, z, bound, 2 * U32 * mag


def act(t, kind):
    if kind == "gelu":
        return torch.nn.functional.gelu(t, approximate="tanh")
    return torch.nn.functional.silu(t) if kind == "silu" else t


def product(a, w, bias=None, kind="none"):
    """(t, bound before its rounding) in 64 bits of Matrix8 operands: t = act(a w^T + bias)."""
    x, v = values(a), values(w)
    t, mag = x @ v.T, x.abs() @ v.abs().T
    k = x.shape[1]
    # products are exact (4 by 4 bits of significand, scales powers of two). A step of the tensor cores adds 32 of them to the sum, 33 terms each cut
    # to 2^-24 of the largest at worst: (k + k / 32 + 33) roundings of the magnitudes; shares of k and the scaling, 40 more
    bound = (1.04 * k + 73) * U32 * mag
    if bias is not None:
        t = t + bias.double()
        bound = bound + U32 * t.abs()
    if kind != "none":
        # both are t s(t) with a slope of at most 1.13; the exponential and the reciprocal of the special function unit are good to 2^-22, the
        # exponent x (|x| <= 1.45 |t| (1 + 0.08 t^2), of weight s (1 - s) <= 2^-x) to 4 roundings: together below 64 roundings of |t|; and where x
        # exceeds 63 the factor stays at 2^-63
        bound = 1.13 * bound + 64 * U32 * t.abs() + 2.0 ** -62 * t.abs()
        t = act(t, kind)
    return t, bound
