"""Definitions in 64 bits of the verification layer's operators, and bounds on what 32-bit arithmetic and the
storage type's rounding may move an element by. Plain torch, no code of the library."""
import math

import torch

U32 = 2.0 ** -24
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}  # largest relative error of one rounding


def offsets(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return out


def modulate(off, x, branch, gate, scale, shift, eps):
    """(y, x', bound of y, bound of x' before its rounding) in 64 bits, each [rows, dim]."""
    seq = torch.repeat_interleave(torch.arange(len(off) - 1, device=x.device),
                                  torch.tensor([b - a for a, b in zip(off, off[1:])], device=x.device))
    z = x.double()
    mag = z.abs()
    if branch is not None:
        t = branch.double() * (gate.double()[seq] if gate is not None else 1.0)
        z, mag = z + t, mag + t.abs()
    n = z.shape[1]
    mean = z.mean(1, keepdim=True)
    var = ((z - mean) ** 2).mean(1, keepdim=True)
    r = 1.0 / torch.sqrt(var + eps)
    s = 1.0 + scale.double()[seq] if scale is not None else torch.ones_like(z)
    t = shift.double()[seq] if shift is not None else torch.zeros_like(z)
    y = (z - mean) * r * s + t
    # each x' is off by at most 2 roundings; a sum over n terms in any order by log2(n) + the terms a thread adds
    # one after another (at most 32), each rounding relative to the summed magnitudes
    depth = math.log2(max(n, 2)) + 40
    dz = 2 * U32 * mag + depth * U32 * mag.mean(1, keepdim=True)
    # rstd: relative error of half the variance's, which the mean's error enters with its square only
    dvar = (depth + 4) * U32 + 2 * (dz * (z - mean).abs()).mean(1, keepdim=True) / (var + eps)
    bound = (dz * r + (z - mean).abs() * r * (dvar + 6 * U32)) * s.abs() + 4 * U32 * (y.abs() + t.abs())
    return y, z, bound, 2 * U32 * mag


def rope(x, weight, pos, axes, theta, halves, eps):
    """(rotated, bound before rounding) of [rows, heads, hd] in 64 bits."""
    hd, r = x.shape[-1], sum(axes)
    u = x.double()
    if weight is not None:
        u = u / torch.sqrt((u * u).mean(-1, keepdim=True) + eps) * weight.double()
    angle = torch.cat([pos[:, a:a + 1].double() * torch.tensor([theta ** (-2.0 * i / d) for i in range(d // 2)],
                                                               dtype=torch.float64, device=x.device)
                       for a, d in enumerate(axes)], 1)[:, None]
    first = list(range(0, r // 2)) if halves else list(range(0, r, 2))
    second = list(range(r // 2, r)) if halves else list(range(1, r, 2))
    out, bound = u.clone(), u.abs().clone()
    a, b = u[..., first], u[..., second]
    out[..., first] = a * torch.cos(angle) - b * torch.sin(angle)
    out[..., second] = a * torch.sin(angle) + b * torch.cos(angle)
    bound[..., first] = bound[..., second] = a.abs() + b.abs()
    # the norm: a sum of hd squares and three more roundings; the turn: an angle off by one rounding of at most
    # half a turn (pi * 2^-24), sine and cosine to 2 units, a product and a sum
    n_norm = (hd + 6) if weight is not None else 0
    return out, (n_norm + 8) * U32 * bound


def attention(off, koff, q, k, v, causal, scale, kv_len=None, lse=False):
    """(o, bound of o before its rounding, lse, bound of lse), rows that see nothing are zero (-inf)."""
    rows, h, hd = q.shape
    group = h // k.shape[1]
    o = torch.zeros(rows, h, hd, dtype=torch.float64, device=q.device)
    bound = torch.zeros_like(o)
    ls = torch.full((h, rows), -math.inf, dtype=torch.float64, device=q.device)
    lb = torch.zeros_like(ls)
    weight_unit = 0.0 if q.dtype == torch.float32 else 2.0 ** -8
    for s in range(len(off) - 1):
        nq, nk = off[s + 1] - off[s], koff[s + 1] - koff[s]
        if kv_len is not None:
            nk = max(0, min(nk, int(kv_len[s])))
        if nq == 0 or nk == 0:
            continue
        kk, vv = k[koff[s]:koff[s] + nk].double(), v[koff[s]:koff[s] + nk].double()
        hidden = torch.zeros(nq, nk, dtype=torch.bool, device=q.device)
        if causal:
            hidden = torch.arange(nk, device=q.device)[None] > (torch.arange(nq, device=q.device) + nk - nq)[:, None]
        empty = hidden.all(1)
        for j in range(h):
            qq, kj, vj = q[off[s]:off[s + 1], j].double(), kk[:, j // group], vv[:, j // group]
            z = (qq @ kj.T) * scale
            size = (qq.abs() @ kj.abs().T) * scale  # what the products of a score add up from
            z = z.masked_fill(hidden, -math.inf)
            p = torch.softmax(z, 1)
            p[empty] = 0.0
            mag = p @ vj.abs()
            # a score is off by hd roundings of its magnitudes and a few of its value, the exponential by as much
            # absolutely and 4 units; sums of up to nk weights, numerator and denominator alike; the weights' own rounding
            ds = ((hd + 6) * U32 * size.masked_fill(hidden, 0.0).amax(1, keepdim=True))
            rel = 2 * (ds + (nk + 40) * U32 + weight_unit)
            o[off[s]:off[s + 1], j] = p @ vj
            bound[off[s]:off[s + 1], j] = rel * mag + 8 * U32 * mag
            ls[j, off[s]:off[s + 1]] = torch.logsumexp(z, 1)
            # weight_unit: the sum is over the rounded weights
            lb[j, off[s]:off[s + 1]] = (ds + (nk + 40) * U32 + weight_unit)[:, 0] + 8 * U32 * ls[j, off[s]:off[s + 1]].abs().nan_to_num(0, 0, 0)
    return o, bound, ls, lb


def check(got, want, bound, what=""):
    """Every element within `bound` of the 64-bit value, plus one rounding to its own type."""
    g, w = got.double(), want
    inf = torch.isinf(w)
    assert torch.equal(g[inf], w[inf]), what
    allow = bound + UNIT[got.dtype] * (w.abs() + bound) + 1e-38
    bad = ~inf & ~((g - w).abs() <= allow)
    if bool(bad.any()):
        i = tuple(bad.nonzero()[0].tolist())
        raise AssertionError("%s: %d of %d elements off, first at %s: got %r, want %r, allowed %.3g" % (
            what, int(bad.sum()), bad.numel(), i, float(g[i]), float(w[i]), float(allow[i])))
