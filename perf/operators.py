"""Workloads of the verification layer's operators: adaptive layer norm, rotary positions over several
axes, attention over packed sequences. Plain torch forms in 32 bits, the library's calls, and the
definitions in 64 bits."""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6
THETA = 10000.0


# ---- cases -----------------------------------------------------------------------------------------

def listed():
    return [
        # the entry of the verification layer of a FLUX.1-dev-shaped step: residual add of the branch, norm, modulation
        dict(name="modulate_flux", op="modulate", lens="4608", dim=3072, dtype="bf16", branch=True, active=""),
        # DiT-XL/2, 8 images x CFG pair, every third sample rejected and masked out
        dict(name="modulate_dit_masked", op="modulate", lens=" ".join(["256"] * 16), dim=1152, dtype="bf16", branch=False,
             active="1101101101101101"),
        # the fp32 DiT-S-like cache: the smallest call, latency counts
        dict(name="modulate_tiny_f32", op="modulate", lens="64 64", dim=384, dtype="f32", branch=True, active=""),
        # FLUX-shaped q and k out of the fused projection: RMS norm per head, 512 text tokens at the origin, 64 x 64 image
        dict(name="rope_flux", op="rope", lens="4608", heads=24, kv_heads=24, head_dim=128, axes="16 56 56", grid="1 64 64",
             text=512, pairing="interleaved", norm=True, dtype="bf16", active=""),
        # HunyuanVideo-shaped: 13 x 30 x 53 video tokens and 256 text tokens
        dict(name="rope_hunyuan", op="rope", lens="20926", heads=24, kv_heads=24, head_dim=128, axes="16 56 56",
             grid="13 30 53", text=256, pairing="interleaved", norm=True, dtype="bf16", active=""),
        # one new token per sequence of a grouped-head text model, half-split pairs, one axis
        dict(name="rope_single_tokens", op="rope", lens="1 1 1 1", heads=32, kv_heads=8, head_dim=128, axes="128",
             grid="1 1 4096", text=0, pairing="halves", norm=False, dtype="bf16", active=""),
        # DiT-XL/2: 16 heads of 72, sixteen samples of 256 tokens
        dict(name="attention_dit", op="attention", q_lens=" ".join(["256"] * 16), kv_lens="", valid="", heads=16, kv_heads=16,
             head_dim=72, dtype="bf16", causal=False, sharp=1.0, active=""),
        # FLUX-shaped joint attention over 512 + 4096 tokens
        dict(name="attention_flux", op="attention", q_lens="4608", kv_lens="", valid="", heads=24, kv_heads=24, head_dim=128,
             dtype="bf16", causal=False, sharp=1.5, active=""),
        # HunyuanVideo-shaped: 20670 video tokens + 256 text tokens, of which 77 are not padding
        dict(name="attention_hunyuan", op="attention", q_lens="20926", kv_lens="", valid="20747", heads=24, kv_heads=24,
             head_dim=128, dtype="bf16", causal=False, sharp=1.0, active=""),
        # prompts of a grouped-head text encoder, packed, causal, ragged, from one token on
        dict(name="attention_prompts", op="attention", q_lens="1 77 256 1023 2048 4096 333 512", kv_lens="", valid="",
             heads=32, kv_heads=8, head_dim=128, dtype="bf16", causal=True, sharp=2.0, active=""),
        # one new token per sequence against caches of different fill
        dict(name="attention_single_tokens", op="attention", q_lens="1 1 1 1 1 1 1 1",
             kv_lens="4096 8192 16384 32768 4096 8192 16384 32768", valid="4000 8192 12345 32767 1 5000 16383 20000",
             heads=32, kv_heads=8, head_dim=128, dtype="bf16", causal=True, sharp=2.0, active=""),
        # the fp32 DiT-S-like model: 6 heads of 64, two samples
        dict(name="attention_tiny_f32", op="attention", q_lens="64 64", kv_lens="", valid="", heads=6, kv_heads=6, head_dim=64,
             dtype="f32", causal=False, sharp=1.0, active=""),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _split(rng, total, parts):
    """`parts` lengths of at least one that add up to about `total`."""
    w = [rng.uniform(0.05, 1.0) for _ in range(parts)]
    return [max(1, int(total * x / sum(w))) for x in w]


def _mask(rng, n):
    if n < 2 or rng.random() < 0.6:
        return ""
    bits = [rng.random() < 0.6 for _ in range(n)]
    bits[rng.randrange(n)] = True
    return "".join("1" if b else "0" for b in bits)


def _text(xs):
    return " ".join(str(x) for x in xs)


def draw(rng):
    op = rng.choice(["modulate", "rope", "attention", "attention"])
    if op == "modulate":
        n = rng.choice([1, 1, 2, 5, 16])
        dim = _log(rng, 64, 8192)
        if rng.random() < 0.6:
            dim = max(64, dim // 64 * 64)
        lens = _split(rng, min(_log(rng, n, 20926), (1 << 26) // dim), n)
        return dict(op=op, lens=_text(lens), dim=dim, dtype=rng.choice(["bf16", "bf16", "f32"]),
                    branch=rng.random() < 0.5, active=_mask(rng, n))
    if op == "rope":
        hd = rng.choice([64, 72, 96, 128])
        grid = [rng.randint(1, 16), rng.randint(1, 64), rng.randint(1, 64)]
        axes = rng.choice([[hd], [hd // 2], [hd // 8, (hd - hd // 8) // 4 * 2, hd - hd // 8 - (hd - hd // 8) // 4 * 2],
                           [hd // 4 * 2, hd - hd // 4 * 2]])
        axes = [a for a in axes if a]
        if any(a % 2 for a in axes):
            axes = [hd]
        kv = rng.choice([1, 2, 8, 12, 24])
        heads = kv * rng.choice([1, 1, 2, 4])
        n = rng.choice([1, 1, 3, 8])
        lens = _split(rng, min(_log(rng, n, 20926), (1 << 27) // ((heads + kv) * hd)), n)
        return dict(op=op, lens=_text(lens), heads=heads, kv_heads=kv, head_dim=hd, axes=_text(axes), grid=_text(grid),
                    text=rng.choice([0, 0, 77]), pairing=rng.choice(["interleaved", "halves"]), norm=rng.random() < 0.5,
                    dtype=rng.choice(["bf16", "bf16", "f32"]), active=_mask(rng, n))
    kind = rng.choice(["full", "full", "prompts", "few", "f32"])
    kv = rng.choice([1, 2, 3, 8, 16])
    heads = kv * rng.choice([1, 1, 3, 4, 7])
    hd = rng.choice([32, 64, 72, 80, 96, 128, 128])
    sharp = rng.choice([0.5, 1.0, 2.0, 4.0])
    kv_lens, valid = "", ""
    if kind == "full":
        n = rng.choice([1, 1, 2, 16])
        q = _split(rng, _log(rng, 4 * n, 12000), n)
        if rng.random() < 0.3:
            k = _split(rng, _log(rng, 4 * n, 12000), n)
            kv_lens = _text(k)
        causal = False
    elif kind == "prompts":
        n = rng.choice([1, 3, 8, 24])
        q = _split(rng, _log(rng, 2 * n, 16000), n)
        causal = True
    elif kind == "few":
        n = rng.choice([1, 1, 4, 32])
        q = [rng.choice([1, 1, 1, 2, 5]) for _ in range(n)]
        k = [max(8, x) for x in _split(rng, _log(rng, 64 * n, 400000), n)]
        kv_lens = _text(k)
        valid = _text([rng.randint(min(x, 5), x) for x in k]) if rng.random() < 0.7 else ""
        causal = True
    else:
        n = rng.choice([1, 2, 4])
        heads = kv = rng.choice([1, 3, 6])
        q = _split(rng, _log(rng, 2 * n, 2000), n)
        hd = rng.choice([hd, 36, 64])
        causal = rng.random() < 0.5
    return dict(op=op, q_lens=_text(q), kv_lens=kv_lens, valid=valid, heads=heads, kv_heads=kv, head_dim=hd,
                dtype="f32" if kind == "f32" else "bf16", causal=causal, sharp=sharp, active=_mask(rng, n))


# ---- inputs ----------------------------------------------------------------------------------------

def _ints(text):
    return [int(x) for x in text.split()]


def _offsets(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return out


def _on(case, n):
    return [c == "1" for c in case["active"]] if case["active"] else [True] * n


def _inputs(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32)

    if case["op"] == "modulate":
        off = _offsets(_ints(case["lens"]))
        dim, n = case["dim"], len(off) - 1
        x = normal(off[-1], dim)
        # a few outlier channels, as in the activations of diffusion transformers
        x[:, torch.randperm(dim, generator=g, device=DEV)[:max(1, dim // 1000)]] *= 50.0
        mod = 0.3 * normal(n, 3, dim)
        s = dict(off=off, x=x.to(dt), mod=mod.to(dt), branch=normal(off[-1], dim).to(dt) if case["branch"] else None)
    elif case["op"] == "rope":
        off = _offsets(_ints(case["lens"]))
        h, kv, hd = case["heads"], case["kv_heads"], case["head_dim"]
        axes, grid = _ints(case["axes"]), _ints(case["grid"])
        start = [int(x) for x in torch.randint(0, max(grid), (len(off),), generator=g, device=DEV).tolist()]
        pos = torch.zeros(off[-1], len(axes), device=DEV, dtype=torch.float32)
        for i in range(len(off) - 1):
            t = torch.arange(off[i + 1] - off[i], device=DEV) - case["text"]
            t = torch.where(t >= 0, t + (start[i] if len(axes) == 1 else 0), torch.zeros_like(t))
            where = [t // (grid[1] * grid[2]), t // grid[2] % grid[1], t % grid[2]]
            cols = [t] if len(axes) == 1 else where[3 - len(axes):]
            pos[off[i]:off[i + 1]] = torch.stack(cols, 1).to(torch.float32)
        s = dict(off=off, qkv=normal(off[-1], h + 2 * kv, hd).to(dt), pos=pos,
                 wq=(1 + 0.2 * normal(hd)).to(dt) if case["norm"] else None,
                 wk=(1 + 0.2 * normal(hd)).to(dt) if case["norm"] else None)
    else:
        ql = _ints(case["q_lens"])
        kl = _ints(case["kv_lens"]) if case["kv_lens"] else ql
        off, koff = _offsets(ql), _offsets(kl)
        h, kv, hd = case["heads"], case["kv_heads"], case["head_dim"]
        q = (case["sharp"] * normal(off[-1], h, hd)).to(dt)
        k = (normal(koff[-1], kv, hd) + normal(1, kv, hd)).to(dt)
        # values stay where the projection left them: a strided part of its output
        v = (normal(koff[-1], 2 * kv, hd) + 0.25 * normal(1, 2 * kv, hd)).to(dt)[:, kv:]
        s = dict(off=off, koff=koff, q=q, k=k, v=v, valid=_ints(case["valid"]) if case["valid"] else None)
    n = len(s["off"]) - 1
    s["on"] = _on(case, n)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"], s["own"] = case, own
    if not own:
        return s
    from paper_2509_11628_b200 import binding as S
    dtype = S.SPECA_BF16 if case["dtype"] == "bf16" else S.SPECA_F32
    kw = dict(dtype=dtype, device="cuda:%d" % torch.cuda.current_device())
    s["active"] = torch.tensor(s["on"], dtype=torch.uint8, device=DEV) if case["active"] else None
    if case["op"] == "modulate":
        s["layer"] = S.SpecaLayer(s["off"], norm_eps=EPS, **kw)
        s["y"] = torch.zeros_like(s["x"])
        s["x_out"] = torch.zeros_like(s["x"]) if case["branch"] else None
    elif case["op"] == "rope":
        h, kv = case["heads"], case["kv_heads"]
        pairing = S.SPECA_ROPE_INTERLEAVED if case["pairing"] == "interleaved" else S.SPECA_ROPE_HALVES
        s["layer"] = S.SpecaLayer(s["off"], n_heads=h, n_kv_heads=kv, head_dim=case["head_dim"], axis_dims=_ints(case["axes"]),
                                  theta=THETA, pairing=pairing, norm_eps=EPS, **kw)
        t, hd = s["off"][-1], case["head_dim"]
        s["q_out"] = torch.zeros(t, h, hd, dtype=s["qkv"].dtype, device=DEV)
        s["k_out"] = torch.zeros(t, kv, hd, dtype=s["qkv"].dtype, device=DEV)
    else:
        s["layer"] = S.SpecaLayer(s["off"], kv_start=s["koff"], n_heads=case["heads"], n_kv_heads=case["kv_heads"],
                                  head_dim=case["head_dim"], causal=case["causal"], **kw)
        s["out"] = torch.zeros_like(s["q"])
        s["kv_len"] = torch.tensor(s["valid"], dtype=torch.int32, device=DEV) if s["valid"] else None
    return s


# ---- one pass --------------------------------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    if s["own"]:
        layer = s["layer"]
        if op == "modulate":
            gate, scale, shift = s["mod"][:, 0], s["mod"][:, 1], s["mod"][:, 2]
            layer.modulate(s["x"], s["y"], branch=s["branch"], gate=gate if s["branch"] is not None else None, scale=scale,
                           shift=shift, x_out=s["x_out"], active=s["active"])
            return {"y": s["y"]} if s["branch"] is None else {"y": s["y"], "x": s["x_out"]}
        if op == "rope":
            h, kv = s["case"]["heads"], s["case"]["kv_heads"]
            layer.rope(s["qkv"][:, :h], s["q_out"], s["qkv"][:, h:h + kv], s["k_out"], s["pos"], q_weight=s["wq"],
                       k_weight=s["wk"], active=s["active"])
            return {"q": s["q_out"], "k": s["k_out"]}
        layer.attention(s["q"], s["k"], s["v"], s["out"], kv_len=s["kv_len"], active=s["active"])
        return {"o": s["out"]}
    return {"modulate": _plain_modulate, "rope": _plain_rope, "attention": _plain_attention}[op](s)


def _plain_modulate(s):
    y = torch.zeros_like(s["x"])
    x_out = torch.zeros_like(s["x"])
    for i, on in enumerate(s["on"]):
        if not on:
            continue
        rows = slice(s["off"][i], s["off"][i + 1])
        gate, scale, shift = s["mod"][i].float()
        x = s["x"][rows].float()
        if s["branch"] is not None:
            x = x + gate * s["branch"][rows].float()
            x_out[rows] = x.to(x_out.dtype)
        d = x - x.mean(-1, keepdim=True)
        u = d * torch.rsqrt((d * d).mean(-1, keepdim=True) + EPS)
        y[rows] = (u * (1 + scale) + shift).to(y.dtype)
    return {"y": y} if s["branch"] is None else {"y": y, "x": x_out}


def _plain_rope(s):
    case = s["case"]
    h, kv = case["heads"], case["kv_heads"]
    axes = _ints(case["axes"])
    angle = torch.cat([s["pos"][:, a:a + 1] * THETA ** (-2.0 * torch.arange(d // 2, device=DEV, dtype=torch.float32) / d)
                       for a, d in enumerate(axes)], 1)[:, None]
    c, sn = torch.cos(angle), torch.sin(angle)
    r = sum(axes)
    keep = torch.cat([torch.full((s["off"][i + 1] - s["off"][i],), on, device=DEV) for i, on in enumerate(s["on"])])

    def turn(x, w):
        u = x.float()
        if w is not None:
            u = u * torch.rsqrt((u * u).mean(-1, keepdim=True) + EPS) * w.float()
        out = u.clone()
        if case["pairing"] == "interleaved":
            a, b = u[..., 0:r:2], u[..., 1:r:2]
            out[..., 0:r:2], out[..., 1:r:2] = a * c - b * sn, a * sn + b * c
        else:
            a, b = u[..., :r // 2], u[..., r // 2:r]
            out[..., :r // 2], out[..., r // 2:r] = a * c - b * sn, a * sn + b * c
        return torch.where(keep[:, None, None], out, torch.zeros_like(out)).to(x.dtype)

    return {"q": turn(s["qkv"][:, :h], s["wq"]), "k": turn(s["qkv"][:, h:h + kv], s["wk"])}


def _plain_attention(s):
    case = s["case"]
    h, kv, hd = case["heads"], case["kv_heads"], case["head_dim"]
    group = h // kv
    out = torch.zeros_like(s["q"])
    for i, on in enumerate(s["on"]):
        nq = s["off"][i + 1] - s["off"][i]
        nk = s["koff"][i + 1] - s["koff"][i]
        if s["valid"]:
            nk = s["valid"][i]
        if not on or not nq or not nk:
            continue
        # [kv head, query x group, hd]; as many heads at once as a 2 GB score matrix holds
        q = s["q"][s["off"][i]:s["off"][i + 1]].float().view(nq, kv, group, hd).permute(1, 2, 0, 3).reshape(kv, group * nq, hd)
        k = s["k"][s["koff"][i]:s["koff"][i] + nk].float().permute(1, 2, 0)
        v = s["v"][s["koff"][i]:s["koff"][i] + nk].float().permute(1, 0, 2)
        hidden = None
        if case["causal"]:
            last = torch.arange(nq, device=DEV) + (nk - nq)
            hidden = (torch.arange(nk, device=DEV)[None] > last[:, None]).repeat(group, 1)
        o = torch.empty(kv, group * nq, hd, device=DEV)
        step = max(1, (1 << 29) // (group * nq * nk))
        for a in range(0, kv, step):
            e = torch.matmul(q[a:a + step], k[a:a + step]) * (hd ** -0.5)
            if hidden is not None:
                e = e.masked_fill(hidden, float("-inf"))
            top = e.amax(-1, keepdim=True)
            e = torch.exp(e - torch.where(torch.isfinite(top), top, torch.zeros_like(top)))
            o[a:a + step] = torch.matmul(e, v[a:a + step]) / e.sum(-1, keepdim=True).clamp_min(1e-37)
        out[s["off"][i]:s["off"][i + 1]] = o.view(kv, group, nq, hd).permute(2, 0, 1, 3).reshape(nq, h, hd).to(out.dtype)
    return {"o": out}


# ---- the floor -------------------------------------------------------------------------------------

def _visible(nq, nk, causal):
    """Query-key pairs that are not masked."""
    if not causal:
        return nq * nk
    first = max(0, nq - nk)  # rows before this one see nothing
    rows = nq - first
    return rows * (nk - nq + first + 1) + rows * (rows - 1) // 2


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "attention":
        ql = _ints(case["q_lens"])
        kl = _ints(case["valid"]) if case["valid"] else _ints(case["kv_lens"]) if case["kv_lens"] else ql
        on = _on(case, len(ql))
        h, kv, hd = case["heads"], case["kv_heads"], case["head_dim"]
        nbytes = sum(size * hd * (2 * a * h + 2 * b * kv) for a, b, o in zip(ql, kl, on) if o)
        return {"bytes": nbytes, "flops": sum(4 * hd * h * _visible(a, b, case["causal"]) for a, b, o in zip(ql, kl, on) if o)}
    lens = _ints(case["lens"])
    rows = sum(n for n, o in zip(lens, _on(case, len(lens))) if o)
    if case["op"] == "modulate":
        words = (4 if case["branch"] else 2) * rows + 3 * len(lens)
        return {"bytes": size * words * case["dim"], "flops": (11 if case["branch"] else 9) * rows * case["dim"]}
    width = (case["heads"] + case["kv_heads"]) * case["head_dim"]
    return {"bytes": 2 * size * rows * width + 4 * rows * len(_ints(case["axes"])), "flops": (7 if case["norm"] else 3) * rows * width}


# ---- the definitions in 64 bits --------------------------------------------------------------------

def exact(case, seed):
    s = _inputs(case, seed)
    return {"modulate": _exact_modulate, "rope": _exact_rope, "attention": _exact_attention}[case["op"]](case, s)


def _exact_modulate(case, s):
    n = [b - a for a, b in zip(s["off"], s["off"][1:])]
    per_row = torch.repeat_interleave(torch.arange(len(n), device=DEV), torch.tensor(n, device=DEV))
    on = torch.tensor(s["on"], device=DEV)[per_row][:, None]
    y, z = [], []
    for a in range(0, s["off"][-1], 4096):
        seq = per_row[a:a + 4096]
        x = s["x"][a:a + 4096].double()
        m = s["mod"].double()
        if s["branch"] is not None:
            x = x + m[seq, 0] * s["branch"][a:a + 4096].double()
        var, mean = torch.var_mean(x, -1, correction=0, keepdim=True)
        z.append(x)
        y.append((x - mean) / torch.sqrt(var + EPS) * (1 + m[seq, 1]) + m[seq, 2])
    y, z = torch.cat(y) * on, torch.cat(z) * on
    return {"y": y} if s["branch"] is None else {"y": y, "x": z}


def _exact_rope(case, s):
    axes, hd = _ints(case["axes"]), case["head_dim"]
    t, r = s["off"][-1], sum(axes)
    turn = torch.ones(t, hd // 2, dtype=torch.complex128, device=DEV)  # one rotation per pair of the head
    p = 0
    for a, d in enumerate(axes):
        for i in range(d // 2):
            angle = s["pos"][:, a].double() * math.pow(THETA, -2.0 * i / d)
            turn[:, p] = torch.polar(torch.ones_like(angle), angle)
            p += 1
    if case["pairing"] == "interleaved":
        first = list(range(0, hd, 2))
        second = list(range(1, hd, 2))
    else:
        first = list(range(r // 2)) + list(range(r, hd, 2))
        second = list(range(r // 2, r)) + list(range(r + 1, hd, 2))
    on = torch.zeros(t, dtype=torch.float64, device=DEV)
    for i, o in enumerate(s["on"]):
        on[s["off"][i]:s["off"][i + 1]] = float(o)

    def one(x, w):
        out = torch.empty(x.shape, dtype=torch.float64, device=DEV)
        for head in range(x.shape[1]):
            u = x[:, head].double()
            if w is not None:
                u = u / torch.sqrt(u.pow(2).sum(-1, keepdim=True) / hd + EPS) * w.double()
            z = torch.complex(u[:, first], u[:, second]) * turn
            out[:, head, first], out[:, head, second] = z.real, z.imag
        return out * on[:, None, None]

    h, kv = case["heads"], case["kv_heads"]
    return {"q": one(s["qkv"][:, :h], s["wq"]), "k": one(s["qkv"][:, h:h + kv], s["wk"])}


def _exact_attention(case, s):
    h, kv, hd = case["heads"], case["kv_heads"], case["head_dim"]
    out = torch.zeros(s["off"][-1], h, hd, dtype=torch.float64, device=DEV)
    for i, on in enumerate(s["on"]):
        if not on:
            continue
        a, b, ka = s["off"][i], s["off"][i + 1], s["koff"][i]
        nk = s["valid"][i] if s["valid"] else s["koff"][i + 1] - ka
        for head in range(h):
            k = s["k"][ka:ka + nk, head * kv // h].double()
            v = s["v"][ka:ka + nk, head * kv // h].double()
            for r in range(a, b, 8192):
                q = s["q"][r:min(b, r + 8192), head].double()
                z = q @ k.T / math.sqrt(hd)
                if case["causal"]:
                    row = torch.arange(r - a, r - a + q.shape[0], device=DEV)[:, None]
                    z[torch.arange(nk, device=DEV)[None] - row > nk - (b - a)] = float("-inf")
                p = torch.softmax(z, -1).nan_to_num(0.0)
                out[r:r + q.shape[0], head] = p @ v
    return {"o": out}
