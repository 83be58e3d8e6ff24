"""Workloads of the block's 8-bit operators: norms with the residual's addition and an output in 8 bits, quantising rows,
matrix products in 8 bits with one scale for each 128 elements. Plain torch forms in 32 bits, the library's calls, and
the definitions in 64 bits."""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6
BLOCK = 128   # elements of a row that share a scale
TOP = 448.0   # the largest e4m3 value


# ---- cases -----------------------------------------------------------------------------------------

def listed():
    return [
        # one new token for each of eight sequences of a text model: the smallest call, latency counts
        dict(name="norm8_single_tokens", op="norm8", lens=" ".join(["1"] * 8), dim=4096, kind="rms", parts="branch weight", dtype="bf16",
             active=""),
        # DiT-XL/2, 8 images x CFG pair, every third sample rejected and masked out: adaptive layer norm with the gated residual
        dict(name="norm8_dit_masked", op="norm8", lens=" ".join(["256"] * 16), dim=1152, kind="layer",
             parts="branch gate scale shift", dtype="bf16", active="1101101101101101"),
        # a video's tokens, pre-norm block with an RMS norm's weight
        dict(name="norm8_video", op="norm8", lens="20926", dim=4096, kind="rms", parts="branch gate weight", dtype="bf16", active=""),
        # fp32 rows that divide into nothing
        dict(name="norm8_odd_f32", op="norm8", lens="77 1 333", dim=1155, kind="rms", parts="weight", dtype="f32", active=""),
        # the attention's output on its way to the output projection: 16 heads of 128, packed prompts, one sample masked out
        dict(name="quantize8_prompts", op="quantize8", lens="1 77 256 1023 2048 4096 333 512", dim=2048, dtype="bf16", weights=False,
             active="11110111"),
        # a weight matrix when a model is loaded
        dict(name="quantize8_weight", op="quantize8", lens="16384", dim=4096, dtype="bf16", weights=True, active=""),
        # one new token for each of four sequences: query, key and value projection with 32 heads and 8 key heads of 128
        dict(name="matmul8_single_tokens", op="matmul8", lens="1 1 1 1", k=4096, n=6144, act="none", parts="", out="same",
             dtype="bf16", active=""),
        # DiT-XL/2 MLP, first product: 4608 features, GELU, straight into the second product's 8 bits
        dict(name="matmul8_dit_up", op="matmul8", lens=" ".join(["256"] * 16), k=1152, n=4608, act="gelu", parts="bias", out="8bit",
             dtype="bf16", active=""),
        # DiT-XL/2 MLP, second product with the gated residual, rejected samples masked out
        dict(name="matmul8_dit_down_masked", op="matmul8", lens=" ".join(["256"] * 16), k=4608, n=1152, act="none",
             parts="bias residual gate", out="same", dtype="bf16", active="1101101101101101"),
        # packed ragged prompts of a text model, first product of its MLP
        dict(name="matmul8_prompts", op="matmul8", lens="1 77 256 1023 2048 4096 333 512", k=4096, n=14336, act="silu", parts="", out="same",
             dtype="bf16", active=""),
        # a video's tokens, first product of the MLP: the largest
        dict(name="matmul8_video_up", op="matmul8", lens="20926", k=4096, n=16384, act="gelu", parts="bias", out="8bit", dtype="bf16",
             active=""),
        # fp32 model, sizes that divide into nothing
        dict(name="matmul8_odd_f32", op="matmul8", lens="77 1 133", k=1155, n=333, act="none", parts="bias", out="same", dtype="f32",
             active=""),
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


def _width(rng, lo, hi):
    n = _log(rng, lo, hi)
    return max(64, n // 64 * 64) if rng.random() < 0.65 else n


def draw(rng):
    op = rng.choice(["norm8", "quantize8", "matmul8", "matmul8"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    n = rng.choice([1, 1, 2, 5, 16])
    if op == "matmul8":
        k, wide = _width(rng, 64, 16384), _width(rng, 64, 16384)
        k = min(k, (1 << 26) // wide)
        rows = min(_log(rng, n, 20926), (1 << 40) // (k * wide))
        out = rng.choice(["same", "same", "8bit"])
        parts = [p for p in ("bias", "residual") if rng.random() < 0.5 and (p == "bias" or out == "same")]
        if "residual" in parts and rng.random() < 0.6:
            parts.append("gate")
        return dict(op=op, lens=_text(_split(rng, rows, n)), k=k, n=wide, act=rng.choice(["none", "gelu", "silu"]), parts=" ".join(parts),
                    out=out, dtype=dtype, active=_mask(rng, n))
    dim = _width(rng, 64, 8192)
    lens = _text(_split(rng, min(_log(rng, n, 20926), (1 << 26) // dim), n))
    if op == "quantize8":
        weights = rng.random() < 0.3
        return dict(op=op, lens=lens, dim=dim, dtype=dtype, weights=weights, active="" if weights else _mask(rng, n))
    parts = [p for p in ("branch", "scale", "shift", "weight") if rng.random() < 0.5]
    if "branch" in parts and rng.random() < 0.6:
        parts.append("gate")
    return dict(op=op, lens=lens, dim=dim, kind=rng.choice(["rms", "layer"]), parts=" ".join(parts), dtype=dtype, active=_mask(rng, n))


# ---- inputs ----------------------------------------------------------------------------------------

def _ints(text):
    return [int(x) for x in text.split()]


def _offsets(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return out


def _grouped(scales):
    """[rows, blocks] scale bytes as the library lays them out: [blocks / 4, rows, 4]; bytes behind the last block are zero."""
    rows, blocks = scales.shape
    groups = (blocks + 3) // 4
    full = torch.zeros(rows, groups * 4, dtype=torch.uint8, device=scales.device)
    full[:, :blocks] = scales
    return full.view(rows, groups, 4).transpose(0, 1).contiguous().view(torch.float8_e8m0fnu)


def _padded(x):
    """x in blocks: [rows, blocks, 128], zeros behind the end."""
    rows, dim = x.shape
    blocks = -(-dim // BLOCK)
    if dim % BLOCK:
        x = torch.nn.functional.pad(x, (0, blocks * BLOCK - dim))
    return x.view(rows, blocks, BLOCK)


def _to8(x):
    """Codes [rows, dim] and scale bytes [rows, blocks]: the smallest power of two that brings a block's largest finite value
    to 448 or less (1 for a block of zeros), and the block divided by it; what is not finite is NaN."""
    rows, dim = x.shape
    y = _padded(x)
    top = torch.where(torch.isfinite(y), y, torch.zeros_like(y)).abs().amax(-1)
    m, e = torch.frexp(top)
    e = torch.where(top > 0, (e - 9 + (m > 0.875)).clamp(-126, 127), torch.zeros_like(e))
    codes = torch.ldexp(y, -e[..., None]).to(torch.float8_e4m3fn)
    return codes.view(rows, -1)[:, :dim], (e + 127).to(torch.uint8)


def _from8(codes, scales):
    """The values of codes [rows, dim] with scales [groups, rows, 4], in fp32."""
    rows, dim = codes.shape
    e = scales.view(torch.uint8).transpose(0, 1).reshape(rows, -1)[:, :-(-dim // BLOCK)].to(torch.int32) - 127
    return torch.ldexp(_padded(codes.float()), e[..., None]).view(rows, -1)[:, :dim]


def _rows16(codes):
    """The same codes in rows of a multiple of 16 bytes."""
    rows, dim = codes.shape
    out = torch.zeros(rows, -(-dim // 16) * 16, dtype=torch.uint8, device=codes.device)
    out[:, :dim] = codes.view(torch.uint8)
    return out[:, :dim].view(torch.float8_e4m3fn)


def _inputs(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32)

    def activations(rows, dim):
        # a few outlier channels, as in the activations of transformers
        x = normal(rows, dim)
        x[:, torch.randperm(dim, generator=g, device=DEV)[:max(1, dim // 1000)]] *= 50.0
        return x

    lens = _ints(case["lens"])
    off = _offsets(lens)
    n, rows = len(lens), off[-1]
    on = torch.tensor([c == "1" for c in case["active"]] or [True] * n, device=DEV)
    s = dict(off=off, on=on, seq=torch.repeat_interleave(torch.arange(n, device=DEV), torch.tensor(lens, device=DEV)))
    s["live"] = on[s["seq"]][:, None]
    parts = case.get("parts", "").split()
    if case["op"] == "quantize8":
        s["x"] = activations(rows, case["dim"]).to(dt)
        return s
    if case["op"] == "norm8":
        dim = case["dim"]
        s["x"] = activations(rows, dim).to(dt)
        mod = (0.3 * normal(n, 3, dim)).to(dt)
        s["branch"] = normal(rows, dim).to(dt) if "branch" in parts else None
        s["gate"], s["scale"], s["shift"] = (mod[:, i] if p in parts else None for i, p in enumerate(("gate", "scale", "shift")))
        s["weight"] = (1 + 0.2 * normal(dim)).to(dt) if "weight" in parts else None
        return s
    k, wide = case["k"], case["n"]
    for name, m in (("a", activations(rows, k)), ("w", normal(wide, k) / math.sqrt(k))):
        codes, scales = _to8(m)
        s[name] = (_rows16(codes), _grouped(scales))
        del m, codes, scales
    s["bias"] = (0.2 * normal(wide)).to(dt) if "bias" in parts else None
    s["residual"] = normal(rows, wide).to(dt) if "residual" in parts else None
    s["gate"] = (0.5 * normal(n, 2, wide)).to(dt)[:, 1] if "gate" in parts else None
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"], s["own"] = case, own
    if not own:
        return s
    from paper_2509_11628_b200 import binding as S
    device = "cuda:%d" % torch.cuda.current_device()
    rows, dt = s["off"][-1], DTYPES[case["dtype"]]
    s["S"] = S
    s["layer"] = S.SpecaLayer(s["off"], S.SPECA_BF16 if case["dtype"] == "bf16" else S.SPECA_F32, norm_eps=EPS, device=device)
    s["active"] = s["on"].to(torch.uint8) if case["active"] else None
    if case["op"] == "matmul8":
        s["a8"], s["w8"] = S.Matrix8(*s["a"]), S.Matrix8(*s["w"])
        s["out"] = S.Matrix8.empty(rows, case["n"], device) if case["out"] == "8bit" else torch.zeros(rows, case["n"], dtype=dt, device=DEV)
        s["act"] = {"none": S.SPECA_ACT_NONE, "gelu": S.SPECA_ACT_GELU, "silu": S.SPECA_ACT_SILU}[case["act"]]
    else:
        s["out"] = S.Matrix8.empty(rows, case["dim"], device)
    if case["op"] == "norm8":
        s["kind"] = S.SPECA_NORM_RMS if case["kind"] == "rms" else S.SPECA_NORM_LAYER
        s["x_out"] = torch.zeros_like(s["x"]) if s["branch"] is not None else None
    return s


# ---- one pass --------------------------------------------------------------------------------------

def run(s):
    case = s["case"]
    op = case["op"]
    if not s["own"]:
        return {"norm8": _plain_norm8, "quantize8": _plain_quantize8, "matmul8": _plain_matmul8}[op](s)
    layer, out = s["layer"], s["out"]
    if op == "matmul8":
        layer.matmul8(s["a8"], s["w8"], out, bias=s["bias"], activation=s["act"], residual=s["residual"], gate=s["gate"], active=s["active"])
        return {"o": out} if case["out"] == "same" else {"codes": out.codes, "scales": out.scales}
    if op == "norm8":
        layer.norm8(s["x"], out, kind=s["kind"], branch=s["branch"], gate=s["gate"], scale=s["scale"], shift=s["shift"],
                    weight=s["weight"], x_out=s["x_out"], active=s["active"])
        got = {"codes": out.codes, "scales": out.scales}
        return got if s["x_out"] is None else {**got, "x": s["x_out"]}
    if case["weights"]:
        s["S"].quantize8(s["x"], out)
    else:
        layer.quantize8(s["x"], out, active=s["active"])
    return {"codes": out.codes, "scales": out.scales}


def _eight(s, y):
    """y in 8 bits, zeros (codes and scale bytes) in the rows of samples that are masked out."""
    codes, scales = _to8(y)
    codes = torch.where(s["live"], codes.view(torch.uint8), 0).view(torch.float8_e4m3fn)
    return {"codes": codes, "scales": _grouped(torch.where(s["live"], scales, 0))}


def _plain_quantize8(s):
    return _eight(s, s["x"].float())


def _plain_norm8(s):
    x = s["x"].float()
    if s["branch"] is not None:
        t = s["branch"].float()
        x = x + (t if s["gate"] is None else s["gate"].float()[s["seq"]] * t)
    d = x - x.mean(-1, keepdim=True) if s["case"]["kind"] == "layer" else x
    y = d * torch.rsqrt((d * d).mean(-1, keepdim=True) + EPS)
    if s["weight"] is not None:
        y = y * s["weight"].float()
    if s["scale"] is not None:
        y = y * (1 + s["scale"].float()[s["seq"]])
    if s["shift"] is not None:
        y = y + s["shift"].float()[s["seq"]]
    got = _eight(s, y)
    return got if s["branch"] is None else {**got, "x": torch.where(s["live"], x, torch.zeros_like(x)).to(s["x"].dtype)}


def _activate(t, act):
    if act == "gelu":
        return 0.5 * t * (1 + torch.tanh(math.sqrt(2 / math.pi) * (t + 0.044715 * t * t * t)))
    return t / (1 + torch.exp(-t)) if act == "silu" else t


def _plain_matmul8(s):
    t = torch.matmul(_from8(*s["a"]), _from8(*s["w"]).T)
    if s["bias"] is not None:
        t = t + s["bias"].float()
    t = _activate(t, s["case"]["act"])
    if s["case"]["out"] == "8bit":
        return _eight(s, t)
    if s["gate"] is not None:
        t = t * s["gate"].float()[s["seq"]]
    if s["residual"] is not None:
        t = t + s["residual"].float()
    return {"o": torch.where(s["live"], t, torch.zeros_like(t)).to(DTYPES[s["case"]["dtype"]])}


# ---- the floor -------------------------------------------------------------------------------------

def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    lens = _ints(case["lens"])
    on = [c == "1" for c in case["active"]] or [True] * len(lens)
    rows = sum(n for n, o in zip(lens, on) if o)
    parts = case.get("parts", "").split()

    def eight(r, dim):
        return r * (dim + -(-dim // BLOCK))

    if case["op"] == "matmul8":
        k, wide = case["k"], case["n"]
        nbytes = eight(rows + wide, k) + (eight(rows, wide) if case["out"] == "8bit" else size * rows * wide)
        nbytes += size * wide * (("bias" in parts) + ("residual" in parts) * rows + ("gate" in parts) * sum(on))
        return {"bytes": nbytes, "flops": 2 * rows * k * wide}
    dim = case["dim"]
    nbytes = size * rows * dim * (3 if "branch" in parts else 1) + eight(rows, dim)
    nbytes += size * dim * (("weight" in parts) + sum(p in parts for p in ("gate", "scale", "shift")) * sum(on))
    return {"bytes": nbytes, "flops": rows * dim * (12 if case["op"] == "norm8" else 3)}


# ---- the definitions in 64 bits --------------------------------------------------------------------

def _exact8(s, y):
    """The same format from the definition: the exponent by its inequality, the codes by torch's rounding of the quotient."""
    rows, dim = y.shape
    blocks = -(-dim // BLOCK)
    codes = torch.zeros(rows, dim, dtype=torch.float64, device=DEV)
    scales = torch.full((-(-blocks // 4), rows, 4), 2.0 ** -127, dtype=torch.float64, device=DEV)
    live = s["live"][:, 0]
    for b in range(blocks):
        part = y[:, b * BLOCK:(b + 1) * BLOCK]
        top = part.abs().amax(1)
        e = torch.ceil(torch.log2(top.clamp_min(1e-300) / TOP))
        e = torch.where(top > TOP * torch.exp2(e), e + 1, e)
        e = torch.where(top <= TOP * torch.exp2(e - 1), e - 1, e).clamp(-126, 127)
        e = torch.where(top > 0, e, torch.zeros_like(e))
        q = part / torch.exp2(e)[:, None]
        # e4m3: steps of 2^-3 of the value's binade, of 2^-9 below 2^-6
        step = torch.exp2(torch.floor(torch.log2(q.abs().clamp_min(2.0 ** -6))) - 3)
        codes[live, b * BLOCK:(b + 1) * BLOCK] = (torch.round(q / step) * step)[live]
        scales[b // 4, live, b % 4] = torch.exp2(e)[live]
    return {"codes": codes, "scales": scales}


def exact(case, seed):
    s = _inputs(case, seed)
    live = s["live"]
    if case["op"] == "quantize8":
        return _exact8(s, s["x"].double())
    if case["op"] == "norm8":
        x = s["x"].double()
        if s["branch"] is not None:
            x = torch.addcmul(x, s["branch"].double(), s["gate"].double()[s["seq"]] if s["gate"] is not None else torch.ones_like(x))
        mean = x.mean(1, keepdim=True) if case["kind"] == "layer" else 0.0
        y = (x - mean) / torch.sqrt((x - mean).square().sum(1, keepdim=True) / x.shape[1] + EPS)
        if s["weight"] is not None:
            y *= s["weight"].double()
        if s["scale"] is not None:
            y += y * s["scale"].double()[s["seq"]]
        if s["shift"] is not None:
            y += s["shift"].double()[s["seq"]]
        got = _exact8(s, y)
        return got if s["branch"] is None else {**got, "x": x * live}

    def values(codes, scales):
        rows, k = codes.shape
        out = torch.empty(rows, k, dtype=torch.float64, device=DEV)
        for b in range(-(-k // BLOCK)):
            cols = slice(b * BLOCK, (b + 1) * BLOCK)
            out[:, cols] = codes[:, cols].double() * scales[b // 4, :, b % 4].double()[:, None]
        return out

    t = values(*s["a"]) @ values(*s["w"]).T
    if s["bias"] is not None:
        t += s["bias"].double()
    if case["act"] == "gelu":
        t = torch.nn.functional.gelu(t, approximate="tanh")
    elif case["act"] == "silu":
        t = torch.nn.functional.silu(t)
    if case["out"] == "8bit":
        return _exact8(s, t)
    if s["gate"] is not None:
        t *= s["gate"].double()[s["seq"]]
    if s["residual"] is not None:
        t += s["residual"].double()
    return {"o": t * live}
