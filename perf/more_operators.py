"""The operators of a layer around its matrix products that this library is measured on:
root-mean-square norm with the residual's addition and an output in 8 bits,
activations kept in 8 bits and read by the backward pass, and rotary positions
with several axes.

A case names the operator (``op``), its sizes, its type and what is asked of it.
Sizes follow the modules of the synthetic workloads: hidden 4096 and FFN 14336
(language model, 32 heads and 8 of keys of 128), 1792 and 15360 (vision encoder,
16 heads of 112), 3584 and 10240 (diffusion transformer, 28 heads of 128), FFN
divided by a tensor-parallel degree of 4; 576 tokens an image, texts up to 8192
tokens, prompts of about 150 and latent videos of up to 64 frames of 1024 patches.

    rms      t = x + residual, y = gamma t rstd, rstd = 1 / sqrt(mean(t^2) + eps),
             y in the inputs' type and in 8 bits
    pack     a matrix to 8 bits and back, through an activation where it was kept before one
    linear   y = residual + act(x w^T + bias) with the value before the activation
             kept in 8 bits, and the gradients from that and from an x kept so
    rotary   queries and keys turned by their tokens' positions along every axis

8 bits: 32 consecutive columns of a row share a scale, the smallest power of two
(2^-126 at least) by which the largest of them divides to at most 448; values are
rounded to nearest even with three bits behind the leading one and steps of at least
2^-9.  A scale is a byte, its exponent plus 127.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}
POSITIONS = {"int32": torch.int32, "int64": torch.int64, "fp32": torch.float32}
EPS = 1e-5
BASE = 10000.0


def listed():
    return [
        # the smallest norm: one token of the language model joins its residual
        dict(name="norm token", op="rms", dtype="bf16", m=1, c=4096, residual=True, packed=False, train=False),
        # a prompt: what the next product's backward needs leaves in 8 bits with it
        dict(name="norm prompt", op="rms", dtype="bf16", m=149, c=4096, residual=True, packed=True, train=True),
        # rows that fill no vector and start at odd addresses, in 32 bits
        dict(name="norm ragged", op="rms", dtype="fp32", m=1201, c=1795, residual=False, packed=True, train=True),
        # the longest video
        dict(name="norm video", op="rms", dtype="bf16", m=65536, c=3584, residual=True, packed=True, train=True),
        # two images' FFN kept before its GELU and restored behind it
        dict(name="pack images", op="pack", dtype="bf16", m=1152, n=3840, act="gelu"),
        # the longest video's FFN
        dict(name="pack video", op="pack", dtype="fp16", m=65536, n=2560, act="none"),
        # sizes that fill no tile, rows that start at odd addresses
        dict(name="kept linear ragged", op="linear", dtype="fp16", m=1201, k=1795, n=1027, act="relu",
             x_act="none", bias=True, residual=True),
        # two images through the vision encoder's FFN-in
        dict(name="kept linear images", op="linear", dtype="bf16", m=1152, k=1792, n=3840, act="gelu",
             x_act="none", bias=True, residual=False),
        # a text at the cap through FFN-out, whose x is the activation of what is kept
        dict(name="kept linear text out", op="linear", dtype="bf16", m=8192, k=3584, n=4096, act="none",
             x_act="silu", bias=False, residual=True),
        # one token far into a text that images precede
        dict(name="rotary token", op="rotary", dtype="bf16", t=1, heads=32, keys=8, dim=128, axes=3,
             interleaved=False, shared=True, positions="int32", start=1000003, train=False),
        # two images by row and column, a head that is no power of two
        dict(name="rotary images", op="rotary", dtype="fp16", t=1152, heads=16, keys=16, dim=112, axes=2,
             interleaved=True, shared=False, positions="int64", start=0, train=True),
        # the longest video by frame, row and column
        dict(name="rotary video", op="rotary", dtype="bf16", t=65536, heads=28, keys=28, dim=128, axes=3,
             interleaved=False, shared=False, positions="fp32", start=0, train=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """Spread over the logarithm; one in three as it falls, the others in whole 64s."""
    v = _log(rng, lo, hi)
    return v if v < 64 or rng.random() < 0.34 else max(64, v // 64 * 64)


def draw(rng):
    op = rng.choice(("rms", "rms", "pack", "linear", "linear", "rotary", "rotary"))
    half = ("bf16", "bf16", "fp16")
    if op == "rms":
        m, c = _size(rng, 1, 65536), _size(rng, 16, 16384)
        dtype = rng.choice(half + ("fp32",))
        m = max(1, min(m, 65536 * 3584 // (c * BYTES[dtype] // 2)))
        return dict(op=op, dtype=dtype, m=m, c=c, residual=rng.random() < 0.6, packed=rng.random() < 0.6,
                    train=rng.random() < 0.7)
    if op == "pack":
        m, n = _size(rng, 1, 65536), _size(rng, 16, 16384)
        dtype = rng.choice(half + ("fp32",))
        m = max(1, min(m, 65536 * 2560 // (n * BYTES[dtype] // 2)))
        return dict(op=op, dtype=dtype, m=m, n=n, act=rng.choice(("none", "none", "relu", "silu", "gelu")))
    if op == "linear":
        m, k, n = _size(rng, 1, 32768), _size(rng, 64, 14336), _size(rng, 64, 15360)
        m = max(1, min(m, 8192 * 3584 * 4096 // (k * n)))
        return dict(op=op, dtype=rng.choice(half), m=m, k=k, n=n, act=rng.choice(("none", "relu", "silu", "gelu")),
                    x_act=rng.choice(("none", "none", "silu", "gelu")), bias=rng.random() < 0.7,
                    residual=rng.random() < 0.4)
    t, heads = _size(rng, 1, 65536), rng.randint(1, 64)
    keys = rng.choice([k for k in range(1, heads + 1) if heads % k == 0])
    dim, axes = 2 * rng.choice((8, 16, 32, 36, 40, 48, 56, 64, 64, 80, 96, 128)), rng.randint(1, 4)
    dtype = rng.choice(half + ("fp32",))
    t = max(1, min(t, 65536 * 56 * 128 // ((heads + keys) * dim * BYTES[dtype] // 2)))
    return dict(op=op, dtype=dtype, t=t, heads=heads, keys=keys, dim=dim, axes=axes, interleaved=rng.random() < 0.5,
                shared=rng.random() < 0.5, positions=rng.choice(("int32", "int32", "int64", "fp32")),
                start=rng.choice((0, 0, 4096, 1000003)), train=rng.random() < 0.7)


def _sections(pairs, axes):
    """Pairs of a head that turn with each axis: even shares, the first axes the larger."""
    return [pairs // axes + (i < pairs % axes) for i in range(axes)]


def _frequencies(case):
    """(axis, radians a position) of each pair: powers of one base over all pairs, or over each axis' own."""
    pairs = case["dim"] // 2
    axis, freq = [], []
    for a, n in enumerate(_sections(pairs, case["axes"])):
        for i in range(n):
            axis.append(a)
            freq.append(BASE ** -(len(freq) / pairs) if case["shared"] else BASE ** -(i / n))
    return axis, freq


def _to8(v):
    """(values, scales) of a float32 matrix."""
    m, n = v.shape
    g = torch.nn.functional.pad(v, (0, -n % 32)).reshape(m, -1, 32)
    f, e = torch.frexp(g.abs().amax(2))                                   # f in [1/2, 1)
    e = torch.clamp_min(torch.where(f > 0.875, e - 8, torch.where(f > 0, e - 9, -126)), -126)
    q = torch.ldexp(g, -e[:, :, None]).reshape(m, -1)[:, :n].to(torch.float8_e4m3fn)
    return q.contiguous(), (e + 127).to(torch.uint8)


def _from8(values, scales):
    n = values.shape[1]
    s = torch.exp2(scales.float() - 127).repeat_interleave(32, 1)[:, :n]
    return values.float() * s


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = DTYPES[case["dtype"]]

    def normal(*shape, scale=1.0, shift=0.0):
        return torch.randn(shape, generator=g, device="cuda").mul_(scale).add_(shift).to(t)

    s = dict(case)
    if case["op"] == "rms":
        m, c = case["m"], case["c"]
        wide = 1 + 3 * torch.rand(c, generator=g, device="cuda").pow_(8)       # a few channels stand out
        s["x"] = (torch.randn((m, c), generator=g, device="cuda") * wide).to(t)
        s["r"] = normal(m, c, scale=2.0) if case["residual"] else None
        s["gamma"] = normal(c, scale=0.2, shift=1.0)
        s["dy"] = normal(m, c, scale=0.1) if case["train"] else None
        s["dt"] = normal(m, c, scale=0.1) if case["train"] and case["residual"] else None
    elif case["op"] == "pack":
        s["x"] = normal(case["m"], case["n"])
    elif case["op"] == "linear":
        m, k, n = case["m"], case["k"], case["n"]
        z = normal(m, k)
        s["x"] = _act(z.float(), case["x_act"]).to(t)
        s["x8"], s["xs"] = _to8(z.float())                                  # kept before x_act
        s["w"] = normal(n, k, scale=1.0 / math.sqrt(k))
        s["b"] = normal(n, scale=0.5) if case["bias"] else None
        s["r"] = normal(m, n) if case["residual"] else None
        s["dy"] = normal(m, n, scale=0.1)
    else:
        tokens, h, k, d = case["t"], case["heads"], case["keys"], case["dim"]
        qkv = normal(tokens, h + 2 * k, d)
        s["q"], s["k"] = qkv[:, :h], qkv[:, h:h + k]
        if case["train"]:
            grad = normal(tokens, h + k, d, scale=0.1)
            s["dq"], s["dk"] = grad[:, :h], grad[:, h:]
        # frames of patches in rows and columns; texts and odd axes count tokens
        i = torch.arange(tokens, device="cuda")
        of = {1: (i,), 2: (i // 24 % 24, i % 24), 3: (i // 1024, i // 32 % 32, i % 32),
              4: (i // 1024, i // 32 % 32, i % 32, i // 1024 % 7)}[case["axes"]]
        s["pos"] = (torch.stack(of, 1) + case["start"] + seed % 5).to(POSITIONS[case["positions"]])
        if case["positions"] == "fp32":
            s["pos"] = s["pos"] * 0.5                                       # frames at half the trained rate
        axis, freq = _frequencies(case)
        s["axis"] = torch.tensor(axis, dtype=torch.int32, device="cuda")
        s["freq"] = torch.tensor(freq, dtype=torch.float64, device="cuda")
    return s


# ------------------------------------------------------------ the plain form

def _act(z, act):
    if act == "relu":
        return torch.clamp_min(z, 0)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.tanh(0.7978845608028654 * (z + 0.044715 * z * z * z)))
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        e = 1 / (1 + torch.exp(-z))
        return e * (1 + z * (1 - e))
    if act == "gelu":
        h = torch.tanh(0.7978845608028654 * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + h) + 0.5 * z * (1 - h * h) * 0.7978845608028654 * (1 + 0.134145 * z * z)
    return torch.ones_like(z)


def _turn(x, cos, sin, interleaved):
    x = x.float()
    a, b = (x[..., 0::2], x[..., 1::2]) if interleaved else x.chunk(2, -1)
    u, v = a * cos - b * sin, a * sin + b * cos
    return torch.stack((u, v), -1).flatten(-2) if interleaved else torch.cat((u, v), -1)


def _plain(s):
    if s["op"] == "rms":
        t = s["x"].dtype
        total = s["x"] if s["r"] is None else (s["x"].float() + s["r"].float()).to(t)
        v, gamma = total.float(), s["gamma"].float()
        rstd = torch.rsqrt((v * v).mean(1, keepdim=True) + EPS)
        xh = v * rstd
        y = xh * gamma
        out = {"y": y.to(t)}
        if s["r"] is not None:
            out["total"] = total
        if s["packed"]:
            out["kept"] = _from8(*_to8(y)).to(torch.bfloat16)
        if s["train"]:
            dy = s["dy"].float()
            h = dy * gamma
            dx = rstd * (h - xh * (h * xh).mean(1, keepdim=True))
            out["dx"] = (dx if s["dt"] is None else dx + s["dt"].float()).to(t)
            out["dgamma"] = (dy * xh).sum(0).to(t)
        return out
    if s["op"] == "pack":
        return {"x": _act(_from8(*_to8(s["x"].float())), s["act"]).to(s["x"].dtype)}
    if s["op"] == "linear":
        t = s["x"].dtype
        w = s["w"].float()
        z = s["x"].float() @ w.T
        if s["b"] is not None:
            z = z + s["b"].float()
        y = _act(z, s["act"])
        if s["r"] is not None:
            y = y + s["r"].float()
        g = s["dy"].float()
        if s["act"] != "none":
            g = g * _act_grad(_from8(*_to8(z)), s["act"])
        x = _act(_from8(s["x8"], s["xs"]), s["x_act"])
        out = {"y": y.to(t), "dx": (g @ w).to(t), "dw": (g.T @ x).to(t)}
        if s["b"] is not None:
            out["db"] = g.sum(0).to(t)
        return out
    angle = s["pos"].double()[:, s["axis"].long()] * s["freq"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    out = {n: _turn(s[n], cos, sin, s["interleaved"]).to(s[n].dtype) for n in ("q", "k")}
    if s["train"]:
        out |= {n: _turn(s[n], cos, -sin, s["interleaved"]).to(s[n].dtype) for n in ("dq", "dk")}
    return out


# ------------------------------------------------------- the library's calls

def _library(s):
    from paper_2504_14145_amd import ops
    if s["op"] == "rms":
        y, total, rstd, kept = ops.rms_norm(s["x"], s["gamma"], EPS, residual=s["r"], packed=s["packed"])
        out = {"y": y}
        if s["r"] is not None:
            out["total"] = total
        if s["packed"]:
            out["kept"] = ops.unpack8(kept, torch.bfloat16)
        if s["train"]:
            out["dx"], out["dgamma"] = ops.rms_norm_backward(s["dy"], total, rstd, s["gamma"], dtotal=s["dt"])
        return out
    if s["op"] == "pack":
        return {"x": ops.unpack8(ops.pack8(s["x"]), s["x"].dtype, act=s["act"])}
    if s["op"] == "linear":
        pre = ops.Packed8.empty(s["m"], s["n"], s["x"].device) if s["act"] != "none" else None
        out = {"y": ops.linear(s["x"], s["w"], s["b"], act=s["act"], residual=s["r"], pre=pre)}
        dx, dw, db = ops.linear_backward(s["dy"], ops.Packed8(s["x8"], s["xs"]), s["w"], act=s["act"], pre=pre,
                                         bias=s["b"] is not None, x_act=s["x_act"])
        out["dx"], out["dw"] = dx, dw
        if db is not None:
            out["db"] = db
        return out
    out = {}
    out["q"], out["k"] = ops.rotary(s["q"], s["pos"], s["freq"], s["axis"], k=s["k"], interleaved=s["interleaved"])
    if s["train"]:
        out["dq"], out["dk"] = ops.rotary_backward(s["dq"], s["pos"], s["freq"], s["axis"], dk=s["dk"],
                                                   interleaved=s["interleaved"])
    return out


def run(state):
    return _library(state) if own else _plain(state)


def work(case):
    e = BYTES[case["dtype"]]
    if case["op"] == "rms":
        mc, c = case["m"] * case["c"], case["c"]
        values = mc * (4 if case["residual"] else 2) + c
        more = 2 * mc if case["packed"] else 0                               # the kept values, in 16 bits
        if case["train"]:
            values += mc * (3 if case["residual"] else 2) + c
        return {"bytes": e * values + more, "flops": mc * (4 + (2 if case["packed"] else 0) + (9 if case["train"] else 0))}
    if case["op"] == "pack":
        return {"bytes": 2 * e * case["m"] * case["n"], "flops": 4 * case["m"] * case["n"]}
    if case["op"] == "linear":
        m, k, n = case["m"], case["k"], case["n"]
        values = 2 * m * k + 2 * n * k + m * n * (3 if case["residual"] else 2) + (2 * n if case["bias"] else 0)
        return {"bytes": e * values + m * k + m * ((k + 31) // 32), "flops": 6 * m * n * k}
    all_ = case["t"] * (case["heads"] + case["keys"]) * case["dim"] * (2 if case["train"] else 1)
    return {"bytes": 2 * e * all_ + case["t"] * case["axes"] * (8 if case["positions"] == "int64" else 4),
            "flops": 3 * all_}


# ------------------------------------------------- the definition in 64 bits

def _round8(v):
    """The values that 8 bits hold of a 64-bit matrix, by arithmetic."""
    m, n = v.shape
    most = torch.zeros((m, -(-n // 32)), dtype=torch.float64, device=v.device)
    most.scatter_reduce_(1, (torch.arange(n, device=v.device) // 32).expand(m, n), v.abs(), "amax")
    e = torch.ceil(torch.log2(most / 448)).clamp_(-126, 127)                # log2 rounds: put right below
    e = torch.where(most > 448 * torch.exp2(e), e + 1, torch.where((most <= 224 * torch.exp2(e)) & (e > -126), e - 1, e))
    scale = torch.exp2(e).repeat_interleave(32, 1)[:, :n]
    q = v / scale
    step = torch.exp2(torch.floor(torch.log2(q.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(q / step) * step * scale


def _sigmoid64(z):
    return torch.where(z >= 0, 1 / (1 + torch.exp(-z.abs())), torch.exp(-z.abs()) / (1 + torch.exp(-z.abs())))


def _act64(z, act):
    """act(z) and its derivative."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return torch.where(z > 0, z, 0.0), torch.where(z > 0, 1.0, 0.0).double()
    if act == "silu":
        e = _sigmoid64(z)
        return z * e, e + z * e * (1 - e)
    a = math.sqrt(2 / math.pi)                # 1/2 (1 + tanh u) = sigmoid(2 u)
    e = _sigmoid64(2 * a * (z + 0.044715 * z ** 3))
    return z * e, e + z * e * (1 - e) * 2 * a * (1 + 3 * 0.044715 * z ** 2)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rms":
        v = s["x"].double()
        out = {}
        if s["r"] is not None:
            out["total"] = v + s["r"].double()
            v = (s["x"].double() + s["r"].double()).to(s["x"].dtype).double()      # the norm is that of what is stored
        gamma = s["gamma"].double()
        inv = 1 / torch.sqrt((v ** 2).sum(1, keepdim=True) / case["c"] + EPS)
        y = v * inv * gamma
        out["y"] = y
        if case["packed"]:
            out["kept"] = _round8(y)
        del y
        if case["train"]:
            h = s["dy"].double() * gamma
            dot = (h * v).sum(1, keepdim=True) / case["c"]
            out["dx"] = inv * h - v * (inv ** 3 * dot)
            if s["dt"] is not None:
                out["dx"] += s["dt"].double()
            out["dgamma"] = (s["dy"].double() * v * inv).sum(0)
        return out
    if case["op"] == "pack":
        return {"x": _act64(_round8(s["x"].double()), case["act"])[0]}
    if case["op"] == "linear":
        x, w = s["x"].double(), s["w"].double()
        z = torch.mm(x, w.t().contiguous())
        if s["b"] is not None:
            z += s["b"].double()
        y = _act64(z, case["act"])[0]
        if s["r"] is not None:
            y = y + s["r"].double()
        g = s["dy"].double()
        if case["act"] != "none":
            g = g * _act64(_round8(z), case["act"])[1]
        scale = torch.pow(2.0, s["xs"].double() - 127)
        kept = s["x8"].double() * scale[:, torch.arange(case["k"], device="cuda") // 32]
        kept = _act64(kept, case["x_act"])[0]
        out = {"y": y, "dx": torch.mm(g, w), "dw": torch.mm(g.t().contiguous(), kept)}
        if s["b"] is not None:
            out["db"] = g.sum(0)
        return out
    out = {}
    pairs = case["dim"] // 2
    first = torch.arange(pairs, device="cuda") * (2 if case["interleaved"] else 1)
    second = first + (1 if case["interleaved"] else pairs)
    place = s["pos"].double().index_select(1, s["axis"])
    turn = torch.polar(torch.ones_like(place), place * s["freq"])[:, None]
    for name in ("q", "k") + (("dq", "dk") if case["train"] else ()):
        v = s[name].double()
        z = torch.complex(v[..., first], v[..., second]) * (turn.conj() if name[0] == "d" else turn)
        v[..., first], v[..., second] = z.real, z.imag
        out[name] = v
    return out
