"""What stands around a linear layer with narrow operands when it is a block of a model that is trained and served: norms with the residual
stream, products with an epilogue, the clipping of gradients.

`listed()` names twelve passes over the range of real use, `draw()` draws more of the same ranges, `prepare()` makes what
the program holds before the call, `run()` is one pass (the plain form in 32 bits, or with `own` the library's entry
points), `exact()` the same outputs from the definitions in 64 bits, `work()` what a pass cannot do without.

A case's "op" is one of
  norm     s = r + scale gate after y / rms(y), then before s / rms(s) as numbers, in 8 bits, or both
  dnorm    its gradients: of r, y (numbers and 8 bits), both weights and the gate
  linear   y = residual + scale act(z), z = x w^T + bias, of 8-bit operands; z is kept where a backward pass wants it
  dlinear  dz = scale dy act'(z) as numbers and in 8 bits, and dbias, its sums over the rows
  packed   the first of these with packed codebook weights
  clip     the norm of all gradients of a model, and the gradients times min(1, most / norm)

A gate has G rows of D, each for M / G rows of y (G = 0: no gate); `after` and `before` are norm weights of D, or missing.
8-bit blocks of 1 x 128: a = largest finite |x| of a block, e = the smallest integer with a <= top * 2^e (top: the format's
largest number), at least -126, and 0 where a = 0; the scale is 2^e, an element's code is x / 2^e rounded to nearest even.
"""
import math

import torch

own = False

CODE = {"E4M3": torch.float8_e4m3fn, "E5M2": torch.float8_e5m2}
FLOAT = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6


def _norm(name, op, M, D, **more):
    c = dict(name=name, op=op, M=M, D=D, pad=0, y="bf16", r="bf16", G=0, scale=1.0, after=True, before=True, numbers="", fmt="E4M3" if op == "norm" else "E5M2")
    c.update(more)
    return c


def _linear(name, op, M, N, K, **more):
    c = dict(name=name, op=op, M=M, N=N, K=K, pad=0, act="none", bias=True, residual=False, scale=1.0, keep=False, out="bf16", fmt="E5M2" if op == "dlinear" else "E4M3")
    c.update(more)
    return c


def listed():
    return [
        # one token between two blocks: nothing to do but the launch
        _norm("norm_token", "norm", 1, 4096),
        # a full batch of tokens of a 70B-shaped model, residual stream in 32 bits
        _norm("norm_batch", "norm", 8192, 8192, r="f32"),
        # gradients of an odd microbatch, three sequences with a gate each, all in 32 bits
        _norm("dnorm_ragged", "dnorm", 777, 5024, y="f32", r="f32", G=3, scale=0.5),
        # gradients over a full batch, a learnt gate for each channel
        _norm("dnorm_batch", "dnorm", 8192, 4096, G=1),
        # one token through an MLP down-projection onto the residual stream
        _linear("linear_token", "linear", 1, 4096, 11008, residual=True),
        # the up-projection of a training batch: activation in the epilogue, what it took kept for the backward pass
        _linear("linear_batch", "linear", 4096, 11008, 4096, act="gelu", keep=True),
        # gradient of an odd microbatch's activation, in 32 bits
        _linear("dlinear_ragged", "dlinear", 301, 1531, 0, act="gelu_tanh", out="f32"),
        # gradient of a full batch's activation
        _linear("dlinear_batch", "dlinear", 8192, 11008, 0, act="gelu"),
        # one token with the packed pair that the search writes, onto the residual stream
        _linear("packed_token", "packed", 1, 4096, 11008, residual=True, bits=4, g=16, word="S1E5M5", two=True, k=2),
        # a prompt with it, activation in the epilogue
        _linear("packed_prompt", "packed", 2048, 11008, 4096, act="silu", bits=4, g=16, word="UE4M3", two=True, k=0),
        # gradients of two small layers: latency
        dict(name="clip_small", op="clip", layers=2, width=768, hidden=2048, dtype="f32", out="f32", most=1.0, level=1e-3),
        # gradients of eight layers, 1.1 G of them, into bf16 for an optimizer that holds them so
        dict(name="clip_large", op="clip", layers=8, width=4096, hidden=11008, dtype="f32", out="bf16", most=1.0, level=1e-3),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above: sizes spread over their logarithm, odd ones among them."""
    op = rng.choice(["norm", "dnorm", "linear", "dlinear", "packed", "clip"])
    odd = lambda n: n if rng.random() < 0.5 else max(64, n // 64 * 64)  # noqa: E731
    pad, M = rng.choice([0, 0, 8 * rng.randrange(1, 16)]), _log_int(rng, 1, 8192)
    scale = rng.choice([1.0, 1.0, 0.5, 0.1])
    if op == "clip":
        c = dict(name="", op=op, layers=rng.randrange(1, 9), width=odd(_log_int(rng, 64, 4096)), hidden=odd(_log_int(rng, 128, 11008)), dtype=rng.choice(["f32", "f32", "bf16"]),
                 out="", most=rng.choice([1.0, 1e3]), level=1e-3)
        c.update(out=rng.choice([c["dtype"], "bf16"]))
    elif op in ("norm", "dnorm"):
        G = rng.choice([0, 0, 1, 2, 4, M])
        M, D = max(1, M // max(G, 1)) * max(G, 1), odd(_log_int(rng, 64, 12288))
        M = M if M * D <= 1 << 26 else G * max(1, (1 << 26) // D // G) if G else (1 << 26) // D
        G = M if G > 4 else G
        after, before = rng.random() < 0.7, rng.random() < 0.8
        y = rng.choice(["bf16", "bf16", "f32"])
        c = _norm("", op, M, D, pad=pad, y=y, r=rng.choice([y, "f32"]), G=G, scale=scale, after=after, before=before)
        if op == "norm":
            c.update(numbers=rng.choice(["", "", "bf16", "f32"]) if before else "", fmt=rng.choice(["E4M3", "E4M3", "E5M2"]) if before else "")
    elif op == "dlinear":
        c = _linear("", op, M, odd(_log_int(rng, 256, 12288)), 0, pad=pad, act=rng.choice(["relu", "silu", "gelu", "gelu_tanh"]), scale=scale, out=rng.choice(["bf16", "bf16", "f32"]),
                    bias=rng.random() < 0.8, fmt=rng.choice(["E4M3", "E5M2"]))
    else:
        K, N = odd(_log_int(rng, 256, 12288)), odd(_log_int(rng, 256, 12288))
        N = max(64, min(N, int(1.5e11 / M / K)))
        c = _linear("", op, M, N, K, pad=pad, act=rng.choice(["none", "relu", "silu", "gelu", "gelu_tanh"]), bias=rng.random() < 0.7, residual=rng.random() < 0.5, scale=scale)
        if op == "linear":
            c.update(keep=rng.random() < 0.3, out=rng.choice(["bf16", "bf16", "f32"]), fmt=rng.choice(["E4M3", "E4M3", "E5M2"]))
        else:
            g, two = rng.choice([8, 16, 16, 32, 64]), rng.random() < 0.7
            c.update(K=max(1, K // g) * g, g=g, bits=rng.choice([3, 4, 4, 4, 5]), two=two, word=rng.choice(["UE4M3", "S1E5M5"] if two else ["UE4M3", "UE4M4", "S1E5M5"]), k=rng.randrange(0, 4))
    del c["name"]
    return c


# ---- inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rows(gen, M, K, dtype, pad, scale=1.0):
    """[M, K] with heavy tails and a few columns of outliers, as activations have; `pad` elements between the rows."""
    x = torch.randn((M, K), generator=gen, device="cuda")
    x *= torch.exp(0.5 * torch.randn((1, K), generator=gen, device="cuda")) * scale
    x *= torch.where(torch.rand((1, K), generator=gen, device="cuda") < 0.002, 20.0, 1.0)
    step = -(-(K + pad) // 8) * 8                                       # (rows start on 16 bytes)
    buf = torch.zeros((M, step), dtype=dtype, device="cuda")
    buf[:, :K] = x
    return buf[:, :K]


def _kept(gen, M, K, rows, fmt, scale=1.0):
    """What a program has kept in 8 bits: (codes, scales), rows of codes a multiple of 16 apart, rows of scales of 4."""
    codes, scales = _plain_blocks(_rows(gen, M, K, torch.bfloat16, 0, scale).float(), rows, fmt)
    return _spaced(codes, 16), _spaced(scales, 4)


def _spaced(t, unit):
    buf = torch.zeros((t.shape[0], -(-t.shape[1] // unit) * unit), dtype=torch.uint8, device="cuda")
    buf[:, :t.shape[1]] = t.view(torch.uint8)
    return buf.view(t.dtype)[:, :t.shape[1]]


# scale words of packed weights: sign, exponent and mantissa bits, container bits, bias; a metabit is left where a pair is packed
WORDS = {"UE4M3": (0, 4, 3, 8, 7), "S1E5M5": (1, 5, 5, 12, 15), "UE4M4": (0, 4, 4, 8, 7)}


def _bits_of(case):
    """Bit positions of a scale word: (sign, lowest magnitude bit, selector)."""
    w, x, y, b, _ = WORDS[case["word"]]
    m = b - w - x - y
    return b - 1, m if w else max(m - 1, 0), m - 1 if w else b - 1


def _codebook(alpha, c, bits):
    """A sinh grid of 2^bits entries, largest magnitude 1, ascending."""
    t = torch.linspace(-1, 1, 1 << bits, dtype=torch.float64)
    v = torch.sinh(alpha * t) + c
    return (v / v.abs().max()).float()


def _layer(case, gen):
    N, K, g, n = case["N"], case["K"], case["g"], case["bits"]
    w, x, y, b, bias = WORDS[case["word"]]
    sign, low, sel = _bits_of(case)
    count = N * K // g
    tables = [_codebook(1.5, -0.02, n), _codebook(0.4, 0.05, n)][:2 if case["two"] else 1]
    mid = ((tables[0][1:] + tables[0][:-1]) / 2).cuda()
    codes = torch.bucketize(0.45 * torch.randn((count, g), generator=gen, device="cuda"), mid).long()
    word = torch.randint((bias - 4) << y, (bias + 1) << y, (count,), generator=gen, device="cuda") << low
    if w:
        word |= torch.randint(0, 2, (count,), generator=gen, device="cuda") << sign
    if case["two"]:
        word |= torch.randint(0, 2, (count,), generator=gen, device="cuda") << sel
    eight = (codes.view(count, g // 8, 8) << (n * torch.arange(8, device="cuda"))).sum(-1)
    payload = (eight[..., None] >> (8 * torch.arange(n, device="cuda")) & 255).to(torch.uint8).view(count, g * n // 8)
    return dict(words=word.to(torch.int16), payload=payload, tables=tables)


def prepare(case, seed):
    gen, op, s = _gen(seed), case["op"], dict(case=case)
    if op == "clip":
        shapes = [(case["hidden"], case["width"]), (case["hidden"], case["width"]), (case["width"], case["hidden"]), (case["hidden"],), (case["width"],), (case["width"],)] * case["layers"]
        s["grads"] = [(case["level"] * torch.randn(z, generator=gen, device="cuda") * (1 + i % 5)).to(FLOAT[case["dtype"]]) for i, z in enumerate(shapes)]
        s["outs"] = [torch.empty_like(g, dtype=FLOAT[case["out"]]) for g in s["grads"]]
    elif op in ("norm", "dnorm"):
        M, D, G, pad, ty, tr = case["M"], case["D"], case["G"], case["pad"], FLOAT[case["y"]], FLOAT[case["r"]]
        weight = lambda: 1 + 0.2 * torch.randn(D, generator=gen, device="cuda")  # noqa: E731
        s.update(y=_rows(gen, M, D, ty, pad, 0.3), r=_rows(gen, M, D, tr, pad), after=weight() if case["after"] else None, before=weight() if case["before"] else None)
        s["gate"] = (0.5 * torch.randn((G, D), generator=gen, device="cuda")).to(torch.float32 if G == 1 else ty) if G else None
        if op == "dnorm":                                              # (r stands for the stored sum)
            s.update(ds=_rows(gen, M, D, tr, pad, 1e-4), dn=_rows(gen, M, D, ty, pad, 1e-4) if case["before"] else None)
    else:
        M, N, K, pad, out = case["M"], case["N"], case["K"], case["pad"], FLOAT[case["out"]]
        if op == "dlinear":
            s.update(dy=_rows(gen, M, N, out, pad, 1e-4), z=_rows(gen, M, N, out, pad))
        else:
            if op == "linear":
                s.update(x=_kept(gen, M, K, 1, case["fmt"]), w=_kept(gen, N, K, 128, "E4M3", 0.02))
            else:
                s.update(x=_rows(gen, M, K, torch.bfloat16, pad, 0.1), **_layer(case, gen))
            s["bias"] = 0.5 * torch.randn(N, generator=gen, device="cuda") if case["bias"] else None
            s["residual"] = _rows(gen, M, N, out, pad) if case["residual"] else None
    if own:
        import paper_2605_14929_amd as sop
        s["sop"], s["ctx"] = sop, sop.Context(0)
        if op == "packed":                                             # the layer as a serving program holds it
            s["layer"] = sop.PackedWeights(s["words"], s["payload"], case["N"], case["K"], case["g"], case["bits"], sop.ScaleFmt(*WORDS[case["word"]][:5], -1),
                                           [t.numpy() for t in s["tables"]], k=case["k"])
    return s


# ---- the plain form

def _plain_blocks(x, rows, fmt):
    """32-bit x into (codes, scales)."""
    M, K = x.shape
    R, B = -(-M // rows), -(-K // 128)
    big = torch.where(x.abs() < math.inf, x.abs(), torch.zeros((), device=x.device))
    big = torch.nn.functional.pad(big, (0, B * 128 - K, 0, R * rows - M)).view(R, rows, B, 128).amax((1, 3))
    m, e = torch.frexp(big)                                            # big = m 2^e, m in [1/2, 1); the largest number is 7/8 2^(9 or 16)
    e = torch.where(big > 0, e - (9 if fmt == "E4M3" else 16) + (m > 0.875), 0).clamp(-126, 127)
    up = torch.exp2(-e.float()).repeat_interleave(rows, 0)[:M].repeat_interleave(128, 1)[:, :K]
    return (x * up).to(CODE[fmt]), (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _plain_values(codes, scales, rows):
    M, K = codes.shape
    return codes.float() * scales.float().repeat_interleave(rows, 0)[:M].repeat_interleave(128, 1)[:, :K]


def _plain_packed(s):
    case = s["case"]
    w, x, y, b, bias = WORDS[case["word"]]
    sign, low, sel = _bits_of(case)
    n, g = case["bits"], case["g"]
    word = s["words"].int() & 0xFFFF
    mag = word >> low & (1 << x + y) - 1
    e, f = mag >> y, mag & (1 << y) - 1
    scale = torch.where(e > 0, f + (1 << y), f).float() * torch.exp2((e.clamp(min=1) - bias - y - case["k"]).float())
    if w:
        scale = torch.where(word >> sign & 1 > 0, -scale, scale)
    eight = (s["payload"].view(-1, n).long() << (8 * torch.arange(n, device="cuda"))).sum(-1, keepdim=True)
    codes = (eight >> (n * torch.arange(8, device="cuda")) & (1 << n) - 1).view(-1, g)
    values = s["tables"][0].cuda()[codes]
    if case["two"]:
        values = torch.where((word >> sel & 1 > 0)[:, None], s["tables"][1].cuda()[codes], values)
    return (values * scale[:, None]).view(case["N"], case["K"])


def _gate_rows(s):
    case = s["case"]
    g = case["scale"] * s["gate"].float() if s["gate"] is not None else torch.full((1, case["D"]), case["scale"], device="cuda")
    return g.repeat_interleave(case["M"] // len(g), 0)


def _plain_norm(s):
    case, y = s["case"], s["y"].float()
    v = _gate_rows(s) * y
    if case["after"]:
        v = v * s["after"] * torch.rsqrt((y * y).mean(1, keepdim=True) + EPS)
    total = s["r"].float() + v
    out = [total.to(s["r"].dtype)]
    if case["before"]:
        n = total * torch.rsqrt((total * total).mean(1, keepdim=True) + EPS) * s["before"]
        out += ([n.to(FLOAT[case["numbers"]])] if case["numbers"] else []) + list(_plain_blocks(n, 1, case["fmt"]))
    return out


def _plain_dnorm(s):
    case, total, y, dr = s["case"], s["r"].float(), s["y"].float(), s["ds"].float()
    out = {}
    if case["before"]:
        dn, inv = s["dn"].float(), torch.rsqrt((total * total).mean(1, keepdim=True) + EPS)
        h, p = total * inv, s["before"] * dn
        dr = dr + inv * (p - h * (p * h).mean(1, keepdim=True))
        out["dbefore"] = (dn * h).sum(0)
    gate, x, after = _gate_rows(s), y, 1.0
    if case["after"]:
        inv, after = torch.rsqrt((y * y).mean(1, keepdim=True) + EPS), s["after"]
        x = y * inv
        out["dafter"] = (gate * dr * x).sum(0)
    q = gate * after * dr
    dy = inv * (q - x * (q * x).mean(1, keepdim=True)) if case["after"] else q
    if case["G"]:
        out["dgate"] = (case["scale"] * after * dr * x).view(case["G"], -1, case["D"]).sum(1).to(s["gate"].dtype)
    return dict(out, dr=dr.to(s["r"].dtype), dy=dy.to(s["y"].dtype), dy8=_plain_blocks(dy, 1, case["fmt"]))


def _act(act, z):
    if act == "relu":
        return z.clamp(min=0)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh((2 / math.pi) ** 0.5 * (z + 0.044715 * z ** 3)))
    return z


def _dact(act, z):
    if act == "relu":
        return (z > 0).float()
    if act == "silu":
        q = 1 / (1 + torch.exp(-z))
        return q * (1 + z * (1 - q))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    if act == "gelu_tanh":
        t = torch.tanh((2 / math.pi) ** 0.5 * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * (2 / math.pi) ** 0.5 * (1 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


def _plain(s):
    case = s["case"]
    op = case["op"]
    if op == "norm":
        return _plain_norm(s)
    if op == "dnorm":
        return _plain_dnorm(s)
    if op == "clip":
        norm = torch.stack([g.double().square().sum() for g in s["grads"]]).sum().sqrt()
        c = (case["most"] / norm).clamp(max=1.0).float()
        return [norm.float().view(1)] + [(g.float() * c).to(o.dtype) for g, o in zip(s["grads"], s["outs"])]
    if op == "dlinear":
        dz = case["scale"] * s["dy"].float() * _dact(case["act"], s["z"].float())
        return [dz.to(s["dy"].dtype), *_plain_blocks(dz, 1, case["fmt"])] + ([dz.sum(0)] if case["bias"] else [])
    z = _plain_values(*s["x"], 1) @ _plain_values(*s["w"], 128).t() if op == "linear" else s["x"].float() @ _plain_packed(s).t()
    if case["bias"]:
        z = z + s["bias"]
    y = case["scale"] * _act(case["act"], z)
    if case["residual"]:
        y = y + s["residual"].float()
    return [y.to(FLOAT[case["out"]])] + ([z.to(FLOAT[case["out"]])] if case["keep"] else [])


# ---- the library

def _own(s):
    case, sop, ctx = s["case"], s["sop"], s["ctx"]
    op = case["op"]
    if op == "norm":
        total, n, n8 = ctx.residual_norm(s["r"], s["y"], after=s["after"], gate=s["gate"], scale=case["scale"], before=s["before"], eps=EPS,
                                         dtype=FLOAT.get(case["numbers"]), fmt=CODE.get(case["fmt"]) if case["before"] else None)
        return [total] + ([n] if case["numbers"] else []) + ([n8.codes, n8.scales] if case["before"] else [])
    if op == "dnorm":
        d = ctx.residual_norm_grad(s["ds"], s["dn"], s["r"] if case["before"] else None, before=s["before"], y=s["y"], after=s["after"], gate=s["gate"],
                                   scale=case["scale"], eps=EPS, fmt=CODE[case["fmt"]])
        out = {k: v for k, v in (("dbefore", d.dbefore), ("dafter", d.dafter), ("dgate", d.dgate)) if v is not None}
        return dict(out, dr=d.dr, dy=d.dy, dy8=(d.dy8.codes, d.dy8.scales))
    if op == "clip":
        return [ctx.clip_grads(s["grads"], case["most"], out=s["outs"])] + s["outs"]
    act = {"none": None, "relu": sop.RELU, "silu": sop.SILU, "gelu": sop.GELU, "gelu_tanh": sop.GELU_TANH}[case["act"]]
    if op == "dlinear":
        dz, dz8, dbias = ctx.fp8_linear_grad(s["dy"], s["z"], act=act, scale=case["scale"], bias=case["bias"], fmt=CODE[case["fmt"]])
        return [dz, dz8.codes, dz8.scales] + ([dbias] if case["bias"] else [])
    more = dict(bias=s["bias"], act=act, residual=s["residual"], scale=case["scale"])
    if op == "linear":
        y = ctx.fp8_linear(sop.Fp8Blocks(*s["x"]), sop.Fp8Blocks(*s["w"], rows=128), keep=case["keep"], dtype=FLOAT[case["out"]], **more)
        return list(y) if case["keep"] else [y]
    return [ctx.packed_linear(s["x"], s["layer"], **more)]


def run(state):
    return _own(state) if own else _plain(state)


# ---- in 64 bits, from the definitions

def _exact_blocks(x, fmt):
    """(codes' values, scales' values) of finite 64-bit x."""
    top, least, mant = (448.0, -6, 3) if fmt == "E4M3" else (57344.0, -14, 2)
    col = torch.arange(x.shape[1], device="cuda") // 128
    a = torch.zeros((x.shape[0], int(col[-1]) + 1), dtype=torch.float64, device="cuda").scatter_reduce_(1, col.expand(x.shape), x.abs(), "amax")
    e = torch.ceil(torch.log2(torch.where(a > 0, a, top) / top))
    e = torch.where(a > top * torch.exp2(e), e + 1, e)
    e = torch.where(a <= top * torch.exp2(e - 1), e - 1, e)            # (the logarithm may be off by one at a power of two)
    e = torch.where(a > 0, e.clamp(min=-126), 0.0)
    v = x / torch.exp2(e)[:, col]
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** (least - 1)))).clamp(min=least) - mant)
    return torch.round(v / step) * step, torch.exp2(e)


def _exact_values(codes, scales, rows):
    M, K = codes.shape
    row, col = torch.arange(M, device="cuda") // rows, torch.arange(K, device="cuda") // 128
    return codes.double() * scales.double()[row][:, col]


def _exact_packed(s):
    case = s["case"]
    w, x, y, b, bias = WORDS[case["word"]]
    sign, low, sel = _bits_of(case)
    n, g = case["bits"], case["g"]
    word = s["words"].long() & 0xFFFF
    value = torch.tensor([(q & (1 << y) - 1) * 2.0 ** (1 - bias - y) if q >> y == 0 else (1 + (q & (1 << y) - 1) / 2 ** y) * 2.0 ** ((q >> y) - bias)
                          for q in range(1 << x + y)], dtype=torch.float64, device="cuda") / 2.0 ** case["k"]
    scale = value[(word >> low) % (1 << x + y)]
    if w:
        scale = scale * (1 - 2 * (word >> sign & 1))
    bit = (s["payload"][:, :, None] >> torch.arange(8, device="cuda") & 1).view(-1, g, n)
    code = (bit.short() << torch.arange(n, device="cuda").short()).sum(-1)
    both = torch.stack(s["tables"]).double().cuda()
    pick = (word >> sel & 1) if case["two"] else torch.zeros_like(word)
    return (both[pick[:, None], code] * scale[:, None]).view(case["N"], case["K"])


def _exact_norm(s):
    """A layer of the definitions, with autograd in 64 bits where the case asks for gradients."""
    case, grad = s["case"], s["case"]["op"] == "dnorm"
    M, D, G = case["M"], case["D"], max(case["G"], 1)
    wide = {k: s[k].double().requires_grad_(grad) for k in ("y", "r", "after", "before", "gate") if s[k] is not None}
    unit = lambda t: t / torch.sqrt(t.square().sum(1, keepdim=True) / D + EPS)  # noqa: E731
    with torch.set_grad_enabled(grad):
        y = unit(wide["y"]) * wide["after"] if case["after"] else wide["y"]
        if case["G"]:
            y = (y.view(G, M // G, D) * wide["gate"][:, None]).view(M, D)
        y = case["scale"] * y
        if not grad:
            total = wide["r"] + y
            if not case["before"]:
                return [total]
            n = unit(total) * wide["before"]
            return [total] + ([n] if case["numbers"] else []) + list(_exact_blocks(n, case["fmt"]))
        dr = s["ds"].double()
        if case["before"]:                                             # the sum as it is stored is where the second norm is differentiated
            (unit(wide["r"]) * wide["before"]).backward(s["dn"].double())
            dr = dr + wide["r"].grad
        y.backward(dr)
    out = {"d" + k: wide[k].grad for k in ("before", "after", "gate") if k in wide}
    return dict(out, dr=dr, dy=wide["y"].grad, dy8=_exact_blocks(wide["y"].grad, case["fmt"]))


def _exact_act(act, z):
    if act == "relu":
        return torch.where(z > 0, z, 0.0)
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return z * torch.special.ndtr(z)
    if act == "gelu_tanh":
        return z * torch.sigmoid((8 / math.pi) ** 0.5 * (z + 0.044715 * z * z * z))
    return z * 1.0


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("norm", "dnorm"):
        return _exact_norm(s)
    if op == "clip":
        norm = math.sqrt(math.fsum(float(torch.linalg.vector_norm(g, dtype=torch.float64)) ** 2 for g in s["grads"]))
        return [torch.tensor([norm], dtype=torch.float64)] + [g.double() * min(1.0, case["most"] / norm) for g in s["grads"]]
    if op == "dlinear":
        z = s["z"].double().requires_grad_()
        (case["scale"] * _exact_act(case["act"], z)).backward(s["dy"].double())
        return [z.grad, *_exact_blocks(z.grad, case["fmt"])] + ([z.grad.sum(0)] if case["bias"] else [])
    z = _exact_values(*s["x"], 1) @ _exact_values(*s["w"], 128).t() if op == "linear" else s["x"].double() @ _exact_packed(s).t()
    z = z + (s["bias"].double() if case["bias"] else 0.0)
    y = case["scale"] * _exact_act(case["act"], z) + (s["residual"].double() if case["residual"] else 0.0)
    return [y, z] if case["keep"] else [y]


def work(case):
    """Each input read once, each output written once; two operations a multiply-add, ten to forty an element of the element-wise passes."""
    op = case["op"]
    size = lambda k: 2 if case[k] == "bf16" else 4  # noqa: E731
    tok = 1 + 1 / 128
    if op == "clip":
        n = case["layers"] * (3 * case["width"] * case["hidden"] + case["hidden"] + 2 * case["width"])
        return {"bytes": n * (size("dtype") + size("out")), "flops": 3 * n}
    if op in ("norm", "dnorm"):
        n, gate = case["M"] * case["D"], case["G"] * case["D"] * (4 if case["G"] == 1 else size("y"))
        if op == "norm":
            return {"bytes": n * (size("y") + 2 * size("r") + (size("numbers") if case["numbers"] else 0) + (tok if case["before"] else 0)) + gate, "flops": 16 * n}
        return {"bytes": n * (2 * size("y") + 2 * size("r") + (size("y") + size("r") if case["before"] else 0) + tok) + 2 * gate, "flops": 40 * n}
    M, N, K, o = case["M"], case["N"], case["K"], size("out")
    if op == "dlinear":
        return {"bytes": M * N * (3 * o + tok), "flops": 30 * M * N}
    out = M * N * o * (1 + case["residual"] + case["keep"])
    w, x = (N * K * (1 + 1 / 128 ** 2), M * K * tok) if op == "linear" else (N * K * (case["bits"] / 8 + 2 / case["g"]), M * K * 2)
    return {"bytes": w + x + out, "flops": 2 * M * N * K}
