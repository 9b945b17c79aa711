"""The products of a linear layer with narrow operands, forward and backward, as a user's program calls them.

`listed()` names twelve passes over the range of real use, `draw()` draws more of the same ranges, `prepare()` makes what
the program holds before the call, `run()` is one pass (the plain form in 32 bits, or with `own` the library's entry
points), `exact()` the same outputs from the definitions in 64 bits, `work()` what a pass cannot do without.

A case's "op" is one of
  quantize   8-bit floats with one power-of-two scale for each block of 128 (1 x 128, or 128 x 128 for weights)
  product    y = x w^T of two such operands
  dinput     the input gradient of that product: the output gradient goes to 8 bits, then dx = dy w
  dweight    its weight gradient from the 8-bit checkpoint of x: dw = dy^T x
  gated      h = silu(gate) * up into 8 bits, and checkpoints of gate and up in 8 bits
  dgated     the gradients of gate and up from those checkpoints, as numbers and in 8 bits
  packed     y = x w^T with packed codebook weights (scale words with sign and selector, n-bit codes, one or two codebooks)

Blocks: a = largest finite |x| of a block, e = the smallest integer with a <= top * 2^e (top: the format's largest
number), at least -126, and 0 where a = 0; the scale is 2^e, an element's code is x / 2^e rounded to nearest even.
"""
import math

import torch

own = False

CODE = {"E4M3": torch.float8_e4m3fn, "E5M2": torch.float8_e5m2}
FLOAT = {"bf16": torch.bfloat16, "f32": torch.float32}
# scale words of packed weights: sign, exponent and mantissa bits, container bits, bias; a metabit is left where a pair is packed
WORDS = {"UE4M3": (0, 4, 3, 8, 7), "S1E5M5": (1, 5, 5, 12, 15), "UE4M4": (0, 4, 4, 8, 7)}


def _case(name, op, M, N, K, **more):
    c = dict(name=name, op=op, M=M, N=N, K=K, pad=0, dtype="bf16", fmt="E4M3")
    c.update(more)
    return c


def listed():
    return [
        # one token's activations on their way into a product: nothing to do but the launch
        _case("quantize_token", "quantize", 1, 0, 4096, rows=1, t=False),
        # a 70B-shaped weight after an optimizer step: both layouts that training reads
        _case("quantize_weight_70b", "quantize", 28672, 0, 8192, rows=128, t=True),
        # one token through an MLP down-projection: the weights are read once
        _case("product_token", "product", 1, 4096, 11008, out="bf16"),
        # a few hundred tokens, odd sizes, numbers out in 32 bits
        _case("product_ragged_f32", "product", 301, 1531, 5024, out="f32"),
        # a batch of prompts through the 70B-shaped up-projection
        _case("product_prompt_70b", "product", 8192, 28672, 8192, out="bf16"),
        # input gradient of the up-projection, gradients in E5M2
        _case("dinput_up", "dinput", 4096, 11008, 4096, fmt="E5M2", out="bf16"),
        # weight gradient of a ragged microbatch of a small layer
        _case("dweight_ragged", "dweight", 777, 1531, 5024, out="f32"),
        # weight gradient of the up-projection over a full batch of tokens
        _case("dweight_up", "dweight", 8192, 11008, 4096, out="f32"),
        # the gated unit of the MLP over a batch, gate and up being halves of one product's output
        _case("gated_batch", "gated", 8192, 0, 11008, pad=11008),
        # its gradient over an odd microbatch
        _case("dgated_ragged", "dgated", 1531, 0, 5024, grad="E5M2"),
        # one token with the packed pair that the search writes
        _case("packed_token", "packed", 1, 4096, 11008, bits=4, g=16, word="S1E5M5", two=True, k=2),
        # a prompt with it
        _case("packed_prompt", "packed", 2048, 11008, 4096, bits=4, g=16, word="UE4M3", two=True, k=0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above: sizes spread over their logarithm, odd ones among them."""
    op = rng.choice(["quantize", "product", "product", "dinput", "dweight", "gated", "dgated", "packed", "packed"])
    odd = lambda n: n if rng.random() < 0.5 else max(64, n // 64 * 64)  # noqa: E731
    M = _log_int(rng, 1, 8192)
    K, N = odd(_log_int(rng, 256, 16384)), odd(_log_int(rng, 256, 16384))
    more = dict(dtype=rng.choice(["bf16", "bf16", "f32"]), fmt=rng.choice(["E4M3", "E4M3", "E5M2"]), pad=rng.choice([0, 0, 8 * rng.randrange(1, 16)]))
    if op in ("product", "dinput", "dweight", "packed"):
        N = max(64, min(N, int(6e11 / M / K)))
        more.update(out=rng.choice(["bf16", "f32"]), dtype="bf16")
    if op == "quantize":
        more.update(rows=rng.choice([1, 1, 128]))
        more.update(t=more["rows"] == 128 and rng.random() < 0.7)
        N = 0
    elif op in ("gated", "dgated"):
        N = 0
        if op == "dgated":
            more.update(grad=rng.choice(["E4M3", "E5M2"]), fmt="E4M3")
    elif op == "packed":
        g, bits = rng.choice([8, 16, 16, 32, 64]), rng.choice([3, 4, 4, 4, 5])
        two = rng.random() < 0.7
        K = max(1, K // g) * g
        more.update(g=g, bits=bits, two=two, word=rng.choice(["UE4M3", "S1E5M5"] if two else ["UE4M3", "UE4M4", "S1E5M5"]), k=rng.randrange(0, 4), fmt="", out="bf16")
    case = _case("", op, M, N, K, **more)
    del case["name"]
    return case


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


def _codebook(alpha, c, bits):
    """A sinh grid of 2^bits entries, largest magnitude 1, ascending."""
    t = torch.linspace(-1, 1, 1 << bits, dtype=torch.float64)
    v = torch.sinh(alpha * t) + c
    return (v / v.abs().max()).float()


def _words(case):
    """Bit positions of a scale word: (sign, lowest magnitude bit, selector)."""
    w, x, y, b, _ = WORDS[case["word"]]
    m = b - w - x - y
    return b - 1, m if w else max(m - 1, 0), m - 1 if w else b - 1


def _prepare_packed(case, gen):
    N, K, g, n = case["N"], case["K"], case["g"], case["bits"]
    w, x, y, b, bias = WORDS[case["word"]]
    sign, low, sel = _words(case)
    count = N * K // g
    tables = [_codebook(1.5, -0.02, n), _codebook(0.4, 0.05, n)][:2 if case["two"] else 1]
    # codes: normal weights against the first codebook's midpoints; scales around 2^-2
    mid = ((tables[0][1:] + tables[0][:-1]) / 2).cuda()
    codes = torch.bucketize(0.45 * torch.randn((count, g), generator=gen, device="cuda"), mid).long()
    mag = torch.randint((bias - 4) << y, (bias + 1) << y, (count,), generator=gen, device="cuda")
    word = mag << low
    if w:
        word |= torch.randint(0, 2, (count,), generator=gen, device="cuda") << sign
    if case["two"]:
        word |= torch.randint(0, 2, (count,), generator=gen, device="cuda") << sel
    eight = (codes.view(count, g // 8, 8) << (n * torch.arange(8, device="cuda"))).sum(-1)
    payload = (eight[..., None] >> (8 * torch.arange(n, device="cuda")) & 255).to(torch.uint8).view(count, g * n // 8)
    return dict(x=_rows(gen, case["M"], K, torch.bfloat16, case["pad"]), words=word.to(torch.int16), payload=payload, tables=tables)


def prepare(case, seed):
    gen, op, M, N, K = _gen(seed), case["op"], case["M"], case["N"], case["K"]
    dtype, pad, fmt = FLOAT[case["dtype"]], case["pad"], case["fmt"]
    s = dict(case=case)
    if op == "quantize":
        s["x"] = _rows(gen, M, K, dtype, pad, 0.02 if case["rows"] == 128 else 1.0)
    elif op == "product":
        s["x"], s["w"] = _kept(gen, M, K, 1, fmt), _kept(gen, N, K, 128, "E4M3", 0.02)
    elif op == "dinput":
        codes, scales = _kept(gen, N, K, 128, "E4M3", 0.02)
        s.update(dy=_rows(gen, M, N, dtype, pad, 1e-4), w=(codes, scales), wt=_spaced(codes.view(torch.uint8).t().contiguous().view(codes.dtype), 16))
    elif op == "dweight":
        s.update(dy=_rows(gen, M, N, torch.bfloat16, pad, 1e-4), x=_kept(gen, M, K, 1, fmt))
    elif op == "gated":
        both = _rows(gen, M, 2 * K if pad >= K else K, dtype, 0 if pad >= K else pad)
        s.update(gate=both[:, :K], up=both[:, K:] if pad >= K else _rows(gen, M, K, dtype, pad))
    elif op == "dgated":
        s.update(gate=_kept(gen, M, K, 1, fmt), up=_kept(gen, M, K, 1, fmt), dh=_rows(gen, M, K, dtype, pad, 1e-4))
    else:
        s.update(_prepare_packed(case, gen))
    if own:
        import paper_2605_14929_amd as sop
        s["sop"], s["ctx"] = sop, sop.Context(0)
        if op == "packed":                                             # the layer as a serving program holds it
            s["layer"] = sop.PackedWeights(s["words"], s["payload"], N, K, case["g"], case["bits"], sop.ScaleFmt(*WORDS[case["word"]][:5], -1),
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
    sign, low, sel = _words(case)
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


def _plain(s):
    case = s["case"]
    op, fmt = case["op"], case["fmt"]
    if op == "quantize":
        codes, scales = _plain_blocks(s["x"].float(), case["rows"], fmt)
        return (codes, scales) + ((codes.view(torch.uint8).t().contiguous().view(codes.dtype),) if case["t"] else ())
    if op == "product":
        return (_plain_values(*s["x"], 1) @ _plain_values(*s["w"], 128).t()).to(FLOAT[case["out"]])
    if op == "dinput":
        dy = _plain_values(*_plain_blocks(s["dy"].float(), 1, fmt), 1)
        return (dy @ _plain_values(*s["w"], 128)).to(FLOAT[case["out"]])
    if op == "dweight":
        return (s["dy"].float().t() @ _plain_values(*s["x"], 1)).to(FLOAT[case["out"]])
    if op == "gated":
        g, u = s["gate"].float(), s["up"].float()
        return (*_plain_blocks(g / (1 + torch.exp(-g)) * u, 1, fmt), *_plain_blocks(g, 1, fmt), *_plain_blocks(u, 1, fmt))
    if op == "dgated":
        g, u, dh = _plain_values(*s["gate"], 1), _plain_values(*s["up"], 1), s["dh"].float()
        q = 1 / (1 + torch.exp(-g))
        dg, du = dh * u * q * (1 + g * (1 - q)), dh * g * q
        return (dg.to(s["dh"].dtype), du.to(s["dh"].dtype), *_plain_blocks(dg, 1, case["grad"]), *_plain_blocks(du, 1, case["grad"]))
    return (s["x"].float() @ _plain_packed(s).t()).to(torch.bfloat16)


# ---- the library

def _own(s):
    case, sop, ctx = s["case"], s["sop"], s["ctx"]
    op = case["op"]
    if op == "quantize":
        q = ctx.fp8_quantize(s["x"], rows=case["rows"], fmt=CODE[case["fmt"]], transposed=case["t"])
        return (q.codes, q.scales) + ((q.codes_t,) if case["t"] else ())
    if op == "product":
        return ctx.fp8_matmul(sop.Fp8Blocks(*s["x"]), sop.Fp8Blocks(*s["w"], rows=128), dtype=FLOAT[case["out"]])
    if op == "dinput":
        dy = ctx.fp8_quantize(s["dy"], fmt=CODE[case["fmt"]])
        return ctx.fp8_matmul(dy, sop.Fp8Blocks(*s["w"], rows=128, codes_t=s["wt"]), transposed=True, dtype=FLOAT[case["out"]])
    if op == "dweight":
        return ctx.fp8_weight_grad(s["dy"], sop.Fp8Blocks(*s["x"]), dtype=FLOAT[case["out"]])
    if op == "gated":
        h, g, u = ctx.fp8_gated(s["gate"], s["up"], fmt=CODE[case["fmt"]])
        return h.codes, h.scales, g.codes, g.scales, u.codes, u.scales
    if op == "dgated":
        dg, du, dg8, du8 = ctx.fp8_gated_grad(sop.Fp8Blocks(*s["gate"]), sop.Fp8Blocks(*s["up"]), s["dh"], fmt=CODE[case["grad"]])
        return dg, du, dg8.codes, dg8.scales, du8.codes, du8.scales
    return ctx.packed_matmul(s["x"], s["layer"])


def run(state):
    return _own(state) if own else _plain(state)


# ---- in 64 bits, from the definitions

def _exact_blocks(x, rows, fmt):
    """(codes' values, scales' values) of finite 64-bit x."""
    top, least, mant = (448.0, -6, 3) if fmt == "E4M3" else (57344.0, -14, 2)
    M, K = x.shape
    row, col = torch.arange(M, device="cuda") // rows, torch.arange(K, device="cuda") // 128
    R, B = int(row[-1]) + 1, int(col[-1]) + 1
    a = torch.zeros((M, B), dtype=torch.float64, device="cuda").scatter_reduce_(1, col.expand(M, K), x.abs(), "amax")
    a = torch.zeros((R, B), dtype=torch.float64, device="cuda").scatter_reduce_(0, row[:, None].expand(M, B), a, "amax")
    e = torch.ceil(torch.log2(torch.where(a > 0, a, top) / top))
    e = torch.where(a > top * torch.exp2(e), e + 1, e)
    e = torch.where(a <= top * torch.exp2(e - 1), e - 1, e)            # (the logarithm may be off by one at a power of two)
    e = torch.where(a > 0, e.clamp(min=-126), 0.0)
    v = x / torch.exp2(e)[row][:, col]
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** (least - 1)))).clamp(min=least) - mant)
    return torch.round(v / step) * step, torch.exp2(e)


def _exact_values(codes, scales, rows):
    M, K = codes.shape
    row, col = torch.arange(M, device="cuda") // rows, torch.arange(K, device="cuda") // 128
    return codes.double() * scales.double()[row][:, col]


def _exact_packed(s):
    case = s["case"]
    w, x, y, b, bias = WORDS[case["word"]]
    sign, low, sel = _words(case)
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


def exact(case, seed):
    s = prepare(case, seed)
    op, fmt = case["op"], case["fmt"]
    if op == "quantize":
        codes, scales = _exact_blocks(s["x"].double(), case["rows"], fmt)
        return (codes, scales) + ((codes.t().contiguous(),) if case["t"] else ())
    if op == "product":
        return _exact_values(*s["x"], 1) @ _exact_values(*s["w"], 128).t()
    if op == "dinput":
        codes, scales = _exact_blocks(s["dy"].double(), 1, fmt)
        return _exact_values(codes, scales, 1) @ _exact_values(*s["w"], 128)
    if op == "dweight":
        return s["dy"].double().t() @ _exact_values(*s["x"], 1)
    if op == "gated":
        g, u = s["gate"].double(), s["up"].double()
        return (*_exact_blocks(g * torch.sigmoid(g) * u, 1, fmt), *_exact_blocks(g, 1, fmt), *_exact_blocks(u, 1, fmt))
    if op == "dgated":
        g, u, dh = _exact_values(*s["gate"], 1), _exact_values(*s["up"], 1), s["dh"].double()
        q = torch.sigmoid(g)
        dg, du = dh * u * (q + g * q * (1 - q)), dh * g * q
        return (dg, du, *_exact_blocks(dg, 1, case["grad"]), *_exact_blocks(du, 1, case["grad"]))
    return s["x"].double() @ _exact_packed(s).t()


def work(case):
    """Each input read once, each output written once; two operations a multiply-add, about ten an element of the element-wise passes."""
    op, M, N, K = case["op"], case["M"], case["N"], case["K"]
    b, o = (2 if case["dtype"] == "bf16" else 4), (2 if case.get("out") == "bf16" else 4)
    tok, wgt = 1 + 1 / 128, 1 + 1 / 128 ** 2
    if op == "quantize":
        return {"bytes": M * K * (b + (tok if case["rows"] == 1 else wgt) + case["t"]), "flops": 4 * M * K}
    if op == "product":
        return {"bytes": M * K * tok + N * K * wgt + M * N * o, "flops": 2 * M * N * K}
    if op == "dinput":
        return {"bytes": M * N * b + N * K * wgt + M * K * o, "flops": 2 * M * N * K}
    if op == "dweight":
        return {"bytes": M * N * 2 + M * K * tok + N * K * o, "flops": 2 * M * N * K}
    if op == "gated":
        return {"bytes": M * K * (2 * b + 3 * tok), "flops": 16 * M * K}
    if op == "dgated":
        return {"bytes": M * K * (2 * tok + b + 2 * b + 2 * tok), "flops": 24 * M * K}
    return {"bytes": N * K * (case["bits"] / 8 + 2 / case["g"]) + M * K * 2 + M * N * 2, "flops": 2 * M * N * K}
