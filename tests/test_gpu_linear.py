"""Products of a linear layer with narrow operands on the GPU against the oracle in 64 bits.

Tolerances.  Quantised codes and scales are exact.  A product of two 8-bit floats is exact; a binary32 sum of K terms, in any order, is
off by at most about K units of 2^-24 of the sum of the terms' magnitudes (twice that is allowed: the matrix instruction's own
additions may be truncated).  With a bf16 result the 8-bit instruction adds eight products on a grid of 2^-16 of the largest of them:
2^-13 of the magnitudes' sum at most, and 2^-8 of the result's magnitude for its rounding (bf16 has 8 significant bits: 257 is halfway
between its neighbours 256 and 258).  Sums of small integers are exact whatever the
order: those products are compared for equality.  A packed weight is rounded to bf16 on its way into the matrix instruction: 2^-8 of each
term's magnitude."""
import numpy as np
import pytest

import paper_2605_14929_amd as sop
from oracle import linear as OL
from oracle import pack as OP
from gpu_util import ctx, oracle_fmt

pytestmark = pytest.mark.gpu
FMT = {"E4M3": sop.E4M3, "E5M2": sop.E5M2}


def _t(x, dtype="f32", pad=0, shift=0):
    """A CUDA copy: rows `pad` elements apart, `shift` elements off their allocation."""
    import torch
    M, K = x.shape
    buf = torch.zeros(M * (K + pad) + shift, dtype=torch.float32 if dtype == "f32" else torch.bfloat16, device="cuda")
    v = buf[shift:].view(M, K + pad)[:, :K]
    v.copy_(torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)))
    return v


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _bytes(t):
    import torch
    return t.view(torch.uint8).cpu().numpy()


def _f8(codes, scales, rows, fmt, codes_t=False):
    import torch
    dt = torch.float8_e4m3fn if fmt == "E4M3" else torch.float8_e5m2
    c = torch.from_numpy(np.ascontiguousarray(codes)).cuda().view(dt)
    s = torch.from_numpy(np.ascontiguousarray(scales)).cuda().view(torch.float8_e8m0fnu)
    t = torch.from_numpy(np.ascontiguousarray(codes.T)).cuda().view(dt) if codes_t else None
    return sop.Fp8Blocks(c, s, rows=rows, codes_t=t)


def _bf16(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16).float().numpy()


def _spread(rng, M, K):
    return (rng.standard_normal((M, K)) * np.exp(rng.standard_normal((1, K))) * 2.0 ** rng.integers(-8, 8, (M, 1))).astype(np.float32)


SHAPES = [(1, 1), (1, 128), (1, 4096), (2, 7), (3, 129), (5, 1000), (127, 128), (128, 257), (130, 640), (257, 333), (300, 1531)]


@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("fmt", ["E4M3", "E5M2"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantize(rows, fmt, dtype):
    rng = np.random.default_rng(1)
    for i, (M, K) in enumerate(SHAPES):
        x = _spread(rng, M, K)
        if dtype == "bf16":
            x = _bf16(x)
        for pad, shift in ((0, 0), (5, 1), (8 - K % 8, 0)):
            q = ctx().fp8_quantize(_t(x, dtype, pad, shift), rows=rows, fmt=FMT[fmt], transposed=rows == 128)
            codes, scales = OL.quantize(x, rows, fmt)
            assert np.array_equal(_bytes(q.scales), scales), (M, K, pad)
            assert np.array_equal(_bytes(q.codes), codes), (M, K, pad)
            if rows == 128:
                assert np.array_equal(_bytes(q.codes_t), codes.T), (M, K, pad)


@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("fmt", ["E4M3", "E5M2"])
def test_quantize_at_the_edges(rows, fmt):
    """Blocks of zeros, of one element, of the largest and smallest numbers, on and beside the scale's steps, ties, infinities, NaN."""
    top = OL.TOP[fmt]
    rng = np.random.default_rng(2)
    blocks = [np.zeros(128), np.full(128, 3.4028235e38), np.full(128, 1e-45), np.full(128, 1.1754944e-38)]
    for e in (-100, -3, 0, 50):
        for a in (top, np.nextafter(np.float32(top), np.float32(np.inf)), np.nextafter(np.float32(top), np.float32(0)), top / 2):
            b = rng.standard_normal(128) * a / 4
            b[17] = -a
            blocks.append(np.clip(b, -a, a) * 2.0 ** e)
    vals = OL.code_values(fmt)
    vals = vals[np.isfinite(vals)]
    ties = ((vals[1:] + vals[:-1]) / 2)[:127]
    blocks.append(np.concatenate([ties, np.full(128 - ties.size, top)]))
    for bad in ([np.inf], [np.nan], [-np.inf, np.nan, np.inf], [np.nan] * 128, [np.inf] * 128):
        b = rng.standard_normal(128)
        b[128 - len(bad):] = bad
        blocks.append(b)
        blocks.append(np.where(np.isfinite(b), 0.0, b))
    x = np.stack(blocks).astype(np.float32)
    if rows == 128:
        x = np.concatenate([np.concatenate([b[None], np.zeros((127, 128), np.float32)]) for b in x])
    q = ctx().fp8_quantize(_t(x), rows=rows, fmt=FMT[fmt])
    codes, scales = OL.quantize(x, rows, fmt)
    assert np.array_equal(_bytes(q.scales), scales)
    assert np.array_equal(OL.decode(_bytes(q.codes), fmt), OL.decode(codes, fmt), equal_nan=True)


def _integers(rng, M, K, rows, fmt="E4M3"):
    """Codes of whole numbers up to 4 in magnitude under scales of 1, 2 or 4."""
    v = rng.integers(-4, 5, (M, K)).astype(np.float64)
    e = rng.integers(0, 3, (-(-M // rows), -(-K // 128)))
    return OL.encode(v, fmt), (e + 127).astype(np.uint8)


PRODUCTS = [(1, 1, 1), (1, 16, 128), (1, 4096, 11008), (3, 17, 130), (16, 33, 1000), (17, 100, 257), (33, 130, 384), (64, 200, 129), (65, 129, 512), (100, 1531, 200),
            (128, 128, 128), (300, 333, 777), (2049, 2050, 160), (4096, 4200, 300)]


@pytest.mark.parametrize("fmt", ["E4M3", "E5M2"])
@pytest.mark.parametrize("dims", PRODUCTS)
def test_product_of_whole_numbers_is_exact(dims, fmt):
    import torch
    M, N, K = dims
    rng = np.random.default_rng(3)
    xc, xs = _integers(rng, M, K, 1, fmt)
    wc, ws = _integers(rng, N, K, 128)
    x, w = OL.values(xc, xs, 1, fmt), OL.values(wc, ws, 128, "E4M3")
    ref = (torch.from_numpy(x).cuda() @ torch.from_numpy(w).cuda().t()).cpu().numpy()
    y = ctx().fp8_matmul(_f8(xc, xs, 1, fmt), _f8(wc, ws, 128, "E4M3"), dtype=torch.float32)
    assert np.array_equal(_np(y), ref)
    yb = ctx().fp8_matmul(_f8(xc, xs, 1, fmt), _f8(wc, ws, 128, "E4M3"))
    assert np.array_equal(_np(yb), _bf16(ref))
    # the other index: dx = dy w, the weight being [K, N] here
    vc, vs = _integers(rng, K, N, 128)
    v = OL.values(vc, vs, 128, "E4M3")
    z = ctx().fp8_matmul(_f8(xc, xs, 1, fmt), _f8(vc, vs, 128, "E4M3", codes_t=True), transposed=True, dtype=torch.float32)
    assert np.array_equal(_np(z), (torch.from_numpy(x).cuda() @ torch.from_numpy(v).cuda()).cpu().numpy())


@pytest.mark.parametrize("dims", [(1, 300, 5024), (40, 257, 4096), (130, 260, 1531), (513, 1025, 700), (2300, 4700, 1000)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_product_of_quantised_numbers(dims, dtype):
    import torch
    M, N, K = dims
    rng = np.random.default_rng(4)
    x, w = _spread(rng, M, K), _spread(rng, N, K)
    x[0] = 0
    cx = ctx()
    xq, wq = cx.fp8_quantize(_t(x)), cx.fp8_quantize(_t(w), rows=128)
    xv = torch.from_numpy(OL.values(*OL.quantize(x, 1, "E4M3"), 1, "E4M3")).cuda()
    wv = torch.from_numpy(OL.values(*OL.quantize(w, 128, "E4M3"), 128, "E4M3")).cuda()
    ref, mag = (xv @ wv.t()).cpu().numpy(), (xv.abs() @ wv.abs().t()).cpu().numpy()
    buf = torch.full((M, N + 3), 7.0, dtype=torch.float32 if dtype == "f32" else torch.bfloat16, device="cuda")
    y = cx.fp8_matmul(xq, wq, out=buf[:, :N])
    d = np.abs(_np(y) - ref)
    assert np.all(d <= 2 * K * 2.0 ** -24 * mag + ((2.0 ** -8 + 2.0 ** -17) * np.abs(ref) + 2.0 ** -13 * mag if dtype == "bf16" else 0))
    assert np.all(_np(buf[:, N:]) == 7.0)                              # what lies between the rows stays
    assert np.array_equal(_np(cx.fp8_matmul(xq, wq, out=buf[:, :N])), _np(y))


def test_product_takes_nan_and_infinity_to_their_rows_alone():
    import torch
    rng = np.random.default_rng(5)
    M, N, K = 40, 150, 260
    xc, xs = _integers(rng, M, K, 1, "E5M2")
    wc, ws = _integers(rng, N, K, 128)
    wc[:, 250:] = OL.encode(np.ones((N, K - 250)), "E4M3")
    xc[3, 255], xc[5, 259] = 0x7F, 0x7C                                # NaN, infinity
    y = _np(ctx().fp8_matmul(_f8(xc, xs, 1, "E5M2"), _f8(wc, ws, 128, "E4M3"), dtype=torch.float32))
    assert np.isnan(y[3]).all() and np.isposinf(y[5]).all()
    keep = np.setdiff1d(np.arange(M), [3, 5])
    ref = OL.values(xc, xs, 1, "E5M2")[keep] @ OL.values(wc, ws, 128, "E4M3").T
    assert np.array_equal(y[keep], ref)
    # a scale that stands for NaN
    xc2, xs2 = _integers(rng, M, K, 1)
    xs2[7, 1] = 255
    y = _np(ctx().fp8_matmul(_f8(xc2, xs2, 1, "E4M3"), _f8(wc, ws, 128, "E4M3"), dtype=torch.float32))
    assert np.isnan(y[7]).all() and np.isfinite(np.delete(y, 7, 0)).all()


def test_what_lies_beyond_the_last_column_of_codes_is_not_used():
    import torch
    rng = np.random.default_rng(6)
    for M in (3, 40, 200):
        K, N = 200, 140
        xc, xs = _integers(rng, M, K + 56, 1)
        wc, ws = _integers(rng, N, K + 56, 128)
        xc[:, K:], wc[:, K:] = 0x7F, 0x7F                              # NaN, in rows that go on
        x = _f8(xc, xs, 1, "E4M3")
        w = _f8(wc, ws, 128, "E4M3")
        x, w = sop.Fp8Blocks(x.codes[:, :K], x.scales), sop.Fp8Blocks(w.codes[:, :K], w.scales, rows=128)
        ref = OL.values(xc, xs, 1, "E4M3")[:, :K] @ OL.values(wc, ws, 128, "E4M3")[:, :K].T
        assert np.array_equal(_np(ctx().fp8_matmul(x, w, dtype=torch.float32)), ref)
        dy = rng.integers(-3, 4, (M, 33)).astype(np.float32)
        assert np.array_equal(_np(ctx().fp8_weight_grad(_t(dy, "bf16"), x)), dy.T.astype(np.float64) @ OL.values(xc, xs, 1, "E4M3")[:, :K])


GRADS = [(1, 1, 1), (1, 2, 128), (2, 3, 5), (63, 64, 130), (64, 65, 129), (65, 130, 257), (200, 131, 1000), (777, 300, 640), (130, 2050, 4100), (100, 4224, 4352)]


@pytest.mark.parametrize("fmt", ["E4M3", "E5M2"])
@pytest.mark.parametrize("dims", GRADS)
def test_weight_gradient_of_whole_numbers_is_exact(dims, fmt):
    import torch
    M, N, K = dims
    rng = np.random.default_rng(7)
    xc, xs = _integers(rng, M, K, 1, fmt)
    dy = rng.integers(-8, 9, (M, N)).astype(np.float32)
    ref = (torch.from_numpy(dy).cuda().double().t() @ torch.from_numpy(OL.values(xc, xs, 1, fmt)).cuda()).cpu().numpy()
    x = _f8(xc, xs, 1, fmt)
    for pad, shift in ((0, 0), (3, 1)):
        assert np.array_equal(_np(ctx().fp8_weight_grad(_t(dy, "bf16", pad, shift), x)), ref)
    assert np.array_equal(_np(ctx().fp8_weight_grad(_t(dy, "bf16"), x, dtype=torch.bfloat16)), _bf16(ref))
    had = rng.integers(-9, 10, (N, K + 2)).astype(np.float32)
    for dtype in ("f32", "bf16"):
        out = _t(had, dtype)
        ctx().fp8_weight_grad(_t(dy, "bf16"), x, out=out[:, :K], accumulate=True)
        want = had[:, :K] + ref
        assert np.array_equal(_np(out[:, :K]), want if dtype == "f32" else _bf16(want))
        assert np.array_equal(_np(out[:, K:]), had[:, K:])


def test_weight_gradient_of_quantised_numbers():
    import torch
    rng = np.random.default_rng(8)
    M, N, K = 1000, 300, 500
    x, dy = _spread(rng, M, K), _bf16(_spread(rng, M, N) * 1e-3)
    q = ctx().fp8_quantize(_t(x))
    xv = OL.values(*OL.quantize(x, 1, "E4M3"), 1, "E4M3")
    ref, mag = dy.T.astype(np.float64) @ xv, np.abs(dy.T) @ np.abs(xv)
    assert np.all(np.abs(_np(ctx().fp8_weight_grad(_t(dy, "bf16"), q)) - ref) <= 2 * M * 2.0 ** -24 * mag)
    assert _np(ctx().fp8_weight_grad(_t(dy[:0], "bf16"), ctx().fp8_quantize(_t(x[:0])))).max() == 0      # no rows: zeros
    out = torch.ones((N, K), device="cuda")
    assert _np(ctx().fp8_weight_grad(_t(dy[:0], "bf16"), ctx().fp8_quantize(_t(x[:0])), out=out, accumulate=True)).min() == 1


def test_weight_gradient_takes_every_code_and_scale():
    """All codes of both formats under scales over the whole range: the checkpoint's numbers are exact in bf16."""
    for fmt in ("E4M3", "E5M2"):
        codes = np.tile(np.arange(256, dtype=np.uint8), 1)[None]
        for s in (1, 20, 100, 127, 150, 200, 230):
            scales = np.full((1, 2), s, dtype=np.uint8)
            got = _np(ctx().fp8_weight_grad(_t(np.ones((1, 1)), "bf16"), _f8(codes, scales, 1, fmt)))[0]
            want = OL.values(codes, scales, 1, fmt)[0]
            tiny = np.abs(want) < 2.0 ** -126
            with np.errstate(over="ignore"):
                want32 = want.astype(np.float32).astype(np.float64)
            assert np.array_equal(got[~tiny], want32[~tiny], equal_nan=True), (fmt, s)
            assert np.all(np.abs(got[tiny] - want[tiny]) <= 2.0 ** -134)         # (bf16's spacing there is 2^-133)


def _near_codes(q, value, fmt, rel):
    """The numbers of q are those of `value` rounded to the format under q's own scale, `value` known to `rel`; scales the rule's, unless
    the block's largest is within `rel` of a step."""
    codes, scales = _bytes(q.codes), _bytes(q.scales)
    M, K = value.shape
    e = OL.block_exponents(value, 1, fmt)
    lo, hi = OL.block_exponents(value * (1 - rel), 1, fmt), OL.block_exponents(value * (1 + rel), 1, fmt)
    got = scales.astype(np.int64) - 127
    assert np.all((got == e) | (got == lo) | (got == hi))
    step = 2.0 ** OL.spread(got, 1, M, K)
    v = OL.values(codes, scales, 1, fmt)
    unit = 2.0 ** np.maximum(np.floor(np.log2(np.maximum(np.abs(value) / step, 1e-300))), OL.LEAST[fmt]) * 2.0 ** -OL.MANT[fmt] * step
    assert np.all(np.abs(v - value) <= unit / 2 * (1 + 1e-9) + rel * np.abs(value) + 1e-300)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", ["E4M3", "E5M2"])
def test_gated_unit(dtype, fmt):
    rng = np.random.default_rng(9)
    for M, F in [(1, 1), (1, 4096), (3, 129), (70, 1000), (257, 333)]:
        g, u = _spread(rng, M, F), _spread(rng, M, F)
        if dtype == "bf16":
            g, u = _bf16(g), _bf16(u)
        for pad, shift in ((0, 0), (8 - F % 8, 0), (3, 1)):
            h, g8, u8 = ctx().fp8_gated(_t(g, dtype, pad, shift), _t(u, dtype, pad, shift), fmt=FMT[fmt])
            for q, x in ((g8, g), (u8, u)):
                codes, scales = OL.quantize(x, 1, fmt)
                assert np.array_equal(_bytes(q.codes), codes) and np.array_equal(_bytes(q.scales), scales)
            with np.errstate(over="ignore"):
                want = OL.silu_mul(g.astype(np.float64), u.astype(np.float64))
            want[np.abs(want) < 2.0 ** -120] = 0                       # (binary32 underflow)
            _near_codes(h, want, fmt, 2.0 ** -20)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", ["E4M3", "E5M2"])
def test_gated_gradient(dtype, fmt):
    rng = np.random.default_rng(10)
    for M, F in [(1, 1), (1, 300), (5, 128), (33, 1001), (130, 512)]:
        g, u, dh = rng.standard_normal((M, F)) * 4, rng.standard_normal((M, F)), rng.standard_normal((M, F)) * 1e-3
        if dtype == "bf16":
            dh = _bf16(dh)
        dh = dh.astype(np.float32)
        gq, uq = OL.quantize(g, 1, fmt), OL.quantize(u, 1, fmt)
        gv, uv = OL.values(*gq, 1, fmt), OL.values(*uq, 1, fmt)
        dg, du, dg8, du8 = ctx().fp8_gated_grad(_f8(*gq, 1, fmt), _f8(*uq, 1, fmt), _t(dh, dtype, 5, 1), fmt=FMT[fmt])
        wg, wu = OL.silu_mul_grad(gv, uv, dh.astype(np.float64))
        # dgate's last factor, 1 + g (1 - s), may cancel: its error is one of the two terms
        part = np.abs(dh * uv) * (1 + np.abs(gv)) * (1 / (1 + np.exp(-gv)))
        tol = 2.0 ** -8 if dtype == "bf16" else 0
        assert np.all(np.abs(_np(dg) - wg) <= tol * np.abs(wg) + 2.0 ** -20 * part + 1e-30)
        assert np.all(np.abs(_np(du) - wu) <= (tol + 2.0 ** -20) * np.abs(wu) + 1e-30)
        if dtype == "f32":
            for q, x in ((dg8, _np(dg)), (du8, _np(du))):              # the codes are those of the 32-bit results
                codes, scales = OL.quantize(x, 1, fmt)
                assert np.array_equal(_bytes(q.codes), codes) and np.array_equal(_bytes(q.scales), scales)
        else:
            _near_codes(du8, wu, fmt, 2.0 ** -20)


def test_gated_unit_at_large_and_missing_numbers():
    g = np.array([[0.0, 100.0, -100.0, 3e38, -3e38, np.inf, np.nan, 1.0]], dtype=np.float32)
    u = np.ones_like(g)
    h, g8, u8 = ctx().fp8_gated(_t(g), _t(u), fmt=sop.E5M2)
    hv = OL.values(_bytes(h.codes), _bytes(h.scales), 1, "E5M2")[0]
    assert hv[0] == 0 and hv[2] == 0 and hv[4] == 0 and np.isposinf(hv[5]) and np.isnan(hv[6])
    assert abs(hv[3] - 3e38) <= 3e38 / 8


def _pack(rng, N, K, g, n, word, two, k):
    w, x, y, b = word
    Nb = N * K // g
    codes = rng.integers(0, 1 << n, (Nb, g))
    mag = rng.integers(0, 1 << (x + y), Nb)
    near = rng.integers(((1 << (x - 1)) - 4) << y, (1 << (x - 1)) << y, Nb)
    mag = np.where(rng.random(Nb) < 0.05, np.minimum(mag, (1 << (x - 1)) << y), near)    # some subnormal ones among them
    sc = (mag | np.where((w == 1) & (rng.random(Nb) < 0.5), 0x8000, 0)).astype(np.uint16)
    sel = rng.integers(0, 2, Nb) if two else None
    tabs = [np.sort(rng.uniform(-1, 1, 1 << n)).astype(np.float32) for _ in range(2 if two else 1)]
    return OP.pack_words(sc, sel, w, x, y, b), OP.pack_payload(codes, n), tabs


PACKED = [(1, 16, 128, 16, 4, (1, 5, 5, 12), True, 2), (1, 1, 8, 8, 3, (0, 4, 4, 8), False, 0), (2, 33, 264, 8, 5, (0, 4, 3, 8), True, 1), (5, 4096, 1040, 16, 4, (0, 4, 3, 8), True, 0),
          (16, 50, 320, 64, 6, (1, 4, 7, 12), False, -3), (17, 50, 320, 32, 1, (0, 5, 7, 12), False, 3), (31, 100, 136, 8, 2, (1, 5, 5, 12), True, 0), (33, 65, 200, 8, 4, (0, 4, 4, 8), False, 0),
          (100, 130, 1000, 8, 3, (0, 4, 3, 8), True, 5), (130, 1531, 304, 16, 5, (1, 5, 5, 12), True, 0), (300, 333, 640, 64, 4, (0, 4, 3, 8), True, 0), (2049, 2050, 192, 32, 6, (1, 5, 5, 12), True, 0),
          (4100, 4200, 80, 16, 4, (0, 4, 3, 8), True, 1)]


@pytest.mark.parametrize("case", PACKED)
def test_packed_product(case):
    import torch
    M, N, K, g, n, word, two, k = case
    rng = np.random.default_rng(11)
    words, payload, tabs = _pack(rng, N, K, g, n, word, two, k)
    fmt = sop.ScaleFmt(*word, -1, -1)
    w = OP.reconstruct(words, payload, n, g, N, K, tabs[0], tabs[1] if two else None, oracle_fmt(fmt), k, *word).astype(np.float64)
    x = _bf16(_spread(rng, M, K))
    layer = sop.PackedWeights(torch.from_numpy(words.view(np.int16)).cuda(), torch.from_numpy(payload).cuda(), N, K, g, n, fmt, tabs, k=k)
    xd, wd = torch.from_numpy(x).cuda().double(), torch.from_numpy(w).cuda()
    ref, mag = (xd @ wd.t()).cpu().numpy(), (xd.abs() @ wd.abs().t()).cpu().numpy()
    buf = torch.full((M, N + 1), 7.0, dtype=torch.bfloat16, device="cuda")
    for pad in (0, 8):
        y = ctx().packed_matmul(_t(x, "bf16", pad), layer, out=buf[:, :N])
        assert np.all(np.abs(_np(y) - ref) <= (2.0 ** -8 + 2 * K * 2.0 ** -24) * mag + 2.0 ** -8 * np.abs(ref))
        assert np.all(_np(buf[:, N:]) == 7.0)


def test_packed_product_of_what_a_search_packed():
    import torch
    import sop_inputs as si
    cx = ctx()
    N, K, g = 96, 512, 16
    W = si.student_t_weights(N, K, 4.0, 21)
    c = si.channel_norms(K, 1.0, 22)
    fmt = sop.fmt_by_name("S1E5M5")
    tabs = sop.build_alphabet(["NF4", "SH4"])
    cx.set_alphabet(tabs)
    cx.set_pairs(None)
    out = cx.pair_search(_t(W), torch.from_numpy(c).cuda(), g, fmt, emit=True)
    words, payload, n = cx.pack_blocks(out, N, K, g, fmt, 0, 1)
    layer = sop.PackedWeights(words, payload, N, K, g, n, fmt, tabs)
    eye = torch.eye(K, dtype=torch.bfloat16, device="cuda")
    got = _np(cx.packed_matmul(eye, layer)).T                         # the layer itself, rounded to bf16 once
    want = OP.reconstruct(words.cpu().numpy().view(np.uint16), payload.cpu().numpy(), n, g, N, K, tabs[0], tabs[1], oracle_fmt(fmt), 0, 1, 5, 5, 12)
    assert np.array_equal(got, _bf16(want))
    assert np.mean((want - W) ** 2) < 0.02 * np.mean(W ** 2)


def test_rows_beyond_four_gigabytes():
    import torch
    cx = ctx()
    M, K, N = 540_000, 8192, 64                                       # 4.4e9 codes
    x = sop.Fp8Blocks.empty(M, K, sop.E4M3, torch.device("cuda", 0))
    x.codes.view(torch.uint8).zero_()
    x.scales.view(torch.uint8).fill_(127)
    one = 0x38                                                        # 1.0
    x.codes.view(torch.uint8)[M - 1] = one
    x.codes.view(torch.uint8)[M - 2, 5] = one
    w = cx.fp8_quantize(torch.ones((N, K), device="cuda"), rows=128)
    y = cx.fp8_matmul(x, w, dtype=torch.float32)
    assert float(y[M - 1].min()) == float(y[M - 1].max()) == K and float(y[M - 2].min()) == float(y[M - 2].max()) == 1 and float(y[:M - 2].abs().max()) == 0
    dy = torch.zeros((M, 8), dtype=torch.bfloat16, device="cuda")
    dy[M - 1, 3] = 2
    dw = cx.fp8_weight_grad(dy, x)
    assert float(dw[3].min()) == float(dw[3].max()) == 2 and float(dw.sum()) == 2 * K
    big = torch.zeros((M, K), dtype=torch.bfloat16, device="cuda")    # 8.8e9 bytes
    big[M - 1] = 448
    q = cx.fp8_quantize(big)
    assert int(q.codes.view(torch.uint8)[M - 1].min()) == 0x7E and int(q.scales.view(torch.uint8)[M - 1].min()) == 127 and int(q.codes.view(torch.uint8)[M - 2].max()) == 0


def test_products_on_another_stream_and_in_a_graph():
    import torch
    cx = ctx()
    rng = np.random.default_rng(12)
    M, N, K = 40, 300, 512
    x, w = _t(_spread(rng, M, K), "bf16"), _t(_spread(rng, N, K))
    wq = cx.fp8_quantize(w, rows=128, transposed=True)

    def step():
        q = cx.fp8_quantize(x)
        y = cx.fp8_matmul(q, wq)
        h, g8, u8 = cx.fp8_gated(y[:, :128], y[:, 128:256])
        dg, du, dg8, du8 = cx.fp8_gated_grad(g8, u8, y[:, :128])
        return y, h.codes, dg, du8.codes, cx.fp8_weight_grad(y, q), cx.fp8_matmul(cx.fp8_quantize(y, fmt=sop.E5M2), wq, transposed=True)

    plain = [t.clone() for t in step()]
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        other = step()
    torch.cuda.current_stream().wait_stream(st)
    torch.cuda.synchronize()
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(plain, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for seed in (13, 14, 15):
        x.copy_(_t(_spread(np.random.default_rng(seed), M, K), "bf16"))
        graph.replay()
        torch.cuda.synchronize()
        fresh = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(held, fresh))


def test_no_rows():
    import torch
    cx = ctx()
    w = cx.fp8_quantize(torch.ones((130, 200), device="cuda"), rows=128)
    q = cx.fp8_quantize(torch.empty((0, 200), device="cuda"))
    assert tuple(cx.fp8_matmul(q, w).shape) == (0, 130)
    h, g8, u8 = cx.fp8_gated(torch.empty((0, 200), device="cuda"), torch.empty((0, 200), device="cuda"))
    assert tuple(h.codes.shape) == (0, 200) and cx.fp8_gated_grad(g8, u8, torch.empty((0, 200), device="cuda"))[0].shape == (0, 200)


def test_refusals():
    import torch
    cx = ctx()
    x = torch.ones((4, 256), device="cuda")
    q, w = cx.fp8_quantize(x), cx.fp8_quantize(torch.ones((140, 256), device="cuda"), rows=128)

    def refused(status, f, *a, **k):
        with pytest.raises(sop.SopError) as e:
            f(*a, **k)
        assert e.value.status == status, e.value

    refused(1, cx.fp8_quantize, x.cpu())
    refused(1, cx.fp8_quantize, x.half())
    refused(2, cx.fp8_quantize, x.t())
    refused(1, cx.fp8_quantize, x, rows=2)
    refused(1, cx.fp8_quantize, x, transposed=True)
    refused(1, cx.fp8_matmul, w, w)                                    # square blocks where rows are wanted
    refused(1, cx.fp8_matmul, q, q)
    refused(2, cx.fp8_matmul, cx.fp8_quantize(x[:, :128]), w)
    refused(1, cx.fp8_matmul, q, w, transposed=True)                   # no transposed codes
    refused(1, cx.fp8_matmul, q, cx.fp8_quantize(torch.ones((140, 256), device="cuda"), rows=128, fmt=sop.E5M2))
    refused(2, cx.fp8_matmul, q, w, out=torch.empty((4, 141), device="cuda"))
    refused(1, cx.fp8_matmul, q, w, dtype=torch.float16)
    refused(1, cx.fp8_weight_grad, x, q)                               # fp32 dy
    refused(2, cx.fp8_weight_grad, x[:3].bfloat16(), q)
    refused(1, cx.fp8_weight_grad, x.bfloat16(), q, accumulate=True)
    refused(1, cx.fp8_weight_grad, torch.ones((140, 8), dtype=torch.bfloat16, device="cuda"), w)
    refused(2, cx.fp8_gated, x, x[:, :128])
    refused(2, cx.fp8_gated_grad, q, q, x[:2])
    refused(2, sop.Fp8Blocks, q.codes, q.scales[:, :1])
    refused(1, sop.Fp8Blocks, x, q.scales)
    words, payload = torch.zeros(140 * 16, dtype=torch.int16, device="cuda"), torch.zeros(140 * 128, dtype=torch.uint8, device="cuda")
    tab = np.linspace(-1, 1, 16).astype(np.float32)
    fmt = sop.fmt_by_name("S1E5M5")
    layer = sop.PackedWeights(words, payload, 140, 256, 16, 4, fmt, [tab])
    refused(1, cx.packed_matmul, x, layer)                             # fp32 x
    refused(2, cx.packed_matmul, x[:, :128].bfloat16(), layer)
    refused(1, cx.packed_matmul, torch.ones((4, 260), dtype=torch.bfloat16, device="cuda")[:, :256], layer)
    refused(1, cx.packed_matmul, torch.ones((4, 264), dtype=torch.bfloat16, device="cuda")[:, 1:257], layer)
    refused(2, sop.PackedWeights, words, payload, 140, 256, 8, 4, fmt, [tab])
    refused(3, sop.PackedWeights, words, payload, 140, 256, 16, 4, fmt, [])
    refused(4, cx.packed_matmul, x.bfloat16(), sop.PackedWeights(words, payload, 140, 256, 16, 4, sop.fmt_by_name("UE4M4"), [tab, tab]))
    refused(4, cx.packed_matmul, x.bfloat16(), sop.PackedWeights(words, payload, 140, 256, 16, 4, fmt, [tab], k=65))
    refused(3, cx.packed_matmul, x.bfloat16(), sop.PackedWeights(words, payload, 140, 256, 16, 4, fmt, [np.zeros(65, np.float32)]))


@pytest.mark.parametrize("case", [(4100, 4200, 136, 8, 4, (0, 4, 3, 8), True, 1), (2100, 11000, 208, 16, 4, (1, 5, 5, 12), True, 0), (4097, 8200, 64, 32, 4, (0, 4, 4, 8), False, 0),
                                  (8200, 2049, 320, 64, 4, (0, 4, 3, 8), True, 2)])
def test_packed_product_of_large_layers(case):
    test_packed_product(case)


# the kernels that share a wide output out, and that deal K out, by code width: K ends in the middle of a step, of sixteen codes and on a step
@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 6])
@pytest.mark.parametrize("M, N, K, g", [(1020, 4090, 136, 8), (1020, 4090, 72, 8), (1000, 11000, 152, 8), (4000, 4090, 88, 8), (1020, 4090, 176, 16), (4000, 4090, 64, 64), (1000, 11000, 320, 32)])
def test_packed_product_of_wide_outputs(M, N, K, g, n):
    test_packed_product((M, N, K, g, n, (1, 5, 5, 12), True, 1))


@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 6])
@pytest.mark.parametrize("M, N, K, g", [(20, 100, 8, 8), (17, 33, 1096, 8), (65, 1001, 584, 8), (128, 4097, 600, 8), (128, 4097, 608, 16), (64, 11008, 1040, 16), (61, 11008, 72, 8), (511, 4096, 576, 64), (505, 4090, 520, 8)])
def test_packed_product_of_some_rows(M, N, K, g, n):
    test_packed_product((M, N, K, g, n, (0, 4, 3, 8), True, 0))


# rows of dy on 16 bytes, its columns no multiple of 8: the rows dealt out (32 x 64 and 64 x 64 of dw a workgroup), 128 x 128 and 256 x 256 (sums of at
# most 128 M, which binary32 holds exactly)
@pytest.mark.parametrize("fmt", ["E4M3", "E5M2"])
@pytest.mark.parametrize("M, N, K", [(1, 1, 1), (63, 33, 65), (65, 100, 130), (129, 31, 127), (513, 257, 515), (1100, 300, 500), (2100, 1001, 1000), (65, 1531, 2100), (130, 1027, 4100), (1025, 4090, 4000)])
def test_weight_gradient_of_spaced_rows(M, N, K, fmt):
    import torch
    rng = np.random.default_rng(12)
    xc, xs = _integers(rng, M, K, 1, fmt)
    dy = rng.integers(-8, 9, (M, N)).astype(np.float32)
    ref = (torch.from_numpy(dy).cuda().double().t() @ torch.from_numpy(OL.values(xc, xs, 1, fmt)).cuda()).cpu().numpy()
    x, d = _f8(xc, xs, 1, fmt), _t(dy, "bf16", 8 + -N % 8)
    assert np.array_equal(_np(ctx().fp8_weight_grad(d, x)), ref)
    out = torch.ones((N, K + 1), device="cuda")
    ctx().fp8_weight_grad(d, x, out=out[:, :K], accumulate=True)
    assert np.array_equal(_np(out[:, :K]), ref + 1) and np.all(_np(out[:, K:]) == 1)


@pytest.mark.parametrize("M, N, K", [(3, 40, 200), (70, 300, 600), (777, 1024, 1100), (65, 1536, 2100), (1025, 4096, 4000)])
def test_missing_numbers_stay_in_their_block(M, N, K):
    """A scale that is no number, or a code that is none, makes what it takes part in no number, and nothing else."""
    import torch
    rng = np.random.default_rng(13)
    xc, xs = _integers(rng, M, K, 1)
    wc, ws = _integers(rng, N, K, 128)
    xs[M // 2, 1] = 255                                                 # columns 128 .. 255 of a row of x
    xc[M - 1, K - 1] = 0x7F                                             # one element
    x = _f8(xc, xs, 1, "E4M3")
    dy = rng.integers(-8, 9, (M, N)).astype(np.float32)
    dw = _np(ctx().fp8_weight_grad(_t(dy, "bf16"), x))
    gone = np.zeros(K, bool)
    gone[128:256] = True
    gone[K - 1] = True
    assert np.isnan(dw[:, gone]).all() and np.isfinite(dw[:, ~gone]).all()
    for dtype in (torch.float32, torch.bfloat16):
        y = _np(ctx().fp8_matmul(x, _f8(wc, ws, 128, "E4M3"), dtype=dtype))
        rows = np.isin(np.arange(M), [M // 2, M - 1])
        assert np.isnan(y[rows]).all() and np.isfinite(y[~rows]).all()
    ws[0, 1] = 255                                                      # rows 0 .. 127 of w
    good = _f8(*_integers(rng, M, K, 1), 1, "E4M3")
    for dtype in (torch.float32, torch.bfloat16):
        y = _np(ctx().fp8_matmul(good, _f8(wc, ws, 128, "E4M3"), dtype=dtype))
        assert np.isnan(y[:, :128]).all() and np.isfinite(y[:, 128:]).all()


def test_a_given_stream_holds_the_call_and_its_results():
    """stream=handle: the kernels run there, ordered after what is queued there, and results are that stream's to allocate."""
    import torch
    cx = ctx()
    rng = np.random.default_rng(14)
    M, N, K = 50, 300, 520
    x, w = _t(_spread(rng, M, K), "bf16"), _t(_spread(rng, N, K))

    def step(**kw):
        wq, q = cx.fp8_quantize(w, rows=128, transposed=True, **kw), cx.fp8_quantize(x, **kw)
        y = cx.fp8_matmul(q, wq, **kw)
        h, g8, u8 = cx.fp8_gated(y, y, **kw)
        dg, du, dg8, du8 = cx.fp8_gated_grad(g8, u8, y, **kw)
        return y, h.codes, dg, du8.codes, cx.fp8_weight_grad(y, q, **kw), cx.fp8_matmul(du8, wq, transposed=True, **kw)

    plain = [_bytes(t.contiguous()) if t.element_size() == 1 else _np(t) for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(stream=side.cuda_stream)
    side.synchronize()
    for a, b in zip(plain, got):
        assert np.array_equal(a, _bytes(b.contiguous()) if b.element_size() == 1 else _np(b))
    for a, b in zip(plain, step(stream=0)):                             # the default stream
        assert np.array_equal(a, _bytes(b.contiguous()) if b.element_size() == 1 else _np(b))


# tiles of one row and of one column at the end, K ending inside the last step: 256 x 192 (128 x 128 with 6 bits), 256 x 256, 128 x 128 of y a workgroup
@pytest.mark.parametrize("n", [1, 3, 4, 5, 6])
@pytest.mark.parametrize("K, g", [(72, 8), (136, 8), (80, 16), (96, 32), (192, 64)])
@pytest.mark.parametrize("M, N", [(2049, 3841), (1025, 11009), (4097, 3841)])
def test_packed_product_with_one_row_left(M, N, K, g, n):
    test_packed_product((M, N, K, g, n, (0, 4, 3, 8), True, 0))


# A size for each way of sharing y out: up to four rows, tiles of 32 x 32, 32 x 64, 64 x 64, 64 x 128, 128 x 128 and (bf16 results alone) 256 x 256.
F8_KERNELS = [(3, 130, 300), (40, 150, 300), (301, 1531, 300), (513, 1025, 300), (1001, 4090, 150), (2049, 2050, 150), (2300, 4700, 150)]


# Scales from 2^-127 to 2^127 whose product is moderate: whole numbers, exact in either type of result.
@pytest.mark.parametrize("fmt", ["E4M3", "E5M2"])
@pytest.mark.parametrize("a, b", [(252, 0), (0, 252), (60, 190), (1, 251), (9, 243), (245, 9), (15, 237), (238, 14)])
@pytest.mark.parametrize("M, N, K", F8_KERNELS)
def test_product_under_scales_of_any_size(M, N, K, a, b, fmt):
    import torch
    rng = np.random.default_rng(15)
    (xc, xs), (wc, ws) = _integers(rng, M, K, 1, fmt), _integers(rng, N, K, 128)
    xs, ws = (xs - 127 + a).astype(np.uint8), (ws - 127 + b).astype(np.uint8)
    x, w = OL.values(xc, xs, 1, fmt), OL.values(wc, ws, 128, "E4M3")
    ref = (torch.from_numpy(x).cuda() @ torch.from_numpy(w).cuda().t()).cpu().numpy()
    x, w = _f8(xc, xs, 1, fmt), _f8(wc, ws, 128, "E4M3")
    assert np.array_equal(_np(ctx().fp8_matmul(x, w, dtype=torch.float32)), ref)
    assert np.array_equal(_np(ctx().fp8_matmul(x, w)), _bf16(ref))


def test_product_of_the_smallest_numbers():
    """Results among binary32's subnormal numbers, whole multiples of the least one."""
    import torch
    rng = np.random.default_rng(16)
    for (M, N, K), a in ((d, a) for d in ((3, 130, 300), (40, 150, 300), (513, 1025, 300), (1001, 4090, 150), (2049, 2050, 150)) for a in (1, 50, 80)):
        (xc, xs), (wc, ws) = _integers(rng, M, K, 1), _integers(rng, N, K, 128)
        xs, ws = (xs - 127 + a).astype(np.uint8), (ws - 127 + 105 - a).astype(np.uint8)   # 2^-149 and up, with one small scale or two moderate ones
        x, w = OL.values(xc, xs, 1, "E4M3"), OL.values(wc, ws, 128, "E4M3")
        ref = (torch.from_numpy(x).cuda() @ torch.from_numpy(w).cuda().t()).cpu().numpy()
        y = ctx().fp8_matmul(_f8(xc, xs, 1, "E4M3"), _f8(wc, ws, 128, "E4M3"), dtype=torch.float32)
        assert np.array_equal(y.cpu().numpy().astype(np.float64), ref)


def test_product_in_32_bits_drops_nothing_beside_a_large_product():
    """Two products of 448 x 448 in every 128, of both signs, among products of 1 or 0: sums are whole and below 2^24 in any order, so exact in
    binary32; on a grid of 2^-16 of the largest of eight (2 here) they would not be."""
    import torch
    rng = np.random.default_rng(17)
    for M, N, K in ((3, 130, 4096), (40, 150, 4096), (301, 1531, 4096), (513, 1025, 4096), (1001, 4090, 1024), (2049, 2050, 1024)):
        x, w = np.ones((M, K)), np.ones((N, K))
        x[:, :] = rng.integers(-1, 2, (M, K))
        x[:, ::128], x[:, 8::128], w[:, ::128], w[:, 8::128] = 448, -448, 448, 448
        one = lambda r: np.full((r, K // 128), 127, np.uint8)  # noqa: E731
        y = ctx().fp8_matmul(_f8(OL.encode(x, "E4M3"), one(M), 1, "E4M3"), _f8(OL.encode(w, "E4M3"), one(-(-N // 128)), 128, "E4M3"), dtype=torch.float32)
        assert np.array_equal(_np(y), (torch.from_numpy(x).cuda() @ torch.from_numpy(w).cuda().t()).cpu().numpy())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", ["E4M3", "E5M2"])
def test_gated_unit_far_below_zero(dtype, fmt):
    """Gates from -60 to -130, where the logistic function leaves binary32, beside factors that bring the product back: a row's block has one gate."""
    rng = np.random.default_rng(18)
    M, F = 101, 136
    g = np.repeat(np.linspace(-60, -130, M)[:, None], F, 1)
    u, dh = (rng.uniform(0.5, 2, (M, F)) * rng.choice([-1, 1], (M, F)) * s for s in (1e37, 1e20))
    g, u, dh = (_bf16(t) if dtype == "bf16" else t.astype(np.float32) for t in (g, u, dh))
    for pad, shift in ((0, 0), (3, 1)):
        h, g8, u8 = ctx().fp8_gated(_t(g, dtype, pad, shift), _t(u, dtype, pad, shift), fmt=FMT[fmt])
        _near_codes(h, OL.silu_mul(g.astype(np.float64), u.astype(np.float64)), fmt, 2.0 ** -20)
        gv, uv = (OL.values(_bytes(q.codes), _bytes(q.scales), 1, fmt) for q in (g8, u8))
        dg, du, dg8, du8 = ctx().fp8_gated_grad(g8, u8, _t(dh, dtype, pad, shift), fmt=FMT[fmt])
        wg, wu = OL.silu_mul_grad(gv, uv, dh.astype(np.float64))
        tol = 2.0 ** -20 + (2.0 ** -8 if dtype == "bf16" else 0)
        assert np.all(np.abs(_np(dg) - wg) <= tol * np.abs(wg)) and np.all(np.abs(_np(du) - wu) <= tol * np.abs(wu))
        _near_codes(dg8, wg, fmt, 2.0 ** -20)
        _near_codes(du8, wu, fmt, 2.0 ** -20)


def test_a_result_of_another_type_than_asked_for_is_refused():
    import torch
    cx = ctx()
    x = torch.ones((4, 256), device="cuda")
    q, w = cx.fp8_quantize(x), cx.fp8_quantize(torch.ones((140, 256), device="cuda"), rows=128)
    for f, a, shape in ((cx.fp8_matmul, (q, w), (4, 140)), (cx.fp8_weight_grad, (x.bfloat16(), q), (256, 256))):
        for has, asked in ((torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32)):
            with pytest.raises(sop.SopError) as e:
                f(*a, dtype=asked, out=torch.empty(shape, dtype=has, device="cuda"))
            assert e.value.status == 1
            out = torch.empty(shape, dtype=has, device="cuda")
            assert f(*a, dtype=has, out=out) is out and f(*a, out=out) is out


# tiles of 64 x 32 of y a workgroup
@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 6])
@pytest.mark.parametrize("M, N, K, g", [(100, 4001, 200, 8), (128, 4096, 584, 8), (90, 4030, 1040, 16), (127, 3999, 192, 64)])
def test_packed_product_of_a_hundred_rows(M, N, K, g, n):
    test_packed_product((M, N, K, g, n, (1, 5, 5, 12), True, 0))


def test_more_rows_or_columns_than_one_grid_of_small_tiles_holds():
    """2^28 rows in tiles of 32, 2^27 columns by 16: 2^32 threads and more, so larger tiles take them."""
    import torch
    cx = ctx()
    M, K = (1 << 28) + 5, 16
    x = sop.Fp8Blocks.empty(M, K, sop.E4M3, torch.device("cuda", 0))
    x.codes.view(torch.uint8).fill_(0x38)                             # 1.0
    x.scales.view(torch.uint8).fill_(127)
    x.codes.view(torch.uint8)[M - 1, 3] = 0x40                        # 2.0
    w = cx.fp8_quantize(torch.ones((1, K), device="cuda"), rows=128)
    for dtype in (torch.float32, torch.bfloat16):
        y = cx.fp8_matmul(x, w, dtype=dtype)
        assert float(y[M - 1, 0]) == K + 1 and float(y[:M - 1].min()) == float(y[:M - 1].max()) == K
    del x, y
    w = sop.Fp8Blocks.empty(M, K, sop.E4M3, torch.device("cuda", 0), rows=128)
    w.codes.view(torch.uint8).fill_(0x38)
    w.scales.view(torch.uint8).fill_(127)
    w.codes.view(torch.uint8)[M - 1, 3] = 0x40
    y = cx.fp8_matmul(cx.fp8_quantize(torch.ones((2, K), device="cuda")), w, dtype=torch.float32)
    assert float(y[:, M - 1].min()) == float(y[:, M - 1].max()) == K + 1 and float(y[:, :M - 1].min()) == float(y[:, :M - 1].max()) == K
    del w, y
    N, K, g, n = (1 << 27) + 5, 8, 8, 1
    fmt = sop.ScaleFmt(0, 4, 4, 8, -1, -1)                            # 7 << 4: the scale 1
    words, payload = torch.full((N,), 7 << 4, dtype=torch.int16, device="cuda"), torch.zeros(N, dtype=torch.uint8, device="cuda")
    payload[N - 1] = 1
    layer = sop.PackedWeights(words, payload, N, K, g, n, fmt, [np.array([1.0, 3.0], np.float32)])
    y = cx.packed_matmul(torch.ones((2, K), dtype=torch.bfloat16, device="cuda"), layer)
    assert float(y[:, N - 1].min()) == float(y[:, N - 1].max()) == K + 2 and float(y[:, :N - 1].min()) == float(y[:, :N - 1].max()) == K


def test_packed_products_too_large_for_a_launch():
    """2^29 columns, or rows, of fewer than 64 elements: no tile is large enough, so two launches share them."""
    import torch
    cx = ctx()
    fmt, K = sop.ScaleFmt(0, 4, 4, 8, -1, -1), 8
    for M, N in ((1, (1 << 29) + 5), ((1 << 29) + 5, 1)):
        words, payload = torch.full((N,), 7 << 4, dtype=torch.int16, device="cuda"), torch.zeros(N, dtype=torch.uint8, device="cuda")
        x = torch.ones((M, K), dtype=torch.bfloat16, device="cuda")
        x[M - 1, 0] = 2
        payload[N - 1] = 1
        y = cx.packed_matmul(x, sop.PackedWeights(words, payload, N, K, 8, 1, fmt, [np.array([1.0, 3.0], np.float32)])).view(-1)
        assert float(y[-1]) == 13 and float(y[:-1].min()) == float(y[:-1].max()) == (9 if M == 1 else 10)
        del x, y, words, payload


# the product over the other index, by every kernel, in both formats and both types of result; K ends inside a step
@pytest.mark.parametrize("fmt", ["E4M3", "E5M2"])
@pytest.mark.parametrize("M, N, K", F8_KERNELS + [(2300, 4700, 1001), (1001, 4090, 700)])
def test_transposed_product_of_whole_numbers_is_exact(M, N, K, fmt):
    import torch
    rng = np.random.default_rng(19)
    (xc, xs), (vc, vs) = _integers(rng, M, K, 1, fmt), _integers(rng, K, N, 128)
    ref = (torch.from_numpy(OL.values(xc, xs, 1, fmt)).cuda() @ torch.from_numpy(OL.values(vc, vs, 128, "E4M3")).cuda()).cpu().numpy()
    x, v = _f8(xc, xs, 1, fmt), _f8(vc, vs, 128, "E4M3", codes_t=True)
    assert np.array_equal(_np(ctx().fp8_matmul(x, v, transposed=True, dtype=torch.float32)), ref)
    assert np.array_equal(_np(ctx().fp8_matmul(x, v, transposed=True)), _bf16(ref))


# results of 32 bits in whole lines of 128 bytes, which go past the caches, alone and added to what is there
@pytest.mark.parametrize("M, N, K", [(3, 128, 300), (40, 160, 300), (301, 1536, 300), (513, 1024, 300), (1001, 4096, 150), (2049, 2048, 150), (1025, 4096, 4000)])
def test_product_in_whole_lines(M, N, K):
    import torch
    rng = np.random.default_rng(20)
    (xc, xs), (wc, ws) = _integers(rng, M, K, 1), _integers(rng, N, K, 128)
    ref = (torch.from_numpy(OL.values(xc, xs, 1, "E4M3")).cuda() @ torch.from_numpy(OL.values(wc, ws, 128, "E4M3")).cuda().t()).cpu().numpy()
    buf = torch.full((M, N + 32), 7.0, device="cuda")
    assert buf.data_ptr() % 128 == 0
    ctx().fp8_matmul(_f8(xc, xs, 1, "E4M3"), _f8(wc, ws, 128, "E4M3"), out=buf[:, :N])
    assert np.array_equal(_np(buf[:, :N]), ref) and np.all(_np(buf[:, N:]) == 7)


@pytest.mark.parametrize("spaced", [True, False])
@pytest.mark.parametrize("M, N, K", [(65, 101, 160), (1100, 300, 512), (2100, 1001, 1024), (65, 1531, 2112), (130, 1027, 4096), (1025, 4090, 4000), (130, 2050, 4096)])
def test_weight_gradient_in_whole_lines(M, N, K, spaced):
    import torch
    rng = np.random.default_rng(21)
    xc, xs = _integers(rng, M, K, 1)
    dy, had = rng.integers(-8, 9, (M, N)).astype(np.float32), rng.integers(-9, 10, (N, K + 32)).astype(np.float32)
    ref = (torch.from_numpy(dy).cuda().double().t() @ torch.from_numpy(OL.values(xc, xs, 1, "E4M3")).cuda()).cpu().numpy()
    x, d, out = _f8(xc, xs, 1, "E4M3"), _t(dy, "bf16", 8 + -N % 8 if spaced else 0, 0 if spaced else 1), _t(had)
    assert out.data_ptr() % 128 == 0
    ctx().fp8_weight_grad(d, x, out=out[:, :K], accumulate=True)
    assert np.array_equal(_np(out[:, :K]), ref + had[:, :K]) and np.array_equal(_np(out[:, K:]), had[:, K:])
    ctx().fp8_weight_grad(d, x, out=out[:, :K])
    assert np.array_equal(_np(out[:, :K]), ref) and np.array_equal(_np(out[:, K:]), had[:, K:])


def _near_codes_within(q, value, fmt, err):
    """As _near_codes, `value` being known to `err` element by element."""
    codes, scales = _bytes(q.codes), _bytes(q.scales)
    M, K = value.shape
    got = scales.astype(np.int64) - 127
    lo, hi = OL.block_exponents(np.maximum(np.abs(value) - err, 0), 1, fmt), OL.block_exponents(np.abs(value) + err, 1, fmt)
    assert np.all((got >= lo) & (got <= hi))
    step = 2.0 ** OL.spread(got, 1, M, K)
    unit = 2.0 ** np.maximum(np.floor(np.log2(np.maximum((np.abs(value) + err) / step, 1e-300))), OL.LEAST[fmt]) * 2.0 ** -OL.MANT[fmt] * step
    assert np.all(np.abs(OL.values(codes, scales, 1, fmt) - value) <= unit / 2 + err)


# rows on 16 bytes and off them, rows that end inside eight elements and on them, more rows than the wavefronts of a launch (the last ones are compared)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", ["E4M3", "E5M2"])
@pytest.mark.parametrize("M, F", [(1, 8), (33, 1001), (130, 512), (70, 1000), (9000, 520)])
def test_gated_unit_and_gradient_on_any_alignment(M, F, dtype, fmt):
    rng = np.random.default_rng(22)
    g, u, dh = rng.standard_normal((M, F)) * 4, rng.standard_normal((M, F)), rng.standard_normal((M, F)) * 1e-3
    g, u, dh = (_bf16(t) if dtype == "bf16" else t.astype(np.float32) for t in (g, u, dh))
    end = slice(max(0, M - 150), M)
    for pad, shift in ((0, 0), (-F % 8 + 8, 0), (5, 1)):
        h, g8, u8 = ctx().fp8_gated(_t(g, dtype, pad, shift), _t(u, dtype, pad, shift), fmt=FMT[fmt])
        dg, du, dg8, du8 = ctx().fp8_gated_grad(g8, u8, _t(dh, dtype, pad, shift), fmt=FMT[fmt])
        h, g8, u8, dg8, du8 = (sop.Fp8Blocks(q.codes[end], q.scales[end]) for q in (h, g8, u8, dg8, du8))
        for q, x in ((g8, g), (u8, u)):
            codes, scales = OL.quantize(x[end], 1, fmt)
            assert np.array_equal(_bytes(q.codes), codes) and np.array_equal(_bytes(q.scales), scales)
        _near_codes(h, OL.silu_mul(g[end].astype(np.float64), u[end].astype(np.float64)), fmt, 2.0 ** -20)
        gv, uv = (OL.values(_bytes(q.codes), _bytes(q.scales), 1, fmt) for q in (g8, u8))
        wg, wu = OL.silu_mul_grad(gv, uv, dh[end].astype(np.float64))
        # dgate's last factor, 1 + g (1 - s), may cancel: its error is one of the two terms
        part = np.abs(dh[end] * uv) * (1 + np.abs(gv)) * (1 / (1 + np.exp(-gv)))
        tol = 2.0 ** -8 if dtype == "bf16" else 0
        assert np.all(np.abs(_np(dg[end]) - wg) <= tol * np.abs(wg) + 2.0 ** -20 * part)
        assert np.all(np.abs(_np(du[end]) - wu) <= (tol + 2.0 ** -20) * np.abs(wu))
        _near_codes_within(dg8, wg, fmt, 2.0 ** -20 * part)
        _near_codes(du8, wu, fmt, 2.0 ** -20)
