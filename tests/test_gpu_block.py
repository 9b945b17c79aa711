"""What stands around a linear layer in a block of a model, on the GPU against the oracle in 64 bits: norms with the residual stream and their gradients,
products with an epilogue and its gradient, gradients clipped together.

Tolerances, U = 2^-24 (half a step of binary32).
  A row's sum of D terms is added up by at least 64 threads: chains of D / 64 additions and some 16 to join them, (D / 64 + 16) U of the magnitudes' sum.  1 / rms
  is off by half of that (the sum stands under a root), and by the instruction's and the mean's roundings, 4 U: E = (D / 128 + 12) U of itself.
  The sum s: v = scale gate after y / rms(y) has E and five roundings, then one addition.  n: the relative error of s as a vector goes into its rms.
  Gradients: the same counted along their formulas (see there).  Sums over M rows: at most M U of the magnitudes' sum beside the terms' own errors.
  Activations: the hardware's exponential, reciprocal and the fitted tail are each off by 8 U at most, taken together less than 2^-20 of the value; gelu by tanh
  has an exponent of 1.6 |z + 0.045 z^3| that is itself rounded (three roundings), and so is off by as many 4 U more where it is small because of it.  Where results are
  bf16 the exponent (z^2 / 2 of gelu, |z| of silu) is formed without a low part: a rounding of z^2, of the factor and of the product, 2.5 U of it (1.5 U without z^2).
  A rounding to bf16 is off by 2^-8 of the value at most, one to binary32 by U, and what
  ends below the least normal number 2^-126, where numbers are 2^-149 apart (bf16: 2^-133), by half of that more."""
import numpy as np
import pytest
from scipy import special

import paper_2605_14929_amd as sop
from oracle import block as OB
from oracle import linear as OL
from gpu_util import ctx
from test_gpu_linear import F8_KERNELS, FMT, _bf16, _bytes, _f8, _integers, _np, _t

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
STEP = {"bf16": 2.0 ** -8, "f32": U}
ACT = {"none": None, "relu": sop.RELU, "silu": sop.SILU, "gelu": sop.GELU, "gelu_tanh": sop.GELU_TANH}
TYPES = [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f32", "bf16")]     # y, r


def _type(t):
    import torch
    return torch.float32 if t == "f32" else torch.bfloat16


def _to(x, t):
    return _bf16(x) if t == "bf16" else np.asarray(x, dtype=np.float32)


def _vec(x):
    import torch
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda()


def _close(got, want, err, t):
    """Numbers of type t against what they should be, known to err."""
    got, want = _np(got), np.asarray(want)
    tol = err + STEP[t] * (np.abs(want) + err) + 2.0 ** -149 + (2.0 ** -134 if t == "bf16" else 0)   # (below 2^-126 numbers are 2^-149 apart, bf16 ones 2^-133)
    bad = np.abs(got - want) > tol
    assert not np.any(bad), (np.argwhere(bad)[:5], got[bad][:5], want[bad][:5], np.broadcast_to(tol, want.shape)[bad][:5])


def _near_codes_within(q, value, fmt, err):
    """Codes and scales of what is known to `err` element by element.  A block that may be zero, none of its elements being larger than its error, may have
    the scale of such a block, 1."""
    codes, scales = _bytes(q.codes), _bytes(q.scales)
    M, K = value.shape
    err = err + 2.0 ** -149                                             # (a value below 2^-126 was rounded to a multiple of 2^-149 on its way)
    got = scales.astype(np.int64) - 127
    lo, hi = OL.block_exponents(np.maximum(np.abs(value) - err, 0), 1, fmt), OL.block_exponents(np.abs(value) + err, 1, fmt)
    least = np.maximum(np.abs(value) - err, 0)
    nothing = np.array([[np.all(least[i, 128 * j:128 * j + 128] == 0) for j in range(got.shape[1])] for i in range(M)])
    lo = np.where(nothing, -126, lo)                                    # (what is left of it may be as small as it likes)
    assert np.all(((got >= lo) & (got <= hi)) | (nothing & (got == 0)))
    step = 2.0 ** OL.spread(got, 1, M, K)
    unit = 2.0 ** np.maximum(np.floor(np.log2(np.maximum((np.abs(value) + err) / step, 1e-300))), OL.LEAST[fmt]) * 2.0 ** -OL.MANT[fmt] * step
    assert np.all(np.abs(OL.values(codes, scales, 1, fmt) - value) <= unit / 2 + err)


def _norm_case(rng, M, D, ty, tr, G, after, before, scale=0.7):
    """Operands of a norm: rows and columns of different sizes."""
    size = lambda: np.exp(0.5 * rng.standard_normal((1, D))) * 2.0 ** rng.integers(-4, 5, (M, 1))  # noqa: E731
    c = dict(r=_to(rng.standard_normal((M, D)) * size(), tr), y=_to(rng.standard_normal((M, D)) * size(), ty),
             after=(1 + 0.3 * rng.standard_normal(D)).astype(np.float32) if after else None, before=(1 + 0.3 * rng.standard_normal(D)).astype(np.float32) if before else None,
             gate=_to(rng.standard_normal((G, D)), ty) if G else None, scale=float(np.float32(scale)), eps=1e-6)
    return c


def _gate(c, ty, pad, shift):
    return None if c["gate"] is None else _t(c["gate"], ty, pad, shift)


def _forward_errors(c):
    """(s, its error, n, its error) of a case"""
    D = c["r"].shape[1]
    E = (D / 128 + 12) * U
    s, n = OB.residual_norm(**c)
    es = 0.0 * s if c["y"] is None else np.abs(s - c["r"]) * ((E if c["after"] is not None else 0) + 6 * U) + U * np.abs(s)
    if n is None:
        return s, es, None, None
    unit = OB.unit(s, c["eps"])
    of_rms = np.linalg.norm(es, axis=1, keepdims=True) / np.maximum(np.linalg.norm(s, axis=1, keepdims=True), 1e-300) * (np.abs(s).max(1, keepdims=True) > 0)
    return s, es, n, np.abs(c["before"]) * unit * es + np.abs(n) * (of_rms + E + 4 * U)


def _check_norm(c, ty, tr, fmt="E4M3", numbers="f32", pad=0, shift=0, out=None):
    r, y = _t(c["r"], tr, pad, shift), None if c["y"] is None else _t(c["y"], ty, pad, shift)
    has = c["before"] is not None
    s, n, n8 = ctx().residual_norm(r, y, after=_vec(c["after"]), gate=_gate(c, ty, pad, shift), scale=c["scale"], before=_vec(c["before"]), eps=c["eps"],
                                   dtype=_type(numbers) if has else None, fmt=FMT[fmt] if has else None, out=r if out == "r" else None)
    want, es, wn, en = _forward_errors(c)
    if y is None:
        assert s is r
    else:
        assert s.dtype is _type(tr) and (out is None or s is r)
        _close(s, want, es, tr)
    if not has:
        assert n is None and n8 is None
        return
    _close(n, wn, en, numbers)
    _near_codes_within(n8, wn, fmt, en)


WIDTHS = [1, 7, 8, 64, 129, 512, 513, 1000, 1024, 1025, 2048, 2050, 4096, 4104, 5024, 8192, 8193, 12000, 12288, 12296, 16384, 16385, 20001]


@pytest.mark.parametrize("ty, tr", TYPES)
@pytest.mark.parametrize("D", WIDTHS)
def test_norm(D, ty, tr):
    rng = np.random.default_rng(D)
    for M, G, after, before, pad, shift in ((1, 0, True, True, 0, 0), (6, 3, True, True, 8 + -D % 8, 0), (5, 5, True, True, 3, 1), (9, 1, False, True, 0, 0), (4, 2, True, False, 0, 0), (3, 0, False, False, 5, 1)):
        _check_norm(_norm_case(rng, M, D, ty, tr, G, after, before), ty, tr, "E5M2" if M % 2 else "E4M3", "bf16" if M % 3 else "f32", pad, shift, "r" if M > 5 else None)


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 1000, 4096, 8192, 20000])
def test_norm_of_the_stream_alone(D, t):
    """No block's output: the norm in front of the first block, or the last one."""
    rng = np.random.default_rng(D + 1)
    c = _norm_case(rng, 7, D, t, t, 0, False, True)
    c["y"] = None
    _check_norm(c, t, t, numbers=t)


@pytest.mark.parametrize("D", [100, 1000, 4096, 8192])
def test_norm_of_more_rows_than_are_in_flight(D):
    """Several rows a workgroup (and a wavefront), gates that change between and inside its rows; the last ones are compared, and some from the middle."""
    rng = np.random.default_rng(2)
    for M, G in ((9000, 0), (8194, 2), (8000, 4000), (8001, 2667)):
        c = _norm_case(rng, M, D, "bf16", "f32", G, True, True)
        import torch
        s, n, n8 = ctx().residual_norm(_t(c["r"]), _t(c["y"], "bf16"), after=_vec(c["after"]), gate=_gate(c, "bf16", 0, 0), scale=c["scale"], before=_vec(c["before"]), dtype=torch.float32, fmt=sop.E4M3)
        at = np.concatenate([np.arange(5), np.arange(M // 2 - 20, M // 2 + 20), np.arange(M - 60, M)])
        part = dict(c, r=c["r"][at], y=c["y"][at], gate=None if not G else OB.rows_of(c["gate"], M, D)[at])
        want, es, wn, en = _forward_errors(part)
        idx = torch.from_numpy(at).cuda()
        _close(s[idx], want, es, "f32")
        _close(n[idx], wn, en, "f32")
        _near_codes_within(sop.Fp8Blocks(n8.codes.view(torch.uint8)[idx].view(torch.float8_e4m3fn), n8.scales.view(torch.uint8)[idx].view(torch.float8_e8m0fnu)), wn, "E4M3", en)


@pytest.mark.parametrize("D", [96, 1000, 4096, 8192, 20000])
def test_norm_at_the_edges(D):
    """Rows of zeros, rows whose squares leave binary32 above and below, one large element, infinities and NaN, which stay in their rows."""
    rng = np.random.default_rng(3)
    base = rng.standard_normal((12, D))
    c = _norm_case(rng, 12, D, "f32", "f32", 0, True, True, scale=1.0)
    r, y = base.copy(), rng.standard_normal((12, D))
    r[0], y[0] = 0, 0
    r[1], y[1] = 0, 1e30 * y[1]
    r[2], y[2] = 1e36 * r[2], 1e-30 * y[2]
    r[3], y[3] = 1e-30 * r[3], 1e-25 * y[3]
    r[4, D // 2], y[4, 0] = 3e38, -3e38
    r[5], y[5] = 1e20 * r[5], 1e20 * y[5]
    r[6], y[6] = 0, 1e19 * y[6]
    r[7, 1] = np.nan
    y[8, D - 1] = np.inf
    r[9, 0] = -np.inf
    y[10, 2] = np.nan
    c.update(r=r.astype(np.float32), y=y.astype(np.float32), gate=None)
    import torch
    s, n, n8 = ctx().residual_norm(_t(c["r"]), _t(c["y"]), after=_vec(c["after"]), before=_vec(c["before"]), dtype=torch.float32, fmt=sop.E4M3)
    whole = [0, 1, 2, 3, 4, 5, 6, 11]
    part = dict(c, r=c["r"][whole], y=c["y"][whole])
    want, es, wn, en = _forward_errors(part)
    _close(s[whole], want, es, "f32")
    _close(n[whole], wn, en + 2.0 ** -126, "f32")
    s, n = _np(s), _np(n)
    assert np.isnan(s[7, 1]) and np.isfinite(np.delete(s[7], 1)).all() and np.isnan(n[7]).all()
    assert np.isnan(s[8, D - 1]) and np.array_equal(s[8, :D - 1], c["r"][8, :D - 1]) and np.isnan(n[8]).all()      # the others are y / infinity = 0
    assert s[9, 0] == -np.inf and np.isnan(n[9, 0]) and np.all(n[9, 1:] == 0)
    assert np.isnan(s[10]).all() and np.isnan(n[10]).all()
    codes = OL.decode(_bytes(n8.codes), "E4M3")
    assert np.isnan(codes[[7, 10]]).all() and np.isnan(codes[9, 0]) and np.all(codes[9, 1:] == 0)


# ---- gradients of the norm

def _grad_errors(c, ds, dn, s):
    """Errors of the gradients' formulas.  c = (D / 32 + 60) U covers what a term of a row's result has behind it: twice E (1 / rms, and h within the mean), the sum's own
    (D / 64 + 16) U, and some ten roundings."""
    M, D = c["r"].shape
    k = (D / 32 + 60) * U
    w = OB.residual_norm_grad(ds, dn, s, before=c["before"], y=c["y"], after=c["after"], gate=c["gate"], scale=c["scale"], eps=c["eps"])
    e = {"dr": U * np.abs(w["dr"])}
    if c["before"] is not None:
        u = OB.unit(s.astype(np.float64), c["eps"])
        h, p = np.abs(s) * u, np.abs(c["before"] * dn.astype(np.float64))
        e["dr"] = e["dr"] + k * u * (p + h * np.mean(p * h, 1, keepdims=True))
        e["dbefore"] = (M * U + k) * np.sum(np.abs(dn) * h, 0)
    if c["y"] is None:
        return w, e
    y, g = np.abs(c["y"].astype(np.float64)), np.abs(c["scale"] * OB.rows_of(c["gate"], M, D))
    a = 1.0 if c["after"] is None else np.abs(c["after"].astype(np.float64))
    q, eq = g * a * np.abs(w["dr"]), g * a * (e["dr"] + 4 * U * np.abs(w["dr"]))
    x = y
    e["dy"] = eq
    if c["after"] is not None:
        u = OB.unit(c["y"].astype(np.float64), c["eps"])
        x = y * u
        e["dy"] = u * (eq + k * q + x * (np.mean(eq * x, 1, keepdims=True) + k * np.mean(q * x, 1, keepdims=True)))
        e["dafter"] = np.sum(g * x * (e["dr"] + (M * U + k) * np.abs(w["dr"])), 0)
    if c["gate"] is not None:
        G = c["gate"].shape[0]
        e["dgate"] = np.sum((c["scale"] * a * x * (e["dr"] + (M * U + k) * np.abs(w["dr"]))).reshape(G, M // G, D), 1)
    return w, e


def _check_norm_grad(c, ty, tr, rng, fmt="E5M2", pad=0, shift=0, with_ds=True):
    M, D = c["r"].shape
    s = c["r"]
    ds = _to(rng.standard_normal((M, D)) * 1e-3, tr) if with_ds else None
    dn = _to(rng.standard_normal((M, D)) * 1e-3, ty) if c["before"] is not None else None
    up = lambda x, t: None if x is None else _t(x, t, pad, shift)  # noqa: E731
    got = ctx().residual_norm_grad(up(ds, tr), up(dn, ty), up(s, tr) if dn is not None else None, before=_vec(c["before"]), y=up(c["y"], ty), after=_vec(c["after"]),
                                   gate=_gate(c, ty, pad, shift), scale=c["scale"], eps=c["eps"], fmt=FMT[fmt] if c["y"] is not None else None)
    want, err = _grad_errors(c, ds, dn, s)
    _close(got.dr, want["dr"], err["dr"], tr)
    assert (got.dbefore is None) == (dn is None) and (got.dy is None) == (c["y"] is None) and (got.dafter is None) == (c["after"] is None) and (got.dgate is None) == (c["gate"] is None)
    if dn is not None:
        _close(got.dbefore, want["dbefore"], err["dbefore"], "f32")
    if c["y"] is None:
        assert got.dy8 is None
        return
    _close(got.dy, want["dy"], err["dy"], ty)
    _near_codes_within(got.dy8, want["dy"], fmt, err["dy"])
    if c["after"] is not None:
        _close(got.dafter, want["dafter"], err["dafter"], "f32")
    if c["gate"] is not None:
        _close(got.dgate, want["dgate"], err["dgate"], ty)


@pytest.mark.parametrize("ty, tr", TYPES)
@pytest.mark.parametrize("D", WIDTHS)
def test_norm_gradients(D, ty, tr):
    rng = np.random.default_rng(D + 2)
    for M, G, after, before, pad, shift in ((1, 0, True, True, 0, 0), (6, 3, True, True, 8 + -D % 8, 0), (5, 5, True, True, 3, 1), (9, 1, False, True, 0, 0), (4, 2, True, False, 0, 0), (3, 0, False, False, 5, 1)):
        _check_norm_grad(_norm_case(rng, M, D, ty, tr, G, after, before), ty, tr, rng, "E5M2" if M % 2 else "E4M3", pad, shift, with_ds=not (before and M == 9))


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 1000, 4096, 8192, 20000])
def test_norm_gradients_of_the_stream_alone(D, t):
    rng = np.random.default_rng(D + 3)
    for with_ds in (True, False):
        c = _norm_case(rng, 7, D, t, t, 0, False, True)
        c["y"] = None
        _check_norm_grad(c, t, t, rng, with_ds=with_ds)


# rows of a gate shared out to several workgroups, several gates' rows a workgroup, more groups than workgroups, one row of the gate for each of y
@pytest.mark.parametrize("D", [72, 600, 1100, 3000, 8192, 9000])
@pytest.mark.parametrize("M, G", [(3001, 0), (2000, 1), (2400, 3), (1400, 700), (2100, 2100), (3300, 1100)])
def test_norm_gradients_of_many_rows(M, G, D):
    if D > 4000 and M % 2:
        M, G = M // 2, G // 2 if G == M else G
        M -= M % max(G, 1)
    rng = np.random.default_rng(4)
    _check_norm_grad(_norm_case(rng, M, D, "bf16", "f32", G, True, True), "bf16", "f32", rng)


@pytest.mark.parametrize("D", [96, 1000, 4096, 8192, 20000])
def test_norm_gradients_at_the_edges(D):
    """Rows of zeros, rows whose squares leave binary32; infinities and NaN stay in their rows, but for the sums over rows."""
    rng = np.random.default_rng(5)
    c = _norm_case(rng, 6, D, "f32", "f32", 0, True, True, scale=1.0)
    s, y = rng.standard_normal((6, D)), rng.standard_normal((6, D))
    s[0], y[0] = 0, 0
    s[1], y[1] = 1e30 * s[1], 1e30 * y[1]
    s[2], y[2] = 1e-25 * s[2], 1e36 * y[2]
    s[3, 0], y[3, 5] = 3e38, 3e38
    c.update(r=s.astype(np.float32), y=y.astype(np.float32), gate=None)
    _check_norm_grad(c, "f32", "f32", rng)
    import torch
    ds, dn = rng.standard_normal((6, D)).astype(np.float32), rng.standard_normal((6, D)).astype(np.float32)
    clean = ctx().residual_norm_grad(_t(ds), _t(dn), _t(c["r"]), before=_vec(c["before"]), y=_t(c["y"]), after=_vec(c["after"]), fmt=sop.E5M2)
    for place, bad in (("s", np.nan), ("y", np.inf), ("dn", np.nan), ("ds", -np.inf)):
        m = dict(s=c["r"].copy(), y=c["y"].copy(), dn=dn.copy(), ds=ds.copy())
        m[place][4, 3] = bad
        got = ctx().residual_norm_grad(_t(m["ds"]), _t(m["dn"]), _t(m["s"]), before=_vec(c["before"]), y=_t(m["y"]), after=_vec(c["after"]), fmt=sop.E5M2)
        others = [0, 1, 2, 3, 5]
        assert torch.equal(got.dr[others], clean.dr[others]) and torch.equal(got.dy[others], clean.dy[others]), place
        assert np.isnan(_np(got.dy[4])).any(), place


def test_norms_of_no_rows():
    import torch
    r, w = torch.empty((0, 300), device="cuda"), torch.ones(300, device="cuda")
    s, n, n8 = ctx().residual_norm(r, r, after=w, gate=torch.ones((2, 300), device="cuda"), before=w, dtype=torch.float32, fmt=sop.E4M3)
    assert s.shape == n.shape == (0, 300) and n8.shape == (0, 300)
    d = ctx().residual_norm_grad(r, r, r, before=w, y=r, after=w, gate=torch.ones((40000, 300), dtype=torch.bfloat16, device="cuda"), fmt=sop.E5M2)
    assert d.dr.shape == d.dy.shape == (0, 300)
    for g in (d.dbefore, d.dafter, d.dgate):
        assert float(g.float().abs().max()) == 0
    assert d.dgate.shape == (40000, 300)


def test_norm_refusals():
    import torch
    cx = ctx()
    r, w = torch.ones((4, 64), device="cuda"), torch.ones(64, device="cuda")

    def refused(status, f, *a, **k):
        with pytest.raises(sop.SopError) as e:
            f(*a, **k)
        assert e.value.status == status, e.value

    refused(1, cx.residual_norm, r.cpu(), before=w, fmt=sop.E4M3)
    refused(1, cx.residual_norm, r.half(), before=w, fmt=sop.E4M3)
    refused(2, cx.residual_norm, r.t(), before=w, fmt=sop.E4M3)
    refused(1, cx.residual_norm, r, before=w)                          # nothing asked for
    refused(1, cx.residual_norm, r, fmt=sop.E4M3)
    refused(1, cx.residual_norm, r)
    refused(1, cx.residual_norm, r, after=w, before=w, fmt=sop.E4M3)   # no block's output
    refused(2, cx.residual_norm, r, r[:3], after=w)
    refused(2, cx.residual_norm, r, r, after=w[:63].clone())
    refused(1, cx.residual_norm, r, r, after=w.bfloat16())
    refused(1, cx.residual_norm, r, r, after=torch.ones(128, device="cuda")[::2])
    refused(2, cx.residual_norm, r, r, gate=torch.ones((3, 64), device="cuda"))
    refused(1, cx.residual_norm, r, r, gate=w.half())
    refused(1, cx.residual_norm, r, r, out=r.bfloat16())
    refused(2, cx.residual_norm, r, r, out=torch.empty((4, 65), device="cuda"))
    y = r.clone()
    refused(1, cx.residual_norm, r, y, out=y)                          # the sum in y's place
    refused(1, cx.residual_norm, r, before=w, fmt=sop.E4M3, out=y)
    refused(1, cx.residual_norm, r, before=w, fmt=sop.E4M3, eps=0.0)
    refused(1, cx.residual_norm, r, before=w, dtype=torch.float16)
    refused(1, cx.residual_norm_grad, None)
    refused(1, cx.residual_norm_grad, r, dn=r, before=w)               # no s
    refused(1, cx.residual_norm_grad, r, y=r.clone(), after=w, s=r)
    refused(1, cx.residual_norm_grad, r, r.bfloat16(), r, before=w, y=r.clone(), after=w)
    refused(1, cx.residual_norm_grad, r, r, r.bfloat16(), before=w)
    refused(2, cx.residual_norm_grad, r, r[:3], r, before=w)
    refused(1, cx.residual_norm_grad, r, after=w)
    refused(1, cx.residual_norm_grad, r, r, r, before=w, fmt=sop.E5M2)


# ---- products with an epilogue

def _z_case(rng, M, N, K, fmt="E4M3"):
    """Whole numbers times 2^-4 with a bias of such: z is exact, and within some tens."""
    (xc, xs), (wc, ws) = _integers(rng, M, K, 1, fmt), _integers(rng, N, K, 128)
    xs = (xs - (7 if K > 600 else 6)).astype(np.uint8)
    x, w = OL.values(xc, xs, 1, fmt), OL.values(wc, ws, 128, "E4M3")
    import torch
    bias = rng.integers(-64, 65, N) / 16
    z = (torch.from_numpy(x).cuda() @ torch.from_numpy(w).cuda().t()).cpu().numpy()
    return _f8(xc, xs, 1, fmt), _f8(wc, ws, 128, "E4M3", codes_t=False), bias, z


def _act_error(name, z, dtype="f32"):
    y = np.abs(OB.act(name, z))
    if name in ("none", "relu"):
        return 0 * y
    exponent = 0.5 * z * z if name == "gelu" else np.abs(z) if name == "silu" else 1.6 * np.abs(z + 0.044715 * z ** 3)
    more = exponent * U * ((4 if name == "gelu_tanh" else 0) + (0 if dtype == "f32" else 2.5))
    return y * np.where(z < 0, 2.0 ** -20 + more, 2.0 ** -20 + more * np.exp(-np.minimum(exponent, 700.0))) + 2.0 ** -148   # (above zero it stands beside 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", OB.ACTS)
@pytest.mark.parametrize("M, N, K", F8_KERNELS + [(1, 1, 1), (1, 16, 128), (33, 1003, 260)])
def test_product_with_an_epilogue(M, N, K, name, dtype):
    import torch
    rng = np.random.default_rng(6)
    x, w, bias, z = _z_case(rng, M, N, K, "E5M2" if M % 2 else "E4M3")
    for has_bias, has_residual, keep, scale, in_place, pad in ((True, True, False, 0.7, True, 3), (True, False, True, 1.0, False, 0), (False, True, True, -0.3, False, 0)):
        if M * N > 4_000_000 and not keep:
            continue
        zz = z + (bias if has_bias else 0)
        res = _to(rng.standard_normal((M, N)) * 4, dtype) if has_residual else None
        r = None if res is None else _t(res, dtype, pad, pad & 1)
        got = ctx().fp8_linear(x, w, bias=_vec(bias) if has_bias else None, act=ACT[name], residual=r, scale=scale, keep=keep, dtype=_type(dtype), out=r if in_place else None)
        y, kept = got if keep else (got, None)
        assert not in_place or y is r
        f = float(np.float32(scale))
        want = f * OB.act(name, zz) + (0 if res is None else res)
        _close(y, want, abs(f) * _act_error(name, zz, dtype) + U * np.abs(want) + U * np.abs(f * OB.act(name, zz)), dtype)
        if keep:
            assert np.array_equal(_np(kept), _bf16(zz) if dtype == "bf16" else zz)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_transposed_product_with_an_epilogue(dtype):
    rng = np.random.default_rng(7)
    for M, N, K in ((3, 130, 300), (301, 1531, 300), (2300, 4700, 150)):
        (xc, xs), (vc, vs) = _integers(rng, M, K, 1, "E5M2"), _integers(rng, K, N, 128)
        import torch
        z = (torch.from_numpy(OL.values(xc, xs, 1, "E5M2")).cuda() @ torch.from_numpy(OL.values(vc, vs, 128, "E4M3")).cuda()).cpu().numpy()
        res = rng.integers(-64, 65, (M, N)).astype(np.float32)
        y = ctx().fp8_linear(_f8(xc, xs, 1, "E5M2"), _f8(vc, vs, 128, "E4M3", codes_t=True), residual=_t(res, dtype), scale=0.5, transposed=True, dtype=_type(dtype))
        assert np.array_equal(_np(y), _to(0.5 * z + res, dtype))        # (whole numbers and halves)


def test_epilogue_at_infinities_and_nan():
    """Activations over all of binary32, through a product whose one column is z itself by its bias."""
    import torch
    rng = np.random.default_rng(8)
    z = np.concatenate([np.linspace(-20, 20, 801), -np.geomspace(1e-30, 3e38, 200), np.geomspace(1e-30, 3e38, 200), [0.0, -0.0, np.inf, -np.inf, np.nan, -87.4, -100.0, -103.5, -13.9]]).astype(np.float32)
    N = z.size
    x = _f8(np.zeros((2, 16), np.uint8), np.full((2, 1), 127, np.uint8), 1, "E4M3")
    w = _f8(np.zeros((N, 16), np.uint8), np.full((-(-N // 128), 1), 127, np.uint8), 128, "E4M3")
    ok = ~np.isnan(z)
    zw = z.astype(np.float64)
    for name in OB.ACTS:
        y = _np(ctx().fp8_linear(x, w, bias=_vec(z), act=ACT[name], dtype=torch.float32))
        want = OB.act(name, zw)
        assert np.isnan(y[:, ~ok]).all() and np.array_equal(y[0], y[1], equal_nan=True), name
        if name == "none":
            assert np.array_equal(y[0], zw, equal_nan=True)
            continue
        assert np.array_equal(np.isinf(y[0]), np.isinf(want))
        f = ok & np.isfinite(want)
        err = _act_error(name, np.clip(zw[f], -1e4, 1e4)) + 2.0 ** -20 * np.abs(want[f])
        assert np.all(np.abs(y[0][f] - want[f]) <= err), (name, zw[f][np.abs(y[0][f] - want[f]) > err][:5], y[0][f][np.abs(y[0][f] - want[f]) > err][:5])
        # and the slopes there
        for dtype in ("f32", "bf16"):
            zz, dy = _to(z[None].repeat(3, 0), dtype), _to(rng.standard_normal((3, N)), dtype)
            dz, dz8, db = ctx().fp8_linear_grad(_t(dy, dtype), _t(zz, dtype), act=ACT[name], scale=0.5)
            wz = np.float64(zz)
            k = np.isfinite(wz) | np.isinf(wz)
            want_dz = 0.5 * dy * OB.slope(name, wz)
            _close(dz[:, torch.from_numpy(k[0])], want_dz[:, k[0]], (0.5 * np.abs(dy) * _slope_error(name, wz, dtype))[:, k[0]], dtype)
            if name != "relu":
                assert np.isnan(_np(dz)[~k]).all()


PACKED = [(1, 4096, 400, 16), (16, 100, 264, 8), (32, 330, 192, 64), (50, 8000, 136, 8), (64, 11000, 96, 32), (128, 4096, 584, 8), (512, 4096, 96, 16), (1000, 4000, 72, 8), (2049, 3841, 80, 16), (4097, 3841, 72, 8)]


@pytest.mark.parametrize("n", [1, 3, 4, 6])
@pytest.mark.parametrize("M, N, K, g", PACKED)
def test_packed_product_with_an_epilogue(M, N, K, g, n):
    """Against the product without one, whose own error its tests hold: entries and scales are powers of two, x whole numbers, so sums are exact."""
    import torch
    rng = np.random.default_rng(9)
    count = N * K // g
    words = torch.from_numpy(((7 << 4) + 16 * rng.integers(-2, 1, count)).astype(np.int16)).cuda()              # scales of 1, 1/2, 1/4
    payload = torch.from_numpy(rng.integers(0, 256, count * g * n // 8).astype(np.uint8)).cuda()
    table = np.sort(rng.choice([-2.0, -1.0, -0.5, 0.5, 1.0, 2.0], 1 << n)).astype(np.float32)
    layer = sop.PackedWeights(words, payload, N, K, g, n, sop.ScaleFmt(0, 4, 4, 8, -1, -1), [table])
    x = _t(rng.integers(-2, 3, (M, K)) / 16.0, "bf16")
    codes = ((payload.view(count, g * n // 8, 1) >> torch.arange(8, device="cuda")) & 1).view(count, g, n).long()
    codes = (codes << torch.arange(n, device="cuda")).sum(-1)
    v = (torch.from_numpy(table).cuda().double()[codes] * torch.exp2((words.double() - 112)[:, None] / 16)).view(N, K)
    z = (x.double() @ v.t()).cpu().numpy()
    assert np.array_equal(_np(ctx().packed_matmul(x, layer)), _bf16(z))
    bias = rng.integers(-64, 65, N) / 16
    res = _bf16(rng.standard_normal((M, N)) * 4)
    for name, keep, in_place in (("gelu", True, False), ("silu", False, True)):
        r = _t(res, "bf16", 5, 1)
        got = ctx().packed_linear(x, layer, bias=_vec(bias), act=ACT[name], residual=r, scale=0.7, keep=keep, out=r if in_place else None)
        y, kept = got if keep else (got, None)
        f = float(np.float32(0.7))
        a = OB.act(name, z + bias)
        want = f * a + res
        _close(y, want, f * _act_error(name, z + bias, "bf16") + U * np.abs(want) + U * np.abs(f * a), "bf16")
        if keep:
            assert np.array_equal(_np(kept), _bf16(z + bias))


def test_epilogue_refusals():
    import torch
    cx = ctx()
    x = torch.ones((4, 256), device="cuda")
    q, w = cx.fp8_quantize(x), cx.fp8_quantize(torch.ones((140, 256), device="cuda"), rows=128)
    b, r = torch.ones(140, device="cuda"), torch.ones((4, 140), dtype=torch.bfloat16, device="cuda")

    def refused(status, f, *a, **k):
        with pytest.raises(sop.SopError) as e:
            f(*a, **k)
        assert e.value.status == status, e.value

    refused(1, cx.fp8_linear, q, w, act=7)
    refused(2, cx.fp8_linear, q, w, bias=b[:139].clone())
    refused(1, cx.fp8_linear, q, w, bias=b.bfloat16())
    refused(1, cx.fp8_linear, q, w, bias=b.cpu())
    refused(2, cx.fp8_linear, q, w, residual=r[:3])
    refused(1, cx.fp8_linear, q, w, residual=r.float())
    refused(1, cx.fp8_linear, q, w, residual=r, dtype=torch.float32)
    refused(2, cx.fp8_linear, q, w, residual=r.t().contiguous().t())
    refused(1, cx.fp8_linear, q, w, transposed=True)
    refused(1, cx.fp8_linear_grad, r, act=sop.GELU)                    # no z
    refused(1, cx.fp8_linear_grad, r, r.float(), act=sop.GELU)
    refused(2, cx.fp8_linear_grad, r, r[:3], act=sop.GELU)
    refused(1, cx.fp8_linear_grad, r, r, act=9)
    refused(1, cx.fp8_linear_grad, r.half(), r.half(), act=1)
    refused(1, cx.fp8_linear_grad, r.cpu(), r, act=1)


# ---- gradient of an epilogue

def _slope_error(name, z, dtype="f32"):
    """The slope's two terms, each to 2^-20 (and what an exponent's roundings add; of bf16 numbers gelu's is formed without a low part: 2.5 U of z^2 / 2)."""
    if name in ("none", "relu"):
        return np.zeros_like(z)
    c = np.clip(z, -1e4, 1e4)
    if name == "gelu":
        terms = np.abs(OB.act(name, c) / np.where(c == 0, 1, c)) + np.abs(c) * np.exp(-0.5 * c * c) * 0.4 + 0.5 * (c == 0)
        tail = special.ndtr(-np.abs(c)) + np.abs(c) * np.exp(-0.5 * c * c) * 0.4
        return 2.0 ** -19 * terms + (0 if dtype == "f32" else 2.5 * U * 0.5 * c * c) * tail + 2.0 ** -148
    v = c if name == "silu" else 1.6 * np.abs(c + 0.044715 * c ** 3)
    inner = np.abs(c) if name == "silu" else 1.6 * np.abs(c) * (1 + 3 * 0.044715 * c * c)
    q = special.expit(np.where(c < 0, -np.abs(v), np.abs(v)))
    return q * (1 + inner * special.expit(-np.abs(v) * np.sign(c))) * (2.0 ** -20 + 8 * U * np.minimum(np.abs(v), 200)) + 2.0 ** -148


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", OB.ACTS)
@pytest.mark.parametrize("M, N", [(1, 1), (1, 4096), (3, 7), (5, 513), (129, 1000), (301, 1531), (128, 200), (1000, 520), (4001, 96)])
def test_gradient_of_an_epilogue(M, N, name, dtype):
    rng = np.random.default_rng(10)
    z, dy = _to(rng.standard_normal((M, N)) * 4, dtype), _to(rng.standard_normal((M, N)) * 1e-3 * np.exp(rng.standard_normal((1, N))), dtype)
    for scale, pad, shift, bias, fmt in ((1.0, 0, 0, True, "E5M2"), (-0.7, 8 + -N % 8, 0, True, "E4M3"), (0.3, 3, 1, False, "E5M2")):
        d = _t(dy, dtype, pad, shift)
        dz, dz8, db = ctx().fp8_linear_grad(d, _t(z, dtype, pad, shift) if name != "none" else None, act=ACT[name], scale=scale, bias=bias, fmt=FMT[fmt])
        f = float(np.float32(scale))
        want = f * dy.astype(np.float64) * OB.slope(name, z)
        err = abs(f) * np.abs(dy) * _slope_error(name, z.astype(np.float64), dtype) + 4 * U * np.abs(want)
        assert (dz is d) == (name == "none" and scale == 1.0)
        _close(dz, want, err, dtype)
        _near_codes_within(dz8, want, fmt, err)
        assert (db is None) == (not bias)
        if bias:
            _close(db, want.sum(0), err.sum(0) + (M + 4) * U * np.abs(want).sum(0), "f32")


def test_gradient_of_an_epilogue_of_no_rows():
    import torch
    e = torch.empty((0, 200), device="cuda")
    dz, dz8, db = ctx().fp8_linear_grad(e, e, act=sop.GELU)
    assert dz.shape == dz8.shape == (0, 200) and float(db.abs().max()) == 0


# ---- clipping

def _check_clip(tensors, most, types, in_place, shift=0):
    """tensors: flat arrays; types: (type, out's type) of each"""
    import torch
    gs = [_t(_to(x[None], a), a, 0, shift).view(-1) if x.size else torch.empty(0, dtype=_type(a), device="cuda") for x, (a, _) in zip(tensors, types)]
    flat = [_np(g) for g in gs]
    outs = None if in_place else [torch.full((x.size + 9,), 7.0, dtype=_type(b), device="cuda")[3:x.size + 3] for x, (_, b) in zip(tensors, types)]
    alone = ctx().grad_norm(gs)
    norm = ctx().clip_grads(gs, most, out=outs)
    want, clipped = OB.clip(flat, float(np.float32(most)))
    assert norm.shape == (1,) and norm.dtype is torch.float32 and torch.equal(alone, norm)
    assert abs(float(norm) - want) <= U * 1.01 * want or (np.isinf(np.float32(want)) and float(norm) == np.inf)   # (rounded to binary32)
    for g, o, x, w, (a, b) in zip(gs, outs or gs, flat, clipped, types):
        _close(o, w, 2.1 * U * np.abs(w), a if in_place else b)
        if not in_place:
            assert np.array_equal(_np(g), x)
            whole = o._base if o._base is not None else o
            assert float(whole[:3].float().min()) == 7 and (float(whole[3 + x.size:].float().min()) == 7)


@pytest.mark.parametrize("most", [0.0, 1e-3, 5.0, 1e9, float("inf")])
def test_clip(most):
    rng = np.random.default_rng(11)
    sizes = [1, 0, 7, 8, 255, 2047, 8191, 8192, 8193, 100003]
    tensors = [rng.standard_normal(n) for n in sizes]
    for shift in (0, 1):
        for kinds in ([("f32", "f32")], [("bf16", "bf16")], [("f32", "bf16"), ("bf16", "f32"), ("bf16", "bf16")]):
            types = [kinds[i % len(kinds)] for i in range(len(sizes))]
            _check_clip(tensors, most, types, False, shift)
            if all(a == b for a, b in kinds):
                _check_clip(tensors, most, types, True, shift)


def test_clip_of_many_tensors():
    rng = np.random.default_rng(12)
    tensors = [rng.standard_normal(int(n)) for n in rng.integers(0, 3000, 500)]
    _check_clip(tensors, 1.0, [("f32", "f32")] * 500, True)
    _check_clip(tensors[:97], 1.0, [("bf16", "f32")] * 97, False)


def test_clip_of_large_and_small_numbers():
    """Squares beyond binary32 on both sides."""
    rng = np.random.default_rng(13)
    for size in (1e30, 1e-30, 3e37):
        _check_clip([size * rng.uniform(0.1, 1, 5000), size * rng.uniform(0.1, 1, 70)], float(np.float32(size)), [("f32", "f32")] * 2, True)


def test_clip_of_what_is_no_number():
    import torch
    a, b = torch.ones(3000, device="cuda"), torch.ones(500, device="cuda")
    a[7] = float("nan")
    assert np.isnan(float(ctx().clip_grads([a, b], 1.0))) and bool(a.isnan().all()) and bool(b.isnan().all())
    a, b = torch.ones(3000, device="cuda"), torch.ones(500, device="cuda")
    a[7] = -float("inf")
    assert float(ctx().clip_grads([a, b], 1.0)) == float("inf") and bool(a[7].isnan()) and float(b.abs().max()) == 0 and float(a[8:].abs().max()) == 0


def test_clip_of_matrices_in_any_order_of_their_dimensions():
    import torch
    rng = np.random.default_rng(14)
    x = torch.from_numpy(rng.standard_normal((30, 50)).astype(np.float32)).cuda()
    t = x.t()
    want = x.t() * (1.0 / x.double().norm()).float()
    ctx().clip_grads([t, None], 1.0)
    assert torch.allclose(t, want, rtol=4 * U, atol=0) and x.stride() == (50, 1)
    y = torch.empty((2, 3, 4), device="cuda").permute(2, 0, 1)
    assert float(ctx().grad_norm([y.fill_(2.0)])) == pytest.approx((24 * 4) ** 0.5, rel=4 * U)
    for bad in ([x[:, :40]], [x[:, ::2]], [x[:1].expand(4, 50)]):
        with pytest.raises(sop.SopError):
            ctx().clip_grads(bad, 1.0)


def test_clip_refusals():
    import torch
    cx = ctx()
    x = torch.ones(100, device="cuda")

    def refused(status, f, *a, **k):
        with pytest.raises(sop.SopError) as e:
            f(*a, **k)
        assert e.value.status == status, e.value

    refused(1, cx.clip_grads, [x.cpu()], 1.0)
    refused(1, cx.clip_grads, [x.half()], 1.0)
    refused(1, cx.clip_grads, [3.0], 1.0)
    refused(1, cx.clip_grads, [x], -1.0)
    refused(1, cx.clip_grads, [x], float("nan"))
    refused(1, cx.clip_grads, [x, x], 1.0)                             # the same tensor twice
    refused(1, cx.clip_grads, [x, x[50:]], 1.0)
    refused(2, cx.clip_grads, [x], 1.0, out=[])
    refused(2, cx.clip_grads, [x], 1.0, out=[x[:50]])
    refused(1, cx.clip_grads, [x[:50], x[50:]], 1.0, out=[x[50:], torch.empty(50, device="cuda")])
    assert float(x.min()) == 1 and float(cx.grad_norm([x, x])) == pytest.approx(200 ** 0.5, rel=4 * U) and float(cx.grad_norm([])) == 0


def test_clip_takes_elements_beyond_four_gigabytes():
    import torch
    n = (1 << 31) + 5003
    x = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    x[n - 1], x[5], x[1 << 31] = 3.0, 4.0, 12.0
    assert float(ctx().clip_grads([x], 6.5)) == 13
    assert float(x[n - 1]) == 1.5 and float(x[5]) == 2 and float(x[1 << 31]) == 6 and int((x != 0).sum()) == 3


# ---- rows far apart

def _apart(buf, stride, *mats):
    """Copies of matrices side by side in one buffer, their rows `stride` elements apart."""
    wide, at, out = buf.view(-1, stride), 3, []
    for x in mats:
        v = wide[:x.shape[0], at:at + x.shape[1]]
        v.copy_(x)
        out.append(v)
        at += x.shape[1] + 5
    return out


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("D", [100, 1000, 4096, 8200, 16392])
def test_norms_of_rows_far_apart(D, t):
    """Five rows 2^30 elements apart, beyond what 32 bits address, give the bits of rows that follow each other."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(D)
    new = lambda *z: torch.randn(z, generator=gen, device="cuda").to(_type(t))  # noqa: E731
    buf = torch.empty(5 << 30, dtype=_type(t), device="cuda")
    r, y, ds, dn, gate, w = new(5, D), new(5, D), new(5, D), new(5, D), new(5, D), new(D).float()
    fr, fy, fds, fdn, fgate, out = _apart(buf, 1 << 30, r, y, ds, dn, gate, r)
    near = ctx().residual_norm(r, y, after=w, gate=gate, scale=0.5, before=w, dtype=_type(t), fmt=sop.E4M3)
    far = ctx().residual_norm(fr, fy, after=w, gate=fgate, scale=0.5, before=w, dtype=_type(t), fmt=sop.E4M3, out=out)
    assert far[0] is out and torch.equal(near[0], out) and torch.equal(near[1], far[1])
    assert torch.equal(near[2].codes, far[2].codes) and torch.equal(near[2].scales, far[2].scales)
    g = ctx().residual_norm_grad(ds, dn, near[0], before=w, y=y, after=w, gate=gate, scale=0.5, fmt=sop.E5M2)
    h = ctx().residual_norm_grad(fds, fdn, out, before=w, y=fy, after=w, gate=fgate, scale=0.5, fmt=sop.E5M2)
    assert all(torch.equal(a, b) for a, b in ((g.dr, h.dr), (g.dy, h.dy), (g.dy8.codes, h.dy8.codes), (g.dbefore, h.dbefore), (g.dafter, h.dafter), (g.dgate, h.dgate)))


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("M, N, K, apart", [(5, 300, 200, 30), (300, 1531, 300, 23), (2300, 4700, 150, 21)])
def test_epilogue_of_rows_far_apart(M, N, K, apart, t):
    """... and so do residual, y, z and dy of a product with an epilogue, where their offsets pass 32 bits."""
    import torch
    x, w, bias, z = _z_case(np.random.default_rng(11), M, N, K)
    gen = torch.Generator(device="cuda").manual_seed(M)
    res, dy = (torch.randn((M, N), generator=gen, device="cuda").to(_type(t)) for _ in range(2))
    fres, fy, fz, fdy = _apart(torch.empty(M << apart, dtype=_type(t), device="cuda"), 1 << apart, res, res, res, dy)
    kw = dict(bias=_vec(bias), act=sop.GELU, scale=0.5, dtype=_type(t))
    y, kept = ctx().fp8_linear(x, w, residual=res, keep=True, **kw)
    assert torch.equal(y, ctx().fp8_linear(x, w, residual=fres, out=fy, **kw))
    assert torch.equal(y, ctx().fp8_linear(x, w, residual=fres, out=fres, **kw))
    fz.copy_(kept)
    a, b = ctx().fp8_linear_grad(dy, kept, act=sop.GELU), ctx().fp8_linear_grad(fdy, fz, act=sop.GELU)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1].codes, b[1].codes) and torch.equal(a[2], b[2])


# ---- all of it together

def _block(cx, v, x, ds):
    """A block from norm to norm, forward and backward, as a training step runs it: the tensors that come out."""
    w1, w2 = (cx.fp8_quantize(w, rows=128, transposed=True) for w in (v["w1"], v["w2"]))
    _, _, n8 = cx.residual_norm(x, before=v["first"], fmt=sop.E4M3)
    h, z = cx.fp8_linear(n8, w1, bias=v["b1"], act=sop.GELU, keep=True)
    h8 = cx.fp8_quantize(h)
    y = cx.fp8_linear(h8, w2, bias=v["b2"])
    s, n, _ = cx.residual_norm(x, y, after=v["after"], gate=v["gate"], scale=0.5, before=v["last"], dtype=y.dtype)
    g = cx.residual_norm_grad(None, ds, s, before=v["last"], y=y, after=v["after"], gate=v["gate"], scale=0.5, fmt=sop.E5M2)
    dy, dy8, db2 = cx.fp8_linear_grad(g.dy)
    dw2 = cx.fp8_weight_grad(dy, h8)
    dh = cx.fp8_matmul(dy8, w2, transposed=True)
    dz, dz8, db1 = cx.fp8_linear_grad(dh, z, act=sop.GELU)
    dw1 = cx.fp8_weight_grad(dz, n8)
    dn = cx.fp8_matmul(dz8, w1, transposed=True)
    first = cx.residual_norm_grad(g.dr, dn, x, before=v["first"])
    grads = [dw1, db1, dw2, db2, g.dafter, g.dgate, g.dbefore, first.dbefore]
    norm = cx.clip_grads(grads, 1.0)
    return [s, n, first.dr, norm] + grads


def _block_case(seed, M=300, D=384, H=1000):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda *z: torch.randn(z, generator=gen, device="cuda")  # noqa: E731
    v = dict(w1=new(H, D) / D ** 0.5, w2=new(D, H) / H ** 0.5, b1=0.1 * new(H), b2=0.1 * new(D), first=1 + 0.1 * new(D), after=1 + 0.1 * new(D), last=1 + 0.1 * new(D), gate=new(3, D))
    return v, new(M, D).bfloat16(), new(M, D).bfloat16()


def test_a_block_forward_and_backward():
    """Against autograd in 64 bits.  Operands in 8 bits are off by 2^-4 (E4M3) or 2^-3 (E5M2) at most, element by element, and a result in its norm by less than the sum of
    what went into it: n has two 8-bit matrices and the two before them behind it, a gradient those and up to two in E5M2."""
    import torch
    v, x, ds = _block_case(1)
    s, n, dx, norm, *grads = _block(ctx(), v, x, ds)
    wide = {k: t.double().cpu().requires_grad_() for k, t in v.items()}
    xw = x.double().cpu().requires_grad_()
    unit = lambda t: t / torch.sqrt(t.square().mean(1, keepdim=True) + 1e-6)  # noqa: E731
    h = torch.nn.functional.gelu(unit(xw) * wide["first"] @ wide["w1"].t() + wide["b1"])
    y = unit(h @ wide["w2"].t() + wide["b2"]) * wide["after"]
    total = xw + 0.5 * (y.view(3, 100, -1) * wide["gate"][:, None]).view(y.shape)
    out = unit(total) * wide["last"]
    out.backward(ds.double().cpu())
    off = lambda a, b: float((a.double().cpu() - b).norm() / b.norm())  # noqa: E731
    assert off(s, total.detach()) < 4 / 16 and off(n, out.detach()) < 4 / 16
    names = ["w1", "b1", "w2", "b2", "after", "gate", "last", "first"]
    scale = torch.sqrt(sum(wide[k].grad.square().sum() for k in names))
    assert abs(float(norm) / float(scale) - 1) < 4 / 16 + 2 / 8
    for k, g in zip(names, grads):
        assert off(g * norm.double().item(), wide[k].grad) < 4 / 16 + 2 / 8, k
    assert off(dx, xw.grad) < 4 / 16 + 2 / 8


def test_a_block_on_other_streams_and_in_graphs():
    """The same bits on another stream, under a given one, and from a captured graph that is replayed between eager steps, with a second graph of the same step beside it."""
    import torch
    cx = ctx()
    v, x, ds = _block_case(2)
    same = lambda a, b: all(torch.equal(p.view(torch.uint8), q.view(torch.uint8)) for p, q in zip(a, b))  # noqa: E731
    plain = [t.clone() for t in _block(cx, v, x, ds)]
    assert same(plain, _block(cx, v, x, ds))
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        other = _block(cx, v, x, ds)
    st.synchronize()
    assert same(plain, other)

    class Given:                                                        # every call with stream=...
        def __getattr__(self, name):
            return lambda *a, **k: getattr(cx, name)(*a, stream=st.cuda_stream, **k)
    st.wait_stream(torch.cuda.current_stream())
    given = _block(Given(), v, x, ds)
    st.synchronize()
    assert same(plain, given)
    graphs, held = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held.append(_block(cx, v, x, ds))
        graphs.append(graph)
    for seed in (3, 4, 5):
        _, x1, ds1 = _block_case(seed)
        x.copy_(x1)
        ds.copy_(ds1)
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        fresh = _block(cx, v, x, ds)
        torch.cuda.synchronize()
        assert same(held[0], fresh) and same(held[1], fresh)
