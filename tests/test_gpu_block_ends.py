"""What stands around a linear layer in a block of a model, at the ends of binary32: gradients as large as it holds under slopes that vanish, rows full of its largest numbers.
Against the oracle in 64 bits; tolerances are those of test_gpu_block, and what the ends add to them is counted at each test."""
import numpy as np
import pytest

import paper_2605_14929_amd as sop
from oracle import block as OB
from gpu_util import ctx
from test_gpu_block import ACT, U, _forward_errors, _grad_errors, _near_codes_within, _norm_case, _slope_error, _t, _to, _vec
from test_gpu_block import _close as _near, _np

pytestmark = pytest.mark.gpu
BIG = float(np.float32(3e38))


def _close(got, want, err, t):
    """Numbers of type t against what they should be, known to err, none of them infinite or NaN."""
    assert np.isfinite(_np(got)).all()
    _near(got, want, err, t)


@pytest.mark.parametrize("M", [1, 200])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", OB.ACTS)
def test_large_gradients_under_any_slope(name, dtype, M):
    """dz = scale dy act'(z) is finite wherever the slope is at most 1.13 and scale 1/2, however large dy is: no step on the way may leave binary32 (what is beside the result
    overflows for z far below zero).  One row has the gradients, so dbias is that row."""
    z = np.concatenate([np.linspace(-60, 20, 801), -np.geomspace(1e-30, 3e38, 200), np.geomspace(1e-30, 3e38, 200), [0.0, -0.0, -np.inf, np.inf, -87.4, -174.0, -1200.0]])
    N, at = z.size, M // 2
    for size in (1e20, 1e30, 1e33, 1e35, 1e37, BIG):
        zz = _to(np.repeat(z[None].astype(np.float32), M, 0), dtype)
        dy = np.zeros((M, N))
        dy[at] = size * np.where(np.arange(N) % 3 == 1, -1.0, 1.0)
        dy = _to(dy, dtype)
        dz, dz8, db = ctx().fp8_linear_grad(_t(dy, dtype), _t(zz, dtype), act=ACT[name], scale=0.5)
        wz = zz.astype(np.float64)
        want = 0.5 * dy.astype(np.float64) * OB.slope(name, wz)
        err = 0.5 * np.abs(dy) * _slope_error(name, wz, dtype) + 4 * U * np.abs(want)
        _close(dz, want, err, dtype)
        _near_codes_within(dz8, want, "E5M2", err)
        _close(db, want[at], err[at] + 2 * U * np.abs(want[at]), "f32")


def _large_rows(rng, M, D):
    """Rows of one size each, from where their squares leave binary32 to where they all but do themselves; the last has a single such element."""
    x = np.where(rng.random((M, D)) < 0.5, -1.0, 1.0) * rng.uniform(0.5, 1, (M, D)) * np.resize([1e19, 2e18, 1e25, 1e36, 2e37, 1e38, BIG, BIG], M)[:, None]
    x[M - 2] = np.where(x[M - 2] < 0, -BIG, BIG)
    x[M - 1, : D - 1] *= 1e-25
    return x.astype(np.float32)


def _of_unit(unit):
    """What 1 / rms is rounded by where it is no normal number (rms beyond 2^126), of itself: half of 2^-149."""
    return 2.0 ** -150 / unit


@pytest.mark.parametrize("D", [96, 1000, 4096, 8192, 8200, 16384, 20000, 1 << 20])
def test_norm_of_rows_of_large_numbers(D):
    """x after and before h are of size 1 however large the row is."""
    import torch
    rng = np.random.default_rng(21)
    c = _norm_case(rng, 8, D, "f32", "f32", 0, True, True, scale=0.25)
    c["y"] = _large_rows(rng, 8, D)
    want, es, wn, en = _forward_errors(c)
    u = _of_unit(OB.unit(c["y"].astype(np.float64), c["eps"]))
    s, n, n8 = ctx().residual_norm(_t(c["r"]), _t(c["y"]), after=_vec(c["after"]), scale=c["scale"], before=_vec(c["before"]), dtype=torch.float32, fmt=sop.E4M3)
    _close(s, want, es + u * np.abs(want - c["r"]), "f32")
    c["r"], c["y"], c["after"] = c["y"], None, None
    want, es, wn, en = _forward_errors(c)
    s, n, n8 = ctx().residual_norm(_t(c["r"]), before=_vec(c["before"]), dtype=torch.float32, fmt=sop.E4M3)
    en = en + u * np.abs(wn)
    _close(n, wn, en, "f32")
    _near_codes_within(n8, wn, "E4M3", en)


@pytest.mark.parametrize("D", [96, 1000, 4096, 8192, 8200, 16384, 20000])
def test_norm_gradients_of_rows_of_large_numbers(D):
    """... and so the weights' gradients are; those of the rows themselves vanish.  Errors are those of rows of any size, whose k is 60 U at least, and twice a rounding of 1 / rms (4.3 U)
    more: a quarter of them covers that."""
    rng = np.random.default_rng(22)
    for what in ("s", "y"):
        c = _norm_case(rng, 8, D, "f32", "f32", 2, True, True)
        c["r" if what == "s" else "y"] = _large_rows(rng, 8, D)
        ds, dn = (rng.standard_normal((8, D)).astype(np.float32) for _ in range(2))
        want, err = _grad_errors(c, ds, dn, c["r"])
        got = ctx().residual_norm_grad(_t(ds), _t(dn), _t(c["r"]), before=_vec(c["before"]), y=_t(c["y"]), after=_vec(c["after"]), gate=_t(c["gate"]), scale=c["scale"], fmt=sop.E5M2)
        for k in ("dr", "dy", "dbefore", "dafter", "dgate"):
            _close(getattr(got, k), want[k], 1.25 * err[k], "f32")


@pytest.mark.parametrize("D", [96, 4096, 12000, 20000])
def test_norm_under_a_large_eps(D):
    """eps beside a sum of squares that leaves binary32."""
    import torch
    rng = np.random.default_rng(23)
    c = _norm_case(rng, 4, D, "f32", "f32", 0, False, True)
    c.update(r=(1e18 * rng.standard_normal((4, D))).astype(np.float32), y=None, eps=float(np.float32(3e36)))
    c["r"][1:] *= np.float32(10)
    want, es, wn, en = _forward_errors(c)
    _close(ctx().residual_norm(_t(c["r"]), before=_vec(c["before"]), dtype=torch.float32, eps=c["eps"])[1], wn, en, "f32")
    dn = rng.standard_normal((4, D)).astype(np.float32)
    want, err = _grad_errors(c, None, dn, c["r"])
    got = ctx().residual_norm_grad(None, _t(dn), _t(c["r"]), before=_vec(c["before"]), eps=c["eps"])
    _close(got.dr, want["dr"], err["dr"], "f32")
    _close(got.dbefore, want["dbefore"], err["dbefore"], "f32")


@pytest.mark.parametrize("D", [96, 1000, 2050, 4096, 8192, 8200, 16384, 20000])
def test_norm_gradients_from_large_gradients(D):
    """The means of p h and q x are no larger than what they are means of: gradients of 1e35 to 1e37, all of one sign beside h or x, have sums that leave binary32 and means that do not.
    By rows: small s under a large 1 / rms, s of size 1, s and its gradient beside it, y of size 1, y small."""
    rng = np.random.default_rng(24)
    c = _norm_case(rng, 5, D, "f32", "f32", 0, True, True, scale=0.5)
    c.update(after=rng.uniform(0.5, 1, D).astype(np.float32), before=rng.uniform(0.5, 1, D).astype(np.float32))
    s, y, a = rng.standard_normal((5, D)), rng.standard_normal((5, D)), rng.uniform(0.5, 1, (5, D))
    s[0] *= 1e-3
    y[4] *= 1e-3
    c.update(r=s.astype(np.float32), y=y.astype(np.float32))
    dn, ds = a * np.sign(s) * np.array([1e35, 1e37, 1e37, 0, 0])[:, None], a * np.sign(y) * np.array([0, 0, 1e37, 1e37, 1e34])[:, None]
    ds, dn = ds.astype(np.float32), dn.astype(np.float32)
    want, err = _grad_errors(c, ds, dn, c["r"])
    got = ctx().residual_norm_grad(_t(ds), _t(dn), _t(c["r"]), before=_vec(c["before"]), y=_t(c["y"]), after=_vec(c["after"]), scale=c["scale"], fmt=sop.E5M2)
    assert max(np.abs(want[k]).max() for k in want) < 2e38
    for k in ("dr", "dy", "dbefore", "dafter"):
        _close(getattr(got, k), want[k], err[k], "f32")
    _near_codes_within(got.dy8, want["dy"], "E5M2", err["dy"])
