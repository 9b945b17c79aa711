"""What stands around a linear layer in a block of a model, at the ends of binary32: gradients as large as it holds under slopes that vanish, rows full of its largest numbers.
Against the oracle in 64 bits; tolerances are those of test_gpu_block, and what the ends add to them is counted at each test."""
import numpy as np
import pytest

import paper_2605_14929_amd as sop
from oracle import block as OB
from gpu_util import ctx
from test_gpu_block import ACT, U, _near_codes_within, _slope_error, _t, _to
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
