"""The oracle's 8-bit floats, block scales and gated unit against definitions they were not written from."""
import numpy as np
import pytest
import torch

from oracle import linear as OL

TORCH = {"E4M3": torch.float8_e4m3fn, "E5M2": torch.float8_e5m2}


@pytest.mark.parametrize("fmt", ["E4M3", "E5M2"])
def test_code_values_are_the_format_s(fmt):
    mine = OL.decode(np.arange(256, dtype=np.uint8), fmt)
    ref = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(TORCH[fmt]).double().numpy()
    assert np.array_equal(mine, ref, equal_nan=True)


@pytest.mark.parametrize("fmt", ["E4M3", "E5M2"])
def test_encode_is_nearest_with_ties_to_even(fmt):
    vals = OL.code_values(fmt)
    vals = vals[np.isfinite(vals)]
    mid = (vals[1:] + vals[:-1]) / 2
    x = np.concatenate([vals, mid, np.nextafter(mid, 0), np.nextafter(mid, np.inf)]).astype(np.float64)
    x = np.concatenate([x, -x])
    got = OL.decode(OL.encode(x, fmt), fmt)
    for v, y in zip(x, got):
        d = np.abs(np.abs(v) - vals)
        best = np.flatnonzero(d == d.min())
        want = best[0] if best.size == 1 else best[best % 2 == 0][0]
        assert y == np.copysign(vals[want], v), v


@pytest.mark.parametrize("fmt", ["E4M3", "E5M2"])
def test_no_element_saturates_and_no_smaller_scale_would_do(fmt):
    rng = np.random.default_rng(5)
    x = rng.standard_normal((9, 300)) * 2.0 ** rng.integers(-60, 60, (9, 1))
    e = OL.spread(OL.block_exponents(x, 1, fmt), 1, *x.shape)
    assert np.all(np.abs(x) <= OL.TOP[fmt] * 2.0 ** e)
    for j in range(0, 300, 128):
        assert np.all(np.abs(x[:, j:j + 128]).max(1) > OL.TOP[fmt] * 2.0 ** (e[:, j] - 1))


def test_gated_gradient_against_differences():
    rng = np.random.default_rng(6)
    g, u, dh = (rng.standard_normal(200) * 3 for _ in range(3))
    dg, du = OL.silu_mul_grad(g, u, dh)
    h = 1e-5
    assert np.allclose(dg, dh * (OL.silu_mul(g + h, u) - OL.silu_mul(g - h, u)) / (2 * h), rtol=1e-7, atol=1e-8)
    assert np.allclose(du, dh * (OL.silu_mul(g, u + h) - OL.silu_mul(g, u - h)) / (2 * h), rtol=1e-7, atol=1e-8)
