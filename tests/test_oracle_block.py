"""The oracle of norms with the residual stream, epilogues and clipping: gradients against differences, activations against published values."""
import numpy as np
import pytest

from oracle import block as OB


def _differences(f, x, h=1e-5):
    """The gradient of f, a number, at x, by central differences."""
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        a, b = x.copy(), x.copy()
        a[i] += h
        b[i] -= h
        g[i] = (f(a) - f(b)) / (2 * h)
    return g


@pytest.mark.parametrize("name", OB.ACTS[1:])
def test_slopes_are_the_activations_derivatives(name):
    z = np.concatenate([np.linspace(-9, 9, 181) + 0.013, [-40.0, 40.0]])
    h = 1e-5
    d = (OB.act(name, z + h) - OB.act(name, z - h)) / (2 * h)
    assert np.allclose(OB.slope(name, z), d, rtol=0, atol=1e-8)


def test_activations_at_known_points():
    assert OB.act("gelu", np.array([1.0]))[0] == pytest.approx(0.8413447460685429, abs=1e-15)           # Phi(1)
    assert OB.act("silu", np.array([1.0]))[0] == pytest.approx(1 / (1 + np.exp(-1)), abs=1e-15)
    v = np.sqrt(2 / np.pi) * (0.7 + 0.044715 * 0.343)
    assert OB.act("gelu_tanh", np.array([0.7]))[0] == pytest.approx(0.35 * (1 + np.tanh(v)), abs=1e-15)
    for name in OB.ACTS[1:]:
        y = OB.act(name, np.array([-np.inf, np.inf, np.nan, 0.0]))
        assert y[0] == 0 and y[1] == np.inf and np.isnan(y[2]) and y[3] == 0
        s = OB.slope(name, np.array([-np.inf, np.inf]))
        assert s[0] == 0 and s[1] == 1


@pytest.mark.parametrize("G", [None, 1, 2, 6])
@pytest.mark.parametrize("after", [False, True])
@pytest.mark.parametrize("before", [False, True])
def test_norm_gradients_against_differences(G, after, before):
    rng = np.random.default_rng(1)
    M, D, scale, eps = 6, 5, 0.7, 1e-3
    v = dict(r=rng.standard_normal((M, D)), y=rng.standard_normal((M, D)), after=rng.standard_normal(D) if after else None,
             before=rng.standard_normal(D) if before else None, gate=rng.standard_normal((G, D)) if G else None)
    ds, dn = rng.standard_normal((M, D)), rng.standard_normal((M, D)) if before else None

    def loss(**new):
        s, n = OB.residual_norm(**dict(v, **new), scale=scale, eps=eps)
        return float(np.sum(ds * s) + (np.sum(dn * n) if before else 0.0))

    s, _ = OB.residual_norm(**v, scale=scale, eps=eps)
    got = OB.residual_norm_grad(ds, dn, s if before else None, before=v["before"], y=v["y"], after=v["after"], gate=v["gate"], scale=scale, eps=eps)
    assert set(got) == {"dr", "dy"} | ({"dbefore"} if before else set()) | ({"dafter"} if after else set()) | ({"dgate"} if G else set())
    for k, g in got.items():
        name = k[1:]
        assert np.allclose(g, _differences(lambda x: loss(**{name: x}), v[name]), rtol=0, atol=1e-7), k


def test_clip():
    a, b = np.array([3.0, 0.0]), np.array([[4.0]])
    norm, (x, y) = OB.clip([a, b], 10.0)
    assert norm == 5 and np.array_equal(x, a) and np.array_equal(y, b)
    norm, (x, y) = OB.clip([a, b], 1.0)
    assert norm == 5 and np.allclose(x, a / 5) and np.allclose(y, b / 5)
    assert OB.clip([], 1.0)[0] == 0
