"""What stands around a linear layer in a block of a model, in the oracle: activations and their slopes, norms with the residual stream and their gradients,
the clipping of gradients, in binary64.

TEST INFRASTRUCTURE ONLY; shares no code with the HIP library.
"""
from __future__ import annotations

import numpy as np
from scipy import special

ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh")


def act(name: str, z: np.ndarray) -> np.ndarray:
    z = np.asarray(z, dtype=np.float64)
    if name == "relu":
        return np.where(z < 0, 0.0, z)
    if name == "none":
        return z
    with np.errstate(invalid="ignore", over="ignore"):
        if name == "silu":
            y = z * special.expit(z)
        elif name == "gelu":
            y = z * special.ndtr(z)
        else:
            y = z * special.expit((8 / np.pi) ** 0.5 * (z + 0.044715 * z ** 3))
    return np.where(z == -np.inf, 0.0, y)                              # (the limit)


def slope(name: str, z: np.ndarray) -> np.ndarray:
    z = np.asarray(z, dtype=np.float64)
    if name == "none":
        return np.ones_like(z)
    if name == "relu":
        return np.where(z <= 0, 0.0, 1.0)
    c = np.clip(z, -1e4, 1e4)                                           # (far out both ends are flat; NaN stays)
    if name == "silu":
        q = special.expit(c)
        return q * (1 + c * special.expit(-c))
    if name == "gelu":
        return special.ndtr(c) + c * np.exp(-0.5 * c * c) / (2 * np.pi) ** 0.5
    v = (8 / np.pi) ** 0.5
    q = special.expit(v * (c + 0.044715 * c ** 3))
    return q * (1 + c * special.expit(-v * (c + 0.044715 * c ** 3)) * v * (1 + 3 * 0.044715 * c * c))


def rows_of(gate, M: int, D: int) -> np.ndarray:
    """A gate of G rows as one row for each of M (ones without a gate)."""
    if gate is None:
        return np.ones((M, D))
    g = np.asarray(gate, dtype=np.float64).reshape(-1, D)
    return np.repeat(g, M // len(g), 0) if M else np.zeros((0, D))


def unit(x: np.ndarray, eps: float) -> np.ndarray:
    """1 / rms of every row, as a column."""
    return 1 / np.sqrt(np.mean(x * x, 1, keepdims=True) + eps)


def residual_norm(r, y=None, after=None, gate=None, scale=1.0, before=None, eps=1e-6):
    """(s, n or None)"""
    s = r.astype(np.float64)
    if y is not None:
        x = y.astype(np.float64)
        if after is not None:
            x = x * unit(x, eps) * after
        s = s + scale * rows_of(gate, *r.shape) * x
    return s, None if before is None else s * unit(s, eps) * before


def residual_norm_grad(ds, dn=None, s=None, before=None, y=None, after=None, gate=None, scale=1.0, eps=1e-6):
    """dict of dr, dy, dbefore, dafter, dgate (where there is such a thing)"""
    out = {}
    dr = 0.0 if ds is None else ds.astype(np.float64)
    if before is not None:
        s, dn = s.astype(np.float64), dn.astype(np.float64)
        u = unit(s, eps)
        h, p = s * u, before * dn
        dr = dr + u * (p - h * np.mean(p * h, 1, keepdims=True))
        out["dbefore"] = np.sum(dn * h, 0)
    out["dr"] = dr
    if y is None:
        return out
    y = y.astype(np.float64)
    M, D = y.shape
    g = rows_of(gate, M, D)
    w = 1.0 if after is None else np.asarray(after, dtype=np.float64)
    q = scale * g * w * dr
    if after is None:
        x, out["dy"] = y, q
    else:
        u = unit(y, eps)
        x = y * u
        out["dy"] = u * (q - x * np.mean(q * x, 1, keepdims=True))
        out["dafter"] = np.sum(scale * g * dr * x, 0)
    if gate is not None:
        G = np.asarray(gate).reshape(-1, D).shape[0]
        out["dgate"] = np.sum((scale * w * dr * x).reshape(G, M // G, D), 1)
    return out


def clip(tensors, most):
    """(norm, tensors times min(1, most / norm)); every tensor as a flat array of binary64."""
    norm = np.sqrt(sum(float(np.sum(t * t)) for t in tensors))
    with np.errstate(invalid="ignore"):
        c = 1.0 if norm <= most else most / norm
        return norm, [t * c for t in tensors]
