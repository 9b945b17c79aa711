"""The example of the linear-layer operators, at small sizes: its gradients against autograd in 64 bits, its training, its packed products."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


def _example():
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "gated_layer.py")
    spec = importlib.util.spec_from_file_location("gated_layer", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_gradients_of_the_layer():
    """Operands are off by 2^-4 at most (E4M3; E5M2 2^-3), element by element; a result's error, in its norm, stays below the sum of its
    operands' and of what went into them: y has four roundings behind it, a weight's gradient up to seven, one of them E5M2's."""
    import torch
    import paper_2605_14929_amd as sop
    ex = _example()
    rows, width, hidden = 300, 264, 520
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn((rows, width), generator=gen, device="cuda").bfloat16()
    dy = torch.randn((rows, width), generator=gen, device="cuda").bfloat16()
    weights = ex.make_weights(width, hidden, 6)
    layer = ex.GatedLayer(sop.Context(0), *(w.clone() for w in weights))
    y = layer.forward(x)
    grads, dx = layer.backward(dy)
    wide = [w.double().cpu().requires_grad_() for w in weights]
    xw = x.double().cpu().requires_grad_()
    want = ex.plain(wide, xw)
    want.backward(dy.double().cpu())
    assert ex.off(y.cpu(), want) < 4 / 16
    for g, w in zip(grads + [dx], wide + [xw]):
        assert ex.off(g.cpu(), w.grad) < 6 / 16 + 1 / 8


def test_training_and_serving():
    losses, error8, error4 = _example().main(["--rows", "512", "--width", "256", "--hidden", "640", "--steps", "12"])
    assert losses[-1] < 0.8 * losses[0]
    assert error8 < 4 / 16
    assert error4 < 0.35                                                # three matrices of 4-bit codes, each off by a tenth or so
