"""The example of the operators around a linear layer, at small sizes: its gradients against autograd in 64 bits, and that it runs."""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu


def _example():
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "residual_block.py")
    spec = importlib.util.spec_from_file_location("residual_block", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("rows, width, hidden", [(300, 264, 520), (1, 128, 300), (77, 1000, 640)])
def test_gradients_of_the_block(rows, width, hidden):
    """Operands are off by 2^-4 at most (E4M3; E5M2 2^-3), element by element; a result's error, in its norm, stays below the sum of its operands' and of what went into
    them: y has four such roundings behind it, a gradient those and up to two of E5M2's."""
    import torch
    import paper_2605_14929_amd as sop
    ex = _example()
    gen = torch.Generator(device="cuda").manual_seed(5)
    x, ds = (torch.randn((rows, width), generator=gen, device="cuda").bfloat16() for _ in range(2))
    params = ex.make_params(width, hidden, 6)
    block = ex.ResidualBlock(sop.Context(0), {k: v.clone() for k, v in params.items()})
    s = block.forward(x)
    grads, dx = block.backward(ds)
    wide = {k: v.double().cpu().requires_grad_() for k, v in params.items()}
    xw = x.double().cpu().requires_grad_()
    want = ex.plain(wide, xw)
    want.backward(ds.double().cpu())
    off = lambda a, b: float((a.double().cpu() - b.detach()).norm() / b.detach().norm())  # noqa: E731
    assert off(s, want) < 4 / 16 and torch.equal(s, block.forward(x, keep=False))
    for k in ex.NAMES:
        assert grads[k].shape == params[k].shape and off(grads[k], wide[k].grad) < 4 / 16 + 2 / 8, k
    assert off(dx, xw.grad) < 4 / 16 + 2 / 8
    norm = block.step(grads, 0.1, most=0.5)
    total = math.sqrt(sum(float(g.double().square().sum()) for g in grads.values()))
    assert total <= 0.5 * (1 + 2.0 ** -20) and (float(norm) <= 0.5 or total >= 0.5 * (1 - 2.0 ** -20))


def test_training_and_serving():
    losses, norms, error = _example().main(["--rows", "200", "--width", "256", "--hidden", "640", "--steps", "5"])
    assert len(losses) == len(norms) == 5 and all(math.isfinite(v) for v in losses + norms)
    assert error < 4 / 16
