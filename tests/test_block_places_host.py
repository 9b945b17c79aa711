"""Results of the entry points around a linear layer in their operands' places: which calls are refused, and which go through (on the host, with stubs in the kernels' place)."""
import pytest

from test_block_api_host import AT, EINVAL, OK, _act_grad, _norm_grad, _opts, _said, lib  # noqa: F401


def test_gradient_of_an_epilogue_in_place(lib):  # noqa: F811
    dy, z = AT, AT + (1 << 30)
    for dz in (dy, z):
        assert _act_grad(lib, dy=dy, z=z, dz=dz)[0] == OK
        assert _act_grad(lib, dy=dy, z=z, dz=dz, lddz=608)[0] == EINVAL and b"row stride" in lib.stub_error()
        assert _act_grad(lib, dy=dy, lddy=608, z=z, ldz=608, dz=dz, lddz=608)[0] == OK
        assert _act_grad(lib, 1, dy=dy, z=z, dz=dz, lddz=608)[0] == OK   # (of one row the stride says nothing)
    assert _act_grad(lib, act=0, dy=dy, z=z, dz=z, lddz=608)[0] == OK    # (z is not looked at)
    _said(lib)


@pytest.mark.parametrize("groups", [1, 2, 6])
def test_gradients_of_a_norm_where_its_weights_are(lib, groups):  # noqa: F811
    """Weights and gate are read by the workgroups that join sums while others write theirs."""
    o = _opts(before=AT + (1 << 20), after=AT + (1 << 21), gate=AT + (1 << 22), ld_gate=300, groups=groups)
    assert _norm_grad(lib, o=o)[0] == OK
    for more in (dict(dbefore=o.before), dict(dafter=o.after), dict(dgate=o.gate)):
        assert _norm_grad(lib, o=o, **more)[0] == EINVAL and b"memory of their own" in lib.stub_error(), more
    _said(lib)
