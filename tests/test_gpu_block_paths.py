"""What stands around a linear layer in a block of a model, on the ways through its kernels that sizes and alignment choose: whole tiles that leave by windows (matrices whose rows start on
four elements), with and without a residual and a kept z, and rows of more than 16384 elements, several to a workgroup.  Against the oracle in 64 bits, tolerances as in test_gpu_block."""
import numpy as np
import pytest

import paper_2605_14929_amd as sop
from oracle import block as OB
from gpu_util import ctx
from test_gpu_block import ACT, U, _act_error, _forward_errors, _gate, _grad_errors, _near_codes_within, _norm_case, _t, _to, _type, _vec, _z_case
from test_gpu_block_ends import _close
from test_gpu_linear import _bf16, _np

pytestmark = pytest.mark.gpu
# M, N, K and the kernel (by bf16 and fp32 results) that the rules choose on 256 compute units: N a multiple of four, some tiles whole and some not
F8_TILES = [(1000, 2052, 300, "64x128", "64x128"), (1000, 4700, 150, "128x128", "128x128"), (2300, 5000, 150, "256x256", "128x128"), (192, 2560, 260, "32x64", "32x64")]
# M, N, K, g, bits
PACKED_TILES = [(1000, 3500, 72, 8, 4, "128x128"), (2000, 5000, 80, 16, 3, "256x192"), (2000, 5000, 80, 16, 4, "256x192"), (2000, 5000, 72, 8, 5, "256x192"), (3000, 5000, 72, 8, 4, "256x256"),
                (3000, 5000, 96, 32, 1, "256x256"), (3000, 5000, 80, 16, 5, "256x256"), (1000, 3500, 72, 8, 6, "128x128")]
FORMS = [(False, False, False), (True, False, False), (True, False, True), (False, True, False), (True, True, False)]   # residual, z, y in the residual's place


def _apart(t, rows, stride, *mats):
    """Matrices side by side in one buffer, their rows `stride` elements apart, all of them on four elements."""
    import torch
    wide, at, out = torch.empty(rows * stride, dtype=_type(t), device="cuda").view(rows, stride), 4, []
    for x in mats:
        v = wide[:, at:at + x.shape[1]]
        v.copy_(x)
        out.append(v)
        at += -(-x.shape[1] // 4) * 4 + 8
    assert at <= stride
    return out


def _on_four(x):
    return x.data_ptr() % (4 * x.element_size()) == 0 and x.stride(0) % 4 == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M, N, K, by_bf16, by_f32", F8_TILES)
def test_epilogue_of_whole_tiles(M, N, K, by_bf16, by_f32, dtype):
    import torch
    x, w, bias, z = _z_case(np.random.default_rng(31), M, N, K)
    z = z + bias
    gen = torch.Generator(device="cuda").manual_seed(M)
    res = (4 * torch.randn((M, N), generator=gen, device="cuda")).to(_type(dtype))
    rw = _np(res)
    f = float(np.float32(-0.7))
    for name in ("gelu", "silu"):
        a = f * OB.act(name, z)
        ea = abs(f) * _act_error(name, z, dtype) + U * np.abs(a)
        for has_residual, keep, in_place in FORMS:
            r = res.clone() if has_residual else None
            out = r if in_place else torch.empty((M, N), dtype=_type(dtype), device="cuda")
            assert _on_four(out) and (r is None or _on_four(r))
            got = ctx().fp8_linear(x, w, bias=_vec(bias), act=ACT[name], residual=r, scale=f, keep=keep, out=out)
            y, kept = got if keep else (got, None)
            want = a + (rw if has_residual else 0)
            assert y is out
            _close(y, want, ea + U * np.abs(want), dtype)
            if keep:
                assert _on_four(kept) and np.array_equal(_np(kept), _bf16(z) if dtype == "bf16" else z)


@pytest.mark.parametrize("M, N, K, g, n, by", PACKED_TILES)
def test_packed_epilogue_of_whole_tiles(M, N, K, g, n, by):
    """Entries and scales are powers of two, x whole numbers, so sums are exact."""
    import torch
    rng = np.random.default_rng(32)
    count = N * K // g
    words = torch.from_numpy(((7 << 4) + 16 * rng.integers(-2, 1, count)).astype(np.int16)).cuda()              # scales of 1, 1/2, 1/4
    payload = torch.from_numpy(rng.integers(0, 256, count * g * n // 8).astype(np.uint8)).cuda()
    table = np.sort(rng.choice([-2.0, -1.0, -0.5, 0.5, 1.0, 2.0], 1 << n)).astype(np.float32)
    layer = sop.PackedWeights(words, payload, N, K, g, n, sop.ScaleFmt(0, 4, 4, 8, -1, -1), [table])
    x = _t(rng.integers(-2, 3, (M, K)) / 16.0, "bf16")
    codes = ((payload.view(count, g * n // 8, 1) >> torch.arange(8, device="cuda")) & 1).view(count, g, n).long()
    codes = (codes << torch.arange(n, device="cuda")).sum(-1)
    v = (torch.from_numpy(table).cuda().double()[codes] * torch.exp2((words.double() - 112)[:, None] / 16)).view(N, K)
    bias = rng.integers(-64, 65, N) / 16
    z = (x.double() @ v.t()).cpu().numpy() + bias
    gen = torch.Generator(device="cuda").manual_seed(M)
    res = (4 * torch.randn((M, N), generator=gen, device="cuda")).bfloat16()
    rw = _np(res)
    f = float(np.float32(0.7))
    a = f * OB.act("silu", z)
    ea = f * _act_error("silu", z, "bf16") + U * np.abs(a)
    for has_residual, keep, in_place in FORMS:
        r = res.clone() if has_residual else None
        out = r if in_place else torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
        assert _on_four(out) and (r is None or _on_four(r))
        got = ctx().packed_linear(x, layer, bias=_vec(bias), act=sop.SILU, residual=r, scale=f, keep=keep, out=out)
        y, kept = got if keep else (got, None)
        want = a + (rw if has_residual else 0)
        _close(y, want, ea + U * np.abs(want), "bf16")
        if keep:
            assert _on_four(kept) and np.array_equal(_np(kept), _bf16(z))


# the stride that a window still takes is below 2^30 bytes divided by the rows of a wavefront's part: 128 x 2, 64 x 4, 32 x 2 and 32 x 4 bytes
@pytest.mark.parametrize("M, N, K, t, stride", [(2300, 5000, 150, "bf16", (1 << 22) - 4), (2300, 5000, 150, "bf16", 1 << 22), (1000, 4700, 150, "f32", (1 << 22) - 4), (1000, 4700, 150, "f32", 1 << 22),
                                                (1000, 2052, 300, "bf16", (1 << 24) - 4), (1000, 2052, 300, "f32", (1 << 23) - 4)])
def test_epilogue_of_whole_tiles_far_apart(M, N, K, t, stride):
    """Rows on four elements whose offsets pass 32 bits, by windows of nearly 2^30 bytes and just beyond: the bits of rows that follow each other."""
    import torch
    x, w, bias, _ = _z_case(np.random.default_rng(33), M, N, K)
    gen = torch.Generator(device="cuda").manual_seed(M)
    res = torch.randn((M, N), generator=gen, device="cuda").to(_type(t))
    fres, fy = _apart(t, M, stride, res, res)
    assert _on_four(fres) and _on_four(fy)
    kw = dict(bias=_vec(bias), act=sop.GELU, scale=0.5, dtype=_type(t))
    y, kept = ctx().fp8_linear(x, w, residual=res, keep=True, **kw)
    again, far_kept = ctx().fp8_linear(x, w, residual=fres, out=fy, keep=True, **kw)
    assert torch.equal(y, fy) and torch.equal(kept, far_kept) and again is fy
    assert torch.equal(y, ctx().fp8_linear(x, w, residual=fres, out=fres, **kw))


@pytest.mark.parametrize("D", [16392, 20001])
@pytest.mark.parametrize("M, G", [(1100, 0), (1101, 3), (1100, 550), (1100, 1100)])
def test_long_rows_several_to_a_workgroup(M, G, D):
    """More rows than workgroups (512 on 256 compute units), several rows a wavefront of the sums over rows, several groups a workgroup."""
    import torch
    rng = np.random.default_rng(34)
    c = _norm_case(rng, M, D, "bf16", "f32", G, True, True)
    up = dict(after=_vec(c["after"]), gate=_gate(c, "bf16", 0, 0), scale=c["scale"], before=_vec(c["before"]))
    s, n, n8 = ctx().residual_norm(_t(c["r"]), _t(c["y"], "bf16"), dtype=torch.float32, fmt=sop.E4M3, **up)
    at = np.concatenate([np.arange(3), np.arange(505, 525), np.arange(1018, 1034), np.arange(M - 10, M)])
    part = dict(c, r=c["r"][at], y=c["y"][at], gate=None if not G else OB.rows_of(c["gate"], M, D)[at])
    want, es, wn, en = _forward_errors(part)
    idx = torch.from_numpy(at).cuda()
    _close(s[idx], want, es, "f32")
    _close(n[idx], wn, en, "f32")
    _near_codes_within(sop.Fp8Blocks(n8.codes.view(torch.uint8)[idx].view(torch.float8_e4m3fn), n8.scales.view(torch.uint8)[idx].view(torch.float8_e8m0fnu)), wn, "E4M3", en)
    ds, dn = (rng.standard_normal((M, D)) * 1e-3).astype(np.float32), _to(rng.standard_normal((M, D)) * 1e-3, "bf16")
    want, err = _grad_errors(c, ds, dn, c["r"])
    got = ctx().residual_norm_grad(_t(ds), _t(dn, "bf16"), _t(c["r"]), y=_t(c["y"], "bf16"), **up)
    for k, t in (("dr", "f32"), ("dy", "bf16"), ("dbefore", "f32"), ("dafter", "f32"), ("dgate", "bf16")):
        if k in want:
            _close(getattr(got, k), want[k], err[k], t)
