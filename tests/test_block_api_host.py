"""The entry points around a linear layer on the host: what they refuse, and what they would launch (stubs in the kernels' place write it down)."""
import ctypes as C
import os
import re
import subprocess

import pytest

import paper_2605_14929_amd as sop
from paper_2605_14929_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NAMES = ("sop_fp8_linear", "sop_packed_linear", "sop_fp8_linear_grad_workspace", "sop_fp8_linear_grad", "sop_residual_norm", "sop_residual_norm_grad_workspace",
         "sop_residual_norm_grad", "sop_clip_grads_workspace", "sop_grad_norm", "sop_clip_grads")
OK, EINVAL, ESHAPE, ENOMEM = 0, 1, 2, 5
AT = 1 << 20                                                            # an address that nothing is read from


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("stubs") / "stubs.so")
    src = os.path.join(ROOT, "paper_2605_14929_amd", "csrc")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-Wno-unused-result", "-fsanitize=undefined",
                           "-fno-sanitize=enum", "-fno-sanitize-recover=all", "-static-libubsan", "-o", so, os.path.join(ROOT, "tests", "host_block_stubs.cpp"), os.path.join(src, "sop_block_api.cpp"),
                           os.path.join(src, "sop_linear_api.cpp")])
    L = C.CDLL(so)
    for n in NAMES:
        getattr(L, n).argtypes = getattr(sop.lib(), n).argtypes
    L.stub_ctx.restype, L.stub_error.restype, L.stub_record.restype = C.c_void_p, C.c_char_p, C.c_char_p
    L.ctx = C.c_void_p(L.stub_ctx(256))
    return L


def _said(lib):
    return [line.split() for line in lib.stub_record().decode().splitlines()]


def _f8(M, K, rows=1, fmt=0, ld=None, lds=None):
    up = lambda n, u: -(-n // u) * u  # noqa: E731
    return B._F8Matrix(AT, up(K, 16) if ld is None else ld, AT, up(-(-K // 128), 4) if lds is None else lds, fmt, rows)


def _linear(lib, M=4, N=200, K=256, x=None, w=None, y=AT, dtype=B.BF16, ldy=None, **e):
    e = B._Epilogue(**dict(dict(bias=None, residual=None, ldr=0, z=None, ldz=0, act=0, scale=1.0), **e))
    return lib.sop_fp8_linear(lib.ctx, x or _f8(M, K), w or _f8(N, K, 128), 0, M, N, K, e, y, dtype, N if ldy is None else ldy, None)


def test_product_with_an_epilogue(lib):
    assert _linear(lib, act=3, scale=0.5, bias=AT) == OK and _said(lib) == [["f8mm_epilogue", "4", "200", "3", "0.5"]]
    assert _linear(lib, M=0) == OK and _said(lib) == []
    for more in (dict(act=5), dict(act=-1), dict(bias=AT + 2), dict(residual=AT, ldr=199), dict(residual=AT + 1, ldr=200), dict(residual=AT, ldr=208), dict(z=AT + 4096, ldz=100),
                 dict(z=AT, ldz=200), dict(residual=AT + 4096, ldr=200, z=AT + 4096, ldz=200)):
        assert _linear(lib, **more) == EINVAL and lib.stub_error().startswith(b"sop_fp8_linear: "), more
    assert _linear(lib, residual=AT, ldr=200) == OK                    # y itself
    assert lib.sop_fp8_linear(lib.ctx, _f8(4, 256), _f8(200, 256, 128), 0, 4, 200, 256, None, AT, B.BF16, 200, None) == EINVAL
    _said(lib)


def _packed(N, K, g=16, bits=4):
    table = (C.c_float * 16)()
    return B._Packed(AT, AT, N, K, g, bits, sop.ScaleFmt(0, 4, 4, 8, -1, -1), 0, C.cast(table, C.POINTER(C.c_float)), 16, None, 0)


def test_packed_product_with_an_epilogue_in_two_launches(lib):
    """2^29 columns, or 2^30 rows, of 8 elements: halves, each with its part of bias, residual and z."""
    e = B._Epilogue(bias=AT, residual=1 << 40, ldr=1 << 30, z=1 << 50, ldz=(1 << 30) + 8, act=0, scale=1.0)
    N = (1 << 29) + 4
    assert lib.sop_packed_linear(lib.ctx, AT, 8, _packed(N, 8, 8), 1, e, 1 << 45, 1 << 30, None) == OK
    a, b = ([int(v) for v in s[1:]] for s in _said(lib))
    half = N // 2
    assert a == [1, half, AT, 1 << 40, 1 << 50, 1 << 45] and b == [1, N - half, AT + 4 * half, (1 << 40) + 2 * half, (1 << 50) + 2 * half, (1 << 45) + 2 * half]
    e.ldr, e.ldz, N = 3, 5, 1 << 30
    half = N // 2
    assert lib.sop_packed_linear(lib.ctx, AT, 8, _packed(1, 8, 8), N, e, 1 << 45, 1, None) == OK
    a, b = ([int(v) for v in s[1:]] for s in _said(lib))
    assert a == [half, 1, AT, 1 << 40, 1 << 50, 1 << 45] and b == [N - half, 1, AT, (1 << 40) + 6 * half, (1 << 50) + 10 * half, (1 << 45) + 2 * half]
    e.act = 9
    assert lib.sop_packed_linear(lib.ctx, AT, 8, _packed(1, 8, 8), 4, e, AT, 1, None) == EINVAL


def _act_grad(lib, M=1000, N=600, dy=AT, lddy=None, z=AT, ldz=None, dtype=B.F32, act=3, dz=AT + 4, lddz=None, dz8=None, db=AT, ws=1 << 30, size=None):
    n = C.c_size_t()
    assert lib.sop_fp8_linear_grad_workspace(lib.ctx, M, N, C.byref(n)) == OK
    return lib.sop_fp8_linear_grad(lib.ctx, dy, N if lddy is None else lddy, z, N if ldz is None else ldz, dtype, M, N, act, 1.0, dz, N if lddz is None else lddz,
                                   dz8 or _f8(M, N), db, ws, n.value if size is None else size, None), n.value


def test_gradient_of_an_epilogue(lib):
    for M in (1, 4, 5, 100, 128, 129, 8192, 100000):
        for N in (1, 512, 513, 11008, 1 << 20, 1 << 23):
            status, size = _act_grad(lib, M, N)
            assert status == OK
            said = {s[0]: [int(v) for v in s[1:]] for s in _said(lib)}
            m, n, words, strips, part = said["act_grad"]
            assert (m, n, strips) == (M, N, -(-N // 512)) and words * strips <= max(strips, 2048) and 1 <= words <= -(-M // 4)
            few = M <= 128                                             # a workgroup has all of a column
            assert size == (0 if few else words * N * 4) and part == (0 if few else 1 << 30)
            assert ("join" in said) != few
            if not few:
                assert said["join"] == [0, 1, words, 1 << 30, AT]
    assert _act_grad(lib, 0)[0] == OK and _said(lib) == [["join", "0", "1", "0", "0", str(AT)]]   # no rows: zeros
    assert _act_grad(lib, 0, db=None)[0] == OK and _said(lib) == []
    assert _act_grad(lib, act=0, z=None, dz=None)[0] == OK
    for more in (dict(dtype=2), dict(act=5), dict(dy=None), dict(dy=AT + 2), dict(z=None), dict(lddy=599), dict(lddz=599), dict(ldz=1), dict(db=AT + 1), dict(dz8=_f8(1000, 600, 128)),
                 dict(dz8=_f8(1000, 600, fmt=3)), dict(dz8=_f8(1000, 600, ld=592)), dict(dz8=_f8(1000, 600, ld=600))):
        assert _act_grad(lib, **more)[0] == EINVAL, more
    for more in (dict(ws=None), dict(ws=(1 << 30) + 8), dict(size=0)):
        assert _act_grad(lib, **more)[0] == ENOMEM, more
    assert _act_grad(lib, ws=None, db=None)[0] == OK
    assert lib.sop_fp8_linear_grad_workspace(lib.ctx, 1, 0, C.byref(C.c_size_t())) == ESHAPE and lib.sop_fp8_linear_grad_workspace(lib.ctx, 1, 1, None) == EINVAL
    _said(lib)


def _opts(**kw):
    return B._NormOpts(**dict(dict(after=AT, before=AT, gate=None, ld_gate=0, gate_dtype=0, groups=0, scale=1.0, eps=1e-6), **kw))


def _norm(lib, M=6, D=300, o=None, y=AT, ldy=300, ty=B.BF16, r=AT + 4096, ldr=300, tr=B.F32, s=AT + 8192, lds=300, n=None, ldn=300, tn=B.F32, n8=True):
    return lib.sop_residual_norm(lib.ctx, o or _opts(), M, D, y, ldy, ty, r, ldr, tr, s, lds, n, ldn, tn, _f8(M, D) if n8 is True else n8, None)


def test_norm(lib):
    assert _norm(lib) == OK and _said(lib) == [["norm", "6", "300", "6", "1", "0"]]
    assert _norm(lib, o=_opts(gate=AT, ld_gate=300, groups=3)) == OK and _said(lib) == [["norm", "6", "300", "2", "1", "0"]]
    assert _norm(lib, M=0, y=None, r=None, s=None, n8=None, n=AT, o=_opts(after=None)) == OK and _said(lib) == []
    assert _norm(lib, M=0, y=None, r=None, s=None, n8=None, o=_opts(gate=AT, ld_gate=300, groups=5)) == OK and _said(lib) == []   # (no rows: no addresses either)
    assert _norm(lib, s=AT + 4096) == OK                               # in r's place
    assert _norm(lib, y=None, s=None, o=_opts(after=None)) == OK
    gate = dict(gate=AT, ld_gate=300, groups=2)
    for more in (dict(ty=2), dict(tr=-1), dict(n=AT, tn=7), dict(o=_opts(eps=0.0)), dict(o=_opts(eps=float("nan"))), dict(o=_opts(eps=float("inf"))), dict(o=_opts(eps=1e-30)),
                 dict(o=_opts(after=AT + 2)), dict(o=_opts(before=AT + 1)), dict(o=_opts(**dict(gate, groups=4))), dict(o=_opts(**dict(gate, groups=0))),
                 dict(o=_opts(**dict(gate, ld_gate=299))), dict(o=_opts(**dict(gate, gate_dtype=3))), dict(n8=None), dict(o=_opts(before=None)), dict(y=None), dict(y=None, s=None),
                 dict(y=None, s=None, o=_opts(after=None, **gate)), dict(y=None, s=None, o=_opts(after=None, before=None), n8=None), dict(r=None), dict(s=None), dict(ldy=299),
                 dict(lds=299), dict(s=AT + 4096, lds=304), dict(s=AT), dict(n=AT), dict(n=AT + 4096), dict(n=AT + 8192), dict(n=AT + 2, tn=B.F32), dict(n8=_f8(6, 300, 128)),
                 dict(n8=_f8(6, 300, lds=2))):
        assert _norm(lib, **more) == EINVAL and lib.stub_error().startswith(b"sop_residual_norm: "), more
    assert _norm(lib, D=0) == ESHAPE and _norm(lib, D=(1 << 20) + 1) == ESHAPE and _norm(lib, M=-1) == ESHAPE
    _said(lib)


def _norm_grad(lib, M=6, D=300, o=None, ws=1 << 32, size=None, fmt=True, **kw):
    ld = dict(ld_ds=D, ld_dn=D, ld_s=D, ld_y=D, ld_dr=D, ld_dy=D, ld_dgate=D)
    at = {n: AT + (i << 12) for i, n in enumerate(("ds", "dn", "s", "y", "dr", "dy", "dbefore", "dafter"))}
    o = o or _opts()
    q = _f8(M, D)
    t = B._NormGrads(**dict(dict(at, r_dtype=B.F32, y_dtype=B.BF16, dy8=C.pointer(q) if fmt is True else fmt, dgate=AT + (1 << 16) if o.gate else None), **dict(ld, **kw)))
    n = C.c_size_t()
    status = lib.sop_residual_norm_grad_workspace(lib.ctx, M, D, o.groups if o.gate else 0, C.byref(n))
    if status:
        return status, 0
    return lib.sop_residual_norm_grad(lib.ctx, o, M, D, t, ws, n.value if size is None else size, None), n.value


def test_norm_gradients(lib):
    """Every row of a group is somebody's; partial sums, and what long rows keep, lie in the workspace; every sum has its rows joined."""
    for D in (1, 300, 512, 600, 1025, 2048, 4096, 8192, 8193, 16384, 16385, 20000):
        for M, G in ((1, 1), (6, 3), (777, 3), (5000, 1), (4096, 4096), (1200, 600), (2000, 1000), (3000, 1500), (100000, 2)):
            status, size = _norm_grad(lib, M, D, _opts(gate=AT, ld_gate=D, groups=G, gate_dtype=G % 2), dgate=1 << 62)
            assert status == OK, lib.stub_error()
            said = _said(lib)
            m, d, words, parts, groups, each, a, b, t, st = (int(v) for v in said[0][1:])
            assert (m, d, groups, each) == (M, D, G, M // G)
            row, base = words * D * 4, 1 << 32
            if parts > 1:
                assert words == G * parts and parts <= each
                assert [p * each // parts for p in range(parts + 1)][-1] == each
            else:
                assert words <= G and [w * G // words for w in range(words + 1)][-1] == G and all((w + 1) * G // words > w * G // words for w in range(words))
            assert words <= 2048 and (a, t, b) == (base, base, base + row)
            end = base + 2 * row
            assert size == end - base + (12 * M if D > 16384 else 0) and (D <= 16384 or st == end)
            joins = {int(s[1]): [int(v) for v in s[2:]] for s in said[1:]}
            assert (0 not in joins if parts > 1 and G == 1 else joins[0][:3] == [1, words, a])          # (a gate of one row: dafter comes of its set)
            assert joins[1][:3] == [1, words, b] and (2 in joins) == (parts > 1)
            if parts > 1:
                assert joins[2] == [G, parts, t, 1 << 62]
    assert _norm_grad(lib, 0, o=_opts(gate=AT, ld_gate=300, groups=70000), ds=None, y=None)[0] == OK         # no rows: zeros, in as many launches as they take
    said = [[int(v) for v in s[1:]] for s in _said(lib)]
    assert [s[1] for s in said if s[0] == 2] == [32768, 32768, 4464] and all(s[2] == 0 for s in said) and {s[0] for s in said} == {0, 1, 2}
    assert [s[4] - said[0][4] for s in said if s[0] == 2] == [0, 32768 * 1200, 65536 * 1200]


def test_norm_gradients_refuse(lib):
    gate = dict(gate=AT, ld_gate=300, groups=2)
    plain = _opts(after=None, before=None)
    assert _norm_grad(lib, o=plain, dbefore=None, dafter=None, s=None, dn=None)[0] == OK
    assert _norm_grad(lib, o=_opts(after=None), y=None, dy=None, dafter=None, fmt=None)[0] == OK
    assert _norm_grad(lib, ds=None)[0] == OK
    for more in (dict(r_dtype=2), dict(y_dtype=2), dict(y=None), dict(dr=None), dict(dy=None), dict(s=None), dict(dn=None), dict(ld_s=299), dict(ld_ds=1), dict(ds=AT + 2),
                 dict(dr=AT), dict(dy=AT + (2 << 12)), dict(dy=AT + (4 << 12)), dict(dbefore=AT + 2), dict(dafter=AT + 1), dict(o=plain), dict(o=plain, ds=None, dbefore=None, dafter=None),
                 dict(dgate=AT), dict(o=_opts(**gate), ld_dgate=299), dict(o=_opts(**gate), dgate=AT + 2), dict(o=_opts(eps=0.0)), dict(fmt=C.pointer(_f8(6, 300, 128))),
                 dict(o=_opts(after=None), y=None, dafter=None)):
        assert _norm_grad(lib, **more)[0] == EINVAL, more
    for more in (dict(ws=None), dict(ws=(1 << 32) + 4), dict(size=16)):
        assert _norm_grad(lib, **more)[0] == ENOMEM, more
    assert _norm_grad(lib, D=(1 << 20) + 1)[0] == ESHAPE and _norm_grad(lib, M=7, o=_opts(**gate))[0] == ESHAPE
    _said(lib)


def _clip(lib, tensors, most=1.0, norm=AT, ws=AT, size=None):
    n = C.c_size_t()
    assert lib.sop_clip_grads_workspace(lib.ctx, len(tensors), C.byref(n)) == OK
    packed = b"".join(B._GRAD.pack(*t) for t in tensors)
    return lib.sop_clip_grads(lib.ctx, packed, len(tensors), most, norm, ws, n.value if size is None else size, None), n.value


def test_clipping(lib):
    """Chunks of every tensor, lists of at most 96 tensors, partial sums within the workspace, the norm written once."""
    for count in (1, 3, 96, 97, 500, 3000):
        tensors = [((i + 1) << 36, (i + 1) << 36, 0 if i % 7 == 5 else (i + 1) * 7919 % 100000, i & 1, i & 1) for i in range(count)]
        status, size = _clip(lib, tensors)
        assert status == OK
        said = _said(lib)
        sizes, first, seen = [t[2] for t in tensors if t[2]], 0, {"square_sum": [], "clip": []}
        parts = sum(int(s[3]) for s in said if s[0] == "square_sum")
        assert 8 * parts <= size
        n = 0
        for s in said:
            if s[0] == "entry":
                seen[kind].append((int(s[1]), int(s[3])))
                end += -(-int(s[1]) // 8192)
                assert int(s[2]) == end
                continue
            kind, end = s[0], 0
            assert int(s[1]) <= 96 and 1 <= int(s[3]) <= int(s[2])
            if kind == "square_sum":
                assert int(s[4]) == first and int(s[5]) == first + int(s[3])
                first += int(s[3])
            else:
                assert int(s[4]) == n and int(s[5]) == parts           # (the first of them, 0, writes the norm)
                n += 1
        for kind in seen.values():
            assert kind == [(t[2], 3 * t[3]) for t in tensors if t[2]]
        assert len(sizes) == len(seen["clip"])
    assert _clip(lib, [])[0] == OK and _said(lib) == [["norm_of_parts", "0"]]
    assert _clip(lib, [(0, 0, 0, 0, 0)])[0] == OK and _said(lib) == [["norm_of_parts", "0"]]


def test_clipping_refuses(lib):
    one = (1 << 20, 1 << 20, 1000, 0, 0)
    assert _clip(lib, [one])[0] == OK
    assert _clip(lib, [one, (1 << 30, (1 << 20) + 4000, 1000, 0, 0)])[0] == OK   # side by side
    for tensors in ([(0, 1 << 20, 4, 0, 0)], [(1 << 20, 0, 4, 0, 0)], [(1 << 20, 1 << 21, -1, 0, 0)], [(1 << 20, 1 << 21, (1 << 36) + 1, 0, 0)], [((1 << 20) + 2, 1 << 21, 4, 0, 0)],
                    [(1 << 20, (1 << 21) + 1, 4, 0, 1)], [(1 << 20, 1 << 21, 4, 2, 0)], [(1 << 20, 1 << 21, 4, 0, 2)], [(1 << 20, 1 << 20, 4, 0, 1)],
                    [one, one],                                                        # the same tensor twice, in its own place
                    [(1 << 20, 1 << 22, 1000, 0, 0), (1 << 21, 1 << 22, 1000, 0, 0)],    # one out for two
                    [(1 << 20, 1 << 22, 1000, 0, 0), (1 << 21, (1 << 22) + 3996, 1000, 0, 0)], [(1 << 20, (1 << 20) + 4, 1000, 0, 0)], [(1 << 20, (1 << 20) - 4, 1000, 0, 0)],
                    [one, (1 << 30, (1 << 20) - 4, 2, 0, 0)], [(1 << 20, 1 << 25, 1000, 0, 0), (1 << 24, (1 << 20) + 2000, 10, 0, 1)]):
        assert _clip(lib, tensors)[0] == EINVAL, tensors
    assert _clip(lib, [(1 << 20, 1 << 22, 1000, 0, 0), (1 << 20, 1 << 23, 1000, 0, 0)])[0] == OK              # read twice, written apart
    packed = B._GRAD.pack(*one) * 2
    assert lib.sop_grad_norm(lib.ctx, packed, 2, AT, AT, 1 << 20, None) == OK                                # only read
    assert lib.sop_grad_norm(lib.ctx, None, 2, AT, AT, 1 << 20, None) == EINVAL
    for most in (-1.0, float("nan")):
        assert _clip(lib, [one], most=most)[0] == EINVAL
    for more in (dict(norm=None), dict(norm=AT + 2)):
        assert _clip(lib, [one], **more)[0] == EINVAL
    for more in (dict(ws=None), dict(ws=AT + 4), dict(size=64)):
        assert _clip(lib, [one], **more)[0] == ENOMEM
    assert lib.sop_clip_grads_workspace(lib.ctx, -1, C.byref(C.c_size_t())) == EINVAL and lib.sop_clip_grads_workspace(lib.ctx, 1, None) == EINVAL
    _said(lib)


def test_packed_tensor_is_the_headers():
    """The binding packs sop_grad by hand: two addresses, a count, two enumerations."""
    text = open(os.path.join(ROOT, "include", "sop.h")).read()
    assert re.search(r"typedef struct \{ const void\* x; void\* out; int64_t n; sop_dtype x_dtype, out_dtype; \} sop_grad;", text)
    assert B._GRAD.size == 32
