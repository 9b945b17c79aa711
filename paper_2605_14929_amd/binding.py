"""ctypes binding of include/sop.h.  Names follow the C entry points; no arithmetic lives here."""
from __future__ import annotations

import ctypes as C
import os
import struct
from dataclasses import dataclass
from typing import NamedTuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
F32, BF16 = 0, 1
SCALE_ABSMAX, SCALE_ARGMAX = 0, 1
SEL_WSE, SEL_COS, SEL_MSE = 0, 1, 2
MAX_ATOMS, MAX_ENTRIES = 8, 64
_STATUS = {1: "SOP_EINVAL", 2: "SOP_ESHAPE", 3: "SOP_EATOM", 4: "SOP_EFMT", 5: "SOP_ENOMEM", 6: "SOP_EHIP"}


class SopError(RuntimeError):
    def __init__(self, status: int, text: str):
        super().__init__(f"{_STATUS.get(status, status)}: {text}")
        self.status = status


class ScaleFmt(C.Structure):
    """sop_scale_fmt: SwExMy scale word in a b-bit container."""
    _fields_ = [("sign_bits", C.c_int), ("exp_bits", C.c_int), ("man_bits", C.c_int), ("container_bits", C.c_int),
                ("bias", C.c_int), ("max_code", C.c_int)]


class _Layer(C.Structure):
    """sop_layer: one linear layer of a model-wide search."""
    _fields_ = [("W", C.c_void_p), ("M", C.c_int64), ("K", C.c_int64), ("ldw", C.c_int64), ("c", C.c_void_p),
                ("k", C.c_int), ("sel_words", C.c_void_p)]


class WeightFmt(C.Structure):
    """sop_weight_fmt: ExMy weight grid."""
    _fields_ = [("exp_bits", C.c_int), ("man_bits", C.c_int), ("bias", C.c_int), ("max_code", C.c_int)]


class _Atom(C.Structure):
    _fields_ = [("n_entries", C.c_int), ("values", C.POINTER(C.c_float))]


LAYER_MAX_P = 7
LAYER_MAX_ATOMS = 16
LAYER_MAX_PAIRS = 120


class _LayerOpts(C.Structure):
    """sop_layer_opts"""
    _fields_ = [("n_p", C.c_int), ("p_percent", C.c_double * LAYER_MAX_P), ("fit_entries", C.c_int), ("fit_iters", C.c_int),
                ("fit_bins", C.c_int), ("fit_init", C.POINTER(C.c_float)), ("weighted_fit", C.c_int),
                ("fit_grid", C.POINTER(C.c_double)), ("n_fit_grid", C.c_int), ("pack", C.c_int)]


class _LayerResult(C.Structure):
    """sop_layer_result"""
    _fields_ = [("kind", C.c_int), ("a", C.c_int), ("b", C.c_int), ("j", C.c_int), ("p_percent", C.c_double), ("acos", C.c_double),
                ("n_entries_b", C.c_int), ("table_b", C.c_float * MAX_ENTRIES), ("acos_fixed", C.c_double * LAYER_MAX_PAIRS),
                ("acos_atom", C.c_double * LAYER_MAX_ATOMS), ("acos_fitted", (C.c_double * LAYER_MAX_P) * LAYER_MAX_ATOMS), ("n_bits", C.c_int)]


class _Outputs(C.Structure):
    _fields_ = [("acos_pair", C.c_void_p), ("acos_atom", C.c_void_p), ("sel_words", C.c_void_p),
                ("scale_code", C.c_void_p), ("codes", C.c_void_p), ("blk_cos", C.c_void_p), ("blk_err", C.c_void_p),
                ("blk_rank", C.c_void_p)]


class _F8Matrix(C.Structure):
    """sop_f8_matrix"""
    _fields_ = [("codes", C.c_void_p), ("ld_codes", C.c_int64), ("scales", C.c_void_p), ("ld_scales", C.c_int64), ("format", C.c_int), ("block_rows", C.c_int)]


class _Packed(C.Structure):
    """sop_packed_weights"""
    _fields_ = [("words", C.c_void_p), ("payload", C.c_void_p), ("N", C.c_int64), ("K", C.c_int64), ("g", C.c_int), ("n_bits", C.c_int),
                ("fmt", ScaleFmt), ("k", C.c_int), ("table_a", C.POINTER(C.c_float)), ("entries_a", C.c_int), ("table_b", C.POINTER(C.c_float)), ("entries_b", C.c_int)]


def lib_path() -> str:
    return os.path.join(_HERE, "libsop_hip.so")


_lib = None


def lib():
    """Load libsop_hip.so; fails loudly when it has not been built."""
    global _lib
    if _lib is None:
        path = lib_path()
        if not os.path.exists(path):
            raise SopError(6, f"{path} is missing: build it with `python -c 'import __graft_entry__ as g; g.build()'` "
                              "(the pair search has no CPU fallback)")
        # PyTorch ships its own HIP runtime; two HIP runtimes in one process cannot both own the GPU.
        # Importing torch first makes the loader resolve this library's libamdhip64.so.7 dependency
        # to the copy torch already mapped (same soname), so both sides share one runtime.
        import torch  # noqa: F401
        L = C.CDLL(path)
        L.sop_create.argtypes = [C.POINTER(C.c_void_p), C.c_int]
        L.sop_destroy.argtypes = [C.c_void_p]
        L.sop_set_alphabet.argtypes = [C.c_void_p, C.POINTER(_Atom), C.c_int]
        L.sop_check_alphabet.argtypes = [C.POINTER(_Atom), C.c_int, C.POINTER(C.c_int), C.POINTER(C.c_int64)]
        L.sop_set_pairs.argtypes = [C.c_void_p, C.POINTER(C.c_int), C.c_int]
        L.sop_set_scale_rule.argtypes = [C.c_void_p, C.c_int]
        L.sop_workspace_bytes.argtypes = [C.c_void_p, C.c_int64, C.c_int64, C.c_int, C.POINTER(C.c_size_t)]
        L.sop_pair_search.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int64, C.c_int64, C.c_int64, C.c_void_p, C.c_int,
                                      ScaleFmt, C.c_int, C.c_int, C.c_void_p, C.c_size_t, C.POINTER(_Outputs), C.c_void_p]
        L.sop_pair_search_static.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int64, C.c_int64, C.c_int64, C.c_void_p, C.c_int,
                                             ScaleFmt, C.c_int, C.c_int, C.POINTER(_Outputs), C.c_void_p]
        L.sop_search_layer_workspace.argtypes = [C.c_void_p, C.c_int64, C.c_int64, C.c_int, C.c_int, C.POINTER(_LayerOpts), C.POINTER(C.c_size_t)]
        L.sop_search_layer.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int64, C.c_int64, C.c_int64, C.c_void_p, C.c_int, ScaleFmt, C.c_int,
                                       C.c_int, C.POINTER(_Atom), C.c_int, C.POINTER(_LayerOpts), C.c_void_p, C.c_size_t,
                                       C.POINTER(_LayerResult), C.c_void_p, C.c_void_p, C.c_void_p]
        L.sop_prepare_scale.argtypes = [C.c_void_p, ScaleFmt, C.c_int, C.c_void_p]
        L.sop_last_error.argtypes = [C.c_void_p]
        L.sop_last_error.restype = C.c_char_p
        L.sop_atom_nf.argtypes = [C.c_int, C.POINTER(C.c_float)]
        L.sop_atom_sh.argtypes = [C.c_int, C.c_double, C.c_double, C.POINTER(C.c_float)]
        L.sop_atom_negate.argtypes = [C.POINTER(C.c_float), C.c_int, C.POINTER(C.c_float)]
        L.sop_lloyd_1d.argtypes = [C.POINTER(C.c_double), C.POINTER(C.c_double), C.c_int64, C.POINTER(C.c_double), C.c_int, C.c_int]
        L.sop_atom_bof.argtypes = [C.c_int, C.POINTER(C.c_double), C.c_int64, C.c_int, C.c_int, C.POINTER(C.c_float)]
        L.sop_dd_histogram.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int64, C.c_int64, C.c_int64, C.c_void_p, C.c_int, C.c_int,
                                       C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p]
        L.sop_dd_fit.argtypes = [C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_void_p]     # (host arrays by address: the fit is called in loops)
        L.sop_dd_fit_grid.argtypes = [C.c_void_p, C.c_int, C.c_void_p, C.c_int, C.c_int, C.c_void_p, C.c_void_p]
        L.sop_weight_grid.argtypes = [WeightFmt, C.c_double, C.c_void_p, C.c_void_p]
        L.sop_scale_histogram.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int64, C.c_int64, C.c_int64, C.c_int, C.c_float, C.c_float,
                                          ScaleFmt, C.c_void_p, C.c_void_p]
        L.sop_layer_scope_error.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int64, C.c_int64, C.c_int64, C.c_void_p, WeightFmt, ScaleFmt,
                                            C.c_int, C.c_void_p, C.c_void_p, C.c_void_p]
        L.sop_sum_f32.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]
        L.sop_read_probe.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]
        L.sop_issue_probe.argtypes = [C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_float, C.c_float, C.c_void_p, C.POINTER(C.c_int), C.c_void_p]
        L.sop_pair_search_layers.argtypes = [C.c_void_p, C.POINTER(_Layer), C.c_int, C.c_int, C.c_int, ScaleFmt, C.c_int,
                                             C.c_void_p, C.c_void_p, C.c_void_p]
        L.sop_partition.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_int64, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.sop_partition_levels.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.POINTER(C.c_int64), C.c_int, C.c_int, C.c_void_p, C.c_void_p,
                                           C.c_void_p, C.c_void_p]
        L.sop_dd_histogram_levels.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int64, C.c_int64, C.c_int64, C.c_void_p, C.c_int, C.c_int,
                                              C.c_int64, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p]
        L.sop_pack_blocks.argtypes = [C.c_void_p, C.c_int64, C.c_int64, C.c_int, ScaleFmt, C.c_void_p, C.c_void_p, C.c_int,
                                      C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_int, C.c_int, C.c_void_p, C.c_void_p,
                                      C.POINTER(C.c_int), C.c_void_p]
        L.sop_fp8_quantize.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int64, C.c_int64, C.c_int64, C.POINTER(_F8Matrix), C.c_void_p, C.c_int64, C.c_void_p]
        L.sop_fp8_matmul.argtypes = [C.c_void_p, C.POINTER(_F8Matrix), C.POINTER(_F8Matrix), C.c_int, C.c_int64, C.c_int64, C.c_int64, C.c_void_p, C.c_int,
                                     C.c_int64, C.c_void_p]
        L.sop_fp8_weight_grad.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.POINTER(_F8Matrix), C.c_int64, C.c_int64, C.c_int64, C.c_void_p, C.c_int,
                                          C.c_int64, C.c_int, C.c_void_p]
        L.sop_fp8_gated.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_int, C.c_int64, C.c_int64, C.POINTER(_F8Matrix),
                                    C.POINTER(_F8Matrix), C.POINTER(_F8Matrix), C.c_void_p]
        L.sop_fp8_gated_grad.argtypes = [C.c_void_p, C.POINTER(_F8Matrix), C.POINTER(_F8Matrix), C.c_void_p, C.c_int64, C.c_int, C.c_int64, C.c_int64,
                                         C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.POINTER(_F8Matrix), C.POINTER(_F8Matrix), C.c_void_p]
        L.sop_packed_matmul.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.POINTER(_Packed), C.c_int64, C.c_void_p, C.c_int64, C.c_void_p]
        epilogue = [C.POINTER(_Epilogue)]
        L.sop_fp8_linear.argtypes = L.sop_fp8_matmul.argtypes[:7] + epilogue + L.sop_fp8_matmul.argtypes[7:]
        L.sop_packed_linear.argtypes = L.sop_packed_matmul.argtypes[:5] + epilogue + L.sop_packed_matmul.argtypes[5:]
        L.sop_fp8_linear_grad_workspace.argtypes = [C.c_void_p, C.c_int64, C.c_int64, C.POINTER(C.c_size_t)]
        L.sop_fp8_linear_grad.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_int, C.c_int64, C.c_int64, C.c_int, C.c_float, C.c_void_p,
                                          C.c_int64, C.POINTER(_F8Matrix), C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.sop_residual_norm.argtypes = [C.c_void_p, C.POINTER(_NormOpts), C.c_int64, C.c_int64, C.c_void_p, C.c_int64, C.c_int, C.c_void_p, C.c_int64, C.c_int,
                                        C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_int, C.POINTER(_F8Matrix), C.c_void_p]
        L.sop_residual_norm_grad_workspace.argtypes = [C.c_void_p, C.c_int64, C.c_int64, C.c_int64, C.POINTER(C.c_size_t)]
        L.sop_residual_norm_grad.argtypes = [C.c_void_p, C.POINTER(_NormOpts), C.c_int64, C.c_int64, C.POINTER(_NormGrads), C.c_void_p, C.c_size_t, C.c_void_p]
        L.sop_clip_grads_workspace.argtypes = [C.c_void_p, C.c_int64, C.POINTER(C.c_size_t)]
        L.sop_grad_norm.argtypes = [C.c_void_p, C.c_char_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]   # (sop_grad, packed)
        L.sop_clip_grads.argtypes = [C.c_void_p, C.c_char_p, C.c_int64, C.c_float, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.sop_layer_shift.argtypes = [C.POINTER(C.c_int64), C.c_int64, ScaleFmt, C.POINTER(C.c_int), C.POINTER(C.c_double)]
        _lib = L
    return _lib


def _fp(a, t=C.c_float):
    return a.ctypes.data_as(C.POINTER(t))


def _check(status, ctx=None):
    if status != 0:
        raise SopError(status, (lib().sop_last_error(ctx) or b"").decode())


# ---- host atom builders (C implementations) ----
def sop_atom_nf(n_bits: int) -> np.ndarray:
    out = np.empty(2 ** n_bits, dtype=np.float32)
    _check(lib().sop_atom_nf(n_bits, _fp(out)))
    return out


def sop_atom_sh(n_bits: int, alpha: float = 1.5, c: float = -0.02) -> np.ndarray:
    out = np.empty(2 ** n_bits, dtype=np.float32)
    _check(lib().sop_atom_sh(n_bits, alpha, c, _fp(out)))
    return out


def sop_atom_negate(values: np.ndarray) -> np.ndarray:
    v = np.ascontiguousarray(values, dtype=np.float32)
    out = np.empty_like(v)
    _check(lib().sop_atom_negate(_fp(v), v.size, _fp(out)))
    return out


def sop_lloyd_1d(samples: np.ndarray, weights, init: np.ndarray, iters: int) -> np.ndarray:
    x = np.ascontiguousarray(samples, dtype=np.float64)
    w = None if weights is None else np.ascontiguousarray(weights, dtype=np.float64)
    cent = np.array(init, dtype=np.float64).copy()
    _check(lib().sop_lloyd_1d(_fp(x, C.c_double), None if w is None else _fp(w, C.c_double), x.size, _fp(cent, C.c_double), cent.size, iters))
    return cent


def sop_atom_bof(n_bits: int, draws: np.ndarray, g: int = 16, iters: int = 50) -> np.ndarray:
    d = np.ascontiguousarray(draws, dtype=np.float64)
    out = np.empty(2 ** n_bits, dtype=np.float32)
    _check(lib().sop_atom_bof(n_bits, _fp(d, C.c_double), d.size, g, iters, _fp(out)))
    return out


def sop_dd_fit(hist: np.ndarray, n_entries: int, iters: int, init: np.ndarray) -> np.ndarray:
    """Weighted Lloyd fit on an [H] int64 histogram (host)."""
    h = np.ascontiguousarray(hist, dtype=np.int64).reshape(-1)
    ini = np.ascontiguousarray(init, dtype=np.float32)
    out = np.empty(n_entries, dtype=np.float32)
    _check(lib().sop_dd_fit(h.ctypes.data, h.size, n_entries, iters, ini.ctypes.data, out.ctypes.data))
    return out


def sop_dd_fit_grid(hist: np.ndarray, cand: np.ndarray, n_entries: int):
    """Best n_entries of the ascending candidate values for an [H] int64 histogram (host):
    (indices into cand, cost)."""
    h = np.ascontiguousarray(hist, dtype=np.int64).reshape(-1)
    g = np.ascontiguousarray(cand, dtype=np.float64).reshape(-1)
    chosen = np.empty(n_entries, dtype=np.int32)
    cost = C.c_double(0.0)
    _check(lib().sop_dd_fit_grid(h.ctypes.data, h.size, g.ctypes.data, g.size, n_entries, chosen.ctypes.data, C.byref(cost)))
    return chosen.astype(np.int64), cost.value


def sop_weight_grid(wfmt: "WeightFmt", top: float = 0.0) -> np.ndarray:
    """Distinct values of an ExMy weight grid, ascending (host)."""
    out = np.empty(2 * (1 << (wfmt.exp_bits + wfmt.man_bits)) + 1, dtype=np.float64)
    n = C.c_int(0)
    _check(lib().sop_weight_grid(wfmt, C.c_double(top), out.ctypes.data, C.byref(n)))
    return out[:n.value].copy()


def sop_layer_shift(hist: np.ndarray, n_blocks: int, fmt: "ScaleFmt"):
    """(k*, fraction of block scales in the normal range) from a [2, 320] int64 exponent histogram (host)."""
    h = np.ascontiguousarray(hist, dtype=np.int64).reshape(-1)
    if h.size != 640:
        raise SopError(1, "the exponent histogram has 2 x 320 entries")
    k, frac = C.c_int(), C.c_double()
    _check(lib().sop_layer_shift(_fp(h, C.c_int64), n_blocks, fmt, C.byref(k), C.byref(frac)))
    return k.value, frac.value


def sop_check_alphabet(tables):
    """Host-only check of the search table built for these atoms; returns (n_bins, n_checked)."""
    tabs = [np.ascontiguousarray(t, dtype=np.float32) for t in tables]
    arr = (_Atom * len(tabs))()
    for i, t in enumerate(tabs):
        arr[i].n_entries = t.size
        arr[i].values = _fp(t)
    nb, nc = C.c_int(), C.c_int64()
    _check(lib().sop_check_alphabet(arr, len(tabs), C.byref(nb), C.byref(nc)))
    return nb.value, nc.value


_FMTS = {
    "UE4M4": (0, 4, 4, 8, -1, -1), "E4M3": (1, 4, 3, 8, -1, -1), "UE4M3": (0, 4, 3, 8, -1, -1),
    "UE4M6": (0, 4, 6, 10, -1, -1), "E4M5": (1, 4, 5, 10, -1, -1), "UE5M7": (0, 5, 7, 12, -1, -1),
    "E5M6": (1, 5, 6, 12, -1, -1), "E4M7": (1, 4, 7, 12, -1, -1), "S1E5M5": (1, 5, 5, 12, -1, -1),
    "S0E6M5": (0, 6, 5, 12, -1, -1), "UE5M3": (0, 5, 3, 8, -1, -1),
    # bf16-like 16-bit scale kept inside binary32's normal range (values 2^-125 .. < 2^126)
    "E8M7": (1, 8, 7, 16, 119, 244 * 128 + 127),
}


def fmt_by_name(name: str) -> ScaleFmt:
    return ScaleFmt(*_FMTS[name])


def build_alphabet(names, bof_draws=None) -> list:
    """Tables for names such as "NF4", "SH5", "BOF4", "-NF4" using the library's own builders."""
    out = []
    for nm in names:
        neg = nm.startswith("-")
        base = nm[1:] if neg else nm
        kind, n = base[:-1], int(base[-1])
        if kind == "NF":
            t = sop_atom_nf(n)
        elif kind == "SH":
            t = sop_atom_sh(n)
        elif kind == "BOF":
            if bof_draws is None:
                raise ValueError("BOF atoms need N(0,1) draws")
            t = sop_atom_bof(n, bof_draws)
        else:
            raise ValueError(f"unknown atom {nm}")
        out.append(sop_atom_negate(t) if neg else t)
    return out


@dataclass
class Outputs:
    """Device tensors produced by Context.pair_search (None when not requested)."""
    acos_pair: object = None
    acos_atom: object = None
    sel_words: object = None
    scale_code: object = None
    codes: object = None
    code_planes: list = None
    blk_cos: object = None
    blk_err: object = None
    blk_rank: object = None


E4M3, E5M2 = 0, 1
RELU, SILU, GELU, GELU_TANH = 1, 2, 3, 4


class _Epilogue(C.Structure):
    """sop_epilogue"""
    _fields_ = [("bias", C.c_void_p), ("residual", C.c_void_p), ("ldr", C.c_int64), ("z", C.c_void_p), ("ldz", C.c_int64), ("act", C.c_int), ("scale", C.c_float)]


class _NormOpts(C.Structure):
    """sop_residual_norm_opts"""
    _fields_ = [("after", C.c_void_p), ("before", C.c_void_p), ("gate", C.c_void_p), ("ld_gate", C.c_int64), ("gate_dtype", C.c_int), ("groups", C.c_int64),
                ("scale", C.c_float), ("eps", C.c_float)]


class _NormGrads(C.Structure):
    """sop_residual_norm_grads"""
    _fields_ = [("ds", C.c_void_p), ("ld_ds", C.c_int64), ("dn", C.c_void_p), ("ld_dn", C.c_int64), ("s", C.c_void_p), ("ld_s", C.c_int64), ("y", C.c_void_p), ("ld_y", C.c_int64),
                ("dr", C.c_void_p), ("ld_dr", C.c_int64), ("dy", C.c_void_p), ("ld_dy", C.c_int64), ("dy8", C.POINTER(_F8Matrix)), ("dbefore", C.c_void_p), ("dafter", C.c_void_p),
                ("dgate", C.c_void_p), ("ld_dgate", C.c_int64), ("r_dtype", C.c_int), ("y_dtype", C.c_int)]


_GRAD = struct.Struct("@QQqii")                                       # sop_grad


class ResidualNormGrads(NamedTuple):
    """What Context.residual_norm_grad returns; None where there is nothing of it."""
    dr: object
    dy: object
    dy8: object
    dbefore: object
    dafter: object
    dgate: object


def _up(n, unit):
    return -(-n // unit) * unit


def _spaced(t, unit, what):
    """A 2-D tensor of bytes as the library reads it: rows that start on a multiple of `unit` bytes (and may so be read to one: such a piece
    with a byte of the tensor in it lies on a page of its memory).  The tensor itself if it is laid out so, else a copy that is; and the
    distance of its rows."""
    import torch
    if t.dim() != 2 or t.element_size() != 1 or not t.is_cuda:
        raise SopError(1, f"{what} must be a 2-D CUDA tensor of one byte an element")
    R, Cc = t.shape
    ld, step = t.stride()
    if R <= 1:
        ld = _up(Cc, unit)
    if (step == 1 or Cc <= 1) and ld >= Cc and ld % unit == 0 and t.data_ptr() % unit == 0:
        return t, ld
    ld = _up(Cc, unit)
    buf = torch.zeros((R, ld), dtype=torch.uint8, device=t.device)
    buf[:, :Cc] = t.contiguous().view(torch.uint8)
    return buf.view(t.dtype)[:, :Cc], ld


def _room(torch, R, Cc, unit, dtype, device):
    """An uninitialised [R, Cc] of bytes laid out so, and the distance of its rows."""
    ld = -(-Cc // unit) * unit
    return torch.empty_strided((R, Cc), (ld, 1), dtype=dtype, device=device), ld


def _dense(t):
    """Whether a tensor's elements fill a range of memory, in whatever order of its dimensions."""
    n = 1
    for size, step in sorted(zip(t.shape, t.stride()), key=lambda d: (d[1], d[0])):
        if size != 1:
            if step != n:
                return False
            n *= size
    return True


class Fp8Blocks:
    """A matrix in 8 bits: codes (torch.float8_e4m3fn or float8_e5m2, [R, C]) and one power-of-two scale (torch.float8_e8m0fnu) for
    each block of `rows` x 128 (rows = 1: activations and gradients; rows = 128: weights).  codes_t: the same codes as a [C, R]
    matrix, where the product over the other index is wanted too.  Tensors that are not laid out as the library reads them (rows of
    codes 16 bytes apart, of scales 4) are copied, once."""
    __slots__ = ("codes", "scales", "rows", "codes_t", "shape", "device", "_m", "_t")

    def __init__(self, codes, scales, rows: int = 1, codes_t=None):
        import torch
        fmt = E4M3 if codes.dtype is torch.float8_e4m3fn else E5M2 if codes.dtype is torch.float8_e5m2 else None
        if fmt is None:
            raise SopError(1, "codes must be float8_e4m3fn or float8_e5m2")
        if scales.dtype is not torch.float8_e8m0fnu and scales.dtype is not torch.uint8:
            raise SopError(1, "scales must be float8_e8m0fnu (or its bytes)")
        if rows not in (1, 128):
            raise SopError(1, "blocks have 1 or 128 rows")
        self.codes, ld = _spaced(codes, 16, "codes")
        self.scales, lds = _spaced(scales, 4, "scales")
        R, K = codes.shape
        if tuple(scales.shape) != (-(-R // rows), -(-K // 128)):
            raise SopError(2, f"codes of {R} x {K} in blocks of {rows} x 128 have scales of {-(-R // rows)} x {-(-K // 128)}")
        self.device = codes.get_device()
        if scales.get_device() != self.device:
            raise SopError(1, "codes and scales must be on one GPU")
        self.rows, self.shape, self.codes_t, self._t = rows, (R, K), None, None
        self._m = _F8Matrix(self.codes.data_ptr(), ld, self.scales.data_ptr(), lds, fmt, rows)
        if codes_t is not None:
            if rows != 128 or codes_t.dtype is not codes.dtype or tuple(codes_t.shape) != (K, R) or codes_t.get_device() != self.device:
                raise SopError(2, "codes_t must be the codes of 128 x 128 blocks, transposed")
            self.codes_t, ldt = _spaced(codes_t, 16, "codes_t")
            self._t = _F8Matrix(self.codes_t.data_ptr(), ldt, self.scales.data_ptr(), lds, fmt, rows)

    @classmethod
    def empty(cls, R, K, fmt, device, rows: int = 1, transposed: bool = False):
        """Uninitialised, to be written by a call of the library.  fmt: E4M3, E5M2 or the torch type."""
        import torch
        if fmt == E4M3 or fmt is torch.float8_e4m3fn:
            fmt, dt = E4M3, torch.float8_e4m3fn
        elif fmt == E5M2 or fmt is torch.float8_e5m2:
            fmt, dt = E5M2, torch.float8_e5m2
        else:
            raise SopError(1, "the format must be E4M3 or E5M2")
        if rows != 1 and rows != 128:
            raise SopError(1, "blocks have 1 or 128 rows")
        q = cls.__new__(cls)
        q.codes, ld = _room(torch, R, K, 16, dt, device)
        q.scales, lds = _room(torch, -(-R // rows), -(-K // 128), 4, torch.float8_e8m0fnu, device)
        q.rows, q.shape, q.device, q.codes_t, q._t = rows, (R, K), q.codes.get_device(), None, None
        at = q.scales.data_ptr()
        q._m = _F8Matrix(q.codes.data_ptr(), ld, at, lds, fmt, rows)
        if transposed:
            q.codes_t, ldt = _room(torch, K, R, 16, dt, device)
            q._t = _F8Matrix(q.codes_t.data_ptr(), ldt, at, lds, fmt, rows)
        return q


class PackedWeights:
    """A packed layer [N, K] as it is held for products: what pack_blocks / search_layer(pack=True) wrote (words, payload, n_bits), its
    codebooks (one table, or two where the words carry a selector) and the scale format and layer shift k of the search."""
    __slots__ = ("words", "payload", "shape", "tables", "device", "_w")

    def __init__(self, words, payload, N, K, g, n_bits, fmt: ScaleFmt, tables, k: int = 0):
        import torch
        if not (words.is_cuda and payload.is_cuda) or words.device != payload.device:
            raise SopError(1, "words and payload must be CUDA tensors on one GPU (no CPU fallback)")
        if words.element_size() != 2 or payload.dtype != torch.uint8 or not (words.is_contiguous() and payload.is_contiguous()):
            raise SopError(1, "words must be contiguous 16-bit integers, payload contiguous uint8")
        if N < 1 or K < 1 or g < 1 or K % g or words.numel() != N * K // g or payload.numel() != N * K * n_bits // 8:
            raise SopError(2, "words and payload do not hold N x K weights in blocks of g with n_bits codes")
        if not 1 <= len(tables) <= 2:
            raise SopError(3, "one codebook or two")
        self.words, self.payload, self.shape, self.device = words, payload, (N, K), words.get_device()
        self.tables = [np.ascontiguousarray(t, dtype=np.float32) for t in tables]
        a, b = self.tables[0], self.tables[1] if len(tables) == 2 else None
        self._w = _Packed(words.data_ptr(), payload.data_ptr(), N, K, g, n_bits, fmt, k, _fp(a), a.size, None if b is None else _fp(b), 0 if b is None else b.size)


class Context:
    """sop_ctx with PyTorch tensors for device memory and the current stream."""

    def __init__(self, device: int = 0):
        self._h = C.c_void_p()
        _check(lib().sop_create(C.byref(self._h), device))
        self.device = device
        self.n_atoms = 0
        self.n_entries = []
        self.n_pairs = 0
        self._ws = None
        import torch
        self._lib, self._bf16, self._f32 = lib(), torch.bfloat16, torch.float32
        self._dtypes = {torch.float32: F32, torch.bfloat16: BF16}
        # the current stream's handle, without an object around it where torch can give it so
        self._raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda d: torch.cuda.current_stream(d).cuda_stream)

    def close(self):
        if self._h:
            lib().sop_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_alphabet(self, tables):
        tabs = [np.ascontiguousarray(t, dtype=np.float32) for t in tables]
        arr = (_Atom * len(tabs))()
        for i, t in enumerate(tabs):
            arr[i].n_entries = t.size
            arr[i].values = _fp(t)
        _check(lib().sop_set_alphabet(self._h, arr, len(tabs)), self._h)
        self.n_atoms = len(tabs)
        self.n_entries = [t.size for t in tabs]
        self.n_pairs = self.n_atoms * (self.n_atoms - 1) // 2

    def set_pairs(self, pairs):
        if pairs is None or len(pairs) == 0:
            _check(lib().sop_set_pairs(self._h, None, 0), self._h)
            self.n_pairs = self.n_atoms * (self.n_atoms - 1) // 2
            return
        p = np.ascontiguousarray(pairs, dtype=np.int32).reshape(-1, 2)
        _check(lib().sop_set_pairs(self._h, _fp(p, C.c_int), p.shape[0]), self._h)
        self.n_pairs = p.shape[0]

    def workspace_bytes(self, M, K, g) -> int:
        n = C.c_size_t()
        _check(lib().sop_workspace_bytes(self._h, M, K, g, C.byref(n)), self._h)
        return n.value

    def alloc_outputs(self, M, K, g, emit=False, sel=True) -> Outputs:
        """Allocate output tensors for a layer (device memory comes from PyTorch)."""
        import torch
        dev = torch.device("cuda", self.device)
        A, P, Bk = self.n_atoms, self.n_pairs, K // g
        Nb = M * Bk
        o = Outputs()
        o.acos_atom = torch.empty(A, dtype=torch.float64, device=dev)
        o.acos_pair = torch.empty(max(P, 1), dtype=torch.float64, device=dev)
        if sel and P:
            # one selector word per block: 16-bit words up to 16 pairs, 32-bit words beyond
            o.sel_words = torch.empty(Nb, dtype=torch.int16 if P <= 16 else torch.int32, device=dev)
        if emit:
            o.scale_code = torch.empty((A, Nb), dtype=torch.int16, device=dev)
            planes = [M * K // 2 if n <= 16 else M * K for n in self.n_entries]
            o.codes = torch.empty(sum(planes), dtype=torch.uint8, device=dev)
            offs = np.concatenate([[0], np.cumsum(planes)])
            o.code_planes = [o.codes[int(offs[a]):int(offs[a + 1])] for a in range(A)]
            o.blk_cos = torch.empty((A, Nb), dtype=torch.float32, device=dev)
            o.blk_err = torch.empty((A, Nb), dtype=torch.float32, device=dev)
            o.blk_rank = torch.empty((A, Nb), dtype=torch.float32, device=dev)
        return o

    def layer_scope_error(self, W, c, wfmt: WeightFmt, sfmt: ScaleFmt, k: int = 0, want_codes: bool = False, stream=None):
        """sop_layer_scope_error on torch CUDA tensors; returns (out [4] float64 device tensor, codes or None)."""
        import torch
        if not W.is_cuda or (c is not None and not c.is_cuda):
            raise SopError(1, "W and c must be CUDA tensors (no CPU fallback)")
        if W.dim() != 2 or W.stride(1) != 1:
            raise SopError(2, "W must be a 2-D tensor with contiguous rows")
        dt = BF16 if W.dtype == torch.bfloat16 else (F32 if W.dtype == torch.float32 else None)
        if dt is None:
            raise SopError(1, "W must be float32 or bfloat16")
        M, K = W.shape
        out = torch.empty(4, dtype=torch.float64, device=W.device)
        codes = torch.empty((M, K), dtype=torch.int16, device=W.device) if want_codes else None
        st = torch.cuda.current_stream(W.device).cuda_stream if stream is None else stream
        _check(lib().sop_layer_scope_error(self._h, C.c_void_p(W.data_ptr()), dt, M, K, W.stride(0),
                                           None if c is None else C.c_void_p(c.data_ptr()), wfmt, sfmt, k, C.c_void_p(out.data_ptr()),
                                           None if codes is None else C.c_void_p(codes.data_ptr()), C.c_void_p(st)), self._h)
        return out, codes

    def sum_f32(self, x, stream=None):
        """sop_sum_f32 on a contiguous float32 CUDA tensor; returns a [1] float64 device tensor."""
        import torch
        if not x.is_cuda or x.dtype != torch.float32 or not x.is_contiguous():
            raise SopError(1, "x must be a contiguous float32 CUDA tensor")
        out = torch.empty(1, dtype=torch.float64, device=x.device)
        st = torch.cuda.current_stream(x.device).cuda_stream if stream is None else stream
        _check(lib().sop_sum_f32(self._h, C.c_void_p(x.data_ptr()), x.numel(), C.c_void_p(out.data_ptr()), C.c_void_p(st)), self._h)
        return out

    def read_probe(self, x, out=None, stream=None):
        """sop_read_probe on a contiguous CUDA tensor whose size is a multiple of 16 bytes; returns the
        [2048] int32 device tensor of per-workgroup checksums."""
        import torch
        if not x.is_cuda or not x.is_contiguous():
            raise SopError(1, "x must be a contiguous CUDA tensor")
        if out is None:
            out = torch.empty(2048, dtype=torch.int32, device=x.device)
        st = torch.cuda.current_stream(x.device).cuda_stream if stream is None else stream
        _check(lib().sop_read_probe(self._h, C.c_void_p(x.data_ptr()), x.numel() * x.element_size(), C.c_void_p(out.data_ptr()), C.c_void_p(st)), self._h)
        return out

    def issue_probe(self, kind: int, waves_per_simd: int, iters: int, a: float = 0.5, b: float = 0.25, out=None, stream=None):
        """sop_issue_probe: returns the [compute units * waves_per_simd * 256] float32 device tensor of per-lane chain sums."""
        import torch
        dev = torch.device("cuda", self.device)
        n = torch.cuda.get_device_properties(dev).multi_processor_count * int(waves_per_simd) * 256
        if out is None:
            out = torch.empty(n, dtype=torch.float32, device=dev)
        elif out.numel() < n or out.dtype != torch.float32 or not out.is_cuda:
            raise SopError(1, "out must be a CUDA float32 tensor of compute units * waves_per_simd * 256 elements")
        st = torch.cuda.current_stream(dev).cuda_stream if stream is None else stream
        nwg = C.c_int(0)
        _check(lib().sop_issue_probe(self._h, int(kind), int(waves_per_simd), int(iters), float(a), float(b),
                                     C.c_void_p(out.data_ptr()), C.byref(nwg), C.c_void_p(st)), self._h)
        if nwg.value != n:
            raise SopError(6, "the library counts another number of compute units than PyTorch")
        return out

    def pair_search_layers(self, layers, g, fmt: ScaleFmt, metric: int = SEL_WSE, shifts=None, want_sel: bool = False, stream=None):
        """sop_pair_search_layers: layers is a list of (W [M,K], c [K]) CUDA tensors of one dtype.  Returns
        (acos_pair [L,P] float64, acos_atom [L,A] float64, list of selector-word tensors or None);
        asynchronous on the current (or given) stream."""
        import torch
        if not layers:
            raise SopError(1, "no layers")
        dev = layers[0][0].device
        dtypes = {W.dtype for W, _ in layers}
        if dtypes not in ({torch.bfloat16}, {torch.float32}):
            raise SopError(1, "all layers must be bfloat16, or all float32")
        dt = BF16 if torch.bfloat16 in dtypes else F32
        n = len(layers)
        arr = (_Layer * n)()
        sels = [] if want_sel else None
        for i, (W, c) in enumerate(layers):
            if not (W.is_cuda and c.is_cuda) or W.dim() != 2 or W.stride(1) != 1 or c.dtype != torch.float32 or not c.is_contiguous():
                raise SopError(1, f"layer {i}: W must be a 2-D CUDA tensor with contiguous rows, c a contiguous float32 CUDA tensor")
            M, K = W.shape
            arr[i].W, arr[i].M, arr[i].K, arr[i].ldw, arr[i].c = W.data_ptr(), M, K, W.stride(0), c.data_ptr()
            arr[i].k = 0 if shifts is None else int(shifts[i])
            if want_sel:
                sw = torch.empty(M * K // g, dtype=torch.int16 if self.n_pairs <= 16 else torch.int32, device=dev)
                sels.append(sw)
                arr[i].sel_words = sw.data_ptr()
        tp = torch.empty((n, max(self.n_pairs, 1)), dtype=torch.float64, device=dev)
        ta = torch.empty((n, self.n_atoms), dtype=torch.float64, device=dev)
        st = torch.cuda.current_stream(dev).cuda_stream if stream is None else stream
        _check(lib().sop_pair_search_layers(self._h, arr, n, dt, g, fmt, metric,
                                            C.c_void_p(tp.data_ptr()) if self.n_pairs else None, C.c_void_p(ta.data_ptr()),
                                            C.c_void_p(st)), self._h)
        return tp[:, :self.n_pairs], ta, sels

    def search_layer(self, W, c, g, fmt: ScaleFmt, atoms, p_grid=(), k: int = 0, metric: int = SEL_WSE, fit_entries: int = 16,
                     fit_iters: int = 20, fit_bins: int = 1024, fit_init=None, weighted_fit: bool = True, fit_grid=None,
                     pack: bool = False, stream=None):
        """sop_search_layer on torch CUDA tensors.  Returns (result structure, words or None, payload or None); the
        workspace is a torch tensor kept by the context and grown on demand."""
        import torch
        dt = BF16 if W.dtype == torch.bfloat16 else (F32 if W.dtype == torch.float32 else None)
        if dt is None or not (W.is_cuda and c.is_cuda) or W.dim() != 2 or W.stride(1) != 1:
            raise SopError(1, "W must be a 2-D float32 or bfloat16 CUDA tensor with contiguous rows, c a CUDA tensor")
        M, K = W.shape
        tabs = [np.ascontiguousarray(t, dtype=np.float32) for t in atoms]
        arr = (_Atom * len(tabs))()
        for i, t in enumerate(tabs):
            arr[i].n_entries = t.size
            arr[i].values = _fp(t)
        o = _LayerOpts()
        o.n_p = len(p_grid)
        for i, p in enumerate(list(p_grid)[:LAYER_MAX_P]):
            o.p_percent[i] = float(p)
        o.fit_entries, o.fit_iters, o.fit_bins, o.weighted_fit, o.pack = fit_entries, fit_iters, fit_bins, int(bool(weighted_fit)), int(bool(pack))
        keep = []
        if fit_init is not None:
            ini = np.ascontiguousarray(fit_init, dtype=np.float32); keep.append(ini)
            o.fit_init = _fp(ini)
        if fit_grid is not None:
            gr = np.ascontiguousarray(fit_grid, dtype=np.float64); keep.append(gr)
            o.fit_grid = _fp(gr, C.c_double); o.n_fit_grid = gr.size
        need = C.c_size_t()
        _check(lib().sop_search_layer_workspace(self._h, M, K, g, len(tabs), C.byref(o), C.byref(need)), self._h)
        if self._ws is None or self._ws.numel() < need.value:
            self._ws = torch.empty(need.value, dtype=torch.uint8, device=W.device)
        words = payload = None
        if pack:
            n = 1
            while (1 << n) < max(max(t.size for t in tabs), fit_entries if len(p_grid) else 0):
                n += 1                                          # room for the widest codebook that can win
            words = torch.empty(M * K // g, dtype=torch.int16, device=W.device)
            payload = torch.empty((M * K // g, g * n // 8), dtype=torch.uint8, device=W.device)
        res = _LayerResult()
        st = torch.cuda.current_stream(W.device).cuda_stream if stream is None else stream
        _check(lib().sop_search_layer(self._h, C.c_void_p(W.data_ptr()), dt, M, K, W.stride(0), C.c_void_p(c.data_ptr()), g, fmt, k, metric,
                                      arr, len(tabs), C.byref(o), C.c_void_p(self._ws.data_ptr()), self._ws.numel(), C.byref(res),
                                      None if words is None else C.c_void_p(words.data_ptr()),
                                      None if payload is None else C.c_void_p(payload.data_ptr()), C.c_void_p(st)), self._h)
        self.n_atoms = 0
        if pack and payload.shape[1] != g * res.n_bits // 8:
            payload = payload.reshape(-1)[:M * K // g * (g * res.n_bits // 8)].reshape(M * K // g, g * res.n_bits // 8)
        return res, words, payload

    def prepare_scale(self, fmt: ScaleFmt, k: int = 0, stream=None):
        """sop_prepare_scale: write the scale table of (fmt, k) ahead of the searches that use it."""
        import torch
        st = torch.cuda.current_stream(self.device).cuda_stream if stream is None else stream
        _check(lib().sop_prepare_scale(self._h, fmt, k, C.c_void_p(st)), self._h)

    def set_scale_rule(self, rule: int):
        """SCALE_ABSMAX (default) or SCALE_ARGMAX for later pair_search calls."""
        _check(lib().sop_set_scale_rule(self._h, rule), self._h)

    def partition(self, score, n_top: int, higher_is_better: bool = True, stream=None):
        """sop_partition on a contiguous float32 CUDA tensor of per-block scores; returns device
        tensors (pool_b [N_b] uint8, tau [1] float32, n_a [1] int64)."""
        import torch
        if not score.is_cuda or score.dtype != torch.float32 or not score.is_contiguous():
            raise SopError(1, "score must be a contiguous float32 CUDA tensor")
        n = score.numel()
        pool_b = torch.empty(n, dtype=torch.uint8, device=score.device)
        tau = torch.empty(1, dtype=torch.float32, device=score.device)
        n_a = torch.empty(1, dtype=torch.int64, device=score.device)
        st = torch.cuda.current_stream(score.device).cuda_stream if stream is None else stream
        _check(lib().sop_partition(self._h, C.c_void_p(score.data_ptr()), n, n_top, 1 if higher_is_better else 0,
                                   C.c_void_p(pool_b.data_ptr()), C.c_void_p(tau.data_ptr()), C.c_void_p(n_a.data_ptr()),
                                   C.c_void_p(st)), self._h)
        return pool_b, tau, n_a

    def partition_levels(self, score, n_tops, higher_is_better: bool = True, stream=None):
        """sop_partition_levels on a contiguous float32 CUDA tensor of per-block scores; returns device tensors
        (level [N_b] uint8, tau [L] float32, n_a [L] int64)."""
        import torch
        if not score.is_cuda or score.dtype != torch.float32 or not score.is_contiguous():
            raise SopError(1, "score must be a contiguous float32 CUDA tensor")
        n, L = score.numel(), len(n_tops)
        level = torch.empty(n, dtype=torch.uint8, device=score.device)
        tau = torch.empty(L, dtype=torch.float32, device=score.device)
        n_a = torch.empty(L, dtype=torch.int64, device=score.device)
        tops = (C.c_int64 * L)(*[int(t) for t in n_tops])
        st = torch.cuda.current_stream(score.device).cuda_stream if stream is None else stream
        _check(lib().sop_partition_levels(self._h, C.c_void_p(score.data_ptr()), n, tops, L, 1 if higher_is_better else 0,
                                          C.c_void_p(level.data_ptr()), C.c_void_p(tau.data_ptr()), C.c_void_p(n_a.data_ptr()),
                                          C.c_void_p(st)), self._h)
        return level, tau, n_a

    def dd_histogram_levels(self, W, c, g, level, n_levels: int, n_bins: int = 1024, row_step: int = 1, stream=None):
        """sop_dd_histogram_levels on torch CUDA tensors; returns an [n_levels, n_bins] int64 device tensor."""
        import torch
        dt = BF16 if W.dtype == torch.bfloat16 else (F32 if W.dtype == torch.float32 else None)
        if dt is None or not W.is_cuda or W.dim() != 2 or W.stride(1) != 1:
            raise SopError(1, "W must be a 2-D float32 or bfloat16 CUDA tensor with contiguous rows")
        M, K = W.shape
        hist = torch.empty((n_levels, n_bins), dtype=torch.int64, device=W.device)
        st = torch.cuda.current_stream(W.device).cuda_stream if stream is None else stream
        _check(lib().sop_dd_histogram_levels(self._h, C.c_void_p(W.data_ptr()), dt, M, K, W.stride(0),
                                             None if c is None else C.c_void_p(c.data_ptr()), g, n_bins, row_step,
                                             C.c_void_p(level.data_ptr()), n_levels, C.c_void_p(hist.data_ptr()), C.c_void_p(st)), self._h)
        return hist

    def pack_blocks(self, out, M, K, g, fmt: ScaleFmt, a: int, b=None, pair_q: int = 0, stream=None):
        """sop_pack_blocks on the outputs of an emitting pair_search: atom a alone (b None) or the
        pair (a, b) with selector bit pair_q.  Returns (words [N_b] int16, payload [N_b, g*n/8] uint8, n)."""
        import torch
        if out.scale_code is None or out.code_planes is None:
            raise SopError(1, "pack_blocks needs the scale codes and code planes of an emitting search")
        two = b is not None
        if two and out.sel_words is None:
            raise SopError(1, "pack_blocks of a pair needs the selector words")
        ents = self.n_entries
        n = 1
        while (1 << n) < (max(ents[a], ents[b]) if two else ents[a]):
            n += 1
        Nb = M * K // g
        dev = out.scale_code.device
        words = torch.empty(Nb, dtype=torch.int16, device=dev)
        payload = torch.empty((Nb, g * n // 8), dtype=torch.uint8, device=dev)
        nb = C.c_int(0)
        st = torch.cuda.current_stream(dev).cuda_stream if stream is None else stream
        ptr = lambda t: C.c_void_p(t.data_ptr())
        _check(lib().sop_pack_blocks(self._h, M, K, g, fmt, ptr(out.scale_code[a]), ptr(out.code_planes[a]), ents[a],
                                     ptr(out.scale_code[b]) if two else None, ptr(out.code_planes[b]) if two else None, ents[b] if two else 0,
                                     ptr(out.sel_words) if two else None, out.sel_words.element_size() if two else 0, pair_q,
                                     ptr(words), ptr(payload), C.byref(nb), C.c_void_p(st)), self._h)
        assert nb.value == n
        return words, payload, n

    def scale_histogram(self, W, g, t_pos: float, t_neg: float, fmt: ScaleFmt, stream=None):
        """sop_scale_histogram on a torch CUDA tensor; returns a [2, 320] int64 device tensor."""
        import torch
        if not W.is_cuda:
            raise SopError(1, "W must be a CUDA tensor (no CPU fallback)")
        if W.dim() != 2 or W.stride(1) != 1:
            raise SopError(2, "W must be a 2-D tensor with contiguous rows")
        dt = BF16 if W.dtype == torch.bfloat16 else (F32 if W.dtype == torch.float32 else None)
        if dt is None:
            raise SopError(1, "W must be float32 or bfloat16")
        M, K = W.shape
        hist = torch.empty((2, 320), dtype=torch.int64, device=W.device)
        st = torch.cuda.current_stream(W.device).cuda_stream if stream is None else stream
        _check(lib().sop_scale_histogram(self._h, C.c_void_p(W.data_ptr()), dt, M, K, W.stride(0), g, t_pos, t_neg, fmt,
                                         C.c_void_p(hist.data_ptr()), C.c_void_p(st)), self._h)
        return hist

    def dd_histogram(self, W, c, g, n_bins: int = 1024, row_step: int = 1, block_mask=None, stream=None):
        """sop_dd_histogram on torch CUDA tensors; returns an [n_bins] int64 device tensor."""
        import torch
        if not W.is_cuda or (c is not None and not c.is_cuda):
            raise SopError(1, "W and c must be CUDA tensors (no CPU fallback)")
        if W.dim() != 2 or W.stride(1) != 1:
            raise SopError(2, "W must be a 2-D tensor with contiguous rows")
        dt = BF16 if W.dtype == torch.bfloat16 else (F32 if W.dtype == torch.float32 else None)
        if dt is None:
            raise SopError(1, "W must be float32 or bfloat16")
        M, K = W.shape
        hist = torch.empty(n_bins, dtype=torch.int64, device=W.device)
        st = torch.cuda.current_stream(W.device).cuda_stream if stream is None else stream
        _check(lib().sop_dd_histogram(self._h, C.c_void_p(W.data_ptr()), dt, M, K, W.stride(0),
                                      None if c is None else C.c_void_p(c.data_ptr()), g, n_bins, row_step, None if block_mask is None else C.c_void_p(block_mask.data_ptr()),
                                      C.c_void_p(hist.data_ptr()), C.c_void_p(st)), self._h)
        return hist

    def pair_search(self, W, c, g, fmt: ScaleFmt, k: int = 0, metric: int = SEL_WSE, out: Outputs = None,
                    emit: bool = False, stream=None, static: bool = False) -> Outputs:
        """sop_pair_search on torch CUDA tensors: W [M,K] float32 or bfloat16 (row stride = W.stride(0)),
        c [K] float32.  Asynchronous on the current (or given) stream.  static=True calls
        sop_pair_search_static (the caller then passes `out`, so that nothing is allocated)."""
        import torch
        if not (W.is_cuda and c.is_cuda):
            raise SopError(1, "W and c must be CUDA tensors (no CPU fallback)")
        if W.dim() != 2 or W.stride(1) != 1:
            raise SopError(2, "W must be a 2-D tensor with contiguous rows")
        if W.dtype == torch.bfloat16:
            dt = BF16
        elif W.dtype == torch.float32:
            dt = F32
        else:
            raise SopError(1, "W must be float32 or bfloat16")
        if c.dtype != torch.float32 or not c.is_contiguous():
            raise SopError(1, "c must be a contiguous float32 tensor")
        M, K = W.shape
        if out is None:
            out = self.alloc_outputs(M, K, g, emit=emit)
        st = torch.cuda.current_stream(W.device).cuda_stream if stream is None else stream

        def ptr(t):
            return None if t is None else C.c_void_p(t.data_ptr())

        o = _Outputs(ptr(out.acos_pair), ptr(out.acos_atom), ptr(out.sel_words), ptr(out.scale_code), ptr(out.codes),
                     ptr(out.blk_cos), ptr(out.blk_err), ptr(out.blk_rank))
        if static:
            _check(lib().sop_pair_search_static(self._h, C.c_void_p(W.data_ptr()), dt, M, K, W.stride(0), C.c_void_p(c.data_ptr()), g,
                                                fmt, k, metric, C.byref(o), C.c_void_p(st)), self._h)
            return out
        _check(lib().sop_pair_search(self._h, C.c_void_p(W.data_ptr()), dt, M, K, W.stride(0), C.c_void_p(c.data_ptr()), g,
                                     fmt, k, metric, None, 0, C.byref(o),
                                     C.c_void_p(st)), self._h)
        return out

    # ---- products of a linear layer with narrow operands (calls of a few microseconds: their Python side is kept short).  They take tensors' data and
    # know nothing of autograd: results require no gradients, the backward operators are called by who wants them.

    def _on(self, stream, call, *args, **kw):
        """The call with `stream` (a handle) as torch's current stream: what it allocates is then that stream's too."""
        import torch
        with torch.cuda.stream(torch.cuda.ExternalStream(stream, device=self.device)):
            return call(*args, **kw)

    def _here(self, *matrices):
        for q in matrices:
            if q.device != self.device:
                raise SopError(1, "operands must be on the context's GPU (no CPU fallback)")

    def _numbers(self, x, what, bf16_only=False):
        """(sop_dtype, row stride) of a matrix of numbers on the context's GPU."""
        if x.get_device() != self.device:
            raise SopError(1, f"{what} must be on the context's GPU (no CPU fallback)")
        dt = self._dtypes.get(x.dtype)
        if dt is None or (bf16_only and dt != BF16):
            raise SopError(1, f"{what} must be " + ("bfloat16" if bf16_only else "float32 or bfloat16"))
        if x.dim() != 2:
            raise SopError(2, f"{what} must be a 2-D tensor")
        R, Cc = x.shape
        ld, step = x.stride()
        if step != 1 and Cc > 1:
            raise SopError(2, f"{what} must have contiguous rows")
        return dt, (ld if R > 1 else -(-Cc // 8) * 8)                # (of one row the stride says nothing)

    def _result(self, out, M, N, dtype, usual, x):
        """(matrix to write to, its sop_dtype, row stride): `out` if it fits, else a new one beside x, of the type asked for or the usual one."""
        if out is None:
            dtype = dtype or usual
            dt = self._dtypes.get(dtype)
            if dt is None:
                raise SopError(1, "results are float32 or bfloat16")
            return x.new_empty((M, N), dtype=dtype), dt, N
        if tuple(out.shape) != (M, N):
            raise SopError(2, f"out must be {M} x {N}")
        if dtype is not None and out.dtype != dtype:
            raise SopError(1, f"out is {out.dtype}, the result asked for {dtype}")
        return (out, *self._numbers(out, "out"))

    def fp8_quantize(self, x, rows: int = 1, fmt=E4M3, transposed: bool = False, stream=None) -> Fp8Blocks:
        """sop_fp8_quantize: x [M, K] float32 or bfloat16 into 8 bits (fmt: E4M3 / E5M2, or the torch type) with one power-of-two scale for
        each block of rows x 128.  transposed (rows = 128 only): the codes as a [K, M] matrix too."""
        if stream is not None:
            return self._on(stream, self.fp8_quantize, x, rows, fmt, transposed)
        dt, ldx = self._numbers(x, "x")
        if transposed and rows != 128:
            raise SopError(1, "a transposed copy is made of 128 x 128 blocks only")
        M, K = x.shape
        q = Fp8Blocks.empty(M, K, fmt, x.device, rows, transposed)
        s = self._lib.sop_fp8_quantize(self._h, x.data_ptr(), dt, M, K, ldx, q._m, q._t.codes if transposed else None, q._t.ld_codes if transposed else 0,
                                       self._raw_stream(self.device))
        if s:
            _check(s, self._h)
        return q

    def fp8_matmul(self, x: Fp8Blocks, w: Fp8Blocks, transposed: bool = False, dtype=None, out=None, stream=None):
        """sop_fp8_matmul: y = x w^T of x [M, K] (rows = 1) and w [N, K] (rows = 128); transposed: y = x w of x [M, N] and the same w by its
        codes_t (the input gradient).  dtype: bfloat16 (default) or float32; or `out`, a matrix of either type to write to."""
        if stream is not None:
            return self._on(stream, self.fp8_matmul, x, w, transposed, dtype, out)
        self._here(x, w)
        if transposed and w._t is None:
            raise SopError(1, "the transposed product needs the weight's codes_t (fp8_quantize(..., transposed=True))")
        M, K = x.shape
        Kw, N = w.shape if transposed else w.shape[::-1]
        if K != Kw:
            raise SopError(2, f"x has rows of {K} elements, the weight wants {Kw}")
        out, dt, ldy = self._result(out, M, N, dtype, self._bf16, x.codes)
        s = self._lib.sop_fp8_matmul(self._h, x._m, w._t if transposed else w._m, transposed, M, N, K, out.data_ptr(), dt, ldy,
                                     self._raw_stream(self.device))
        if s:
            _check(s, self._h)
        return out

    def fp8_weight_grad(self, dy, x: Fp8Blocks, dtype=None, out=None, accumulate: bool = False, stream=None):
        """sop_fp8_weight_grad: dw [N, K] = dy^T x from dy [M, N] bfloat16 and the 8-bit checkpoint x [M, K] (rows = 1); dtype: float32 (default)
        or bfloat16; accumulate: added to `out`."""
        if stream is not None:
            return self._on(stream, self.fp8_weight_grad, dy, x, dtype, out, accumulate)
        self._here(x)
        _, lddy = self._numbers(dy, "dy", True)
        (M, N), K = dy.shape, x.shape[1]
        if x.shape[0] != M:
            raise SopError(2, f"dy has {M} rows, the checkpoint {x.shape[0]}")
        if accumulate and out is None:
            raise SopError(1, "accumulate needs out")
        out, dt, ldw = self._result(out, N, K, dtype, self._f32, dy)
        s = self._lib.sop_fp8_weight_grad(self._h, dy.data_ptr(), lddy, x._m, M, N, K, out.data_ptr(), dt, ldw, accumulate,
                                          self._raw_stream(self.device))
        if s:
            _check(s, self._h)
        return out

    def fp8_gated(self, gate, up, fmt=E4M3, stream=None):
        """sop_fp8_gated: (h, gate8, up8) of gate, up [M, F]: h = silu(gate) * up in 8 bits, and the 8-bit checkpoints of gate and up."""
        if stream is not None:
            return self._on(stream, self.fp8_gated, gate, up, fmt)
        dt, ldg = self._numbers(gate, "gate")
        du, ldu = self._numbers(up, "up")
        if gate.shape != up.shape or dt != du:
            raise SopError(2, "gate and up must have one shape and type")
        M, F = gate.shape
        dev = gate.device
        h, g8, u8 = Fp8Blocks.empty(M, F, fmt, dev), Fp8Blocks.empty(M, F, fmt, dev), Fp8Blocks.empty(M, F, fmt, dev)
        s = self._lib.sop_fp8_gated(self._h, gate.data_ptr(), ldg, up.data_ptr(), ldu, dt, M, F, h._m, g8._m, u8._m,
                                    self._raw_stream(self.device))
        if s:
            _check(s, self._h)
        return h, g8, u8

    def fp8_gated_grad(self, gate8: Fp8Blocks, up8: Fp8Blocks, dh, fmt=E5M2, stream=None):
        """sop_fp8_gated_grad: (dgate, dup, dgate8, dup8) from the checkpoints of fp8_gated and dh [M, F]: numbers of dh's type, and 8 bits."""
        if stream is not None:
            return self._on(stream, self.fp8_gated_grad, gate8, up8, dh, fmt)
        self._here(gate8, up8)
        dt, ldd = self._numbers(dh, "dh")
        M, F = dh.shape
        if gate8.shape != (M, F) or up8.shape != (M, F):
            raise SopError(2, "the checkpoints and dh must have one shape")
        dev = dh.device
        dgate, dup = dh.new_empty((M, F)), dh.new_empty((M, F))
        g8, u8 = Fp8Blocks.empty(M, F, fmt, dev), Fp8Blocks.empty(M, F, fmt, dev)
        s = self._lib.sop_fp8_gated_grad(self._h, gate8._m, up8._m, dh.data_ptr(), ldd, dt, M, F, dgate.data_ptr(), F, dup.data_ptr(), F, g8._m, u8._m,
                                         self._raw_stream(self.device))
        if s:
            _check(s, self._h)
        return dgate, dup, g8, u8

    def packed_matmul(self, x, w: PackedWeights, out=None, stream=None):
        """sop_packed_matmul: y [M, N] bfloat16 = x w^T of x [M, K] bfloat16 and a packed layer."""
        if stream is not None:
            return self._on(stream, self.packed_matmul, x, w, out)
        self._here(w)
        _, ldx = self._numbers(x, "x", True)
        (M, K), (N, Kw) = x.shape, w.shape
        if K != Kw:
            raise SopError(2, f"x has rows of {K} elements, the layer wants {Kw}")
        out, dt, ldy = self._result(out, M, N, self._bf16, self._bf16, x)
        s = self._lib.sop_packed_matmul(self._h, x.data_ptr(), ldx, w._w, M, out.data_ptr(), ldy, self._raw_stream(self.device))
        if s:
            _check(s, self._h)
        return out

    # ---- what stands around such a layer in a block of a model

    def _vector(self, v, n, what):
        """The address of n float32 on the context's GPU, one after the other; None of None."""
        if v is None:
            return None
        if v.get_device() != self.device:
            raise SopError(1, f"{what} must be on the context's GPU (no CPU fallback)")
        if v.dtype is not self._f32 or not v.is_contiguous():
            raise SopError(1, f"{what} must be contiguous float32")
        if v.numel() != n or v.dim() != 1:
            raise SopError(2, f"{what} must have {n} elements")
        return v.data_ptr()

    def _matrix(self, x, shape, dt, what):
        """(address, row stride) of a matrix of numbers of one shape and sop_dtype."""
        if shape[0] > 1 and x.shape == shape and x.is_contiguous() and self._dtypes.get(x.dtype) == dt and x.get_device() == self.device:
            return x.data_ptr(), shape[1]                                   # (the usual one, sooner)
        xt, ld = self._numbers(x, what)
        if x.shape != shape:
            raise SopError(2, f"{what} must be {shape[0]} x {shape[1]}")
        if xt != dt:
            raise SopError(1, f"{what} is {x.dtype}, which does not go with the other operands")
        return x.data_ptr(), ld

    def _epilogue(self, M, N, out, dt, ldy, bias, act, residual, scale, keep):
        """(sop_epilogue, z or None)"""
        r, ldr = (None, 0) if residual is None else self._matrix(residual, (M, N), dt, "residual")
        z = out.new_empty((M, N)) if keep else None
        return _Epilogue(self._vector(bias, N, "bias"), r, ldr, None if z is None else z.data_ptr(), N, act or 0, scale), z

    def fp8_linear(self, x: Fp8Blocks, w: Fp8Blocks, bias=None, act=None, residual=None, scale: float = 1.0, keep: bool = False, transposed: bool = False, dtype=None,
                   out=None, stream=None):
        """sop_fp8_linear: y = residual + scale act(z), z = x w^T + bias, of x [M, K] (rows = 1) and w [N, K] (rows = 128; transposed as in fp8_matmul).  bias [N]
        float32; act: None, RELU, SILU, GELU (the exact one) or GELU_TANH; residual [M, N] of y's type, which may be `out`; dtype / out as in fp8_matmul.  keep: returns
        (y, z), z of y's type, for fp8_linear_grad."""
        if stream is not None:
            return self._on(stream, self.fp8_linear, x, w, bias, act, residual, scale, keep, transposed, dtype, out)
        self._here(x, w)
        if transposed and w._t is None:
            raise SopError(1, "the transposed product needs the weight's codes_t (fp8_quantize(..., transposed=True))")
        M, K = x.shape
        Kw, N = w.shape if transposed else w.shape[::-1]
        if K != Kw:
            raise SopError(2, f"x has rows of {K} elements, the weight wants {Kw}")
        out, dt, ldy = self._result(out, M, N, dtype, self._bf16, x.codes)
        e, z = self._epilogue(M, N, out, dt, ldy, bias, act, residual, scale, keep)
        s = self._lib.sop_fp8_linear(self._h, x._m, w._t if transposed else w._m, transposed, M, N, K, e, out.data_ptr(), dt, ldy, self._raw_stream(self.device))
        if s:
            _check(s, self._h)
        return (out, z) if keep else out

    def packed_linear(self, x, w: PackedWeights, bias=None, act=None, residual=None, scale: float = 1.0, keep: bool = False, out=None, stream=None):
        """sop_packed_linear: fp8_linear with x [M, K] bfloat16 and a packed layer; y, residual and z are bfloat16."""
        if stream is not None:
            return self._on(stream, self.packed_linear, x, w, bias, act, residual, scale, keep, out)
        self._here(w)
        _, ldx = self._numbers(x, "x", True)
        (M, K), (N, Kw) = x.shape, w.shape
        if K != Kw:
            raise SopError(2, f"x has rows of {K} elements, the layer wants {Kw}")
        out, dt, ldy = self._result(out, M, N, self._bf16, self._bf16, x)
        e, z = self._epilogue(M, N, out, dt, ldy, bias, act, residual, scale, keep)
        s = self._lib.sop_packed_linear(self._h, x.data_ptr(), ldx, w._w, M, e, out.data_ptr(), ldy, self._raw_stream(self.device))
        if s:
            _check(s, self._h)
        return (out, z) if keep else out

    def _workspace(self, size, like, *sizes):
        """(address, bytes, what keeps it) of what a call named by its _workspace entry point needs."""
        n = C.c_size_t()
        st = size(self._h, *sizes, C.byref(n))
        if st:
            _check(st, self._h)
        n = n.value
        if n == 0:
            return None, 0, None
        ws = like.new_empty((n + 3) // 4, dtype=self._f32)
        return ws.data_ptr(), n, ws

    def fp8_linear_grad(self, dy, z=None, act=None, scale: float = 1.0, bias: bool = True, fmt=E5M2, stream=None):
        """sop_fp8_linear_grad: (dz, dz8, dbias) of the epilogue act / scale from dy [M, N] and the z that fp8_linear kept: numbers of dy's type (for fp8_weight_grad; dy
        itself where there is neither activation nor scale), 8 bits (for the input gradient), float32 sums over the rows (bias = False: None)."""
        if stream is not None:
            return self._on(stream, self.fp8_linear_grad, dy, z, act, scale, bias, fmt)
        dt, ldd = self._numbers(dy, "dy")
        M, N = dy.shape
        if act and z is None:
            raise SopError(1, "the gradient of an activation needs z")
        zp, ldz = self._matrix(z, (M, N), dt, "z") if act else (None, 0)
        dz = dy if not act and scale == 1.0 else dy.new_empty((M, N))
        dz8 = Fp8Blocks.empty(M, N, fmt, dy.device)
        db, at, size = None, None, 0
        if bias:
            db = dy.new_empty(N, dtype=self._f32)
            at, size, ws = self._workspace(self._lib.sop_fp8_linear_grad_workspace, dy, M, N)
        s = self._lib.sop_fp8_linear_grad(self._h, dy.data_ptr(), ldd, zp, ldz, dt, M, N, act or 0, scale, None if dz is dy else dz.data_ptr(), N, dz8._m,
                                          None if db is None else db.data_ptr(), at, size, self._raw_stream(self.device))
        if s:
            _check(s, self._h)
        return dz, dz8, db

    def _norm_opts(self, M, D, after, gate, scale, before, eps):
        o = _NormOpts(self._vector(after, D, "after"), self._vector(before, D, "before"), None, 0, F32, 0, scale, eps)
        if gate is not None:
            g = gate.view(1, D) if gate.dim() == 1 and gate.shape[0] == D else gate
            o.gate_dtype, o.ld_gate = self._numbers(g, "gate")
            if g.shape[1] != D or g.shape[0] < 1 or M % g.shape[0]:
                raise SopError(2, f"gate must have rows of {D} elements, and a number of them that divides {M}")
            o.gate, o.groups = g.data_ptr(), g.shape[0]
        return o

    def residual_norm(self, r, y=None, after=None, gate=None, scale: float = 1.0, before=None, eps: float = 1e-6, dtype=None, fmt=None, out=None, stream=None):
        """sop_residual_norm: (s, n, n8) of the residual stream r [M, D] and a block's output y [M, D]: s = r + scale gate y after / rms(y), of r's type (r itself without
        y), and s before / rms(s) as numbers of `dtype` (n) and in 8 bits of `fmt` (n8), each None where it is not asked for.  after, before: [D] float32, or None: no
        such norm.  gate: [D], or [G, D] with G a divisor of M: each row for M / G rows.  out: where s goes; it may be r."""
        if stream is not None:
            return self._on(stream, self.residual_norm, r, y, after, gate, scale, before, eps, dtype, fmt, out)
        dr, ldr = self._numbers(r, "r")
        M, D = r.shape
        o = self._norm_opts(M, D, after, gate, scale, before, eps)
        yp, ldy, dty, sp, lds, s = None, 0, dr, None, 0, r
        if y is not None:
            dty, ldy = self._numbers(y, "y")
            if y.shape != r.shape:
                raise SopError(2, "r and y must have one shape")
            s, _, lds = self._result(out, M, D, r.dtype, r.dtype, r)
            yp, sp = y.data_ptr(), s.data_ptr()
        elif out is not None:
            raise SopError(1, "without y there is no sum to write")
        n, dn = None, F32
        if dtype is not None:
            n, dn, _ = self._result(None, M, D, dtype, None, r)
        n8 = None if fmt is None else Fp8Blocks.empty(M, D, fmt, r.device)
        st = self._lib.sop_residual_norm(self._h, o, M, D, yp, ldy, dty, r.data_ptr(), ldr, dr, sp, lds, None if n is None else n.data_ptr(), D, dn,
                                         None if n8 is None else n8._m, self._raw_stream(self.device))
        if st:
            _check(st, self._h)
        return s, n, n8

    def residual_norm_grad(self, ds, dn=None, s=None, before=None, y=None, after=None, gate=None, scale: float = 1.0, eps: float = 1e-6, fmt=None, stream=None):
        """sop_residual_norm_grad: ResidualNormGrads(dr, dy, dy8, dbefore, dafter, dgate) of residual_norm with these operands, from the gradient ds that s gets elsewhere
        (None: none) and dn.  s: the sum that was returned (with `before`).  Types: s, ds and dr alike, y, dn and dy alike (without y, dn of either type); dy8 is dy in
        8 bits of `fmt` (None: not made); dbefore and dafter are float32, dgate of gate's type and shape."""
        if stream is not None:
            return self._on(stream, self.residual_norm_grad, ds, dn, s, before, y, after, gate, scale, eps, fmt)
        if (before is None) != (dn is None) or (before is None) != (s is None):
            raise SopError(1, "before, dn and s are given together")
        like = ds if ds is not None else s
        if like is None:
            raise SopError(1, "no gradient to go from: neither ds nor dn")
        dt, _ = self._numbers(like, "ds" if ds is not None else "s")
        shape = M, D = like.shape
        o = self._norm_opts(M, D, after, gate, scale, before, eps)
        of_y = y if y is not None else dn
        dty = dt if of_y is None else self._numbers(of_y, "y or dn")[0]
        dsp = sp = dnp = yp = dyp = None
        lds = ls = ldn = ldy = 0
        if ds is not None:
            dsp, lds = self._matrix(ds, shape, dt, "ds")
        if before is not None:
            sp, ls = self._matrix(s, shape, dt, "s")
            dnp, ldn = self._matrix(dn, shape, dty, "dn")
        dr, dy, dy8, m8 = like.new_empty(shape), None, None, None
        if y is not None:
            yp, ldy = self._matrix(y, shape, dty, "y")
            dy = y.new_empty(shape)
            dyp = dy.data_ptr()
            if fmt is not None:
                dy8 = Fp8Blocks.empty(M, D, fmt, like.device)
                m8 = C.pointer(dy8._m)
        elif fmt is not None:
            raise SopError(1, "without y there is no dy8")
        db = None if before is None else before.new_empty(D)
        da = None if after is None else after.new_empty(D)
        dg = None if gate is None else gate.new_empty(gate.shape)
        t = _NormGrads(dsp, lds, dnp, ldn, sp, ls, yp, ldy, dr.data_ptr(), D, dyp, D, m8, None if db is None else db.data_ptr(),
                       None if da is None else da.data_ptr(), None if dg is None else dg.data_ptr(), D, dt, dty)
        at, size, ws = self._workspace(self._lib.sop_residual_norm_grad_workspace, like, M, D, o.groups)
        st = self._lib.sop_residual_norm_grad(self._h, o, M, D, t, at, size, self._raw_stream(self.device))
        if st:
            _check(st, self._h)
        return ResidualNormGrads(dr, dy, dy8, db, da, dg)

    def _grads(self, tensors, outs):
        """The tensors as sop_grad, packed, and how many."""
        import torch
        parts, dev, dts = [], self.device, self._dtypes
        if outs is not None and len(outs) != len(tensors):
            raise SopError(2, "as many outs as tensors")
        for i, x in enumerate(tensors):
            o = x if outs is None else outs[i]
            if x is None and o is None:
                continue                                                    # (a weight without a gradient)
            if not isinstance(x, torch.Tensor) or not isinstance(o, torch.Tensor):
                raise SopError(1, "gradients are tensors")
            dx, do = dts.get(x.dtype), dts.get(o.dtype)
            if dx is None or do is None:
                raise SopError(1, "gradients are float32 or bfloat16")
            if x.get_device() != dev or o.get_device() != dev:
                raise SopError(1, "gradients must be on the context's GPU (no CPU fallback)")
            if x.shape != o.shape:
                raise SopError(2, "a gradient and its out have one shape")
            if not x.is_contiguous() or (o is not x and not o.is_contiguous()):
                if not _dense(x) or (o is not x and o.stride() != x.stride()):
                    raise SopError(2, "a gradient's elements lie one after the other, and its out's in the same order")
            parts.append(_GRAD.pack(x.data_ptr(), o.data_ptr(), x.numel(), dx, do))
        return b"".join(parts), len(parts)

    def grad_norm(self, tensors, stream=None):
        """sop_grad_norm: the norm of all elements of all tensors (float32 or bfloat16; None is passed over), a [1] float32 tensor."""
        if stream is not None:
            return self._on(stream, self.grad_norm, tensors)
        return self._norm_of(tensors, None, None)

    def clip_grads(self, tensors, most: float, out=None, stream=None):
        """sop_clip_grads: the tensors times min(1, most / their norm), in place or into `out` (a tensor for each, float32 or bfloat16, none of them memory of
        another gradient); returns the norm, a [1] float32 tensor."""
        if stream is not None:
            return self._on(stream, self.clip_grads, tensors, most, out)
        return self._norm_of(tensors, float(most), out)

    def _norm_of(self, tensors, most, out):
        import torch
        tensors = list(tensors)
        packed, n = self._grads(tensors, out)
        norm = torch.empty(1, dtype=torch.float32, device=torch.device("cuda", self.device))
        at, size, ws = self._workspace(self._lib.sop_clip_grads_workspace, norm, n)
        st = self._raw_stream(self.device)
        s = (self._lib.sop_grad_norm(self._h, packed, n, norm.data_ptr(), at, size, st) if most is None
             else self._lib.sop_clip_grads(self._h, packed, n, most, norm.data_ptr(), at, size, st))
        if s:
            _check(s, self._h)
        return norm
