"""The rules that share out rows, tensors and columns around a linear layer, evaluated on the host, and the registers of the kernels that they choose."""
import os
import shutil
import subprocess

import pytest

import test_gpu_block as G
import test_linear_resources as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SRC = r"""
#include <cstdio>
#include <cstring>
#include "sop_block_rules.h"
int main()
{
    char op[16];
    long long a, b, c;
    while (std::scanf("%15s %lld %lld %lld", op, &a, &b, &c) == 4) {
        if (!std::strcmp(op, "norm")) { const auto s = sopr::norm_shape(a); std::printf("%d %d\n", s.T, s.C); }
        if (!std::strcmp(op, "grad")) { const auto s = sopr::norm_grad_shape(a); std::printf("%d %d\n", s.T, s.C); }
        if (!std::strcmp(op, "most")) std::printf("%lld 0\n", sopr::norm_grad_most(a, 256));
        if (!std::strcmp(op, "share")) { const auto s = sopr::norm_share(a, b, c); std::printf("%lld %d\n", s.words, s.parts); }
        if (!std::strcmp(op, "act")) std::printf("%lld %d\n", sopr::act_grad_words(a, b, 256), (int)sopr::act_grad_few(a));
        if (!std::strcmp(op, "clip")) std::printf("%lld %lld\n", sopr::clip_launches(a, 96), sopr::clip_words(b, c, 256));
    }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    src, exe = d / "r.cpp", d / "r"
    src.write_text(SRC)
    subprocess.check_call(["g++", "-std=c++17", "-Wall", "-I", os.path.join(ROOT, "paper_2605_14929_amd", "csrc"), "-o", str(exe), str(src)])

    def f(op, *calls):
        text = "".join("%s %d %d %d\n" % ((op,) + tuple(c) + (0,) * (3 - len(c))) for c in calls)
        return [tuple(map(int, line.split())) for line in subprocess.run([str(exe)], input=text, capture_output=True, text=True, check=True).stdout.splitlines()]
    return f


def test_a_row_fits_the_threads_that_share_it(ask):
    widths = list(range(1, 20000, 7)) + [512, 513, 1024, 1025, 2048, 2049, 4096, 8192, 8193, 16384, 16385, 1 << 20]
    for op, end in (("norm", 16384), ("grad", 16384)):
        for D, (T, C) in zip(widths, ask(op, *[(D,) for D in widths])):
            if D > end:
                assert (T, C) == (0, 0)
                continue
            assert T % 64 == 0 and 64 <= T <= 1024 and T * C * 8 >= D
            assert (T == 64) == (D <= (1024 if op == "norm" else 512))     # a wavefront, four of them a workgroup


def test_every_shape_of_a_row_is_compared_at_some_width(ask):
    for op in ("norm", "grad"):
        got = ask(op, *[(D,) for D in G.WIDTHS])
        assert {(T == 64, T == 0, C) for T, C in got} == {(True, False, 1), (False, False, 1), (False, False, 2), (False, True, 0)} | ({(True, False, 2)} if op == "norm" else set())
        assert len({T for T, _ in got}) >= 8


def test_groups_are_shared_out(ask):
    calls = [(G_, each, most) for G_ in (1, 2, 3, 100, 255, 256, 257, 1000, 70000) for each in (1, 2, 259, 10000) for most in (1, 124, 256, 1024)]
    for (G_, each, most), (words, parts) in zip(calls, ask("share", *calls)):
        if parts == 1:
            assert words == min(G_, most)
        else:
            assert words == G_ * parts <= most and 1 < parts <= each
        assert words >= min(most, G_ * each) // 2                       # (no more than half of them idle)


def test_partial_sums_stay_small(ask):
    for D, (most, _) in zip((1, 512, 4096, 8192, 16384, 16385, 1 << 20), ask("most", *[(D,) for D in (1, 512, 4096, 8192, 16384, 16385, 1 << 20)])):
        assert 1 <= most <= 1024 and most * D * 4 <= 17 << 20


def test_columns_and_lists(ask):
    for (M, N), (words, few) in zip([(1, 1), (128, 100), (129, 512), (8192, 11008), (10, 1 << 23)], ask("act", (1, 1), (128, 100), (129, 512), (8192, 11008), (10, 1 << 23))):
        assert 1 <= words <= max(1, (M + 3) // 4) and words * -(-N // 512) <= max(2048, -(-N // 512)) and few == (M <= 128)
    for (count, chunks, launches), got in zip([(0, 1, 1), (96, 5, 1), (97, 10000, 2), (5000, 1 << 20, 53)], ask("clip", (0, 1, 1), (96, 5, 1), (97, 10000, 2), (5000, 1 << 20, 53))):
        assert got[0] == -(-count // 96) and 1 <= got[1] <= chunks and got[1] <= max(64, 2048 // launches)


UNITS = ("norm", "act", "clip", "f8mm_epilogue", "packed_epilogue")


@pytest.mark.skipif(not all(os.path.exists(R._object(u)) for u in UNITS) or not shutil.which(f"{R.LLVM}/clang-offload-bundler"), reason="no objects of a build, or no tools to read them")
@pytest.mark.parametrize("unit", UNITS)
def test_registers(unit, tmp_path):
    """No spills to memory, but for the gradients of a norm that 1024 threads share, who have 128 registers each: a few values at the ends of groups.  (Scalar
    registers are kept in lanes of vector registers there: the kernels' many addresses.)"""
    fat, code = str(tmp_path / "fat"), str(tmp_path / "code")
    subprocess.check_call([f"{R.LLVM}/llvm-objcopy", f"--dump-section=.hip_fatbin={fat}", R._object(unit), str(tmp_path / "copy")], stderr=subprocess.DEVNULL)
    subprocess.check_call([f"{R.LLVM}/clang-offload-bundler", "--unbundle", "--type=o", "--targets=hipv4-amdgcn-amd-amdhsa--gfx950", f"--input={fat}", f"--output={code}"])
    notes = subprocess.run([f"{R.LLVM}/llvm-readobj", "--notes", code], capture_output=True, text=True, check=True).stdout
    seen = 0
    for part in R.re.split(r"\n\s+- \.a", notes)[1:]:
        f = dict(R.re.findall(r"\.?(\w+):\s+(\S+)", part))
        if "symbol" not in f:
            continue
        seen += 1
        name, spilled = f["symbol"], int(f["vgpr_spill_count"])
        most = 48 if "norm_grad_wide" in name else 8 if "norm_grad_kernel" in name else 0
        assert spilled <= most, (name, spilled)
        assert "norm" in name or int(f["sgpr_spill_count"]) == 0, name
        assert int(f["group_segment_fixed_size"]) <= 64 * 1024, name
    assert seen >= 3


@pytest.mark.skipif(not all(os.path.exists(R._object(u)) for u in UNITS + R.UNITS) or not shutil.which(f"{R.LLVM}/clang-offload-bundler"), reason="no objects of a build, or no tools to read them")
@pytest.mark.parametrize("unit", UNITS + R.UNITS)
def test_wide_buffer_stores_have_no_scalar_offset(unit, tmp_path):
    """Beside a scalar offset the compiler lets the instruction after a store of 12 or 16 bytes write the registers that the store still has to read."""
    fat, code = str(tmp_path / "fat"), str(tmp_path / "code")
    subprocess.check_call([f"{R.LLVM}/llvm-objcopy", f"--dump-section=.hip_fatbin={fat}", R._object(unit), str(tmp_path / "copy")], stderr=subprocess.DEVNULL)
    subprocess.check_call([f"{R.LLVM}/clang-offload-bundler", "--unbundle", "--type=o", "--targets=hipv4-amdgcn-amd-amdhsa--gfx950", f"--input={fat}", f"--output={code}"])
    text = subprocess.run([f"{R.LLVM}/llvm-objdump", "-d", code], capture_output=True, text=True, check=True).stdout
    assert "s_endpgm" in text
    stores = [line for line in text.splitlines() if "buffer_store_dwordx4" in line or "buffer_store_dwordx3" in line]
    assert not [line for line in stores if not R.re.search(r"s\[\d+:\d+\], 0 offen", line)]
