"""The rules that choose a kernel for a product with narrow operands, evaluated on the host."""
import os
import subprocess

import pytest

import test_gpu_linear as G

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SRC = r"""
#include <cstdio>
#include <cstring>
#include "sop_linear_rules.h"
int main()
{
    char op[8];
    long long a, b, c, d;
    while (std::scanf("%7s %lld %lld %lld %lld", op, &a, &b, &c, &d) == 5)
        std::printf("%d\n", !std::strcmp(op, "f8mm") ? sopr::f8mm_choice(a, b, d != 0, 256)
                            : !std::strcmp(op, "wgrad") ? sopr::wgrad_choice(a, b, c, d != 0, 256) : sopr::packed_choice(a, b, c, (int)d, 256));
}
"""

F8MM = ["32x32", "32x64", "64x64", "64x128", "128x128", "256x256", "rows"]
WGRAD = ["32x64", "64x64", "128x128", "256x256", "any 64x128", "any 128x128", "any 256x256"]
PACKED = ["32x32", "64x32", "64x64", "128x32", "128x128", "256x192", "256x256", "rows"]
THREADS = {"f8mm": {"64x128": 256, "128x128": 256}, "packed": {"128x128": 256, "256x192": 256, "256x256": 256}}


@pytest.fixture(scope="module")
def choose(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    src, exe = d / "r.cpp", d / "r"
    src.write_text(SRC)
    subprocess.check_call(["g++", "-std=c++17", "-I", os.path.join(ROOT, "paper_2605_14929_amd", "csrc"), "-o", str(exe), str(src)])

    def f(calls):
        text = "".join("%s %d %d %d %d\n" % q for q in calls)
        out = subprocess.run([str(exe)], input=text, capture_output=True, text=True, check=True).stdout.split()
        assert len(out) == len(calls)
        return [None if int(v) < 0 else {"f8mm": F8MM, "wgrad": WGRAD, "packed": PACKED}[q[0]][int(v)] for q, v in zip(calls, out)]
    return f


def test_what_is_chosen_can_be_launched(choose):
    """Fewer than 2^32 threads, for every y that a GPU's 288 GB hold; packed products of fewer than 64 elements from 2^35 numbers on (2^29 rows or columns,
    of tiles of 64) have no such launch, and half of them has."""
    sizes = [1, 3, 16, 17, 100, 4096] + [1 << i for i in range(14, 31)] + [(1 << 27) - 16, (1 << 28) + 1, (1 << 29) - 64]
    for op, ds, itemsize in (("f8mm", (0, 1), (2, 4)), ("packed", (1, 4, 6), (2, 2, 2))):
        for d, z in zip(ds, itemsize):
            for K in (8, 63, 64, 4096):
                calls = [(op, M, N, K, d) for M in sizes for N in sizes if M * N * z <= 288 << 30]
                for (_, M, N, _, _), name in zip(calls, choose(calls)):
                    if name is None:
                        assert op == "packed" and K < 64 and max(M, 64) * max(N, 64) >= 1 << 34
                        continue
                    bm, bn = (16, 16) if name == "rows" else map(int, name.split("x"))
                    assert -(-M // bm) * -(-N // bn) * THREADS[op].get(name, 512) < 1 << 32, (op, M, N, K, name)
                    assert not (name == "256x256" and op == "f8mm" and d == 1)


def test_every_kernel_is_compared_at_some_size(choose):
    """Those of test_gpu_linear.py: the 8-bit product's by result type, the others' by width or alignment."""
    for d in (0, 1):
        got = choose([("f8mm", M, N, K, d) for M, N, K in G.F8_KERNELS])
        assert set(got) == set(F8MM) - ({"256x256"} if d else set()), got
    rows_off = choose([("wgrad", *dims, 0) for dims in G.GRADS])
    assert set(rows_off) == {"any 64x128", "any 128x128", "any 256x256"}
    spaced = [mark.args[1] for mark in G.test_weight_gradient_of_spaced_rows.pytestmark if mark.name == "parametrize" and mark.args[0] == "M, N, K"][0]
    assert set(choose([("wgrad", *dims, 1) for dims in spaced])) == {"32x64", "64x64", "128x128", "256x256"}
    calls = [("packed", case[0], case[1], case[2], case[4]) for case in G.PACKED]
    for f in (G.test_packed_product_of_some_rows, G.test_packed_product_of_a_hundred_rows, G.test_packed_product_of_wide_outputs):
        marks = {mark.args[0]: mark.args[1] for mark in f.pytestmark if mark.name == "parametrize"}
        calls += [("packed", M, N, K, n) for M, N, K, _ in marks["M, N, K, g"] for n in marks["n"]]
    got = list(zip(calls, choose(calls)))
    for n in range(1, 7):
        assert {name for (_, _, _, _, m), name in got if m == n} >= set(PACKED) - {"rows"} - ({"256x192", "256x256"} if n == 6 else set()), n
    assert "rows" in {name for _, name in got}


def test_one_row_left_reaches_every_wide_kernel(choose):
    marks = {mark.args[0]: mark.args[1] for mark in G.test_packed_product_with_one_row_left.pytestmark if mark.name == "parametrize"}
    calls = [("packed", M, N, K, n) for M, N in marks["M, N"] for K, _ in marks["K, g"] for n in marks["n"]]
    ends = set()
    for (_, M, N, _, _), name in zip(calls, choose(calls)):
        bm, bn = map(int, name.split("x"))
        if M % bm == 1:
            ends.add((name, "row"))
        if N % bn == 1:
            ends.add((name, "column"))
    assert ends == {(k, e) for k in ("128x128", "256x192", "256x256") for e in ("row", "column")}
