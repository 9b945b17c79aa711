"""Where the wide packed kernel's loads begin at each step, evaluated on the host: the part of an address that all lanes share stays inside the
window, also where the last tile has a single row, so that what is left of the window, with which a lane's offset is compared, is never negative."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SRC = r"""
#include <cstdio>
#include "sop_linear.h"
int main()
{
    for (int nb = 1; nb <= 6; ++nb)
        for (int lg = 3; lg <= 6; ++lg)
            for (int K = 64; K <= 1200; K += 1 << lg)
                for (int t = 0; t < (K + 63) / 64 + 2; ++t) {
                    const int steps = (K + 63) / 64;
                    const PackedStepAt at = packed_step_at(t, steps, nb, lg, lg == 3 && K % 16 != 0);
                    std::printf("%d %d %d %d %d %d %d\n", nb, lg, K, t, at.x, at.codes, at.words);
                }
}
"""


@pytest.fixture(scope="module")
def places(tmp_path_factory):
    d = tmp_path_factory.mktemp("steps")
    src, exe = d / "s.cpp", d / "s"
    src.write_text(SRC)
    subprocess.check_call(["g++", "-std=c++17", "-I", os.path.join(ROOT, "paper_2605_14929_amd", "csrc"), "-o", str(exe), str(src)])
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout
    return [tuple(int(v) for v in line.split()) for line in out.splitlines()]


def test_no_step_begins_beyond_a_window_of_one_row(places):
    for nb, lg, K, t, x, codes, words in places:
        odd_part = nb // 2 * 4 if nb % 2 else 0                            # codes of an odd width come in two loads, the second this much further on
        assert 0 <= x < 2 * K
        assert 0 <= codes and codes + odd_part < K // 8 * nb
        assert 0 <= words < 2 * K >> lg


def test_steps_follow_each_other(places):
    for nb, lg, K, t, x, codes, words in places:
        if t < K // 64:                                                    # whole steps lie 64 elements apart
            early = nb if lg == 3 and K % 16 and t == (K + 63) // 64 - 1 else 0
            assert (x, codes + early, words) == (128 * t, 8 * nb * t, 2 * (64 * t >> lg))
        elif t >= (K + 63) // 64:                                          # behind the last one: the last one
            last = next(p for p in places if p[:3] == (nb, lg, K) and p[3] == (K + 63) // 64 - 1)
            assert (x, codes, words) == last[4:]
