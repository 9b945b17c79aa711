"""That the shapes of test_gpu_block_paths take the ways through the kernels that they are there for, evaluated on the host."""
import test_gpu_block_paths as P
from test_block_rules_host import ask  # noqa: F401
from test_linear_rules_host import choose  # noqa: F401


def test_products_take_the_kernels_that_are_named(choose):  # noqa: F811
    for d, by in ((0, 3), (1, 4)):
        assert choose([("f8mm", *c[:3], d) for c in P.F8_TILES]) == [c[by] for c in P.F8_TILES]
    assert choose([("packed", M, N, K, n) for M, N, K, g, n, _ in P.PACKED_TILES]) == [c[5] for c in P.PACKED_TILES]
    assert all(c[1] % 4 == 0 for c in P.F8_TILES + P.PACKED_TILES)
    assert {c[3] for c in P.F8_TILES} | {c[4] for c in P.F8_TILES} >= {"64x128", "128x128", "256x256"} and {c[5] for c in P.PACKED_TILES} == {"128x128", "256x192", "256x256"}
    assert {r * 4 + z * 2 + i for r, z, i in P.FORMS} == {0, 4, 5, 2, 6}


def test_long_rows_share_workgroups(ask):  # noqa: F811
    for D in (16392, 20001):
        assert ask("norm", (D,)) == ask("grad", (D,)) == [(0, 0)]
        most = ask("most", (D,))[0][0]
        for G, each in ((1, 1100), (3, 367)):
            words, parts = ask("share", (G, each, most))[0]
            assert parts > 1 and each // parts > 4                     # a second row for each of four wavefronts
        for G in (550, 1100):
            words, parts = ask("share", (G, 1100 // G, most))[0]
            assert parts == 1 and G // words > 1                       # a second group
