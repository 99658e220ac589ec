"""The kernels that sizes of gated layers go to: host arithmetic, compiled alone (no GPU needed)."""
from am_gated_tiles import SIZES
from test_am_plan import run

# the rules of am_launch_gated and am_gated_product, on operands that begin at 0
PROGRAM = r"""
    const auto kernel = [](int64_t m, int64_t k, int64_t n, int el) {
        const AmOperand a{nullptr, k * el, static_cast<int32_t>(m)}, b{nullptr, k * el, static_cast<int32_t>(n)};
        if (m <= 32 || am_tiles(m, 2 * n, 64, 64) <= kComputeUnits / 2) return "no tiles";
        const bool direct = am_gated_direct(a, b, static_cast<int32_t>(k), el);
        const int tile = am_plan(m, 2 * n, k, false, direct, true).tile;
        if (!direct) return tile >= 128 ? "128, staged" : "64, staged";
        if (tile == 256) return "256";
        if (tile == kAmWide) return "128 x 256";
        if (tile == 128) return am_tiles(m, 2 * n, 128, 128) <= kComputeUnits ? "128, one a CU" : "128";
        return "64";
    };
"""


def test_sizes_go_to_the_kernels_that_they_stand_for(tmp_path):
    line = 'printf("%%s/%%s;", kernel(%d, %d, %d, 2), kernel(%d, %d, %d, 1));\n'
    got = " ".join(run(tmp_path, PROGRAM + "".join(line % (s + s) for s in SIZES))).split(";")[:-1]
    assert {s: tuple(g.split("/")) for s, g in zip(SIZES, got)} == SIZES
    kernels = {"256", "128 x 256", "128, one a CU", "128", "64", "128, staged", "64, staged"}
    for i in (0, 1):
        assert {k[i] for k in SIZES.values()} == kernels
