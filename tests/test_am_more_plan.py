"""Plans of the gated layer's products: host arithmetic, compiled alone (no GPU needed)."""
from test_am_plan import run


def test_tiles_of_a_gated_layer(tmp_path):
    # few rows, one tile a CU of 128 x 128, of 128 x 256, several rounds of 256 x 256; only where it is asked for, and
    # only for operands that are fetched straight to LDS
    line = 'printf("%%d %%d %%d ", am_plan(%d, %d, %d, false, true, true).tile, am_plan(%d, %d, %d, false, true).tile, am_plan(%d, %d, %d, false, false, true).tile);\n'
    sizes = {(400, 8192, 1024): 128, (777, 8192, 1024): 192, (1470, 4080, 328): 192, (1921, 3826, 72): 192,
             (1500, 4096, 2048): 192, (777, 4096, 2048): 128, (16384, 8192, 1024): 256}
    got = run(tmp_path, "".join(line % (3 * s) for s in sizes))
    for (s, tile), with_wide, without, staged in zip(sizes.items(), got[::3], got[1::3], got[2::3]):
        assert int(with_wide) == tile, s
        assert int(without) in (64, 128, 256) and int(staged) in (64, 128), s
        if tile == 192:   # at most one a CU
            assert -(-s[0] // 128) * -(-s[1] // 256) <= 256


def test_weights_whose_values_lie_far_behind_are_not_fetched_straight(tmp_path):
    line = "{ const AmOperand a{(const char *)0, 256, 64}, b{(const char *)0, %dll, %d}; printf(\"%%d \", (int)am_gated_direct(a, b, 128, 2)); }\n"
    cases = [((256, 1000), 1), ((1 << 20, 1023), 1), ((1 << 20, 1024), 0), ((1 << 22, 2), 0), ((258, 1000), 0)]
    got = run(tmp_path, "".join(line % c for c, _ in cases))
    assert [int(v) for v in got] == [w for _, w in cases]
