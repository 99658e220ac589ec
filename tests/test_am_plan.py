"""Launches of the acoustic model's products: host arithmetic, compiled alone (no GPU needed)."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1808_00687_amd", "csrc")


def run(tmp_path, body):
    src = tmp_path / "plan.cpp"
    src.write_text('#include <cstdio>\n#include <cstdlib>\n#include "am_plan.h"\nusing namespace wfd;\nint main() {\n%s\nreturn 0;\n}\n' % body)
    exe = str(tmp_path / "plan")
    subprocess.check_call(["g++", "-std=c++20", "-Wall", "-I", CSRC, str(src), "-o", exe])
    return subprocess.check_output([exe], text=True).split()


def test_launches_fit(tmp_path):
    # every block once, in order; fewer than 2^32 threads a launch; runs on the chiplets' turn
    blocks = [1, 2, 255, 4096, (1 << 22) - 1, 1 << 22, (1 << 22) + 1, (1 << 23) + 5, 1 << 24, (1 << 26) + 3, (1 << 31) - 1]
    # the most that the accepted sizes give: 2^30 columns beside 32 rows, and 2^40 results
    for m, n, tile_m, tile_n in ((32, 1 << 30, 16, 16), (1, 1 << 30, 64, 64), (1 << 30, 1, 64, 64), (1 << 30, 1 << 10, 64, 64),
                                 (1 << 20, 1 << 20, 64, 64), (1 << 30, 1 << 10, 128, 128), (1 << 30, 1 << 10, 256, 256)):
        blocks.append(-(-m // tile_m) * -(-n // tile_n))
    one = 'am_in_launches(%dll, [](uint32_t first, uint32_t count) { printf("%%u %%u ", first, count); }); printf("/ ");\n'
    got = " ".join(run(tmp_path, "".join(one % b for b in blocks))).split("/")
    for b, line in zip(blocks, got):
        at, runs = 0, [int(v) for v in line.split()]
        for first, count in zip(runs[::2], runs[1::2]):
            assert first == at and first % 8 == 0 and 0 < count and count * 512 < 1 << 32, b
            at += count
        assert at == b and b < 1 << 32
        assert b > 1 << 22 or len(runs) == 2


def test_the_plan_goes_by_where_operands_lie(tmp_path):
    # A plan for operands on 16 bytes is for those alone: not for a stride, or a first element, beside them.  4,096 x 1,024 of
    # 2,048 is a product whose plans differ.
    line = """{ const AmOperand a{(const char *)%dll, %dll, 4096}, b{(const char *)%dll, %dll, 1024};
    const AmPlan p = am_plan(a, false, b, %s, %d, 2, 1, true); printf("%%d %%d ", p.tile, p.splits); }
    """
    cases = [(0, 4096, 0, 4096, "false", 2048), (16, 4112, 64, 8192, "false", 2048), (0, 4096, 0, 2048, "true", 2048),
             (0, 4098, 0, 4096, "false", 2048), (0, 4096, 0, 2050, "true", 2048), (8, 4096, 0, 4096, "false", 2048),
             (0, 4096, 2, 2048, "true", 2048), (0, 4096, 0, 4096, "false", 2044), (0, 1 << 23, 0, 4096, "false", 2048)]
    plain = """{ const AmPlan p = am_plan(4096, 1024, 2048, true, %s); printf("%%d %%d ", p.tile, p.splits); }
    """
    got = run(tmp_path, "".join(line % c for c in cases) + plain % "true" + plain % "false"
              + 'printf("%lld", (long long)am_most_partial_bytes(4096, 1024, 2048));')
    plans = list(zip(got[:-1:2], got[1:-1:2]))
    whole, other = plans[-2:]
    assert whole != other
    assert plans[:3] == [whole] * 3 and plans[3:-2] == [other] * 6
    assert int(got[-1]) >= max(4 * 4096 * 1024 * int(s) if int(s) > 1 else 0 for _, s in (whole, other))


def test_the_workspace_does_not_depend_on_where_operands_lie():
    pytest.importorskip("torch")
    import ctypes as C
    from paper_1808_00687_amd import acoustic as am
    sizes = set()
    for at, pad in ((0, 0), (2, 0), (0, 1), (8, 3)):
        a = am._LinearBackwardArgs()
        for f, rows, cols in (("dy", 4096, 1024), ("x", 4096, 1024), ("w", 1024, 1024), ("dx", 4096, 1024), ("dw", 1024, 1024)):
            setattr(a, f, am._Matrix(4096 + at, rows, cols, cols + pad, am.WFST_BF16, 0))
        n = C.c_int64()
        assert am._lib.wfst_am_linear_backward_workspace(bytes(a), C.byref(n)) == 0
        sizes.add(n.value)
    assert len(sizes) == 1


@pytest.mark.gpu
@pytest.mark.parametrize("m,n", [(1, (1 << 28) + 33), ((1 << 30) - 5, 1)])
def test_as_many_rows_or_columns_as_are_taken(m, n):
    torch = pytest.importorskip("torch")
    assert torch.cuda.is_available(), "no GPU"
    from paper_1808_00687_amd import acoustic as am
    g = torch.Generator(device="cuda").manual_seed(1)
    long = torch.empty(max(m, n), 1, dtype=torch.bfloat16, device="cuda")
    long.copy_(torch.randint(-99, 100, (1 << 20,), generator=g, device="cuda").repeat(max(m, n) // (1 << 20) + 1)[:max(m, n), None])
    one = torch.full((1, 1), 1.5, dtype=torch.bfloat16, device="cuda")
    y = am.wfst_am_linear(one, long) if m == 1 else am.wfst_am_linear(long, one)
    torch.cuda.synchronize()
    assert y.shape == (m, n)
    long *= 1.5                                  # one rounding as well
    assert torch.equal(y.flatten(), long.flatten())
