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
