"""The layer norm, the gated layer and the clipping at the limits of what they take: host code, compiled alone (no GPU
needed)."""
import os
import subprocess

import pytest

from paper_1808_00687_amd.csrc import build
from test_am_plan import run


def test_columns_of_a_join_fit_their_launches(tmp_path):
    # 32 columns a workgroup of 1,024 threads: every block once, in order, fewer than 2^32 threads a launch, up to the
    # most columns that a norm takes
    columns = [1, 33, (1 << 26) - 1, 1 << 26, (1 << 27) - 32, 1 << 27, (1 << 27) + 33, (1 << 31) - 1]
    one = 'am_in_launches((%dll + 31) / 32, [](uint32_t first, uint32_t count) { printf("%%u %%u ", first, count); }, 1024); printf("/ ");\n'
    got = " ".join(run(tmp_path, "".join(one % n for n in columns))).split("/")
    for n, line in zip(columns, got):
        at, runs = 0, [int(v) for v in line.split()]
        for first, count in zip(runs[::2], runs[1::2]):
            assert first == at and 0 < count and count * 1024 < 1 << 32, n
            at += count
        assert at == -(-n // 32)
        assert n > 1 << 26 or len(runs) == 2


def test_the_gradients_products_do_not_ask_for_their_grid(tmp_path):
    # it lies behind the arguments in memory: one more read, 0.4 us, before a workgroup knows its tile
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    src = tmp_path / "tile.hip"
    src.write_text("""#include "am_tile.h"
namespace wfd {
template __global__ void am_tile_kernel<bf16, true, true, false, AmSmallMajorStaged, false, false, false>(AmProduct);
template __global__ void am_tile_kernel<bf16, false, true, true, AmSmallMajor, false, true, false>(AmProduct);
}
""")
    flags = [f for f in build.FLAGS if f != "-fPIC"]
    text = subprocess.check_output([build.HIPCC, "-x", "hip", *flags, "--cuda-device-only", "-S", "-emit-llvm", str(src), "-o", "-"],
                                   text=True, stderr=subprocess.DEVNULL)
    assert text.count("define protected amdgpu_kernel void @") == 2
    assert "llvm.amdgcn.implicitarg.ptr" not in text
