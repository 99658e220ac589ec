"""Which of the norms' kernels the library holds: those of the shapes that some row takes, each of them, and no other (no GPU
needed)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_1808_00687_amd.csrc import build

# (threads a row, chunks a thread, columns of a chunk) up to a row's end, for 16-bit rows and for 32-bit ones
HALF = [(64, 1, 8), (64, 2, 8), (64, 4, 8), (256, 2, 8), (256, 3, 8), (256, 4, 8), (1024, 2, 8), (1024, 0, 8)]
FULL = [(64, 2, 4), (64, 4, 4), (64, 8, 4), (256, 4, 4), (256, 6, 4), (256, 8, 4), (1024, 4, 4), (1024, 0, 4)]
SHORT_HALF, SHORT_FULL = [(8, 1, 8), (16, 1, 8), (32, 1, 8)], [(8, 2, 4), (16, 2, 4), (32, 2, 4)]


def but(shapes, without, with_):
    return set(shapes) - set(without) | set(with_)


LEAN_HALF = but(HALF, [(64, 4, 8), (256, 4, 8)], [(256, 1, 8), (1024, 1, 8), (1024, 4, 8)])
LEAN_FULL = but(FULL, [(64, 8, 4), (256, 8, 4)], [(256, 2, 4), (1024, 2, 4), (1024, 8, 4)])
# kernel -> (16-bit types' shapes, float32's); forward, a 16-bit row to float32 takes float32's shapes, too
WANT = {"norm_kernel": (set(HALF) | set(FULL), set(FULL)),
        "norm_backward_kernel": (LEAN_HALF, LEAN_FULL),
        "layer_norm_kernel": (set(HALF + SHORT_HALF + [(64, 3, 8)]) | set(FULL + SHORT_FULL), set(FULL + SHORT_FULL)),
        "layer_norm_backward_kernel": (set(HALF + SHORT_HALF + [(64, 3, 8)]), but(FULL, [(64, 8, 4)], SHORT_FULL + [(256, 2, 4)]))}


def test_the_norms_kernels_are_those_that_rows_take():
    if not shutil.which("nm"):
        pytest.skip("no nm")
    if not os.path.exists(build.OUT):
        build.build()
    got = {}
    for line in subprocess.check_output(["nm", build.OUT], text=True).splitlines():
        m = re.search(r"\d+__device_stub__(\w*norm\w*_kernel)I(f|DF16_|DF16b)NS_8RowShapeILi(\d+)ELi(\d+)ELi(\d+)EEE", line)
        if m:
            got.setdefault((m.group(1), m.group(2)), set()).add(tuple(int(v) for v in m.groups()[2:]))
    want = {(k, t): shapes[t == "f"] for k, shapes in WANT.items() for t in ("f", "DF16_", "DF16b")}
    assert got == want
