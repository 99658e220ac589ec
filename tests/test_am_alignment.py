"""Wide accesses of the acoustic model's kernels promise the compiler no more alignment than their operands have: an
element's.  (From a promise of 16 bytes it may take a scalar load for an address that a wave's threads share, and that one
drops the low bits.)  Compiled to the compiler's intermediate form for gfx950; no GPU needed."""
import os
import re
import subprocess

import pytest

from paper_1808_00687_amd.csrc import build

SOURCE = """
#include "am_rows.h"
#include "am_tile.h"
using namespace wfd;
template <typename T, int C> __global__ void chunks(const T *p, T *q, int64_t n)
{
    float x[C];
    load_floats<T, C>(p, n, x);
    store_floats<T, C>(q, n, x);
}
template <typename T, int N> __global__ void rows(wfst_matrix in, wfst_matrix out, int64_t i, int64_t j)
{
    float v[N] = {};
    am_add_row<T>(in, i, j, v, true);
    am_store_row<T>(out, i, j, v, true);
}
__global__ void bytes(const float *p, f8 *q, int64_t n)
{
    float x[8];
    load_floats<float, 8>(p, n, x);
    store_floats<8>(q, n, x);
}
#define EACH(T) template __global__ void chunks<T, 8>(const T *, T *, int64_t); \\
    template __global__ void chunks<T, 4>(const T *, T *, int64_t); \\
    template __global__ void rows<T, 8>(wfst_matrix, wfst_matrix, int64_t, int64_t); \\
    template __global__ void rows<T, 16>(wfst_matrix, wfst_matrix, int64_t, int64_t); \\
    template __global__ void rows<T, 2>(wfst_matrix, wfst_matrix, int64_t, int64_t);
EACH(float) EACH(f16) EACH(bf16)
__global__ void fetch(AmOperand o, i32x4 *q)
{
    i32x4 r[1];
    AmSide<bf16, 64, 64, 4, false, 1, false>{}.load(o, 0, 64, 0, r, 0, threadIdx.x);
    *(AM_GLOBAL i32x4_any *)q = r[0];
}
"""


ELEMENTS = {"float": 4, "half": 2, "bfloat": 2, "i32": 1, "i128": 2}   # words stand for bytes at any address


def accesses(source):
    """(kind, values, element, alignment) of the wide accesses to global memory in a source's kernels."""
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    flags = [f for f in build.FLAGS if f != "-fPIC"]
    cmd = [build.HIPCC, "-x", "hip", *flags, "--cuda-device-only", "-S", "-emit-llvm", source, "-o", "-"]
    seen = set()
    for line in subprocess.check_output(cmd, text=True, stderr=subprocess.DEVNULL).splitlines():
        m = re.search(r"(load|store) (?:<(\d+) x (float|half|bfloat|i32)>|(i128)).*addrspace\(1\).* align (\d+)", line)
        if m:
            seen.add((m.group(1), int(m.group(2) or 1), m.group(3) or m.group(4), int(m.group(5))))
    return seen


def test_wide_accesses_promise_an_elements_alignment(tmp_path):
    src = tmp_path / "wide.hip"
    src.write_text(SOURCE)
    seen = accesses(str(src))
    assert {s for s in seen if s[3] > ELEMENTS[s[2]]} == set()
    assert {s[:3] for s in seen} >= {(k, n, e) for k in ("load", "store") for e in ("float", "half", "bfloat") for n in (2, 4, 8)
                                     if (n, e) != (8, "float")}
    assert ("store", 2, "i32", 1) in seen and ("load", 4, "i32", 1) in seen


@pytest.mark.parametrize("name", ["am_clip.hip", "am_layer_norm.hip"])
def test_an_operators_wide_accesses(name):
    seen = accesses(os.path.join(build.HERE, name))
    assert {s for s in seen if s[3] > ELEMENTS[s[2]]} == set()
    assert len(seen) >= 4


def test_no_alias_asks_for_an_alignment():
    # the compiler drops it without a word from a `using`, and keeps it in a typedef
    for name in sorted(os.listdir(build.HERE)):
        if name.endswith((".h", ".hip", ".cpp")):
            with open(os.path.join(build.HERE, name)) as f:
                assert not re.findall(r"using\s+\w+\s*=[^;]*aligned\s*\(", f.read()), name
