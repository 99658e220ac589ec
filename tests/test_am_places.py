"""The check that outputs lie apart, as the clipping makes it for many tensors: host arithmetic, compiled alone (no GPU
needed)."""
import subprocess

import pytest

from test_am_plan import CSRC

PROGRAM = r"""
#include <chrono>
#include <cstdio>
#include <cstdlib>
#include <random>
#include "am_places.h"
using namespace wfd;

static bool by_pairs(const std::vector<Span> &v)
{
    for (size_t i = 0; i < v.size(); i++)
        for (size_t j = 0; j < i; j++)
            if ((v[i].written || v[j].written) && v[i].r.lo < v[i].r.hi && v[j].r.lo < v[j].r.hi && !disjoint(v[i].r, v[j].r)) return false;
    return true;
}
static Range matrix(uintptr_t at, uintptr_t rows, uintptr_t stride, uintptr_t width)
{
    if (!rows) return {0, 0};
    return {at, at + (rows - 1) * stride + width, rows > 1 ? stride : 0, width};
}

static int random_sets()
{
    std::mt19937 g(7);
    const auto of = [&](int a, int b) { return std::uniform_int_distribution<int>(a, b)(g); };
    int apart = 0, meet = 0;
    for (int round = 0; round < 400000; round++) {
        const int n = of(1, 9), stride = of(1, 2) * 12, other = of(0, 9) ? stride : stride + 2, room = of(0, 3) * 40 + 30;
        const int most_written = of(0, 3), most_width = of(1, 3) * 2;
        std::vector<Span> v;
        for (int i = 0; i < n; i++) {
            const int width = of(1, most_width), rows = of(0, 20) ? of(1, 5) : 0;
            v.push_back({matrix(1000 + of(0, room), rows, of(0, 3) ? stride : other, width), of(0, 3) < most_written});
            if (!of(0, 3)) v.push_back({v[of(0, (int)v.size() - 1)].r, false});   // read twice
            if (!of(0, 5)) {   // the same columns, some rows on
                Range r = v.back().r;
                if (r.stride) r.lo += r.stride, r.hi += r.stride, v.push_back({r, false});
            }
        }
        const bool want = by_pairs(v);
        std::vector<Span> w = v;
        if (spans_apart(w) != want) {
            printf("differs, want %d:", (int)want);
            for (const Span &s : v) printf(" [%zu %zu) %zu %zu %d", (size_t)s.r.lo, (size_t)s.r.hi, (size_t)s.r.stride, (size_t)s.r.width, (int)s.written);
            return 1;
        }
        (want ? apart : meet)++;
    }
    printf("%d %d", apart, meet);
    return 0;
}

// 65,536 tensors, all columns of one buffer, or one of them read again and again: as many outputs
static int many(bool slices)
{
    constexpr uintptr_t n = 65536, rows = 7, width = 16;
    std::vector<Span> v;
    for (uintptr_t i = 0; i < n; i++) {
        v.push_back({slices ? matrix(4096 + i * width, rows, 2 * n * width, width) : matrix(64, rows, 24, width), false});
        v.push_back({slices ? matrix(4096 + (n + i) * width, rows, 2 * n * width, width) : matrix(4096 + i * rows * width, rows, width, width), true});
    }
    const auto start = std::chrono::steady_clock::now();
    std::vector<Span> w = v;
    const bool apart = spans_apart(w);
    v.push_back({matrix(4096 + n * width + 5, 1, 1, 1), true});
    const bool meet = !spans_apart(v);
    const std::chrono::duration<double> t = std::chrono::steady_clock::now() - start;
    printf("%d %d %f", (int)apart, (int)meet, t.count());
    return 0;
}

int main(int, char **a) { return a[1][0] == 'r' ? random_sets() : many(a[1][0] == 's'); }
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("places")
    src = d / "places.cpp"
    src.write_text(PROGRAM)
    subprocess.check_call(["g++", "-std=c++20", "-O1", "-Wall", "-D_GLIBCXX_ASSERTIONS", "-I", CSRC, str(src), "-o", str(d / "places")])
    return str(d / "places")


def test_as_pair_by_pair(program):
    r = subprocess.run([program, "random"], stdout=subprocess.PIPE, text=True)
    assert r.returncode == 0, r.stdout
    apart, meet = (int(v) for v in r.stdout.split())
    assert apart > 20000 and meet > 20000


@pytest.mark.parametrize("kind", ["slices", "again"])
def test_many_tensors_take_a_moment(program, kind):
    # pair by pair they took half a minute
    apart, meet, seconds = subprocess.check_output([program, kind], text=True, timeout=60).split()
    assert (apart, meet) == ("1", "1") and float(seconds) < 3.0
