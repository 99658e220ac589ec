"""The acoustic-model operators' C structures and refusals (no GPU needed: the
checks come before any device call)."""
import ctypes as C
import math
import os
import subprocess

import pytest

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

STRUCTS = {"wfst_matrix": "_Matrix", "wfst_am_linear_args": "_LinearArgs",
           "wfst_am_linear_backward_args": "_LinearBackwardArgs", "wfst_am_norm_args": "_NormArgs",
           "wfst_am_norm_backward_args": "_NormBackwardArgs", "wfst_am_distill_args": "_DistillArgs",
           "wfst_am_loglikes_args": "_LoglikesArgs"}


@pytest.fixture(scope="module")
def am():
    from paper_1808_00687_amd import acoustic
    return acoustic


def test_structs_match_the_header(am, tmp_path):
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "wfstdec.h"', "int main(void) {"]
    for cname, py in STRUCTS.items():
        lines.append('printf("%s size %%zu\\n", sizeof(%s));' % (cname, cname))
        for f, _ in getattr(am, py)._fields_:
            lines.append('printf("%s %s %%zu\\n", offsetof(%s, %s));' % (cname, f, cname, f))
    lines += ["return 0;", "}"]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines) + "\n")
    subprocess.check_call(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "l")])
    got = {tuple(ln.split()[:2]): int(ln.split()[2]) for ln in
           subprocess.check_output([str(tmp_path / "l")], text=True).splitlines()}
    for cname, py in STRUCTS.items():
        t = getattr(am, py)
        assert got[(cname, "size")] == C.sizeof(t), cname
        for f, _ in t._fields_:
            assert got[(cname, f)] == getattr(t, f).offset, (cname, f)


def test_packed_layouts_are_the_structs(am):
    for name, t in (("linear", am._LinearArgs), ("linear_backward", am._LinearBackwardArgs), ("norm", am._NormArgs),
                    ("norm_backward", am._NormBackwardArgs), ("distill", am._DistillArgs),
                    ("loglikes", am._LoglikesArgs)):
        n = len(am._PACK[name].unpack(bytes(am._PACK[name].size)))
        values = [i + 1 for i in range(n)]
        a = t.from_buffer_copy(am._PACK[name].pack(*values))
        flat = []
        for f, ty in t._fields_:
            v = getattr(a, f)
            flat += [getattr(v, g) for g, _ in am._Matrix._fields_] if ty is am._Matrix else [v]
        assert C.sizeof(t) == am._PACK[name].size and [int(v) for v in flat] == values, name


# Addresses that are never read: a call with one wrong argument returns before the device
A = [0x10000000 * (i + 1) for i in range(12)]


def matrix(am, at, rows, cols, t, stride=None):
    return am._Matrix(A[at], rows, cols, cols if stride is None else stride, t, 0)


def linear(am):
    a = am._LinearArgs()
    a.x, a.w, a.y = matrix(am, 0, 4, 16, 2), matrix(am, 1, 8, 16, 2), matrix(am, 2, 4, 8, 0)
    a.residual, a.pre, a.bias = matrix(am, 3, 4, 8, 0), matrix(am, 4, 4, 8, 0), A[5]
    return a


def linear_backward(am):
    a = am._LinearBackwardArgs()
    a.dy, a.pre, a.x, a.w = (matrix(am, 0, 4, 8, 1), matrix(am, 1, 4, 8, 1), matrix(am, 2, 4, 16, 1),
                             matrix(am, 3, 8, 16, 1))
    a.dx, a.dw, a.dbias = matrix(am, 4, 4, 16, 1), matrix(am, 5, 8, 16, 0), A[6]
    a.workspace, a.workspace_bytes, a.activation = A[7], 1 << 20, 2
    return a


def norm(am):
    a = am._NormArgs()
    a.x, a.residual, a.sum, a.y = (matrix(am, i, 4, 16, t) for i, t in enumerate((2, 2, 2, 3)))
    a.gain, a.y_scale, a.eps = A[4], A[5], 1e-6
    return a


def norm_backward(am):
    a = am._NormBackwardArgs()
    a.dy, a.s, a.dsum, a.dx = (matrix(am, i, 4, 16, 2) for i in range(4))
    a.gain, a.dgain, a.workspace, a.workspace_bytes, a.eps = A[4], A[5], A[6], 1 << 20, 1e-6
    return a


def distill(am):
    a = am._DistillArgs()
    a.logits, a.top_logit, a.dlogits = matrix(am, 0, 4, 16, 2), matrix(am, 1, 4, 3, 0), matrix(am, 2, 4, 16, 2)
    a.top_index, a.weight, a.loss, a.lse, a.temperature = A[3], A[4], A[5], A[6], 1.0
    return a


def loglikes(am):
    a = am._LoglikesArgs()
    a.logits, a.ll, a.log_prior, a.scale = matrix(am, 0, 4, 16, 2), matrix(am, 1, 4, 16, 0), A[2], 1.0
    return a


MAKE = {f.__name__: f for f in (linear, linear_backward, norm, norm_backward, distill, loglikes)}
MAKE["distill_backward"] = distill


def put(a, path, value):
    *head, last = path.split(".")
    for p in head:
        a = getattr(a, p)
    setattr(a, last, value)


REFUSED = [
    ("linear", {"x.data": None}), ("linear", {"w.data": None}), ("linear", {"y.data": None}),
    ("linear", {"x.type": 0, "w.type": 0}), ("linear", {"w.type": 1}), ("linear", {"x.type": 9}),
    ("linear", {"x.type": -1}), ("linear", {"y.type": 3}), ("linear", {"w.cols": 15}), ("linear", {"y.rows": 5}),
    ("linear", {"y.cols": 7}), ("linear", {"x.rows": -1}), ("linear", {"x.rows": 1 << 31}), ("linear", {"x.cols": 0}),
    ("linear", {"w.rows": 0}), ("linear", {"x.rows": (1 << 30) + 1}), ("linear", {"x.cols": (1 << 30) + 1}),
    ("linear_backward", {"dy.cols": (1 << 30) + 1}), ("linear", {"x.row_stride": 15}), ("linear", {"y.row_stride": 1 << 60}),
    ("linear", {"x.data": A[0] + 1}), ("linear", {"bias": A[5] + 2}), ("linear", {"residual.type": 2}),
    ("linear", {"residual.rows": 3}), ("linear", {"pre.cols": 9}), ("linear", {"activation": 4}),
    ("linear", {"activation": -1}), ("linear", {"x_scale": A[6]}), ("linear", {"w_scale": A[6]}),
    ("linear", {"x.type": 3, "w.type": 3}), ("linear", {"x.type": 3, "w.type": 3, "x_scale": A[6]}),
    ("linear", {"y.data": A[0]}), ("linear", {"y.data": A[1] + 64}), ("linear", {"y.data": A[5]}),
    ("linear", {"y.data": A[3] + 4}), ("linear", {"y.data": A[3], "y.row_stride": 9}), ("linear", {"pre.data": A[2]}),
    ("linear", {"pre.data": A[3]}), ("linear", {"pre.data": A[0]}),
    ("linear_backward", {"dy.type": 0}), ("linear_backward", {"pre.data": None}), ("linear_backward", {"pre.type": 2}),
    ("linear_backward", {"x.rows": 3}), ("linear_backward", {"x.type": 2}), ("linear_backward", {"w.rows": 9}),
    ("linear_backward", {"w.data": None}), ("linear_backward", {"dx.type": 3}), ("linear_backward", {"dx.rows": 5}),
    ("linear_backward", {"dw.rows": 7}), ("linear_backward", {"dw.cols": 0}), ("linear_backward", {"activation": 7}),
    ("linear_backward", {"workspace": None}), ("linear_backward", {"workspace_bytes": 8}),
    ("linear_backward", {"workspace": A[7] + 4}), ("linear_backward", {"workspace": A[0]}),
    ("linear_backward", {"dx.data": A[0]}), ("linear_backward", {"dw.data": A[4]}), ("linear_backward", {"dbias": A[2]}),
    ("linear_backward", {"dbias": A[6] + 1}),
    ("norm", {"x.type": 3}), ("norm", {"x.cols": 0}), ("norm", {"residual.type": 0}), ("norm", {"sum.type": 0}),
    ("norm", {"y.cols": 8}), ("norm", {"y_scale": None}), ("norm", {"y.type": 2}), ("norm", {"eps": 0.0}),
    ("norm", {"eps": -1.0}), ("norm", {"eps": math.nan}), ("norm", {"eps": math.inf}), ("norm", {"gain": A[4] + 1}),
    ("norm", {"y.data": A[0]}), ("norm", {"y.data": A[2]}), ("norm", {"y_scale": A[1]}), ("norm", {"sum.data": A[0] + 2}),
    ("norm", {"sum.data": A[4]}), ("norm", {"sum.data": A[0], "sum.row_stride": 20}),
    ("norm_backward", {"s.type": 1}), ("norm_backward", {"dy.rows": 3}), ("norm_backward", {"dsum.cols": 8}),
    ("norm_backward", {"dx.type": 0}), ("norm_backward", {"eps": 0.0}), ("norm_backward", {"workspace": None}),
    ("norm_backward", {"workspace_bytes": 0}), ("norm_backward", {"dx.data": A[1]}), ("norm_backward", {"dgain": A[0]}),
    ("norm_backward", {"dx.data": A[0] + 2}), ("norm_backward", {"dgain": A[6]}),
    ("distill", {"logits.type": 3}), ("distill", {"top_logit.type": 3}), ("distill", {"top_logit.cols": 0}),
    ("distill", {"top_logit.cols": 257, "top_logit.row_stride": 257}), ("distill", {"top_logit.rows": 3}),
    ("distill", {"dlogits.type": 0}), ("distill", {"temperature": 0.0}), ("distill", {"temperature": math.nan}),
    ("distill", {"temperature": math.inf}), ("distill", {"top_index": None}), ("distill", {"loss": A[0]}),
    ("distill", {"dlogits.data": A[0] + 2}), ("distill", {"lse": A[5]}), ("distill", {"dlogits.data": A[1]}),
    ("distill_backward", {"lse": None}), ("distill_backward", {"dlogits.data": None}),
    ("distill_backward", {"dlogits.data": A[6]}), ("distill_backward", {"temperature": -1.0}),
    ("loglikes", {"logits.type": 3}), ("loglikes", {"ll.type": 2}), ("loglikes", {"ll.cols": 15}),
    ("loglikes", {"scale": 0.0}), ("loglikes", {"scale": math.inf}), ("loglikes", {"ll.data": A[0]}),
    ("loglikes", {"log_prior": A[2] + 2}), ("loglikes", {"logits.data": None}), ("loglikes", {"ll.data": A[2]}),
]


@pytest.mark.parametrize("name,change", REFUSED)
def test_refusals(am, name, change):
    from paper_1808_00687_amd import wfstdec
    a = MAKE[name](am)
    for path, v in change.items():
        put(a, path, v)
    assert getattr(am._lib, "wfst_am_" + name)(bytes(a), None) == wfstdec.WFST_EINVAL
    assert wfstdec.wfst_last_error().startswith("wfst_am_" + name)


@pytest.mark.parametrize("name", list(MAKE))
def test_refuses_no_arguments(am, name):
    from paper_1808_00687_amd import wfstdec
    assert getattr(am._lib, "wfst_am_" + name)(None, None) == wfstdec.WFST_EINVAL


@pytest.mark.parametrize("name", ["linear", "norm", "distill", "distill_backward", "loglikes"])
def test_no_rows_is_no_work(am, name):
    # no rows, no pointers: accepted without a device call
    a = MAKE[name](am)
    for f, ty in a._fields_:
        if ty is am._Matrix and (name, f) != ("linear", "w"):
            getattr(a, f).rows = 0
            if f in ("x", "y", "logits", "ll"):
                getattr(a, f).data = None
    assert getattr(am._lib, "wfst_am_" + name)(bytes(a), None) == 0


def test_workspace_queries(am):
    from paper_1808_00687_amd import wfstdec
    n = C.c_int64(-1)
    for name in ("linear_backward", "norm_backward"):
        q = getattr(am._lib, "wfst_am_%s_workspace" % name)
        a = MAKE[name](am)
        assert q(bytes(a), C.byref(n)) == 0 and n.value >= 0
        assert q(None, C.byref(n)) == wfstdec.WFST_EINVAL and q(bytes(a), None) == wfstdec.WFST_EINVAL
        put(a, "dy.rows" if name == "linear_backward" else "s.rows", -1)
        assert q(bytes(a), C.byref(n)) == wfstdec.WFST_EINVAL


def test_binding_refuses_host_tensors(am):
    x = torch.zeros(2, 8)
    for call in (lambda: am.wfst_am_linear(x, x), lambda: am.wfst_am_norm(x), lambda: am.wfst_am_loglikes(x),
                 lambda: am.wfst_am_linear_backward(x, x, x), lambda: am.wfst_am_norm_backward(x, x),
                 lambda: am.wfst_am_distill(x, x, x), lambda: am.wfst_am_distill_backward(x, x, x, x)):
        with pytest.raises(TypeError):
            call()
