"""The C structures and refusals of the layer norm, the gated layer and the clipping
of gradients (no GPU needed: the checks come before any device call)."""
import ctypes as C
import math
import os
import subprocess

import pytest

from test_am_abi import A, ROOT, am, matrix, put  # noqa: F401

torch = pytest.importorskip("torch")

STRUCTS = {"wfst_am_layer_norm_args": ("layer_norm", "_LayerNormArgs"),
           "wfst_am_layer_norm_backward_args": ("layer_norm_backward", "_LayerNormBackwardArgs"),
           "wfst_am_gated_args": ("gated", "_GatedArgs"),
           "wfst_am_gated_backward_args": ("gated_backward", "_GatedBackwardArgs"),
           "wfst_am_clip_args": ("clip", "_ClipArgs")}


def test_structs_match_the_header(am, tmp_path):  # noqa: F811
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "wfstdec.h"', "int main(void) {"]
    for cname, (_, py) in STRUCTS.items():
        lines.append('printf("%s size %%zu\\n", sizeof(%s));' % (cname, cname))
        for f, _ in getattr(am, py)._fields_:
            lines.append('printf("%s %s %%zu\\n", offsetof(%s, %s));' % (cname, f, cname, f))
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ["return 0;", "}"]) + "\n")
    subprocess.check_call(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "l")])
    got = {tuple(ln.split()[:2]): int(ln.split()[2]) for ln in
           subprocess.check_output([str(tmp_path / "l")], text=True).splitlines()}
    for cname, (_, py) in STRUCTS.items():
        t = getattr(am, py)
        assert got[(cname, "size")] == C.sizeof(t), cname
        for f, _ in t._fields_:
            assert got[(cname, f)] == getattr(t, f).offset, (cname, f)


def test_packed_layouts_are_the_structs(am):  # noqa: F811
    for name, py in STRUCTS.values():
        t = getattr(am, py)
        n = len(am._PACK[name].unpack(bytes(am._PACK[name].size)))
        values = [i + 1 for i in range(n)]
        a = t.from_buffer_copy(am._PACK[name].pack(*values))
        flat = []
        for f, ty in t._fields_:
            v = getattr(a, f)
            flat += [getattr(v, g) for g, _ in am._Matrix._fields_] if ty is am._Matrix else [v]
        assert C.sizeof(t) == am._PACK[name].size and [int(v) for v in flat] == values, name


def layer_norm(am):  # noqa: F811
    a = am._LayerNormArgs()
    a.x, a.residual, a.sum, a.y = (matrix(am, i, 4, 16, t) for i, t in enumerate((2, 2, 2, 3)))
    a.gain, a.bias, a.y_scale, a.eps = A[4], A[5], A[6], 1e-5
    return a


def layer_norm_backward(am):  # noqa: F811
    a = am._LayerNormBackwardArgs()
    a.dy, a.s, a.dsum, a.dx = (matrix(am, i, 4, 16, 2) for i in range(4))
    a.gain, a.dgain, a.dbias, a.workspace, a.workspace_bytes, a.eps = A[4], A[5], A[6], A[7], 1 << 20, 1e-5
    return a


def clip(am):  # noqa: F811
    """Two grads in places of their own, outputs in others.  The matrices live as long as the arguments."""
    a = am._ClipArgs()
    a.kept = ((am._Matrix * 2)(matrix(am, 0, 4, 16, 2), matrix(am, 1, 1, 9, 0)),
              (am._Matrix * 2)(matrix(am, 2, 4, 16, 2), matrix(am, 3, 1, 9, 0)))
    a.grads, a.outs = (C.cast(k, C.c_void_p) for k in a.kept)
    a.count, a.max_norm, a.norm, a.workspace, a.workspace_bytes = 2, 1.0, A[5], A[6], 1 << 20
    return a


def gated(am):  # noqa: F811
    a = am._GatedArgs()
    a.x, a.w, a.pre, a.y = matrix(am, 0, 4, 16, 2), matrix(am, 1, 16, 16, 2), matrix(am, 2, 4, 16, 0), matrix(am, 3, 4, 8, 0)
    a.bias, a.activation = A[4], 2
    return a


def gated_backward(am):  # noqa: F811
    a = am._GatedBackwardArgs()
    a.dy, a.pre, a.x, a.w = (matrix(am, 0, 4, 8, 1), matrix(am, 1, 4, 16, 1), matrix(am, 2, 4, 16, 1), matrix(am, 3, 16, 16, 1))
    a.dx, a.dw, a.dbias = matrix(am, 4, 4, 16, 1), matrix(am, 5, 16, 16, 0), A[6]
    a.workspace, a.workspace_bytes, a.activation = A[7], 1 << 20, 2
    return a


MAKE = {f.__name__: f for f in (layer_norm, layer_norm_backward, clip, gated, gated_backward)}

REFUSED = [
    ("layer_norm", {"x.type": 3}), ("layer_norm", {"x.cols": 0}), ("layer_norm", {"x.rows": -1}),
    ("layer_norm", {"x.data": None}), ("layer_norm", {"residual.type": 0}), ("layer_norm", {"sum.type": 0}),
    ("layer_norm", {"sum.rows": 3}), ("layer_norm", {"y.cols": 8}), ("layer_norm", {"y.row_stride": 15}),
    ("layer_norm", {"y_scale": None}), ("layer_norm", {"y.type": 2}), ("layer_norm", {"eps": 0.0}),
    ("layer_norm", {"eps": math.nan}), ("layer_norm", {"eps": math.inf}), ("layer_norm", {"gain": A[4] + 1}),
    ("layer_norm", {"bias": A[5] + 2}), ("layer_norm", {"y.data": A[0]}), ("layer_norm", {"y.data": A[2]}),
    ("layer_norm", {"y.data": A[5]}), ("layer_norm", {"y_scale": A[1]}), ("layer_norm", {"sum.data": A[0] + 2}),
    ("layer_norm", {"sum.data": A[5]}), ("layer_norm", {"sum.data": A[4]}),
    ("layer_norm", {"sum.data": A[0], "sum.row_stride": 20}),
    ("layer_norm_backward", {"s.type": 1}), ("layer_norm_backward", {"s.type": 3, "dy.type": 3}),
    ("layer_norm_backward", {"dy.rows": 3}), ("layer_norm_backward", {"dsum.cols": 8}),
    ("layer_norm_backward", {"dx.type": 0}), ("layer_norm_backward", {"eps": -1.0}),
    ("layer_norm_backward", {"workspace": None}), ("layer_norm_backward", {"workspace_bytes": 0}),
    ("layer_norm_backward", {"workspace": A[7] + 128}), ("layer_norm_backward", {"workspace": A[1]}),
    ("layer_norm_backward", {"dx.data": A[1]}), ("layer_norm_backward", {"dgain": A[0]}),
    ("layer_norm_backward", {"dbias": A[5]}), ("layer_norm_backward", {"dbias": A[2]}),
    ("layer_norm_backward", {"dx.data": A[0] + 2}), ("layer_norm_backward", {"dbias": A[6] + 1}),
    ("layer_norm_backward", {"dgain": A[7]}),
    ("gated", {"x.data": None}), ("gated", {"w.data": None}), ("gated", {"y.data": None}), ("gated", {"x.type": 0, "w.type": 0}),
    ("gated", {"w.type": 1}), ("gated", {"y.type": 3}), ("gated", {"w.rows": 15}), ("gated", {"w.rows": 17}),
    ("gated", {"w.cols": 15}), ("gated", {"y.cols": 9}), ("gated", {"y.cols": 0}), ("gated", {"y.cols": -8}), ("gated", {"y.rows": 5}),
    ("gated", {"pre.cols": 8}), ("gated", {"pre.type": 2}), ("gated", {"pre.data": A[3]}), ("gated", {"pre.data": A[0]}),
    ("gated", {"y.data": A[1]}), ("gated", {"y.data": A[2] + 32}), ("gated", {"y.data": A[4] + 32}),
    ("gated", {"pre.data": A[4] + 60}), ("gated", {"activation": 4}), ("gated", {"activation": -1}), ("gated", {"x.rows": -1}),
    ("gated", {"x_scale": A[5]}), ("gated", {"x.type": 3, "w.type": 3}), ("gated", {"x.type": 3, "w.type": 3, "x_scale": A[5]}),
    ("gated", {"bias": A[4] + 2}), ("gated", {"y.cols": 1 << 30, "y.row_stride": 1 << 30}), ("gated", {"x.row_stride": 15}),
    ("gated_backward", {"dy.type": 0}), ("gated_backward", {"dy.cols": 0}), ("gated_backward", {"dy.cols": 7}),
    ("gated_backward", {"pre.data": None}), ("gated_backward", {"pre.cols": 8}), ("gated_backward", {"pre.type": 2}),
    ("gated_backward", {"x.rows": 3}), ("gated_backward", {"w.rows": 8}), ("gated_backward", {"w.data": None}),
    ("gated_backward", {"x.type": 2}), ("gated_backward", {"dx.type": 3}), ("gated_backward", {"dw.rows": 8}),
    ("gated_backward", {"dw.cols": 0}), ("gated_backward", {"activation": 9}), ("gated_backward", {"round_dz": 2}),
    ("gated_backward", {"round_dz": -1}), ("gated_backward", {"workspace": None}), ("gated_backward", {"workspace_bytes": 8}),
    ("gated_backward", {"workspace": A[7] + 4}), ("gated_backward", {"workspace": A[1]}), ("gated_backward", {"dx.data": A[1]}),
    ("gated_backward", {"dw.data": A[4]}), ("gated_backward", {"dbias": A[3] + 4}), ("gated_backward", {"dbias": A[6] + 1}),
    ("gated_backward", {"dw.data": A[6] + 32}),
]


@pytest.mark.parametrize("name,change", REFUSED)
def test_refusals(am, name, change):  # noqa: F811
    from paper_1808_00687_amd import wfstdec
    a = MAKE[name](am)
    for path, v in change.items():
        put(a, path, v)
    assert getattr(am._lib, "wfst_am_" + name)(bytes(a), None) == wfstdec.WFST_EINVAL
    assert wfstdec.wfst_last_error().startswith("wfst_am_" + name)


CLIP_REFUSED = [
    ({"count": -1}, {}), ({"count": 65537}, {}), ({"max_norm": 0.0}, {}), ({"max_norm": -1.0}, {}),
    ({"max_norm": math.nan}, {}), ({"norm": None}, {}), ({"norm": A[5] + 2}, {}), ({"norm": A[2] + 4}, {}),
    ({"norm": A[1] + 4}, {}), ({"norm": A[6] + 64}, {}), ({"workspace": None}, {}), ({"workspace_bytes": 100}, {}),
    ({"workspace": A[6] + 8}, {}), ({"workspace": A[0]}, {}), ({"workspace": A[3]}, {}), ({"grads": None}, {}),
    ({}, {"grads.0.type": 3}), ({}, {"grads.0.rows": -1}), ({}, {"grads.1.cols": 0}), ({}, {"grads.1.data": None}),
    ({}, {"grads.0.row_stride": 15}), ({}, {"grads.0.data": A[0] + 1}), ({}, {"outs.0.type": 1}),
    ({}, {"outs.0.cols": 15}), ({}, {"outs.1.rows": 2}), ({}, {"outs.1.data": A[3] + 2}),
    # an output over another one, over another's grad, beside its own grad's place, in its place with other rows
    ({}, {"outs.1.data": A[2] + 60}), ({}, {"outs.1.data": A[0]}), ({}, {"outs.0.data": A[0] + 2}),
    ({}, {"outs.0.data": A[0], "outs.0.row_stride": 17}), ({"outs": None}, {"grads.1.data": A[0]}),
]


@pytest.mark.parametrize("change,inner", CLIP_REFUSED)
def test_clip_refusals(am, change, inner):  # noqa: F811
    from paper_1808_00687_amd import wfstdec
    a = clip(am)
    for path, v in change.items():
        put(a, path, v)
    for path, v in inner.items():
        which, i, field = path.split(".")
        setattr(a.kept[which == "outs"][int(i)], field, v)
    assert am._lib.wfst_am_clip(bytes(a), None) == wfstdec.WFST_EINVAL
    assert wfstdec.wfst_last_error().startswith("wfst_am_clip")


def test_clip_workspace(am):  # noqa: F811
    from paper_1808_00687_amd import wfstdec
    n = C.c_int64(-1)
    q = am._lib.wfst_am_clip_workspace
    sizes = []
    for count in (0, 1, 71, 72, 1000, 65536):
        a = am._ClipArgs()
        a.count = count
        assert q(bytes(a), C.byref(n)) == 0 and n.value > 0
        sizes.append(n.value)
    assert sizes == sorted(sizes)
    a.count = 65537
    assert q(bytes(a), C.byref(n)) == wfstdec.WFST_EINVAL
    assert q(None, C.byref(n)) == wfstdec.WFST_EINVAL and q(bytes(a), None) == wfstdec.WFST_EINVAL


def test_clip_binding_refuses(am):  # noqa: F811
    x = torch.zeros(2, 8)
    for grads in (x, [], iter([x]), None):
        with pytest.raises(TypeError, match="list"):
            am.wfst_am_clip(grads, 1.0)
    with pytest.raises(TypeError, match="GPU"):
        am.wfst_am_clip([x], 1.0)
    with pytest.raises(TypeError, match="GPU"):
        am.wfst_am_clip(grads=(x,), max_norm=1.0, stream=0)


@pytest.mark.parametrize("name", list(MAKE))
def test_refuses_no_arguments(am, name):  # noqa: F811
    from paper_1808_00687_amd import wfstdec
    assert getattr(am._lib, "wfst_am_" + name)(None, None) == wfstdec.WFST_EINVAL


FORWARD = ["layer_norm", "gated"]


@pytest.mark.parametrize("name", FORWARD)
def test_no_rows_is_no_work(am, name):  # noqa: F811
    a = MAKE[name](am)
    for f, ty in a._fields_:
        if ty is am._Matrix and f != "w":
            getattr(a, f).rows = 0
            if f in ("x", "y"):
                getattr(a, f).data = None
    assert getattr(am._lib, "wfst_am_" + name)(bytes(a), None) == 0


@pytest.mark.parametrize("name", [n for n in MAKE if n.endswith("_backward")])
def test_workspace_queries(am, name):  # noqa: F811
    from paper_1808_00687_amd import wfstdec
    n = C.c_int64(-1)
    q = getattr(am._lib, "wfst_am_%s_workspace" % name)
    a = MAKE[name](am)
    assert q(bytes(a), C.byref(n)) == 0 and n.value >= 0
    assert q(None, C.byref(n)) == wfstdec.WFST_EINVAL and q(bytes(a), None) == wfstdec.WFST_EINVAL
    put(a, "s.rows" if name == "layer_norm_backward" else "dy.rows", -1)
    assert q(bytes(a), C.byref(n)) == wfstdec.WFST_EINVAL


def test_binding_refuses_host_tensors(am):  # noqa: F811
    x = torch.zeros(2, 8)
    for call in (lambda: am.wfst_am_layer_norm(x), lambda: am.wfst_am_layer_norm_backward(x, x),
                 lambda: am.wfst_am_gated(x, x), lambda: am.wfst_am_gated_backward(x, x, x, x)):
        with pytest.raises(TypeError):
            call()
