"""Gradients of the acoustic model's layers: how close the products come to the
definition where an activation's slope has more bits than the operands' type.

Without a rounding of dz to 16 bits the products differ from float64 by their
float32 sums and by what two 16-bit values leave of dz: 2^-16 of it in bfloat16,
2^-22 or 2^-35 in float16, as independent errors of the terms.
"""
import math

import pytest

import am_reference as R
from test_gpu_am_operators import BF16, F16, F32, far, inside, normal, rng

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

INF = math.inf
LEFT = {BF16: (2.0 ** -16, 0.0), F16: (2.0 ** -22, 2.0 ** -35)}   # of dz in two values: relative, absolute


@pytest.fixture(scope="module")
def am():
    assert torch.cuda.is_available(), "no GPU"
    from paper_1808_00687_amd import acoustic
    return acoustic


def gradients(am, dy, x, w, kind, pre, round_dz=0):
    """dx, dw and dbias, all in float32 (the binding's dx has dy's type)."""
    dx, dw = torch.empty(dy.shape[0], w.shape[1]).cuda(), torch.empty(dy.shape[1], x.shape[1]).cuda()
    db = torch.empty(dy.shape[1]).cuda()
    d = dy.get_device()
    head = []
    for t, name in ((dy, "dy"), (pre, "pre"), (x, "x"), (w, "w"), (dx, "dx"), (dw, "dw")):
        head += am._matrix(t, name, d)
    head.append(db.data_ptr())
    pack, act = am._PACK["linear_backward"].pack, am.ACTIVATIONS[kind]
    need = am._bytes_for("wfst_am_linear_backward_workspace", pack(*head, 0, 0, act, round_dz))
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    am._call("wfst_am_linear_backward", pack(*head, work.data_ptr(), need, act, round_dz),
             torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    return dx, dw, db


def inputs(m, k, n, dt, seed, size=0.1):
    g = rng(seed)
    x, w = normal(g, m, k).to(dt), normal(g, n, k, std=k ** -0.5).to(dt)
    return normal(g, m, n, std=size).to(dt), x, w, normal(g, m, n, std=1.5).to(dt)


def check(got, dy, x, w, kind, z, dt, tag):
    dz = R.d(dy) * R.slope(R.d(z), kind)
    slack = 16 * R.U32 * (1 + R.d(z).abs()) * R.d(dy).abs()   # the slope is good to a few float32 roundings
    rel, least = LEFT[dt]
    for g, a, b, s in ((got[0], dz, R.d(w), slack), (got[1], dz.t(), R.d(x), slack.t())):
        want = a @ b
        err = R.sum_bound(2 * a.shape[1], a.abs() @ b.abs()) + (s + least) @ b.abs()
        err = err + R.LAMBDA * rel * torch.sqrt((a * a) @ (b * b)) + R.TINY[dt] * b.abs().sum(0)
        R.close(g, want, err + R.U32 * want.abs() + R.TINY[F32], tag)
    R.close(got[2], dz.sum(0), R.sum_bound(dz.shape[0], dz.abs().sum(0)) + slack.sum(0) + R.TINY[F32], tag + " dbias")


# every tile and storage: few rows, small, medium and large tiles, k in parts, rows off 16 bytes, no whole stage
SHAPES = [(1, 1, 1), (3, 130, 50), (33, 440, 65), (130, 136, 257), (300, 72, 129), (700, 264, 192), (1500, 1400, 200),
          (1501, 1403, 70), (2040, 1960, 456), (2904, 3016, 136), (136, 2904, 3016), (5000, 40, 24)]


@pytest.mark.parametrize("dt", [BF16, F16])
@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("m,k,n", SHAPES)
def test_dz_is_not_rounded(am, m, k, n, kind, dt):
    dy, x, w, z = inputs(m, k, n, dt, m + k + n)
    got = gradients(am, inside(dy), inside(x), inside(w), kind, inside(z))
    check(got, dy, x, w, kind, z, dt, "gradients %s" % ((m, k, n, kind, str(dt)),))


@pytest.mark.parametrize("dt", [BF16, F16])
@pytest.mark.parametrize("pad,offset", [(1, 0), (8, 8), (0, 3)])
def test_dz_strides(am, dt, pad, offset):
    for m, k, n in ((150, 72, 140), (700, 264, 192)):
        dy, x, w, z = inputs(m, k, n, dt, 4)
        got = gradients(am, *(inside(t, pad, offset) for t in (dy, x, w)), "gelu", inside(z, pad, offset))
        check(got, dy, x, w, "gelu", z, dt, "gradients strided %s" % ((m, pad, offset, str(dt)),))


def test_dz_rows_far_apart(am):
    m, k, n = 70, 72, 130
    dy, x, w, z = inputs(m, k, n, BF16, 22)
    a, b = (torch.empty((m << 26) + (1 << 20), dtype=torch.uint8, device="cuda") for _ in range(2))
    got = gradients(am, far(a, dy), far(b, x), w.cuda(), "silu", z.cuda())
    check(got, dy, x, w, "silu", z, BF16, "gradients far")


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_dz_at_the_ends_of_float16(am, kind):
    # gradients near the type's largest value, whose dz is above it, and near its smallest
    for size in (65504.0, 2.0 ** -12, 2.0 ** -20, 2.0 ** -24):
        dy, x, w, z = inputs(70, 72, 64, F16, 5, 1.0)
        dy = (dy.sign().float() * size).to(F16)
        z[:, ::3] = 2.0
        got = gradients(am, dy.cuda(), x.cuda(), w.cuda(), kind, z.cuda())
        check(got, dy, x, w, kind, z, F16, "gradients of size %g" % size)


@pytest.mark.parametrize("dt", [BF16, F16])
@pytest.mark.parametrize("m,k,n", [(60, 64, 72), (2904, 136, 520)])
def test_infinities_and_nan_by_the_formula(am, m, k, n, dt):
    dy, x, w, z = inputs(m, k, n, dt, 6)
    w[3, 5], w[4, 6] = INF, math.nan
    x[7, 1] = -INF
    dy[9, 8], dy[11, 10] = INF, math.nan
    z = z.clamp(-1, 3)            # a finite slope, and none of zero
    got = gradients(am, dy.cuda(), x.cuda(), w.cuda(), "gelu", z.cuda())
    dz = R.d(dy) * R.slope(R.d(z), "gelu")
    for g, a, b in ((got[0], dz, R.d(w)), (got[1], dz.t(), R.d(x)), (got[2][:, None], dz.t(), torch.ones(m, 1).double())):
        want, g = a @ b, g.cpu()
        assert torch.equal(torch.isnan(g), torch.isnan(want))
        assert torch.equal(torch.isposinf(g), torch.isposinf(want)) and torch.equal(torch.isneginf(g), torch.isneginf(want))


@pytest.mark.parametrize("dt", [BF16, F16])
def test_rounded_dz_on_request(am, dt):
    dy, x, w, z = inputs(300, 264, 136, dt, 7)
    args = inside(dy), inside(x), inside(w)
    dx, dw, db = gradients(am, *args, "silu", inside(z), round_dz=1)
    dz = R.d(dy) * R.slope(R.d(z), "silu")
    one = dz.float().to(dt)                   # what the products read then; a slope's error may round to the next value
    slack = 16 * R.U32 * (1 + R.d(z).abs()) * R.d(dy).abs()
    near = (dz + slack).float().to(dt) != (dz - slack).float().to(dt)
    moved = torch.where(near, 2 * R.U[dt] * dz.abs() + R.TINY[dt], torch.zeros_like(dz))
    for g, a, b, s in ((dx, R.d(one), R.d(w), moved), (dw, R.d(one).t(), R.d(x), moved.t())):
        want = a @ b
        R.close(g, want, R.sum_bound(a.shape[1], a.abs() @ b.abs()) + s @ b.abs() + R.U32 * want.abs(), "rounded")
    assert torch.equal(db, gradients(am, *args, "silu", inside(z))[2])
    # a slope of 0 or 1 leaves dz exact: nothing to choose
    for a, b in zip(gradients(am, *args, "relu", inside(z)), gradients(am, *args, "relu", inside(z), round_dz=1)):
        assert torch.equal(a, b)
    # the binding's argument
    wide = am.wfst_am_linear_backward(*args, activation="silu", pre=inside(z), weight_dtype=F32)[1]
    assert torch.equal(wide, gradients(am, *args, "silu", inside(z))[1])
    wide = am.wfst_am_linear_backward(*args, activation="silu", pre=inside(z), weight_dtype=F32, round_dz=True)[1]
    assert torch.equal(wide, dw)
