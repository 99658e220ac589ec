"""The layer norm and its gradients against their definitions in float64.  Inputs
lie among NaN, outputs among values that have to stay (test_gpu_am_operators.py)."""
import math

import pytest

import am_reference as R
import am_reference_more as Q
from test_gpu_am_operators import BF16, F8, F16, F32, INF, Out, inside, normal, rng

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def am():
    assert torch.cuda.is_available(), "no GPU"
    from paper_1808_00687_amd import acoustic
    return acoustic


WIDTHS = [1, 2, 7, 8, 9, 15, 63, 64, 65, 129, 255, 257, 440, 511, 513, 1000, 1024, 1025, 1300, 1536, 1537, 2048, 2500, 4097, 5000, 6145, 8192, 9001, 16384, 20000]


def check(am, x, r, gain, bias, out, tag, pad=0, offset=0, eps=1e-5, in_place=False):
    m, width = x.shape
    dt = x.dtype
    s, v, err = Q.layer_norm(x, r, gain, bias, eps)
    yo, so = Out(m, width, out, pad, offset), Out(m, width, dt, pad, offset)
    rg = inside(r, pad, offset)
    if in_place:
        so.v.copy_(r)
        rg = so.v
    y, scale, total = am.wfst_am_layer_norm(
        inside(x, pad, offset), None if gain is None else gain.cuda(), None if bias is None else bias.cuda(),
        residual=rg, eps=eps, out=yo.v, sum_out=so.v if r is not None else None)
    torch.cuda.synchronize()
    tag = "layer norm %s %s" % (tag, (m, width, str(dt), str(out), r is not None, pad, offset))
    yo.check(tag)
    if r is not None:
        R.close(total, s, R.U32 * s.abs() + R.U[dt] * (s.abs() * (1 + R.U32)) + R.TINY[dt], tag + " sum")
        so.check(tag)
    else:
        assert total is None
    if out != F8:
        assert scale is None
        R.close(y, v, err + R.U[out] * (v.abs() + err) + R.TINY[out], tag)
        return
    top, e_top = v.abs().amax(1), err.amax(1)
    want = torch.clamp(top / 448, min=2.0 ** -126)
    R.close(scale, want, (e_top + 2 * R.U32 * top) / 448, tag + " scale")
    # y scale is within half an e4m3 spacing of v: 2^-4 relative, 2^-10 of the scale below the normals
    got = R.d(y.float()) * R.d(scale)[:, None]
    step = 2.0 ** -4 * (v.abs() + err) + 2.0 ** -10 * (want + e_top / 448)[:, None]
    R.close(got, v, step * (1 + 2.0 ** -20) + err + (v.abs() / top.clamp(min=1e-300)[:, None]) * e_top[:, None], tag)
    big = R.d(y.float()).abs().amax(1)
    assert bool(((big == 448) | (top < 448 * 2.0 ** -126)).all()), tag


def case(am, m, width, dt, out, seed, residual, affine=True, mean=0.0, **kw):
    g = rng(seed)
    x = (normal(g, m, width) + mean).to(dt)
    r = normal(g, m, width, std=3.0).to(dt) if residual else None
    gain = 1 + normal(g, width, std=0.2) if affine else None
    bias = normal(g, width, std=0.2) if affine else None
    check(am, x, r, gain, bias, out, "seed %d" % seed, **kw)


@pytest.mark.parametrize("dt,out", [(BF16, F8), (F16, F8), (F32, F8), (BF16, BF16), (F16, F16), (F32, F32)])
@pytest.mark.parametrize("width", WIDTHS)
def test_widths(am, width, dt, out):
    for m in (1, 5):
        case(am, m, width, dt, out, width + m, residual=True)
        case(am, m, width, dt, out, width + m, residual=False, affine=False)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("pad,offset", [(1, 0), (8, 8), (0, 1), (3, 5)])
def test_strides(am, dt, pad, offset):
    for width in (63, 250, 1024, 5000):
        case(am, 9, width, dt, F8, 3, True, pad=pad, offset=offset)
        case(am, 9, width, dt, dt, 4, True, pad=pad, offset=offset, in_place=True)


@pytest.mark.parametrize("dt,out", [(BF16, F32), (F16, F32), (F32, BF16), (F32, F16), (BF16, F16), (F16, BF16)])
@pytest.mark.parametrize("width", [1, 7, 64, 1000, 2047, 5000, 9001, 20000])
def test_result_of_another_type(am, width, dt, out):
    case(am, 5, width, dt, out, width, residual=True)
    case(am, 6, width, dt, out, 3, False, pad=3, offset=5)


def test_many_rows(am):
    # workgroups take several rows in turn
    case(am, 40000, 96, BF16, F8, 1, True)
    case(am, 9000, 2048, BF16, BF16, 2, True, in_place=True)
    case(am, 4500, 17000, BF16, F8, 3, False)


@pytest.mark.parametrize("width", [50, 1000, 5000, 20000])
def test_rows_far_from_zero(am, width):
    # the mean's own rounding would be 2^-24 of 1e4 and more; differences are exact but for their own bits
    case(am, 5, width, F32, F32, 7, residual=False, mean=1e4)
    case(am, 5, width, BF16, F32, 8, residual=False, mean=300.0)


@pytest.mark.parametrize("out", [F32, F8])
@pytest.mark.parametrize("width", [1, 30, 1500, 20000])
def test_rows_of_one_value(am, width, out):
    # no deviation: the bias itself; with none, zeros
    g = rng(width)
    x = torch.tensor([0.0, 1.0, -3.5, 1024.0])[:, None].expand(4, width).contiguous()
    check(am, x, None, None, None, out, "constant")
    y, _, _ = am.wfst_am_layer_norm(x.cuda())
    assert not y.any()
    bias = normal(g, width)
    y, _, _ = am.wfst_am_layer_norm(x.cuda(), bias=bias.cuda())
    assert torch.equal(y.cpu(), bias.expand(4, width))


def test_extreme_rows(am):
    g = rng(5)
    x = normal(g, 6, 700)
    x[0] *= 1e-20
    x[1] *= 1e17
    x[2, 1:] = 0
    x[3] = 0
    x[3, 9] = 1e-42
    check(am, x, None, 1 + normal(g, 700, std=0.2), normal(g, 700, std=0.2), F32, "extreme", eps=1e-12)
    check(am, x, None, None, None, F8, "extreme", eps=1e-12)


@pytest.mark.parametrize("width", [40, 700, 9000, 17000])
def test_infinity_and_nan_stay_in_their_rows(am, width):
    g = rng(6)
    x = normal(g, 7, width)
    want, _, _ = am.wfst_am_layer_norm(x.cuda())
    x[1, 3], x[4, width - 1] = INF, math.nan
    y, _, _ = am.wfst_am_layer_norm(x.cuda())
    for m in range(7):
        if m in (1, 4):
            assert torch.isnan(y[m]).all()
        else:
            assert torch.equal(y[m], want[m])
    y, scale, _ = am.wfst_am_layer_norm(x.cuda(), out_dtype=F8)
    assert torch.isnan(scale[[1, 4]]).all() and torch.isfinite(scale[[0, 2, 3, 5, 6]]).all()


def test_no_rows(am):
    y, scale, total = am.wfst_am_layer_norm(torch.empty(0, 8).cuda(), residual=torch.empty(0, 8).cuda(), out_dtype=F8)
    assert y.shape == (0, 8) and scale.shape == (0,) and total.shape == (0, 8)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("width", [65, 1500, 9000, 33000])
def test_sum_in_place(am, width, dt):
    g = rng(width)
    x, r = normal(g, 6, width).to(dt).cuda(), normal(g, 6, width).to(dt).cuda()
    for out in (F8, dt):
        want = am.wfst_am_layer_norm(x, residual=r, out_dtype=out)
        place = x.clone()
        got = am.wfst_am_layer_norm(place, residual=r, out_dtype=out, sum_out=place)
        assert got[2] is place
        for a, b in zip(got, want):
            assert a is None and b is None or torch.equal(a.float(), b.float())


# -- gradients --------------------------------------------------------------

def backward_case(am, m, width, dt, seed, ds, gain=True, pad=0, offset=0, eps=1e-5, mean=0.5):
    g = rng(seed)
    s, dy = (normal(g, m, width, std=2.0) + mean).to(dt), normal(g, m, width, std=0.1).to(dt)
    ds = normal(g, m, width, std=0.1).to(dt) if ds else None
    gn = (1 + normal(g, width, std=0.2)) if gain else None
    dx, dg, db, e_dx, e_dg, e_db = Q.layer_norm_backward(dy, s, gn, ds, eps)
    got, got_g, got_b = am.wfst_am_layer_norm_backward(inside(dy, pad, offset), inside(s, pad, offset),
                                                       None if gn is None else gn.cuda(), dsum=inside(ds, pad, offset), eps=eps)
    torch.cuda.synchronize()
    tag = "layer norm backward %s" % ((m, width, str(dt), pad, offset),)
    R.close(got, dx, e_dx + R.U[dt] * (dx.abs() + e_dx) + R.TINY[dt], tag)
    R.close(got_g, dg, e_dg + R.TINY[F32], tag + " dgain")
    R.close(got_b, db, e_db + R.TINY[F32], tag + " dbias")


@pytest.mark.parametrize("dt", [BF16, F16, F32])
@pytest.mark.parametrize("width", WIDTHS)
def test_backward_widths(am, width, dt):
    for m in (1, 37):
        backward_case(am, m, width, dt, width + m, ds=m == 1)


@pytest.mark.parametrize("dt", [BF16, F16, F32])
@pytest.mark.parametrize("width", [32768, 32769, 40001])
def test_backward_long_rows(am, width, dt):
    for m, ds, gain in ((1, True, True), (7, False, True), (200, True, False)):
        backward_case(am, m, width, dt, width + m, ds, gain=gain, pad=m % 2, offset=m % 3)


@pytest.mark.parametrize("pad,offset", [(1, 0), (8, 8), (0, 1)])
def test_backward_strides(am, pad, offset):
    backward_case(am, 300, 250, BF16, 3, True, pad=pad, offset=offset, gain=False)
    backward_case(am, 5, 1024, F32, 3, True, pad=pad, offset=offset)


def test_backward_many_rows(am):
    backward_case(am, 30000, 64, BF16, 1, True)
    backward_case(am, 3300, 2048, F16, 2, False)
    backward_case(am, 1700, 5000, F32, 3, True)
    backward_case(am, 1700, 33000, BF16, 4, True)


def test_backward_rows_far_from_zero(am):
    for width in (50, 1000, 5000):
        backward_case(am, 9, width, F32, 1, False, mean=1e4)


@pytest.mark.parametrize("width", [8, 33000])
def test_backward_no_rows_and_parts(am, width):
    e = torch.empty(0, width).cuda()
    dx, dg, db = am.wfst_am_layer_norm_backward(e, e.clone())
    assert dx.shape == (0, width) and not dg.any() and not db.any()
    g = rng(1)
    s, dy = normal(g, 70, width).cuda(), normal(g, 70, width).cuda()
    whole = am.wfst_am_layer_norm_backward(dy, s)
    for gain in (True, False):
        for bias in (True, False):
            part = am.wfst_am_layer_norm_backward(dy, s, gain_gradient=gain, bias_gradient=bias)
            assert torch.equal(part[0], whole[0])
            for want, asked, got in ((whole[1], gain, part[1]), (whole[2], bias, part[2])):
                assert got is None if not asked else torch.equal(got, want)


@pytest.mark.parametrize("width", [1, 40])
def test_backward_rows_of_one_value(am, width):
    # h is 0: dx is (u - mean u) / sqrt(eps)
    s, dy = torch.full((3, width), 2.5), normal(rng(2), 3, width)
    dx, dg, db = am.wfst_am_layer_norm_backward(dy.cuda(), s.cuda(), eps=0.25)
    want = 2 * (R.d(dy) - R.d(dy).mean(1, keepdim=True))
    R.close(dx, want, 2 * R.sum_bound(width, R.d(dy).abs().amax()) + 4 * R.U32 * want.abs(), "one value")
    assert not dg.any()


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("m,width", [(6, 65), (900, 1500), (6, 9000), (5, 33000)])
def test_gradient_in_place(am, m, width, dt):
    g = rng(width)
    s, dy, ds = (normal(g, m, width, std=v).to(dt) for v in (2.0, 0.1, 0.1))
    gain = (1 + normal(g, width, std=0.2)).cuda()
    dx, dg, db = am.wfst_am_layer_norm_backward(dy.cuda(), s.cuda(), gain, dsum=ds.cuda())
    for over in ("dy", "dsum"):
        t = {"dy": inside(dy, 5), "s": inside(s, 5), "dsum": inside(ds, 5)}
        got, got_b = torch.empty(width).cuda(), torch.empty(width).cuda()
        head = []
        for name in ("dy", "s", "dsum", over):
            head += am._matrix(t[name], name, 0)
        head += [gain.data_ptr(), got.data_ptr(), got_b.data_ptr()]
        pack = am._PACK["layer_norm_backward"].pack
        need = am._bytes_for("wfst_am_layer_norm_backward_workspace", pack(*head, 0, 0, 1e-5, 0))
        work = torch.empty(need, dtype=torch.uint8, device="cuda")
        am._call("wfst_am_layer_norm_backward", pack(*head, work.data_ptr(), need, 1e-5, 0), torch.cuda.current_stream().cuda_stream)
        assert torch.equal(t[over], dx) and torch.equal(got, dg) and torch.equal(got_b, db), over


def test_gradient_against_differences(am):
    # central differences of L = sum(y w) in float64 around the inputs; the step's error is h^2 of third derivatives
    g = rng(8)
    m, width, eps, h = 3, 12, 1e-5, 1e-4
    x, w, gain = normal(g, m, width).double(), normal(g, m, width).double(), (1 + normal(g, width, std=0.2)).double()

    def loss(x, gain, bias):
        mean = x.mean(1, keepdim=True)
        return (((x - mean) / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + eps) * gain + bias) * w).sum()

    dx, dg, db = am.wfst_am_layer_norm_backward(w.float().cuda(), x.float().cuda(), gain.float().cuda(), eps=eps)
    zero = torch.zeros(width).double()
    for got, at in ((dx, "x"), (dg, "gain"), (db, "bias")):
        base = {"x": x, "gain": gain, "bias": zero}
        want = torch.zeros(got.shape).double()
        for i in range(want.numel()):
            step = torch.zeros_like(base[at]).reshape(-1)
            step[i] = h
            step = step.view(base[at].shape)
            up, down = ({**base, at: base[at] + sign * step} for sign in (1, -1))
            want.view(-1)[i] = (loss(**up) - loss(**down)) / (2 * h)
        # inputs were rounded to float32 for the kernel (2^-24 relative), third derivatives are below 1e3 here
        R.close(got, want, 1e3 * h * h / 6 + 1e-5 * want.abs().max(), at)
