"""The gated layer and its gradients against their definitions in float64.  Inputs
lie among NaN, outputs among values that have to stay (test_gpu_am_operators.py)."""
import math

import pytest

import am_reference as R
import am_reference_more as Q
from test_gpu_am_operators import BF16, F8, F16, F32, INF, Out, far, inside, normal, quantised, rng

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def am():
    assert torch.cuda.is_available(), "no GPU"
    from paper_1808_00687_amd import acoustic
    return acoustic


def case(am, m, k, n, dt, kind, out, seed, pre=False, bias=True, pad=0, offset=0, out_pad=0):
    g = rng(seed)
    x, w = normal(g, m, k), normal(g, 2 * n, k, std=k ** -0.5)
    xs = ws = None
    if dt == F8:
        (x, xs), (w, ws) = quantised(x), quantised(w)
    else:
        x, w = x.to(dt), w.to(dt)
    b = normal(g, 2 * n, std=0.3) if bias else None
    y, z, e_z, e_y = Q.gated(x, w, b, kind, xs, ws)
    yo = Out(m, n, out, out_pad, offset)
    po = Out(m, 2 * n, out, out_pad, offset) if pre else None
    c = lambda t: None if t is None else t.cuda()  # noqa: E731
    am.wfst_am_gated(inside(x, pad, offset), inside(w, pad, offset), c(b), activation=kind, x_scale=c(xs), w_scale=c(ws),
                     pre=po.v if pre else None, out=yo.v)
    torch.cuda.synchronize()
    tag = "gated %s" % ((m, k, n, str(dt), kind, str(out), pre, pad, offset, out_pad),)
    R.close(yo.v, y, e_y + R.U[out] * (y.abs() + e_y) + R.TINY[out], tag)
    yo.check(tag)
    if pre:
        R.close(po.v, z, e_z + R.U[out] * (z.abs() + e_z) + R.TINY[out], tag + " pre")
        po.check(tag)


KINDS = ["none", "relu", "silu", "gelu"]
# few rows, each thin shape, small tiles, odd ends of rows and of columns
SHAPES = [(1, 1, 1), (1, 8, 16), (3, 5, 7), (1, 1024, 200), (2, 264, 80), (7, 40, 64), (15, 512, 33), (16, 64, 128),
          (17, 128, 31), (33, 440, 65), (64, 96, 256), (65, 200, 80), (127, 64, 300), (130, 136, 257), (256, 256, 256),
          (300, 72, 129), (333, 328, 520), (40, 520, 2100), (400, 64, 1000)]


@pytest.mark.parametrize("dt", [BF16, F16, F8])
@pytest.mark.parametrize("m,k,n", SHAPES)
def test_shapes(am, m, k, n, dt):
    seed = m + 3 * k + 7 * n
    out = (BF16 if dt == F8 else dt) if seed % 2 else F32 if dt != F8 else F16
    case(am, m, k, n, dt, KINDS[seed % 4], out, seed, pre=seed % 3 == 0, bias=seed % 5 != 0)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dt,out", [(BF16, BF16), (F16, F32), (BF16, F16), (F8, F16), (F8, BF16), (F8, F32)])
def test_epilogues(am, kind, dt, out):
    for m, k, n in ((9, 100, 70), (200, 100, 333)):
        case(am, m, k, n, dt, kind, out, 5, pre=True)
        case(am, m, k, n, dt, kind, out, 6, bias=False)


@pytest.mark.parametrize("dt", [BF16, F16, F8])
@pytest.mark.parametrize("pad,offset,out_pad", [(1, 0, 1), (8, 8, 8), (16, 3, 0), (0, 1, 5), (3, 0, 0)])
def test_strides_and_alignment(am, dt, pad, offset, out_pad):
    out = BF16 if dt == F8 else dt
    for m, k, n in ((5, 72, 40), (150, 72, 700), (700, 120, 515)):
        case(am, m, k, n, dt, "silu", out, 4, pre=True, pad=pad, offset=offset, out_pad=out_pad)


# 256 x 128 results a workgroup, 128 x 64 in one round and in several, 128 x 128, rows off 16 bytes
LARGE = [(1500, 1400, 100), (2904, 1024, 1500), (2040, 456, 980), (4096, 520, 512), (1501, 1403, 700), (3001, 200, 2005),
         (8200, 136, 2050), (1470, 328, 2040), (1921, 72, 1913)]


@pytest.mark.parametrize("dt", [BF16, F16, F8])
@pytest.mark.parametrize("m,k,n", LARGE)
def test_large_tiles(am, m, k, n, dt):
    case(am, m, k, n, dt, KINDS[(m + k) % 4], BF16 if dt == F8 else dt, 7, pre=m < 2000)


@pytest.mark.parametrize("dt", [BF16, F16, F8])
@pytest.mark.parametrize("width", [1, 7, 9, 15, 17, 63, 71, 127, 129, 145])
def test_ends_of_rows(am, width, dt):
    out = BF16 if dt == F8 else dt
    case(am, 300, width, 300, dt, "gelu", out, width)
    case(am, 300, 300, width, dt, "gelu", out, width, pre=True)
    case(am, 4, width, 50, dt, "silu", out, width)


def test_long_inner(am):
    case(am, 3, 20000, 40, BF16, "silu", F32, 1)
    case(am, 300, 9000, 260, F16, "silu", F32, 2)


@pytest.mark.parametrize("m", [4, 300, 2500])
@pytest.mark.parametrize("dt", [BF16, F16])
def test_infinity_and_nan_stay_where_they_belong(am, m, dt):
    g = rng(9)
    n = 1100
    x, w = normal(g, m, 80).to(dt), normal(g, 2 * n, 80, std=0.1).to(dt)
    want = am.wfst_am_gated(x.cuda(), w.cuda())
    x[1, 3], w[5, 2], w[n + 9, 4] = math.nan, INF, math.nan
    y = am.wfst_am_gated(x.cuda(), w.cuda())
    assert torch.isnan(y[1]).all() and torch.isnan(y[:, 9]).all()
    keep = torch.ones(m, n, dtype=torch.bool)
    keep[1], keep[:, 5], keep[:, 9] = False, False, False
    assert torch.equal(y.cpu()[keep], want.cpu()[keep])
    # an infinite gate: silu(+inf) = inf, silu(-inf) = -inf * 0
    sign = x[:, 2].float()
    for i in (0, 2, 3):
        v = float(y[i, 5])
        assert math.isinf(v) if sign[i] > 0 else math.isnan(v)


def test_no_rows(am):
    w = torch.zeros(10, 6, dtype=BF16).cuda()
    assert am.wfst_am_gated(torch.empty(0, 6, dtype=BF16).cuda(), w).shape == (0, 5)
    with pytest.raises(ValueError, match="row for each"):
        am.wfst_am_gated(torch.zeros(2, 6, dtype=BF16).cuda(), w[:9])


def test_slices_of_one_buffer(am):
    g = rng(10)
    x, w = normal(g, 300, 64).to(BF16), normal(g, 200, 64, std=0.125).to(BF16)
    wide = torch.full((300, 64 + 100 + 200), 26.0, dtype=BF16).cuda()
    wide[:, :64] = x.cuda()
    pre = torch.empty(300, 200, dtype=BF16).cuda()
    want = am.wfst_am_gated(x.cuda(), w.cuda(), pre=pre)
    got = am.wfst_am_gated(wide[:, :64], w.cuda(), out=wide[:, 64:164], pre=wide[:, 164:])
    assert torch.equal(got, want) and torch.equal(wide[:, 164:], pre) and torch.equal(wide[:, :64], x.cuda())


def test_weights_far_apart(am):
    # rows 64 MiB apart; and rows near one another, whose values are more than 1 GiB behind the gates
    g = rng(11)
    m, k = 70, 72
    x = normal(g, m, k).to(BF16)
    for n, step in ((33, 1 << 26), (600, (1 << 21) + 2048)):
        w = normal(g, 2 * n, k, std=k ** -0.5).to(BF16)
        buffer = torch.empty(2 * n * step + (1 << 20), dtype=torch.uint8, device="cuda")
        v = buffer.view(BF16).as_strided(w.shape, (step // 2, 1))
        v.copy_(w)
        many = normal(g, 1000, k).to(BF16).cuda()   # tiles
        for rows in (x.cuda(), many):
            assert torch.equal(am.wfst_am_gated(rows, v, out_dtype=F32), am.wfst_am_gated(rows, w.cuda(), out_dtype=F32))
        del buffer, v
    a, b = (torch.empty((m << 26) + (1 << 20), dtype=torch.uint8, device="cuda") for _ in range(2))
    w = normal(g, 400, k, std=k ** -0.5).to(BF16).cuda()
    out = b.view(BF16).as_strided((m, 200), (1 << 25, 1))
    pre = torch.empty(m, 400, dtype=BF16).cuda()
    want = am.wfst_am_gated(x.cuda(), w, pre=pre)
    assert torch.equal(am.wfst_am_gated(far(a, x), w, out=out), want)
    dy = normal(g, m, 200).to(BF16)
    want = am.wfst_am_gated_backward(dy.cuda(), pre, x.cuda(), w)
    got = am.wfst_am_gated_backward(far(b, dy), pre, far(a, x), w)
    # dx is the same product; dw's plan goes by where x lies: both within their bounds
    assert torch.equal(got[2], want[2])
    backward_check(am, got, dy, pre.cpu(), x, w.cpu(), "silu", "far")


# -- gradients --------------------------------------------------------------

def inputs(m, k, n, dt, seed, size=0.1):
    g = rng(seed)
    x, w = normal(g, m, k).to(dt), normal(g, 2 * n, k, std=k ** -0.5).to(dt)
    pre = normal(g, m, 2 * n, std=1.5).to(dt)
    if m:
        pre[0, 0] = 0.0
    return normal(g, m, n, std=size).to(dt), pre, x, w


def backward_check(am, got, dy, pre, x, w, kind, tag, rounded=False):
    dt = dy.dtype
    rel, least = Q.LEFT[dt]
    if rounded:
        rel, least = R.U[dt], R.TINY[dt]
    dz, slack = Q.gated_dz(dy, pre, kind)
    for v, a, b, s in ((got[0], dz, R.d(w), slack), (got[1], dz.t(), R.d(x), slack.t())):
        want, err = Q.product(a, b, s, rel, least, R.TINY[dt])
        R.close(v, want, err + R.U[v.dtype] * (want.abs() + err) + R.TINY[v.dtype], tag)
    if got[2] is not None:
        R.close(got[2], dz.sum(0), R.sum_bound(dz.shape[0], dz.abs().sum(0)) + slack.sum(0) + R.TINY[F32], tag + " dbias")


def backward_case(am, m, k, n, dt, kind, seed, pad=0, offset=0, weight_dtype=None, round_dz=False):
    dy, pre, x, w = inputs(m, k, n, dt, seed)
    got = am.wfst_am_gated_backward(inside(dy, pad, offset), inside(pre, pad, offset), inside(x, pad, offset),
                                    inside(w, pad, offset), activation=kind, weight_dtype=weight_dtype, round_dz=round_dz)
    torch.cuda.synchronize()
    assert got[0].dtype == dt and got[1].dtype == (weight_dtype or dt)
    backward_check(am, got, dy, pre, x, w, kind, "gated backward %s" % ((m, k, n, str(dt), kind, pad, offset, round_dz),), round_dz)


BACKWARD = [(1, 1, 1), (3, 130, 25), (33, 440, 33), (130, 136, 129), (300, 72, 64), (700, 264, 96), (1500, 1400, 100),
            (1501, 1403, 35), (2040, 1960, 228), (136, 2904, 1508), (5000, 40, 12)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dt", [BF16, F16])
@pytest.mark.parametrize("m,k,n", BACKWARD)
def test_backward_shapes(am, m, k, n, dt, kind):
    backward_case(am, m, k, n, dt, kind, m + k + n, weight_dtype=F32)


@pytest.mark.parametrize("dt", [BF16, F16])
@pytest.mark.parametrize("pad,offset", [(1, 0), (8, 8), (0, 3)])
def test_backward_strides(am, dt, pad, offset):
    for kind in ("none", "gelu"):
        backward_case(am, 150, 72, 70, dt, kind, 4, pad=pad, offset=offset)
        backward_case(am, 3, 130, 51, dt, kind, 5, pad=pad, offset=offset)


@pytest.mark.parametrize("dt", [BF16, F16])
def test_backward_rounded(am, dt):
    for m, k, n in ((50, 72, 40), (700, 264, 96)):
        for kind in KINDS:
            backward_case(am, m, k, n, dt, kind, 6, round_dz=True)


@pytest.mark.parametrize("n", [1, 7, 8, 63, 64, 65, 500, 513])
def test_backward_columns(am, n):
    # the pass over dy: threads side by side, strips of rows
    for m in (1, 40, 3000):
        backward_case(am, m, 24, n, BF16, "silu", n + m)


def test_backward_parts_and_no_rows(am):
    dy, pre, x, w = (t.cuda() for t in inputs(9, 6, 5, BF16, 8))
    whole = am.wfst_am_gated_backward(dy, pre, x, w)
    dx, dw, db = am.wfst_am_gated_backward(dy, pre, None, w, bias_gradient=False)
    assert dw is None and db is None and torch.equal(dx, whole[0])
    dx, dw, db = am.wfst_am_gated_backward(dy, pre, x, None)
    assert dx is None and torch.equal(dw, whole[1]) and torch.equal(db, whole[2])
    dx, dw, db = am.wfst_am_gated_backward(dy, pre, None, None)
    assert dx is None and dw is None and torch.equal(db, whole[2])
    dx, dw, db = am.wfst_am_gated_backward(dy[:0], pre[:0], x[:0], w)
    assert dx.shape == (0, 6) and dw.shape == (10, 6) and not dw.any() and not db.any()


def test_backward_range_of_f16(am):
    # large and small dz are held, up to magnitudes of 131,008: with one above it a row of dw is infinite or NaN
    dy, pre, x, w = inputs(40, 24, 20, F16, 9)
    for scale_dy, scale_v in ((2.0 ** 12, 2.0 ** 6), (2.0 ** -12, 2.0 ** -10)):
        a = (dy.float() * scale_dy).to(F16)
        p = pre.clone()
        p[:, 20:] = (pre[:, 20:].float() * scale_v).to(F16)
        got = am.wfst_am_gated_backward(a.cuda(), p.cuda(), x.cuda(), w.cuda(), weight_dtype=F32)
        dz, slack = Q.gated_dz(a, p, "silu")
        held = (dz.abs() < 131008).all(0)
        assert held.sum() >= 36
        want, err = Q.product(dz.t()[held], R.d(x), slack.t()[held], *Q.LEFT[F16], R.TINY[F16])
        R.close(got[1].cpu()[held], want, err + R.U32 * want.abs(), "range")
        assert not torch.isfinite(got[1].cpu()[~held]).any()
    # above it dx is infinite or NaN, and dbias is not
    a = torch.full((2, 1), 60000.0, dtype=F16).cuda()
    p = torch.tensor([[1.0, 1000.0]] * 2, dtype=F16).cuda()
    dx, dw, db = am.wfst_am_gated_backward(a, p, torch.ones(2, 1, dtype=F16).cuda(), torch.ones(2, 1, dtype=F16).cuda(),
                                           activation="none", weight_dtype=F32)
    assert not torch.isfinite(dw[0]).any() and torch.equal(db.cpu(), torch.tensor([1.2e8, 120000.0]))


def test_gradient_against_differences(am):
    # central differences of L = sum(y c) in float64; inputs are exact in float16
    g = rng(12)
    m, k, n, h = 4, 6, 3, 1e-4
    x, w, c = normal(g, m, k).to(F16).double(), normal(g, 2 * n, k).to(F16).double(), normal(g, m, n).to(F16).double()

    def loss(x, w):
        z = x @ w.t()
        return (R.act(z[:, :n], "silu") * z[:, n:] * c).sum()

    pre = torch.empty(m, 2 * n, dtype=F16).cuda()
    xg, wg = x.to(F16).cuda(), w.to(F16).cuda()
    am.wfst_am_gated(xg, wg, pre=pre)
    dx, dw, _ = am.wfst_am_gated_backward(c.to(F16).cuda(), pre, xg, wg, weight_dtype=F32)
    for t, got in (("x", dx), ("w", dw)):
        base = {"x": x, "w": w}
        want = torch.zeros(got.shape).double()
        for i in range(want.numel()):
            step = torch.zeros_like(base[t]).reshape(-1)
            step[i] = h
            up, down = ({**base, t: base[t] + s * step.view(base[t].shape)} for s in (1, -1))
            want.view(-1)[i] = (loss(**up) - loss(**down)) / (2 * h)
        # pre is rounded to float16: a term dy act' value moves by at most |dy| (|value| act'' + 2 act') times its
        # rounding, |pre| 2^-11; act'' and act' are at most 1.1.  Third derivatives give h^2 times less than 1e3
        big = float(pre.abs().max())
        other = w if t == "x" else x
        slack = float(c.abs().max()) * 1.1 * (big + 2) * big * R.U[F16] * float(other.abs().max()) * max(m, 2 * n)
        R.close(got, want, slack + 1e3 * h * h + R.U[got.dtype] * want.abs().max(), t)


def test_repeats_streams_and_graphs(am):
    s = [t.cuda() for t in inputs(1300, 264, 200, BF16, 1)]
    bias = normal(rng(2), 400).cuda()

    def both(dy, pre, x, w):
        y = am.wfst_am_gated(x, w, bias)
        return (y, *am.wfst_am_gated_backward(dy, pre, x, w))

    want = both(*s)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(both(*s), want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = both(*s)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    for st in (side, side.cuda_stream):
        y = am.wfst_am_gated(s[2], s[3], bias, stream=st)
        side.synchronize()
        assert torch.equal(y, want[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both(*s)
    for seed in (4, 5, 6):
        new = [t.cuda() for t in inputs(1300, 264, 200, BF16, seed)]
        for a, b in zip(s, new):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, both(*new)))
