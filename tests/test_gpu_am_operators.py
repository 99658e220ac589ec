"""The acoustic-model operators against their definitions in float64.

Inputs lie inside larger buffers whose other elements are NaN, outputs inside
buffers whose other elements have to keep their value, so a read or a write
beside a matrix shows.
"""
import math

import pytest

import am_reference as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F32, F16, BF16, F8 = torch.float32, torch.float16, torch.bfloat16, torch.float8_e4m3fn
SENTINEL = 26.0   # a value of every output type
INF = float("inf")


@pytest.fixture(scope="module")
def am():
    assert torch.cuda.is_available(), "no GPU"
    from paper_1808_00687_amd import acoustic
    return acoustic


def rng(seed):
    return torch.Generator().manual_seed(seed)


def normal(g, *shape, std=1.0):
    return torch.randn(*shape, generator=g) * std


def placed(t, fill, pad=0, offset=0, after=3):
    """t on the GPU inside a larger buffer: `offset` elements before it, `pad` between rows, `after` rows behind."""
    m, n = t.shape
    flat = torch.full((offset + (m + after) * (n + pad),), fill, dtype=torch.float32).to(t.dtype).cuda()
    v = flat[offset:].as_strided((m, n), (n + pad, 1), offset)
    v.copy_(t)
    return v, flat


def inside(t, pad=0, offset=0):
    return None if t is None else placed(t, math.nan, pad, offset)[0]


class Out:
    """An output matrix whose surroundings have to stay."""

    def __init__(self, m, n, dtype, pad=0, offset=0):
        self.v, self.flat = placed(torch.full((m, n), SENTINEL).to(dtype), SENTINEL, pad, offset)
        self.pad, self.offset, self.m, self.n = pad, offset, m, n

    def check(self, tag):
        keep = torch.ones_like(self.flat, dtype=torch.bool)
        keep.as_strided((self.m, self.n), (self.n + self.pad, 1), self.offset).fill_(False)
        assert bool((self.flat.float()[keep] == SENTINEL).all()), tag + ": written beside the output"


# --------------------------------------------------------------------------
# matrix product
# --------------------------------------------------------------------------

def quantised(t):
    scale = t.abs().amax(1).clamp(min=1e-30) / R.E4M3_MAX
    return (t / scale[:, None]).clamp(-448, 448).to(F8), scale


def linear_case(am, m, k, n, dt, kind, out, seed, residual=False, pre=False, bias=True, pad=0, offset=0,
                in_place=False, out_pad=0):
    g = rng(seed)
    x, w = normal(g, m, k), normal(g, n, k, std=k ** -0.5)
    xs = ws = None
    if dt == F8:
        (x, xs), (w, ws) = quantised(x), quantised(w)
    else:
        x, w = x.to(dt), w.to(dt)
    b = normal(g, n, std=0.3) if bias else None
    r = normal(g, m, n).to(out) if residual else None
    y, z, err = R.linear(x, w, b, kind, r, xs, ws)
    yo = Out(m, n, out, out_pad, offset)
    po = Out(m, n, out, out_pad, offset) if pre else None
    rg = inside(r, out_pad, offset)
    if in_place:
        yo.v.copy_(r)
        rg = yo.v
    c = lambda t: None if t is None else t.cuda()  # noqa: E731
    am.wfst_am_linear(inside(x, pad, offset), inside(w, pad, offset), c(b), activation=kind, residual=rg, x_scale=c(xs),
                      w_scale=c(ws), pre=po.v if pre else None, out=yo.v)
    torch.cuda.synchronize()
    tag = "linear %s" % ((m, k, n, str(dt), kind, str(out), residual, pre, pad, offset),)
    mag = R.act(z, kind).abs() + (R.d(r).abs() if residual else 0)
    # the activation: its error from z's, and a few roundings of its own
    R.close(yo.v, y, R.ACT_LIPSCHITZ * err + 8 * R.U32 * (mag + z.abs()) + R.U[out] * (y.abs() + err) + R.TINY[out], tag)
    yo.check(tag)
    if pre:
        R.close(po.v, z, err + R.U[out] * (z.abs() + err) + R.TINY[out], tag + " pre")
        po.check(tag)


SHAPES = [(1, 1, 1), (1, 8, 16), (3, 5, 7), (1, 1024, 200), (2, 264, 80), (7, 40, 64), (15, 512, 33), (16, 64, 128),
          (17, 128, 31), (33, 440, 65), (64, 96, 256), (65, 200, 80), (127, 64, 300), (130, 136, 257), (256, 256, 256),
          (300, 72, 129), (333, 328, 520)]


@pytest.mark.parametrize("dt", [BF16, F16, F8])
@pytest.mark.parametrize("m,k,n", SHAPES)
def test_linear_shapes(am, m, k, n, dt):
    seed = m * 7 + k * 3 + n
    kinds = ["none", "relu", "silu", "gelu"]
    out = [F32, F16 if dt == F16 else BF16][seed % 2]
    linear_case(am, m, k, n, dt, kinds[seed % 4], out, seed, residual=seed % 3 == 0, pre=seed % 5 == 0)


@pytest.mark.parametrize("kind", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("dt,out", [(BF16, BF16), (F16, F32), (F8, F16), (F8, BF16)])
def test_linear_epilogues(am, kind, dt, out):
    linear_case(am, 70, 96, 72, dt, kind, out, 5, residual=True, pre=True)
    linear_case(am, 5, 96, 72, dt, kind, out, 6, residual=True, pre=True, in_place=True)
    linear_case(am, 70, 96, 72, dt, kind, out, 7, bias=False)


@pytest.mark.parametrize("dt", [BF16, F16, F8])
@pytest.mark.parametrize("pad,offset,out_pad", [(1, 0, 1), (8, 8, 8), (16, 3, 0), (0, 1, 5), (3, 0, 0)])
def test_linear_strides_and_alignment(am, dt, pad, offset, out_pad):
    for m, k, n in ((1, 130, 50), (20, 64, 96), (150, 192, 140), (260, 100, 264)):
        linear_case(am, m, k, n, dt, "relu", BF16, 11, residual=True, pre=True, pad=pad, offset=offset, out_pad=out_pad)


@pytest.mark.parametrize("dt", [BF16, F16])
def test_linear_long_inner(am, dt):
    linear_case(am, 3, 20000, 20, dt, "none", F32, 1)
    linear_case(am, 140, 8200, 150, dt, "none", F32, 2)


# enough tiles for the larger tile sizes, with ragged edges and a last stage of k that is not full
LARGE = [(1500, 200, 1400), (2900, 144, 3016), (2000, 1040, 2100), (1501, 203, 1403)]


@pytest.mark.parametrize("dt", [BF16, F16, F8])
@pytest.mark.parametrize("m,k,n", LARGE)
def test_linear_large_tiles(am, m, k, n, dt):
    linear_case(am, m, k, n, dt, "silu", BF16, 3, residual=True, pre=True)
    linear_case(am, m, k, n, dt, "gelu", F32, 4, bias=False, out_pad=3)


@pytest.mark.parametrize("dt", [BF16, F16])
@pytest.mark.parametrize("m,k,n", [(1500, 1400, 200), (2904, 3016, 136), (136, 2904, 3016), (1501, 1403, 70)])
def test_linear_backward_large_tiles(am, m, k, n, dt):
    backward_case(am, m, k, n, dt, "relu", 3)
    backward_case(am, m, k, n, dt, "none", 4, pad=8, weight_dtype=F32)


# at most one 128 x 128 tile a compute unit, in each of the three products; 8, 9 and 29 stages of k, the last one not full
@pytest.mark.parametrize("dt", [BF16, F16, F8])
@pytest.mark.parametrize("m,k,n", [(2040, 456, 1960), (2048, 1816, 1928), (1912, 520, 2032)])
def test_linear_one_tile_a_unit(am, m, k, n, dt):
    linear_case(am, m, k, n, dt, "relu", F32, 13, pre=True, pad=16)
    if dt != F8:
        backward_case(am, m, n, k, dt, "none", 14, pad=8)   # inner size k in dx
        backward_case(am, k, n, m, dt, "relu", 15)          # and in dw


# rows that are no whole number of 16-byte chunks, around the lengths of a chunk, a tile and a stage
@pytest.mark.parametrize("dt", [BF16, F16, F8])
@pytest.mark.parametrize("width", [1, 7, 9, 15, 17, 63, 71, 127, 129, 145])
def test_linear_ends_of_rows(am, width, dt):
    linear_case(am, 700, width, 900, dt, "none", F32, width, pad=3)
    linear_case(am, 700, 72, 900 + width, dt, "none", F32, width, offset=1)
    if dt != F8:
        for m, k, n in ((300, 264, width), (300, width, 264), (width, 129, 135)):
            backward_case(am, m, k, n, dt, "none", width, pad=3)


@pytest.mark.parametrize("m", [4, 300])
@pytest.mark.parametrize("dt", [BF16, F16, F8])
def test_linear_infinity_and_nan_stay_in_their_rows(am, m, dt):
    k, n = 200, 90
    g = rng(3)
    x, w = normal(g, m, k), normal(g, n, k)
    x[1, 199] = math.nan
    w[7, 0] = math.nan
    if dt != F8:
        x[2, 5] = INF
    x, w = x.to(dt), w.to(dt)
    one = torch.ones(max(m, n)).cuda() if dt == F8 else None
    y = am.wfst_am_linear(inside(x, 8), inside(w, 8), activation="relu", out_dtype=F32,
                          x_scale=None if one is None else one[:m], w_scale=None if one is None else one[:n])
    want = R.act(R.d(x) @ R.d(w).t(), "relu")
    y = y.cpu()
    assert torch.equal(torch.isnan(y), torch.isnan(want))
    assert torch.equal(torch.isinf(y), torch.isinf(want))


def test_linear_no_rows(am):
    y = am.wfst_am_linear(torch.empty(0, 8, dtype=BF16).cuda(), torch.ones(4, 8, dtype=BF16).cuda())
    assert y.shape == (0, 4)


def backward_case(am, m, k, n, dt, kind, seed, pad=0, offset=0, weight_dtype=None):
    g = rng(seed)
    x, w = normal(g, m, k).to(dt), normal(g, n, k, std=k ** -0.5).to(dt)
    dy, z = normal(g, m, n, std=0.1).to(dt), normal(g, m, n, std=1.5).to(dt)
    if m and n:
        z[0, 0] = 0.0
    dx, dw, db = am.wfst_am_linear_backward(inside(dy, pad, offset), inside(x, pad, offset), inside(w, pad, offset),
                                            activation=kind, pre=inside(z, pad, offset) if kind != "none" else None,
                                            weight_dtype=weight_dtype)
    torch.cuda.synchronize()
    tag = "linear backward %s" % ((m, k, n, str(dt), kind, pad, offset),)
    dz = R.d(dy) * R.slope(R.d(z), kind)
    # a smooth activation's dz is rounded to the operands' type, and its slope is good to a few float32 roundings
    u = R.U[dt] if kind in ("silu", "gelu") else 0.0
    slack = 16 * R.U32 * (1 + R.d(z).abs()) * R.d(dy).abs() if u else torch.zeros_like(dz)
    for got, a, b, s in ((dx, dz, R.d(w), slack), (dw, dz.t(), R.d(x), slack.t())):
        want = a @ b
        err = R.sum_bound(a.shape[1], a.abs() @ b.abs()) + s @ b.abs()
        err = err + R.LAMBDA * u * torch.sqrt((a * a) @ (b * b)) + R.TINY[dt] * b.abs().sum(0)
        R.close(got, want, err + R.U[got.dtype] * (want.abs() + err) + R.TINY[got.dtype], tag)
    R.close(db, dz.sum(0), R.sum_bound(m, dz.abs().sum(0)) + slack.sum(0) + R.TINY[F32], tag + " dbias")


@pytest.mark.parametrize("dt", [BF16, F16])
@pytest.mark.parametrize("m,k,n", SHAPES)
def test_linear_backward_shapes(am, m, k, n, dt):
    seed = m + k * 5 + n * 2
    backward_case(am, m, k, n, dt, ["none", "relu", "silu", "gelu"][seed % 4], seed,
                  weight_dtype=F32 if seed % 3 == 0 else None)


@pytest.mark.parametrize("dt", [BF16, F16])
@pytest.mark.parametrize("pad,offset", [(1, 0), (8, 8), (0, 3)])
def test_linear_backward_strides(am, dt, pad, offset):
    for kind in ("none", "gelu"):
        backward_case(am, 150, 72, 140, dt, kind, 4, pad=pad, offset=offset)
        backward_case(am, 3, 130, 50, dt, kind, 5, pad=pad, offset=offset)


def test_linear_backward_long_batch(am):
    # many frames, few weights: the sum over frames is long
    backward_case(am, 5000, 40, 24, BF16, "relu", 9, weight_dtype=F32)


def test_linear_backward_parts_and_no_rows(am):
    g = rng(8)
    dy, x, w = normal(g, 9, 5).to(BF16).cuda(), normal(g, 9, 6).to(BF16).cuda(), normal(g, 5, 6).to(BF16).cuda()
    whole = am.wfst_am_linear_backward(dy, x, w)
    dx, dw, db = am.wfst_am_linear_backward(dy, None, w, bias_gradient=False)
    assert dw is None and db is None and torch.equal(dx, whole[0])
    dx, dw, db = am.wfst_am_linear_backward(dy, x, None)
    assert dx is None and torch.equal(dw, whole[1]) and torch.equal(db, whole[2])
    dx, dw, db = am.wfst_am_linear_backward(dy[:0], x[:0], w, activation="silu", pre=dy[:0])
    assert dx.shape == (0, 6) and not dw.any() and not db.any()


def test_linear_gradient_against_differences(am):
    # the loss sum(y * c) in float32, its gradient by central differences of the operator's own output
    g = rng(12)
    m, k, n, h = 4, 6, 5, 2.0 ** -4
    x, w, c = normal(g, m, k).to(F16), normal(g, n, k).to(F16), normal(g, m, n).to(F16)
    x, w = (x * 16).round() / 16, (w * 16).round() / 16   # x +- h and w +- h are exact
    run = lambda a, b: float((am.wfst_am_linear(a.cuda(), b.cuda(), activation="silu", out_dtype=F32).double().cpu()  # noqa: E731
                              * c.double()).sum())
    pre = torch.empty(m, n, dtype=F16).cuda()
    am.wfst_am_linear(x.cuda(), w.cuda(), activation="silu", pre=pre, out_dtype=F16)
    dx, dw, _ = am.wfst_am_linear_backward(c.cuda(), x.cuda(), w.cuda(), activation="silu", pre=pre)
    for t, got in ((x, dx), (w, dw)):
        for i in range(t.shape[0]):
            for j in range(t.shape[1]):
                up, dn = t.clone(), t.clone()
                up[i, j] += h
                dn[i, j] -= h
                diff = (run(up, w) - run(dn, w) if t is x else run(x, up) - run(x, dn)) / (2 * h)
                # truncation: |silu'''| < 0.4 of a change of at most |c| |other|^3 h^2 / 6 a term; roundings of 16-bit dz and pre
                other = w if t is x else x
                scale = float(other.abs().max()) * float(c.abs().max()) * max(m, n)
                allowed = scale * (0.4 * h * h / 6 * float(other.abs().max()) ** 2 + 4 * R.U[F16] * 4)
                assert abs(float(got[i, j]) - diff) <= allowed, (i, j, float(got[i, j]), diff, allowed)


# --------------------------------------------------------------------------
# norm
# --------------------------------------------------------------------------

WIDTHS = [1, 2, 7, 8, 63, 64, 129, 440, 512, 1000, 1024, 2047, 4096, 5000, 9001, 20000]


def norm_bounds(s, v, width):
    # mean and root: a sum of squares, relative; then a few roundings
    return (R.LAMBDA * math.sqrt(width) + 12) * R.U32 * v.abs()


def norm_case(am, m, width, dt, out, seed, residual, gain=True, pad=0, offset=0, eps=1e-6, in_place=False, x=None):
    g = rng(seed)
    x = normal(g, m, width).to(dt) if x is None else x.to(dt)
    r = normal(g, m, width, std=3.0).to(dt) if residual else None
    gn = (1 + normal(g, width, std=0.2)) if gain else None
    s, v = R.norm(x, r, gn, eps)
    err = norm_bounds(s, v, width)
    yo, so = Out(m, width, out, pad, offset), Out(m, width, dt, pad, offset)
    rg = inside(r, pad, offset)
    if in_place:
        so.v.copy_(r)
        rg = so.v
    y, scale, total = am.wfst_am_norm(inside(x, pad, offset), None if gn is None else gn.cuda(), residual=rg, eps=eps,
                                      out=yo.v, sum_out=so.v if residual else None)
    torch.cuda.synchronize()
    tag = "norm %s" % ((m, width, str(dt), str(out), residual, pad, offset),)
    yo.check(tag)
    if residual:
        R.close(total, s, R.U32 * s.abs() + R.U[dt] * (s.abs() * (1 + R.U32)) + R.TINY[dt], tag + " sum")
        so.check(tag)
    else:
        assert total is None
    if out != F8:
        R.close(y, v, err + R.U[out] * (v.abs() + err) + R.TINY[out], tag)
        return
    top = v.abs().amax(1)
    want = torch.clamp(top / 448, min=2.0 ** -126)
    R.close(scale, want, (R.LAMBDA * math.sqrt(width) + 16) * R.U32 * want, tag + " scale")
    # y scale is within half an e4m3 spacing of v: 2^-4 relative, 2^-10 of the scale below the normals
    got = R.d(y.float()) * R.d(scale)[:, None]
    R.close(got, v, 2.0 ** -4 * v.abs() + 2.0 ** -10 * want[:, None] + 4 * err, tag)
    # the largest of a row is the largest code
    big = R.d(y.float()).abs().amax(1)
    assert bool(((big == 448) | (top < 448 * 2.0 ** -126)).all()), tag


@pytest.mark.parametrize("dt,out", [(BF16, F8), (F16, F8), (F32, F8), (BF16, BF16), (F16, F16), (F32, F32)])
@pytest.mark.parametrize("width", WIDTHS)
def test_norm_widths(am, width, dt, out):
    for m in (1, 5):
        norm_case(am, m, width, dt, out, width + m, residual=True)
        norm_case(am, m, width, dt, out, width + m, residual=False, gain=False)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("pad,offset", [(1, 0), (8, 8), (0, 1), (3, 5)])
def test_norm_strides(am, dt, pad, offset):
    for width in (65, 512, 3000):
        norm_case(am, 6, width, dt, F8, 3, True, pad=pad, offset=offset)
        norm_case(am, 6, width, dt, dt, 3, True, pad=pad, offset=offset, in_place=True)


def test_norm_many_rows(am):
    norm_case(am, 3001, 96, BF16, F8, 5, True)
    norm_case(am, 1500, 1024, BF16, F8, 6, True)


def test_norm_extreme_rows(am):
    # zeros, values far apart, the smallest, and large ones whose squares still fit float32
    x = torch.zeros(5, 300)
    x[1, 7] = 5.0
    x[2] = 2.0 ** -60
    x[3] = torch.linspace(-1e15, 1e15, 300)
    x[4, :] = 1e-3
    x[4, 0] = 1e4
    norm_case(am, 5, 300, F32, F8, 1, False, x=x)
    norm_case(am, 5, 300, F32, F32, 1, False, x=x)
    norm_case(am, 5, 300, BF16, F8, 1, False, x=x, gain=False)


@pytest.mark.parametrize("width", [40, 700, 9000])
def test_norm_infinity_and_nan_stay_in_their_rows(am, width):
    x = normal(rng(4), 4, width).to(F32)
    x[1, width - 1] = math.nan
    x[2, 3] = INF
    for out in (F8, F32):
        y, scale, _ = am.wfst_am_norm(inside(x), out_dtype=out)
        y = y.float().cpu()
        assert not torch.isnan(y[0]).any() and not torch.isnan(y[3]).any()
        assert torch.isnan(y[1]).all()
        assert torch.isnan(y[2, 3])            # infinity over infinity
        if out == F8:
            assert torch.isnan(scale[1]) and torch.isnan(scale[2]) and torch.isfinite(scale[[0, 3]]).all()
        else:
            assert not y[2, :3].any()          # finite over infinity


def norm_backward_case(am, m, width, dt, seed, ds, gain=True, pad=0, offset=0, eps=1e-6):
    g = rng(seed)
    s, dy = normal(g, m, width, std=2.0).to(dt), normal(g, m, width, std=0.1).to(dt)
    ds = normal(g, m, width, std=0.1).to(dt) if ds else None
    gn = (1 + normal(g, width, std=0.2)) if gain else None
    dx, dg = R.norm_backward(dy, s, gn, ds, eps)
    got, got_g = am.wfst_am_norm_backward(inside(dy, pad, offset), inside(s, pad, offset),
                                          None if gn is None else gn.cuda(), dsum=inside(ds, pad, offset), eps=eps)
    torch.cuda.synchronize()
    tag = "norm backward %s" % ((m, width, str(dt), pad, offset),)
    sd, u = R.d(s), R.d(dy) * (R.d(gn) if gain else 1)
    r = 1 / torch.sqrt((sd * sd).mean(1, keepdim=True) + eps)
    c = R.LAMBDA * math.sqrt(width) + 16
    err = c * R.U32 * (r * u.abs() + r ** 3 * sd.abs() * (u * sd).abs().mean(1, keepdim=True))
    if ds is not None:
        err = err + 2 * R.U32 * R.d(ds).abs()
    R.close(got, dx, err + R.U[dt] * (dx.abs() + err) + R.TINY[dt], tag)
    mag = (R.d(dy) * sd * r).abs().sum(0)
    R.close(got_g, dg, R.sum_bound(m, mag) + c * R.U32 * mag + R.TINY[F32], tag + " dgain")


@pytest.mark.parametrize("dt", [BF16, F16, F32])
@pytest.mark.parametrize("width", WIDTHS)
def test_norm_backward_widths(am, width, dt):
    for m in (1, 37):
        norm_backward_case(am, m, width, dt, width + m, ds=m == 1)


@pytest.mark.parametrize("pad,offset", [(1, 0), (8, 8), (0, 1)])
def test_norm_backward_strides(am, pad, offset):
    norm_backward_case(am, 300, 250, BF16, 3, True, pad=pad, offset=offset, gain=False)
    norm_backward_case(am, 5, 1024, F32, 3, True, pad=pad, offset=offset)


def test_norm_backward_many_rows(am):
    norm_backward_case(am, 3000, 128, BF16, 1, True)
    norm_backward_case(am, 1200, 2048, F16, 2, False)


def test_norm_backward_no_rows_and_parts(am):
    dx, dg = am.wfst_am_norm_backward(torch.empty(0, 8).cuda(), torch.empty(0, 8).cuda())
    assert dx.shape == (0, 8) and not dg.any()
    g = rng(2)
    s, dy = normal(g, 4, 100).cuda(), normal(g, 4, 100).cuda()
    dx, dg = am.wfst_am_norm_backward(dy, s, gain_gradient=False)
    assert dg is None and torch.equal(dx, am.wfst_am_norm_backward(dy, s)[0])


def test_norm_gradient_against_differences(am):
    g = rng(13)
    m, width, h = 2, 12, 2.0 ** -6
    x, gn, c = normal(g, m, width), 1 + normal(g, width, std=0.2), normal(g, m, width)
    run = lambda a, b: float((am.wfst_am_norm(a.cuda(), b.cuda())[0].double().cpu() * c.double()).sum())  # noqa: E731
    dx, dg = am.wfst_am_norm_backward(c.cuda(), x.cuda(), gn.cuda())
    for t, got in ((x, dx), (gn, dg)):
        for at in range(t.numel()):
            up, dn = t.clone().flatten(), t.clone().flatten()
            up[at] += h
            dn[at] -= h
            up, dn = up.view_as(t), dn.view_as(t)
            step = float(up.flatten()[at]) - float(dn.flatten()[at])
            diff = (run(up, gn) - run(dn, gn) if t is x else run(x, up) - run(x, dn)) / step
            # the third derivative of a unit vector's part is at most 15 / |x|^3; the loss has `width` of them
            r = float((x * x).sum(1).min()) ** 0.5 / math.sqrt(width)
            allowed = float(c.abs().max()) * width * (15 / r ** 3 / width * h * h / 6 + 32 * R.U32 / h)
            assert abs(float(got.flatten()[at]) - diff) <= allowed, (at, float(got.flatten()[at]), diff, allowed)


# --------------------------------------------------------------------------
# distillation
# --------------------------------------------------------------------------

def top_entries(g, m, n, k, distinct=True):
    idx = torch.stack([torch.randperm(n, generator=g)[:k] for _ in range(m)]) if distinct else \
        torch.randint(0, n, (m, k), generator=g)
    return idx.to(torch.int32), normal(g, m, k, std=2.0)


def distill_check(am, x, idx, top, t, w, tag, pad=0, offset=0, in_place=False):
    loss, lse, dl = R.distill(x, idx, top, t, w)
    n, dt = x.shape[1], x.dtype
    do = Out(x.shape[0], n, dt, pad, offset)
    xg = inside(x, pad, offset)
    if in_place:
        do.v.copy_(x)
        xg = do.v
    args = (idx.cuda(), inside(top, 1))
    wg = None if w is None else w.cuda()
    got_loss, got_lse, _ = am.wfst_am_distill(xg, *args, temperature=t, weight=wg, dlogits=do.v)
    torch.cuda.synchronize()
    do.check(tag)
    xd = R.d(x) / t
    top_x = xd.abs().masked_fill(xd == -INF, 0).amax(1)
    # log sum exp: roundings of x / t and of each exponent, absolute; a sum of n exponentials, relative
    e_lse = 4 * R.U32 * (2 * top_x + lse.abs().masked_fill(~torch.isfinite(lse), 0) + 1) + (R.LAMBDA * math.sqrt(n) + 4) * R.U32
    R.close(got_lse, lse, e_lse, tag + " lse")
    wd = torch.ones(x.shape[0]).double() if w is None else R.d(w)
    tmax = (R.d(top).abs().masked_fill(R.d(top) == -INF, 0).amax(1)) / t
    e_p = 4 * R.U32 * (2 * tmax + 1) + (R.LAMBDA * math.sqrt(idx.shape[1]) + 8) * R.U32
    e_loss = wd.abs() * t * t * (e_lse + 2 * e_p * (1 + tmax + 2 * top_x + lse.abs().masked_fill(~torch.isfinite(lse), 0)))
    R.close(got_loss, loss, e_loss + R.U32 * loss.abs(), tag + " loss")
    q = torch.exp(xd - lse[:, None]).nan_to_num(0)
    e_d = (wd.abs() * t)[:, None] * ((2 * e_lse + 8 * R.U32 * (1 + 2 * top_x))[:, None] * q + 4 * R.U32)
    hit = torch.zeros_like(q)
    for m in range(x.shape[0]):
        for i in idx[m].tolist():
            if 0 <= i < n:
                hit[m, i] = 1
    e_d = e_d + (wd.abs() * t)[:, None] * hit * (4 * e_p)[:, None]
    R.close(do.v, dl, e_d + R.U[dt] * (dl.abs() + e_d) + R.TINY[dt], tag + " dlogits")
    if not in_place:
        alone = am.wfst_am_distill_backward(xg, *args, got_lse, temperature=t, weight=wg)
        R.close(alone, dl, e_d + R.U[dt] * (dl.abs() + e_d) + R.TINY[dt], tag + " backward alone")
        only, _, none = am.wfst_am_distill(xg, *args, temperature=t, weight=wg)
        assert none is None and torch.equal(only, got_loss)


UNITS = [(1, 1), (2, 2), (7, 3), (64, 8), (80, 8), (129, 64), (500, 20), (1000, 1), (2000, 20), (6000, 256), (9001, 5),
         (33000, 33)]


@pytest.mark.parametrize("dt", [BF16, F16, F32])
@pytest.mark.parametrize("n,k", UNITS)
def test_distill_units(am, n, k, dt):
    g = rng(n + k)
    for m, t in ((1, 1.0), (5, 2.0)):
        idx, top = top_entries(g, m, n, k)
        w = torch.rand(m, generator=g) if m > 1 else None
        distill_check(am, normal(g, m, n, std=3.0).to(dt), idx, top.to([F32, F16, BF16][n % 3]), t, w,
                      "distill %s" % ((m, n, k, str(dt)),))


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("pad,offset", [(1, 0), (8, 8), (0, 1)])
def test_distill_strides_and_in_place(am, dt, pad, offset):
    g = rng(5)
    for n in (81, 2000, 20001):
        idx, top = top_entries(g, 4, n, 9)
        x = normal(g, 4, n, std=3.0).to(dt)
        distill_check(am, x, idx, top, 1.5, None, "distill strided %d" % n, pad, offset)
        distill_check(am, x, idx, top, 1.5, None, "distill in place %d" % n, pad, offset, in_place=True)


@pytest.mark.parametrize("n", [90, 3000, 40000])
def test_distill_entries_not_used_and_repeated(am, n):
    g = rng(6)
    m, k = 7, 12
    idx, top = top_entries(g, m, n, k)
    idx[0, 3:] = -1                      # fewer entries than k
    idx[1, :] = -1                       # none
    idx[2, 0], idx[2, 1] = n, 2 ** 31 - 1  # outside the units
    top[3, 2:] = -INF                    # no probability
    top[4, :] = -INF                     # none at all
    idx[5, :] = idx[5, 0]                # one unit, many times
    idx[6, 4:8] = idx[6, 3]
    x = normal(g, m, n, std=3.0)
    x[1, 5] = math.nan                   # nothing of a row without entries counts, but its lse
    loss, lse, dl = am.wfst_am_distill(inside(x), idx.cuda(), top.cuda(), gradient=True)
    for t in (loss, dl):
        assert not t[[1, 4]].any()
    rows = [0, 2, 3, 5, 6]
    distill_check(am, x[rows], idx[rows], top[rows], 2.0, None, "distill entries %d" % n)


@pytest.mark.parametrize("n", [90, 3000, 40000])
def test_distill_masked_frames_and_units(am, n):
    g = rng(7)
    m, k = 6, 5
    idx, top = top_entries(g, m, n, k)
    x = normal(g, m, n, std=3.0)
    w = torch.tensor([1.0, 0.0, 0.5, 0.0, 2.0, 1.0])
    x[1] = math.nan                      # padded frames hold anything
    x[3] = INF
    x[2, :] = -INF                       # masked units: all but the entries
    x[2, idx[2].long()] = 0.25
    x[4, int(idx[4, 1])] = -INF          # a masked unit that the teacher wants: infinite loss, finite gradient
    loss, lse, dl = am.wfst_am_distill(inside(x), idx.cuda(), top.cuda(), weight=w.cuda(), gradient=True)
    assert not loss[[1, 3]].any() and not dl[[1, 3]].any()
    back = am.wfst_am_distill_backward(inside(x), idx.cuda(), top.cuda(), lse, weight=w.cuda())
    assert not back[[1, 3]].any()
    assert float(loss[4]) == INF and torch.isfinite(dl[4]).all()
    rows = [0, 2, 5]
    distill_check(am, x[rows], idx[rows], top[rows], 1.0, w[rows], "distill masked %d" % n)
    # a masked unit whose share has underflowed costs nothing
    top[0, 1] = -1000.0
    x[0, int(idx[0, 1])] = -INF
    loss, _, _ = am.wfst_am_distill(inside(x[:1]), idx[:1].cuda(), top[:1].cuda())
    assert math.isfinite(float(loss[0]))


def test_distill_gradient_against_differences(am):
    g = rng(14)
    n, k, t, h = 12, 4, 2.0, 2.0 ** -5
    idx, top = top_entries(g, 1, n, k)
    x = normal(g, 1, n)
    run = lambda v: float(am.wfst_am_distill(v.cuda(), idx.cuda(), top.cuda(), temperature=t)[0].double())  # noqa: E731
    _, _, dl = am.wfst_am_distill(x.cuda(), idx.cuda(), top.cuda(), temperature=t, gradient=True)
    for i in range(n):
        up, dn = x.clone(), x.clone()
        up[0, i] += h
        dn[0, i] -= h
        diff = (run(up) - run(dn)) / (float(up[0, i]) - float(dn[0, i]))
        # t^2 times log sum exp of x / t: its third derivative is at most 1 / t^3 / 4
        allowed = t * t * (h * h / 6 / 4 / t ** 3 + 64 * R.U32 / h)
        assert abs(float(dl[0, i]) - diff) <= allowed, (i, float(dl[0, i]), diff, allowed)


# --------------------------------------------------------------------------
# log-likelihood rows
# --------------------------------------------------------------------------

def loglikes_check(am, x, prior, scale, tag, pad=0, offset=0, out_pad=0):
    want = R.loglikes(x, prior, scale)
    n = x.shape[1]
    o = Out(x.shape[0], n, F32, out_pad, offset)
    am.wfst_am_loglikes(inside(x, pad, offset), None if prior is None else prior.cuda(), scale=scale, out=o.v)
    torch.cuda.synchronize()
    o.check(tag)
    xd = R.d(x)
    mag = xd.abs().masked_fill(xd == -INF, 0)
    p = R.d(prior).abs().masked_fill(R.d(prior) == -INF, 0) if prior is not None else 0
    err = scale * R.U32 * (8 * (mag + mag.amax(1, keepdim=True) + math.log(n) + 1 + p) + R.LAMBDA * math.sqrt(n) + 4)
    R.close(o.v, want, err, tag)


@pytest.mark.parametrize("dt", [BF16, F16, F32])
@pytest.mark.parametrize("n", [1, 2, 7, 64, 80, 129, 500, 2000, 5001, 6000, 9001, 33000])
def test_loglikes_units(am, n, dt):
    g = rng(n)
    for m in (1, 9):
        loglikes_check(am, normal(g, m, n, std=3.0).to(dt), torch.log_softmax(normal(g, n), 0) if m > 1 else None,
                       0.3 if m > 1 else 1.0, "loglikes %s" % ((m, n, str(dt)),))


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("pad,offset,out_pad", [(1, 0, 0), (8, 8, 4), (0, 1, 3)])
def test_loglikes_strides(am, dt, pad, offset, out_pad):
    for n in (81, 2000, 12000):
        loglikes_check(am, normal(rng(n), 3, n).to(dt), None, 1.0, "loglikes strided %d" % n, pad, offset, out_pad)


@pytest.mark.parametrize("n", [60, 3000, 40000])
def test_loglikes_masked_units(am, n):
    g = rng(3)
    x = normal(g, 5, n, std=2.0)
    prior = torch.log_softmax(normal(g, n), 0)
    prior[4] = -INF
    x[0, : n // 2] = -INF
    x[1, :] = -INF                       # a row that leaves nothing
    x[2, 4] = -INF
    x[3] = torch.finfo(torch.float32).min  # masked by the type's lowest value
    x[3, 0] = 1.0
    got = am.wfst_am_loglikes(inside(x), prior.cuda(), scale=0.5)
    assert not torch.isnan(got).any() and not (got == INF).any()
    assert (got[1] == -INF).all() and (got[:, 4] == -INF).all()
    rows = [0, 2, 4]
    loglikes_check(am, x[rows], prior, 0.5, "loglikes masked %d" % n)


# --------------------------------------------------------------------------
# rows far apart: byte offsets past 32 bits
# --------------------------------------------------------------------------

def far(buffer, t):
    """t's values in rows 2^26 bytes apart."""
    step = (1 << 26) // t.element_size()
    v = buffer.view(t.dtype).as_strided(t.shape, (step, 1))
    v.copy_(t)
    return v


def test_rows_far_apart(am):
    m, k, n = 70, 72, 64 * 66
    g = rng(21)
    a, b, c = (torch.empty((m << 26) + (1 << 20), dtype=torch.uint8, device="cuda") for _ in range(3))
    x, w = normal(g, m, k).to(BF16), normal(g, n, k, std=k ** -0.5).to(BF16)
    y = am.wfst_am_linear(far(a, x), w.cuda(), out_dtype=F32)          # more tiles than half the chip
    want, _, err = R.linear(x, w, None, "none", None)
    R.close(y, want, err + 2 * R.U32 * want.abs(), "far linear")
    few = w[:50].contiguous().cuda()
    assert torch.equal(am.wfst_am_linear(far(a, x), few), am.wfst_am_linear(x.cuda(), few))
    dy = normal(g, m, 130).to(BF16)
    w2 = normal(g, 130, k).to(BF16).cuda()
    dx, dw, db = am.wfst_am_linear_backward(far(b, dy), far(a, x), w2)
    for got, left, right in ((dx, R.d(dy), R.d(w2)), (dw, R.d(dy).t(), R.d(x)), (db[:, None], R.d(dy).t(), torch.ones(m, 1).double())):
        want, err = left @ right, R.sum_bound(left.shape[1], left.abs() @ right.abs())
        R.close(got, want, err + R.U[got.dtype] * (want.abs() + err), "far backward")
    h, res = normal(g, m, 300).to(BF16), normal(g, m, 300).to(BF16)
    out = c.view(BF16).as_strided((m, 300), ((1 << 26) // 2, 1))
    got = am.wfst_am_norm(far(a, h), residual=far(b, res), sum_out=out, out_dtype=F8)
    for u, v in zip(got, am.wfst_am_norm(h.cuda(), residual=res.cuda(), out_dtype=F8)):
        assert torch.equal(u.float(), v.float())
    got = am.wfst_am_norm_backward(far(a, h), far(b, res))
    for u, v in zip(got, am.wfst_am_norm_backward(h.cuda(), res.cuda())):
        assert torch.equal(u, v)
    idx, top = top_entries(g, m, 300, 4)
    got = am.wfst_am_distill(far(a, h), idx.cuda(), top.cuda(), dlogits=out)
    for u, v in zip(got, am.wfst_am_distill(h.cuda(), idx.cuda(), top.cuda(), gradient=True)):
        assert torch.equal(u, v)
    assert torch.equal(am.wfst_am_loglikes(far(a, h), out=c.view(F32).as_strided((m, 300), ((1 << 26) // 4, 1))),
                       am.wfst_am_loglikes(h.cuda()))


# --------------------------------------------------------------------------
# streams, graphs, repeats
# --------------------------------------------------------------------------

def all_operators(am, s):
    """Every operator once, on the current stream."""
    h, q = s["h"], {}
    y, scale, total = am.wfst_am_norm(h, s["gain"], residual=s["res"], out_dtype=F8)
    q["u"] = am.wfst_am_linear(y, s["w8"], s["b1"], activation="gelu", x_scale=scale, w_scale=s["ws"])
    q["pre"] = torch.empty_like(total)
    q["z"] = am.wfst_am_linear(q["u"], s["w2"], s["b2"], activation="silu", residual=total, pre=q["pre"])
    q["logits"] = am.wfst_am_linear(q["z"], s["w3"], out_dtype=F32)
    q["ll"] = am.wfst_am_loglikes(q["logits"], scale=0.2)
    q["loss"], q["lse"], dl = am.wfst_am_distill(q["logits"], s["idx"], s["top"], gradient=True)
    q["dl"] = am.wfst_am_distill_backward(q["logits"], s["idx"], s["top"], q["lse"])
    q["dz"], q["dw3"], _ = am.wfst_am_linear_backward(q["dl"].to(BF16), q["z"], s["w3"])
    q["du"], q["dw2"], q["db2"] = am.wfst_am_linear_backward(q["dz"], q["u"], s["w2"], activation="silu",
                                                            pre=q["pre"])
    q["dx"], q["dg"] = am.wfst_am_norm_backward(q["dz"], total, s["gain"])
    return q


def operator_state(seed, m=70):
    g = rng(seed)
    w8, ws = quantised(normal(g, 128, 96, std=0.1))
    idx, top = top_entries(g, m, 50, 5)
    s = {"h": normal(g, m, 96).to(BF16), "res": normal(g, m, 96).to(BF16), "gain": 1 + normal(g, 96, std=0.1), "w8": w8,
         "ws": ws, "b1": normal(g, 128), "w2": normal(g, 96, 128, std=0.1).to(BF16), "b2": normal(g, 96),
         "w3": normal(g, 50, 96, std=0.3).to(BF16), "idx": idx, "top": top}
    return {k: v.cuda() for k, v in s.items()}


def same(a, b, tag):
    for k in a:
        assert torch.equal(a[k].float(), b[k].float()), "%s: %s" % (tag, k)


def test_repeats_are_identical(am):
    s = operator_state(1)
    first = all_operators(am, s)
    for _ in range(3):
        same(all_operators(am, s), first, "repeat")


def test_other_streams(am):
    s = operator_state(2)
    want = all_operators(am, s)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = all_operators(am, s)
    side.synchronize()
    same(got, want, "side stream")
    # the stream argument, as a torch stream and as a raw handle, behind work that the stream still has to do
    x = torch.zeros(2000, 512, dtype=BF16).cuda()
    w = torch.eye(512, dtype=BF16).cuda()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            x += 1
    for st in (side, side.cuda_stream):
        y = am.wfst_am_linear(x, w, stream=st)
        side.synchronize()
        assert bool((y == 20).all())


def test_graph_capture(am):
    s = operator_state(3)
    all_operators(am, s)                 # warm-up before capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = all_operators(am, s)
    for seed in (4, 5, 6):
        new = operator_state(seed)
        for k in s:
            s[k].copy_(new[k])
        graph.replay()
        torch.cuda.synchronize()
        same(got, all_operators(am, new), "replay")
