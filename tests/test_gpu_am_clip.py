"""The norm of many tensors and their clipping, against float64.  Inputs lie among
NaN, outputs among values that have to stay (test_gpu_am_operators.py).

Bounds: the squares' sum and the factor are held in float64, so the norm has one
float32 rounding; an output has that of the product and that of its type."""
import math

import pytest

import am_reference as R
from test_gpu_am_operators import BF16, F16, F32, INF, Out, far, inside, normal, rng

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def am():
    assert torch.cuda.is_available(), "no GPU"
    from paper_1808_00687_amd import acoustic
    return acoustic


def reference(ts):
    return math.sqrt(math.fsum(float((R.d(t) ** 2).sum()) for t in ts))


def compare(out, norm, ts, max_norm, tag):
    want = reference(ts)
    assert abs(float(norm) - want) <= R.U32 * want * (1 + 1e-6) + 2.0 ** -150, (tag, float(norm), want)
    factor = max_norm / want if want > max_norm else 1.0
    for i, (o, t) in enumerate(zip(out, ts)):
        v = R.d(t) * factor
        R.close(o, v, R.U32 * v.abs() * 1.001 + (0 if t.dtype == F32 else R.U[t.dtype] * v.abs() * (1 + R.U32)) + 2 * R.TINY[t.dtype],
                "%s tensor %d" % (tag, i))


def check(am, ts, share, tag, pad=0, offset=0):
    """Out of place and in place, matrices inside larger buffers."""
    max_norm = share * reference(ts)
    outs = [Out(*t.shape, t.dtype, pad, offset) for t in ts]
    got, norm = am.wfst_am_clip([inside(t, pad, offset) for t in ts], max_norm, out=[o.v for o in outs])
    torch.cuda.synchronize()
    assert all(g is o.v for g, o in zip(got, outs))
    compare(got, norm, ts, max_norm, tag)
    here = [Out(*t.shape, t.dtype, pad, offset) for t in ts]
    for o, t in zip(here, ts):
        o.v.copy_(t)
    again, norm2 = am.wfst_am_clip([o.v for o in here], max_norm)
    torch.cuda.synchronize()
    assert torch.equal(norm, norm2)
    for i, (o, h, t) in enumerate(zip(outs, here, ts)):
        assert torch.equal(o.v, h.v), "%s: in place differs at %d" % (tag, i)
        o.check("%s %d" % (tag, i))
        h.check("%s %d" % (tag, i))


SHAPES = [(1, 1), (1, 7), (3, 5), (0, 4), (1, 8191), (1, 8192), (1, 8193), (1, 4095), (1, 4096), (1, 4097), (64, 128),
          (65, 129), (1000, 3), (7, 3001), (1, 100003), (300, 300)]


@pytest.mark.parametrize("share", [0.01, 0.5, 3.0])
@pytest.mark.parametrize("dt", [BF16, F16, F32])
def test_shapes(am, dt, share):
    g = rng(1)
    check(am, [normal(g, *s, std=0.1).to(dt) for s in SHAPES], share, "shapes")
    for s in SHAPES:
        if s[0]:
            check(am, [normal(g, *s).to(dt)], share, str(s))


@pytest.mark.parametrize("pad,offset", [(1, 0), (8, 8), (0, 1), (5, 3), (0, 5)])
def test_strides_and_alignment(am, pad, offset):
    g = rng(2)
    for dts in ((BF16,), (F32,), (F16, F32, BF16)):
        check(am, [normal(g, *s).to(dts[i % len(dts)]) for i, s in enumerate(SHAPES)], 0.5, "strides", pad, offset)


@pytest.mark.parametrize("count", [70, 71, 72, 142, 143, 500])
def test_many_tensors(am, count):
    g = rng(count)
    ts = [normal(g, 1 + i % 5, 1 + (i * 37) % 900, std=1.0 + i % 3).to((BF16, F32, F16)[i % 3]) for i in range(count)]
    ts[count // 2] = normal(g, 700, 611).to(BF16)
    ts[3] = torch.empty(0, 5)
    check(am, ts, 0.25, "many")


def test_large_tensors(am):
    # more chunks than workgroups, so each takes a run of them over several tensors
    g = rng(3)
    for count in (1, 90):
        ts = [normal(g, 3000, 7001).to(BF16), normal(g, 1, 40000003 // count, std=0.5), normal(g, 50, 33),
              normal(g, 2048, 8192, std=2.0).to(F16)] + [normal(g, 1, 300) for _ in range(count)]
        check(am, ts, 0.5, "large")


def test_any_shape(am):
    g = rng(4)
    ts = [torch.tensor(0.75).cuda(), normal(g, 5).cuda(), normal(g, 3, 4, 5).cuda(), normal(g, 2, 0, 3).cuda(), normal(g, 9, 1).cuda()]
    want = [t.clone() for t in ts]
    got, norm = am.wfst_am_clip(ts, 0.5)
    assert got is ts
    compare(ts, norm, want, 0.5, "any shape")
    # an input of another order is copied where it is not written
    t = normal(g, 40, 30).cuda()
    out = torch.empty(30, 40).cuda()
    _, norm = am.wfst_am_clip([t.t()], 1.0, out=[out])
    compare([out], norm, [t.t()], 1.0, "transposed")
    with pytest.raises(ValueError, match="adjacent"):
        am.wfst_am_clip([t.t()], 1.0)
    # dense outputs of as many values, and matrices beside dense tensors
    flat = torch.empty(1200).cuda()
    _, norm = am.wfst_am_clip([t], 1.0, out=[flat])
    compare([flat.view(40, 30)], norm, [t], 1.0, "flat")
    wide = torch.empty(40, 35).cuda()
    _, norm = am.wfst_am_clip([t], 1.0, out=[wide[:, :30]])
    compare([wide[:, :30]], norm, [t], 1.0, "into columns")
    wide[:, :30] = t
    _, norm = am.wfst_am_clip([wide[:, :30], t], 1.0, out=[flat.view(40, 30), torch.empty_like(t)])
    compare([flat.view(40, 30)], norm / math.sqrt(2), [t], 1.0 / math.sqrt(2), "from columns")
    from paper_1808_00687_amd import wfstdec
    column = torch.empty(1200, 2).cuda()[:, :1]
    _, norm = am.wfst_am_clip([t], 1.0, out=[column])
    compare([column.reshape(40, 30)], norm, [t], 1.0, "into one column")
    for out in ([torch.empty(30, 39).cuda()], [flat[:1199]], [torch.empty(1201, 2).cuda()[:, :1]]):
        with pytest.raises(wfstdec.WfstError, match="shape"):
            am.wfst_am_clip([t], 1.0, out=out)
    for out in ([flat, flat], flat, []):
        with pytest.raises(ValueError, match="as many"):
            am.wfst_am_clip([t], 1.0, out=out)
    with pytest.raises(wfstdec.WfstError, match="type"):
        am.wfst_am_clip([t], 1.0, out=[t.bfloat16()])
    with pytest.raises(ValueError, match="requires a gradient"):
        am.wfst_am_clip([t, torch.zeros(3, requires_grad=True, device="cuda")], 1.0)
    with pytest.raises(ValueError, match="one GPU"):
        am.wfst_am_clip([t, torch.zeros(3)], 1.0)
    with pytest.raises(TypeError, match="int32"):
        am.wfst_am_clip([t, torch.zeros(3, dtype=torch.int32).cuda()], 1.0)


def test_more_than_31_bits_of_values(am):
    # 2^31 + 26 values of 0.5: the norm is exact but for its root, a factor of 1 / 16 is exact
    t = torch.full((2, (1 << 30) + 13), 0.5, dtype=BF16, device="cuda")
    want = 0.5 * math.sqrt(t.numel())
    _, norm = am.wfst_am_clip([t], want / 16)
    assert abs(float(norm) - want) <= R.U32 * want * 1.001
    assert float(t.min()) == float(t.max()) == 0.5 / 16


def test_what_is_within_the_limit_is_not_written(am):
    g = rng(5)
    t = normal(g, 300, 200).to(BF16).cuda()
    t[0, 0] = -0.0
    bits = t.view(torch.int16).clone()
    for limit in (1e6, INF):
        _, norm = am.wfst_am_clip([t], limit)
        assert torch.equal(t.view(torch.int16), bits)
        out = torch.empty_like(t)
        am.wfst_am_clip([t], limit, out=[out])
        assert torch.equal(out.view(torch.int16), bits)
    # a norm that is the limit itself
    t = torch.full((2, 2), 3.0).cuda()
    _, norm = am.wfst_am_clip([t], 6.0)
    assert float(norm) == 6.0 and bool((t == 3).all())
    _, norm = am.wfst_am_clip([t], math.nextafter(6.0, 0))
    assert float(norm) == 6.0 and bool((t <= 3).all())


def test_zeros_and_no_values(am):
    z = torch.zeros(40, 50).cuda()
    _, norm = am.wfst_am_clip([z], 1e-30)
    assert float(norm) == 0 and not z.any()
    _, norm = am.wfst_am_clip([torch.empty(0, 3).cuda(), torch.empty(0).cuda()], 1.0)
    assert float(norm) == 0


def test_range(am):
    g = rng(6)
    # squares below and above float32, and beside them
    check(am, [normal(g, 30, 40, std=1e-25), normal(g, 3, 4, std=1e-30)], 0.5, "small")
    check(am, [normal(g, 30, 40, std=1e30), normal(g, 3, 400, std=1e-30)], 1e-28, "large")
    check(am, [normal(g, 30, 40, std=1e30).to(BF16), normal(g, 3, 400).to(F16)], 1e-30, "large bf16")
    big = torch.full((4, 4), 3e38)
    out = torch.empty(4, 4).cuda()
    _, norm = am.wfst_am_clip([big.cuda()], 8.0, out=[out])
    assert float(norm) == INF
    R.close(out, torch.full((4, 4), 2.0).double(), 2.0 ** -23, "norm above float32")


def test_infinity_and_nan(am):
    g = rng(7)
    a, b = normal(g, 50, 60), normal(g, 9)
    for dt in (F32, BF16, F16):
        x, y = a.to(dt).cuda(), b.cuda()
        x[3, 5] = INF
        out = [torch.empty_like(x), torch.empty_like(y)]
        _, norm = am.wfst_am_clip([x, y], 1.0, out=out)
        assert float(norm) == INF and torch.isnan(out[0][3, 5])
        out[0][3, 5] = 0
        assert not out[0].any() and not out[1].any()
        _, norm = am.wfst_am_clip([x, y], INF, out=out)
        assert float(norm) == INF and torch.equal(out[0], x) and torch.equal(out[1], y)
        x[3, 5] = math.nan
        _, norm = am.wfst_am_clip([x, y], 1.0, out=out)
        assert torch.isnan(norm).all() and torch.equal(out[1], y) and torch.isnan(out[0][3, 5])
        out[0][3, 5] = x[3, 5] = 1
        assert torch.equal(out[0], x)


def test_a_tensor_twice(am):
    t = normal(rng(8), 30, 40)
    x, out = t.cuda(), [torch.empty(30, 40).cuda() for _ in range(2)]
    _, norm = am.wfst_am_clip([x, x], 1.0, out=out)
    compare(out, norm, [t, t], 1.0, "twice")
    from paper_1808_00687_amd import wfstdec
    with pytest.raises(wfstdec.WfstError, match="overlaps"):
        am.wfst_am_clip([x, x], 1.0)
    with pytest.raises(wfstdec.WfstError, match="overlaps"):
        am.wfst_am_clip([x, x], 1.0, out=[x, out[0]])


def test_slices_of_one_buffer(am):
    g = rng(9)
    whole = normal(g, 100, 64).to(BF16)
    x = whole.cuda()
    parts, at = [], 0
    for w in (1, 7, 8, 16, 32):
        parts.append((at, at + w))
        at += w
    _, norm = am.wfst_am_clip([x[:, a:b] for a, b in parts], 2.0)
    compare([x[:, a:b] for a, b in parts], norm, [whole[:, a:b] for a, b in parts], 2.0, "slices")


def test_rows_far_apart(am):
    t = normal(rng(10), 70, 300).to(BF16)
    a, b = (torch.empty((70 << 26) + (1 << 20), dtype=torch.uint8, device="cuda") for _ in range(2))
    v, o = far(a, t), far(b, t)
    _, norm = am.wfst_am_clip([v], 3.0, out=[o])
    compare([o], norm, [t], 3.0, "far")


def test_repeats_streams_and_graphs(am):
    g = rng(11)
    for count in (5, 100):
        ts = [normal(g, 1 + i % 7, 3000).to((BF16, F32)[i % 2]).cuda() for i in range(count)]
        out = [torch.empty_like(t) for t in ts]
        want, norm = am.wfst_am_clip(ts, 1.0, out=out)
        want = [w.clone() for w in want]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        for st in (side, side.cuda_stream):
            for o in out:
                o.zero_()
            side.wait_stream(torch.cuda.current_stream())
            _, again = am.wfst_am_clip(ts, 1.0, out=out, stream=st)
            side.synchronize()
            assert torch.equal(norm, again) and all(torch.equal(a, b) for a, b in zip(out, want))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            _, captured = am.wfst_am_clip(ts, 1.0, out=out)
        for seed in (1, 2, 3):
            for i, t in enumerate(ts):
                t.copy_(normal(rng(100 * seed + i), *t.shape))
            graph.replay()
            torch.cuda.synchronize()
            want, norm = am.wfst_am_clip(ts, 1.0, out=[torch.empty_like(t) for t in ts])
            assert torch.equal(norm, captured) and all(torch.equal(a, b) for a, b in zip(out, want))


def test_norm_of_several_sizes_is_the_same_every_time(am):
    ts = [normal(rng(12), 2000, 3001).cuda()]
    norms = {float(am.wfst_am_clip(ts, INF)[1]) for _ in range(5)}
    assert len(norms) == 1
