"""Norms: 8-bit values at ties, rows too long to be held in registers, results in
place of inputs, types of the input and the result that differ."""
import pytest

import am_reference as R
from test_gpu_am_operators import BF16, F8, F16, F32, inside, norm_backward_case, norm_case, normal, rng

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def am():
    assert torch.cuda.is_available(), "no GPU"
    from paper_1808_00687_amd import acoustic
    return acoustic


def ties():
    """Values halfway between two e4m3 values, and the one of them whose last bit is 0."""
    v = torch.arange(0x7F, dtype=torch.uint8).view(F8).float()   # 0 to 448
    mid = (v[:-1] + v[1:]) / 2
    even = torch.arange(0x7E)
    return mid, v[even + (even & 1)]


@pytest.mark.parametrize("width", [130, 5000, 33000])
def test_ties_go_to_even(am, width):
    # a row of ones has norm 1, so the gain is what is quantised: the scale, times 448 and times ties
    mid, to = ties()
    n = mid.numel()
    for scale in (3.0, 41.0, 47.0, 61.0, 83.0, 97.0, 109.0, 113.0, 2047.0):
        inv = torch.tensor(1.0) / scale
        gain = torch.ones(width)
        gain[:n] = mid * scale           # exact: at most 5 and 11 bits
        gain[n] = R.E4M3_MAX * scale
        y, got, _ = am.wfst_am_norm(torch.ones(2, width).cuda(), gain.cuda(), eps=1e-30, out_dtype=F8)
        assert (got == scale).all()
        small = am.wfst_am_norm(torch.ones(2, width).cuda(), (gain * 2.0 ** -120).cuda(), eps=1e-30, out_dtype=F8)
        assert torch.equal(small[0].float(), y.float()) and (small[1] == scale * 2.0 ** -120).all()
        assert torch.equal(y.float().cpu()[:, :n], to.expand(2, n)), (scale, int((gain[:n] * inv != mid).sum()))


def test_the_scales_tell_a_division_from_a_product():
    mid, _ = ties()
    assert any(bool(((mid * s) * (torch.tensor(1.0) / s) != mid).any()) for s in (41.0, 47.0, 61.0, 83.0, 97.0, 109.0, 113.0, 2047.0))


# rows are held up to 32,768 columns
LONG = [32768, 32769, 40001]


@pytest.mark.parametrize("dt,out", [(BF16, F8), (F32, F8), (BF16, BF16), (F16, F32), (F32, F32)])
@pytest.mark.parametrize("width", LONG)
def test_long_rows(am, width, dt, out):
    for m in (1, 5):
        norm_case(am, m, width, dt, out, width + m, residual=True)
        norm_case(am, m, width, dt, out, width + m, residual=False, gain=False)
    norm_case(am, 3, width, dt, out, 3, True, pad=1, offset=3, in_place=True)


def test_long_rows_many(am):
    # more rows than workgroups: a row is read again after the one before it was written
    norm_case(am, 4500, 32769, BF16, F8, 1, True, in_place=True)


@pytest.mark.parametrize("dt", [BF16, F16, F32])
@pytest.mark.parametrize("width", LONG)
def test_long_rows_backward(am, width, dt):
    for m, ds, gain in ((1, True, True), (7, False, True), (40, True, False)):
        norm_backward_case(am, m, width, dt, width + m, ds, gain=gain, pad=m % 2, offset=m % 3)
    dx, dg = am.wfst_am_norm_backward(torch.empty(0, width, dtype=dt).cuda(), torch.empty(0, width, dtype=dt).cuda())
    assert dx.shape == (0, width) and not dg.any()


def test_long_rows_backward_many(am):
    norm_backward_case(am, 1700, 32769, BF16, 2, True)


@pytest.mark.parametrize("dt,out", [(BF16, F32), (F16, F32), (F32, BF16), (F32, F16), (BF16, F16), (F16, BF16)])
@pytest.mark.parametrize("width", [1, 7, 64, 440, 1000, 2047, 5000, 6144, 9001, 20000])
def test_result_of_another_type(am, width, dt, out):
    for m in (1, 5):
        norm_case(am, m, width, dt, out, width + m, residual=True)
        norm_case(am, m, width, dt, out, width + m, residual=False, gain=False)
    norm_case(am, 6, width, dt, out, 3, True, pad=3, offset=5)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("width", [65, 1500, 9000, 33000])
def test_sum_in_place_of_x(am, width, dt):
    g = rng(width)
    x, r = normal(g, 6, width).to(dt).cuda(), normal(g, 6, width).to(dt).cuda()
    for out in (F8, dt):
        want = am.wfst_am_norm(x, residual=r, out_dtype=out)
        place = x.clone()
        got = am.wfst_am_norm(place, residual=r, out_dtype=out, sum_out=place)
        assert got[2] is place
        for a, b in zip(got, want):
            assert a is None and b is None or torch.equal(a.float(), b.float())


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("m,width", [(6, 65), (900, 1500), (6, 9000), (5, 33000)])
def test_gradient_in_place(am, m, width, dt):
    g = rng(width)
    s, dy, ds = (normal(g, m, width, std=v).to(dt) for v in (2.0, 0.1, 0.1))
    gain = (1 + normal(g, width, std=0.2)).cuda()
    dx, dg = am.wfst_am_norm_backward(dy.cuda(), s.cuda(), gain, dsum=ds.cuda())
    for over in ("dy", "dsum"):
        t = {"dy": inside(dy, 5), "s": inside(s, 5), "dsum": inside(ds, 5)}
        got = torch.empty(width).cuda()
        head = []
        for name in ("dy", "s", "dsum", over):
            head += am._matrix(t[name], name, 0)
        head += [gain.data_ptr(), got.data_ptr()]
        pack = am._PACK["norm_backward"].pack
        need = am._bytes_for("wfst_am_norm_backward_workspace", pack(*head, 0, 0, 1e-6, 0))
        work = torch.empty(need, dtype=torch.uint8, device="cuda")
        am._call("wfst_am_norm_backward", pack(*head, work.data_ptr(), need, 1e-6, 0), torch.cuda.current_stream().cuda_stream)
        assert torch.equal(t[over], dx) and torch.equal(got, dg), over
