"""Workgroups of the row operators that take several rows in turn: the next
row's fetch, the sets used by turns, the lists handed back, rows of weight 0 or
without entries between others.

What a row gives does not depend on which rows lie around it, so all rows have to
equal, bit by bit, those of calls with few rows (one turn each); sampled rows are
compared with float64.
"""
import pytest

import am_reference as R
from test_gpu_am_operators import BF16, F8, F32, distill_check, loglikes_check, norm_backward_case

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def am():
    assert torch.cuda.is_available(), "no GPU"
    from paper_1808_00687_amd import acoustic
    return acoustic


def slices(rows, most=997):
    return [slice(at, min(at + most, rows)) for at in range(0, rows, most)]


# At most 1,024 workgroups of the operators over units: 3 turns and more, of one row a workgroup (256 and 1,024
# threads, held and not) and of four
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("m,n,k", [(13000, 80, 5), (13001, 500, 70), (3500, 2100, 9), (3500, 3000, 70), (3100, 9001, 12), (3100, 33000, 3)])
def test_distill(am, m, n, k, dt):
    g = torch.Generator(device="cuda").manual_seed(n)
    x = (torch.randn(m, n, generator=g, device="cuda") * 3).to(dt)
    idx = torch.randint(0, n, (m, k), generator=g, device="cuda", dtype=torch.int32)   # units repeat
    top = torch.randn(m, k, generator=g, device="cuda") * 2
    w = torch.rand(m, generator=g, device="cuda") + 0.5
    kind = torch.randint(0, 5, (m,), generator=g, device="cuda")
    w[kind == 1] = 0.0
    idx[kind == 2] = -1
    idx[kind == 3, : (k + 1) // 2] = n
    every = dict(temperature=2.0, weight=w)
    loss, lse, dl = am.wfst_am_distill(x, idx, top, gradient=True, **every)
    only, lse_only, _ = am.wfst_am_distill(x, idx, top, **every)
    back = am.wfst_am_distill_backward(x, idx, top, lse, **every)
    place = x.clone()
    am.wfst_am_distill(place, idx, top, dlogits=place, **every)
    assert torch.equal(only, loss) and torch.equal(lse_only, lse) and torch.equal(place, dl)
    place.copy_(x)
    am.wfst_am_distill_backward(place, idx, top, lse, dlogits=place, **every)
    assert torch.equal(place, back)
    for s in slices(m):
        few = dict(temperature=2.0, weight=w[s])
        a, b, c = am.wfst_am_distill(x[s], idx[s], top[s], gradient=True, **few)
        assert torch.equal(a, loss[s]) and torch.equal(b, lse[s]) and torch.equal(c, dl[s]), s
        assert torch.equal(am.wfst_am_distill_backward(x[s], idx[s], top[s], lse[s], **few), back[s]), s
    assert not loss[(kind == 1) | (kind == 2)].any() and not dl[(kind == 1) | (kind == 2)].any()
    rows = torch.tensor([0, 1, 1024, 1025, 2050, m // 2, m - 2, m - 1])
    distill_check(am, x[rows].cpu(), idx[rows].cpu(), top[rows].cpu(), 2.0, w[rows].cpu(), "distill turns %d" % n)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("m,n", [(13000, 80), (13001, 2000), (3500, 3000), (3100, 9001), (3100, 33000)])
def test_loglikes(am, m, n, dt):
    g = torch.Generator(device="cuda").manual_seed(n)
    x = (torch.randn(m, n, generator=g, device="cuda") * 3).to(dt)
    prior = torch.log_softmax(torch.randn(n, generator=g, device="cuda"), 0)
    ll = am.wfst_am_loglikes(x, prior, scale=0.3)
    for s in slices(m):
        assert torch.equal(am.wfst_am_loglikes(x[s], prior, scale=0.3), ll[s]), s
    rows = torch.tensor([0, 1, 1024, 2050, m // 2, m - 1])
    loglikes_check(am, x[rows].cpu(), prior.cpu(), 0.3, "loglikes turns %d" % n)


# at most 4,096 workgroups forward
@pytest.mark.parametrize("dt,out", [(BF16, F8), (BF16, BF16), (F32, F32)])
@pytest.mark.parametrize("m,width", [(50001, 96), (13000, 2100), (12500, 5000), (12500, 9001)])
def test_norm(am, m, width, dt, out):
    g = torch.Generator(device="cuda").manual_seed(width)
    x = torch.randn(m, width, generator=g, device="cuda").to(dt)
    r = (torch.randn(m, width, generator=g, device="cuda") * 3).to(dt)
    gain = 1 + torch.randn(width, generator=g, device="cuda") * 0.2
    y, scale, total = am.wfst_am_norm(x, gain, residual=r, out_dtype=out)
    for s in slices(m, 3989):
        for a, b in zip(am.wfst_am_norm(x[s], gain, residual=r[s], out_dtype=out), (y, scale, total)):
            assert a is None and b is None or torch.equal(a.float(), b[s].float()), s
    # in place of the residual and of x, beside rows on their way
    for place, args in ((r.clone(), lambda p: (x, p)), (x.clone(), lambda p: (p, r))):
        a, b = args(place)
        again, _, kept = am.wfst_am_norm(a, gain, residual=b, out_dtype=out, sum_out=place)
        assert kept is place and torch.equal(place, total) and torch.equal(again.float(), y.float())
    rows = torch.tensor([0, 4095, 4096, 8200, m - 1])
    s, v = R.norm(x[rows], r[rows], gain, 1e-6)
    if out != F8:
        err = (R.LAMBDA * width ** 0.5 + 12) * R.U32 * v.abs()
        R.close(y[rows], v, err + R.U[out] * (v.abs() + err) + R.TINY[out], "norm turns")
    else:
        got = R.d(y[rows].float()) * R.d(scale[rows])[:, None]
        top = v.abs().amax(1, keepdim=True) / 448
        R.close(got, v, 2.0 ** -4 * v.abs() + 2.0 ** -10 * top + (R.LAMBDA * width ** 0.5 + 16) * 4 * R.U32 * v.abs(), "norm turns")
    R.close(total[rows], s, R.U32 * s.abs() + R.U[dt] * s.abs() * (1 + R.U32) + R.TINY[dt], "norm turns, sum")


# at most 768 workgroups backward
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("m,width", [(9500, 80), (9301, 1000), (2500, 1500), (2500, 3000), (2400, 5000)])
def test_norm_backward(am, m, width, dt):
    norm_backward_case(am, m, width, dt, width, True)
    g = torch.Generator(device="cuda").manual_seed(width)
    s, dy, ds = ((torch.randn(m, width, generator=g, device="cuda") * a).to(dt) for a in (2.0, 0.1, 0.1))
    dx, _ = am.wfst_am_norm_backward(dy, s, dsum=ds)
    for at in slices(m, 761):
        assert torch.equal(am.wfst_am_norm_backward(dy[at], s[at], dsum=ds[at])[0], dx[at]), at
