"""Rows far from zero in the operators over units: a row's softmax does not
depend on an offset, and a mask of a finite value that leaves nothing makes it
uniform.  Bounds hold the roundings relative to the row's maximum."""
import math

import pytest

import am_reference as R
from test_gpu_am_operators import BF16, F16, F32, inside, normal, rng, top_entries

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

INF = math.inf
MOST = torch.finfo(F32).max


@pytest.fixture(scope="module")
def am():
    assert torch.cuda.is_available(), "no GPU"
    from paper_1808_00687_amd import acoustic
    return acoustic


def softmax(x, t):
    """Of finite rows: (x - max) / t, log of the sum, and that log's error bound in float32."""
    y = (R.d(x) - R.d(x).amax(1, keepdim=True)) / t
    log_sum = torch.logsumexp(y, 1, keepdim=True)
    q = torch.exp(y - log_sum)
    # an exponent has three roundings (difference, scale, constant) and an exponential two ulp; a sum; the logarithm
    inner = (q * y.abs()).nan_to_num(0).sum(1, keepdim=True)
    err = R.U32 * (4 * inner + 4 + R.LAMBDA * math.sqrt(x.shape[1]) + 4 + 4 * log_sum.abs())
    return y, log_sum, q, err


def check_loglikes(am, x, prior, scale, tag):
    y, log_sum, _, err = softmax(x, 1.0)
    p = R.d(prior) if prior is not None else torch.zeros(x.shape[1]).double()
    want = scale * (y - log_sum - p)
    got = am.wfst_am_loglikes(inside(x), None if prior is None else prior.cuda(), scale=scale)
    bound = abs(scale) * (err + 4 * R.U32 * (y.abs() + log_sum.abs() + p.abs()))
    R.close(got, want, bound, tag)


def check_distill(am, x, idx, top, t, tag):
    """Entries distinct and used, weights 1."""
    y, log_sum, q, err = softmax(x, t)
    p = torch.softmax(R.d(top) / t, 1)
    at = idx.long()
    log_q = (y - log_sum).gather(1, at)
    want = t * t * (torch.xlogy(p, p) - torch.where(p > 0, p * log_q, torch.zeros_like(p))).sum(1)
    dl = t * (q.scatter_add(1, at, -p))
    loss, lse, got = am.wfst_am_distill(inside(x), idx.cuda(), inside(top), temperature=t, gradient=True)
    e_p = R.U32 * (16 * (R.d(top).abs().amax(1, keepdim=True) / t + 1) + R.LAMBDA * math.sqrt(idx.shape[1]))
    e_q = err + 4 * R.U32 * (y.abs() + 1)
    bound = t * t * (2 * (p * (e_p + e_q.gather(1, at)) + 4 * e_p * p * (log_q.abs() + 1 + torch.log(p).abs().nan_to_num(0, 0, 0))).sum(1))
    bound = bound + R.U32 * want.abs()
    loss = torch.where((loss.cpu() == INF) & (want + bound > MOST), want, loss.cpu().double())   # the loss is a float32
    R.close(loss, want, bound, tag + " loss")
    bound = t * (2 * q * e_q + 4 * R.U32 * (q + dl.abs() / t) + torch.zeros_like(q).scatter_add(1, at, 2 * e_p * p + R.U32 * p))
    R.close(got, dl, bound + R.U[x.dtype] * (dl.abs() + bound) + R.TINY[x.dtype], tag + " dlogits")
    true = (R.d(x).amax(1) / t + log_sum[:, 0]).clamp(-MOST, MOST)
    R.close(lse, true, err[:, 0] + 4 * R.U32 * true.abs(), tag + " lse")
    alone = am.wfst_am_distill_backward(inside(x), idx.cuda(), inside(top), lse, temperature=t)
    assert torch.isfinite(alone).all(), tag + " backward alone"
    # from lse, whose rounding it takes over
    e_l = (R.d(lse) - true).abs()[:, None] + 4 * R.U32 * (R.d(x).abs() / t + true.abs()[:, None] + 1)
    near = (e_l < 0.25).all(1)
    bound = (bound + t * 2 * q * e_l)[near]
    R.close(alone[near.cuda()], dl[near], bound + R.U[x.dtype] * (dl[near].abs() + bound) + R.TINY[x.dtype], tag + " backward alone")


# one wave a row, several, one to four rows of chunks held, rows that are not held
UNITS = [1, 60, 500, 2000, 5001, 9001, 20001, 40000]
FILLS = [-1e4, -1e10, -1e12, -1e30, torch.finfo(F32).min, 1e10, 1e30, torch.finfo(F32).max]


def filled(m, n, dt, g):
    """Rows of one finite value each, and a row that is one but for a unit."""
    x = torch.stack([torch.full((n,), v) for v in FILLS] + [torch.full((n,), torch.finfo(dt).min)])
    x = x.clamp(torch.finfo(dt).min, torch.finfo(dt).max).to(dt)
    if n > 3:
        x[-1, 3] = 1.0
    return x


@pytest.mark.parametrize("dt", [BF16, F16, F32])
@pytest.mark.parametrize("n", UNITS)
def test_loglikes_of_masks_that_leave_nothing(am, n, dt):
    g = rng(n)
    x = filled(len(FILLS), n, dt, g)
    check_loglikes(am, x, None, 1.0, "loglikes filled %d" % n)
    check_loglikes(am, x, torch.log_softmax(normal(g, n), 0), 0.3, "loglikes filled, prior %d" % n)


@pytest.mark.parametrize("dt", [BF16, F16, F32])
@pytest.mark.parametrize("t", [1.0, 0.25, 2.0])
@pytest.mark.parametrize("n", UNITS)
def test_distill_of_masks_that_leave_nothing(am, n, t, dt):
    x = filled(len(FILLS), n, dt, rng(n))
    idx, top = top_entries(rng(n + 1), x.shape[0], n, min(n, 7))
    check_distill(am, x, idx, top, t, "distill filled %s" % ((n, t, str(dt)),))


@pytest.mark.parametrize("offset", [30.0, -300.0, 3e4, 1e6, -1e9])
@pytest.mark.parametrize("n", [60, 2000, 5001, 40000])
def test_offsets_cost_no_bits(am, n, offset):
    g = rng(n)
    x = normal(g, 4, n, std=3.0) + offset
    idx, top = top_entries(g, 4, n, 9)
    check_loglikes(am, x, torch.log_softmax(normal(g, n), 0), 0.7, "loglikes offset %s" % ((n, offset),))
    for t in (1.0, 2.0):
        check_distill(am, x, idx, top, t, "distill offset %s" % ((n, offset),))


def test_filled_rows_are_rows_that_the_search_takes(am):
    from paper_1808_00687_amd import wfstdec, workloads
    wl = workloads.workload(1)
    ll = wl.loglikes[0][:20].copy()
    x = torch.from_numpy(ll).cuda()
    x[7] = torch.finfo(F32).min
    x[11] = -1e12
    graph = wfstdec.load_graph(wl.graph)
    r = wfstdec.wfst_decode(graph, am.wfst_am_loglikes(x), wl.opts.beam, max_active=300, lattice_beam=6.0)
    graph.free()
    assert r.status == 0 and math.isfinite(r.cost) and r.num_decoded == 20


@pytest.mark.parametrize("k", [5, 70])
@pytest.mark.parametrize("t", [1.0, 0.25, 3.0])
def test_teacher_logits_far_from_zero(am, t, k):
    # what the entries add up to does not change with their offset, which these sums hold exactly
    g = rng(k)
    n = 300
    x = normal(g, 1, n).expand(5, n).contiguous()
    idx = top_entries(g, 1, n, k)[0].expand(5, k).contiguous()
    top = torch.randint(-9, 10, (1, k), generator=g).float() + torch.tensor([[0.0], [-2.0 ** 20], [2.0 ** 22], [-77.0], [5e5]])
    loss, _, dl = am.wfst_am_distill(x.cuda(), idx.cuda(), top.cuda(), temperature=t, gradient=True)
    for m in range(1, 5):
        assert torch.equal(loss[m], loss[0]) and torch.equal(dl[m], dl[0]), m
    # entries of one finite value share alike, the type's lowest and largest among them
    top = torch.tensor([0.0, torch.finfo(F32).min, MOST, -1e12, 3e38])[:, None].expand(5, k).contiguous()
    loss, _, dl = am.wfst_am_distill(x.cuda(), idx.cuda(), top.cuda(), temperature=t, gradient=True)
    assert float(loss[0]) > 0
    for m in range(1, 5):
        assert torch.equal(loss[m], loss[0]) and torch.equal(dl[m], dl[0]), m
    # masked by the lowest value, one left
    top[:, :] = torch.finfo(F32).min
    top[:, 3] = 1.0
    loss, _, dl = am.wfst_am_distill(x.cuda(), idx.cuda(), top.cuda(), temperature=t, gradient=True)
    one = am.wfst_am_distill(x.cuda(), idx[:, 3:4].contiguous().cuda(), top[:, 3:4].contiguous().cuda(), temperature=t, gradient=True)
    assert torch.equal(loss, one[0]) and torch.equal(dl, one[2])
