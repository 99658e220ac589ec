"""Operands and results that are column slices of one buffer."""
import pytest

from test_gpu_am_operators import BF16, F32, normal, rng, top_entries

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def am():
    assert torch.cuda.is_available(), "no GPU"
    from paper_1808_00687_amd import acoustic
    return acoustic


class Buffer:
    """Slices side by side; everything between them keeps its value."""

    def __init__(self, rows, width, dtype, gap):
        self.all = torch.full((rows, width), 7.0).to(dtype).cuda()
        self.at, self.gap, self.free = 0, gap, torch.ones(width, dtype=torch.bool)

    def take(self, n, value=None):
        v = self.all[:, self.at:self.at + n]
        self.free[self.at:self.at + n] = False
        self.at += n + self.gap
        assert self.at <= self.all.shape[1]
        if value is not None:
            v.copy_(value)
        return v

    def check(self):
        assert bool((self.all[:, self.free.cuda()] == 7.0).all())


@pytest.mark.parametrize("gap", [0, 3, 8])
@pytest.mark.parametrize("m,k,n", [(5, 64, 40), (300, 72, 200), (700, 264, 300), (1500, 200, 1400)])
def test_layer(am, m, k, n, gap):
    g = rng(m)
    x, w, r = normal(g, m, k).to(BF16).cuda(), normal(g, n, k, std=k ** -0.5).to(BF16).cuda(), normal(g, m, n).to(BF16).cuda()
    pre = torch.empty_like(r)
    y = am.wfst_am_linear(x, w, activation="gelu", residual=r, pre=pre)
    b = Buffer(m, 4 * (n + gap) + k + gap, BF16, gap)
    yo, xi, po, ri = b.take(n), b.take(k, x), b.take(n), b.take(n, r)
    am.wfst_am_linear(xi, w, activation="gelu", residual=ri, pre=po, out=yo)
    assert torch.equal(yo, y) and torch.equal(po, pre) and torch.equal(xi, x) and torch.equal(ri, r)
    b.check()


@pytest.mark.parametrize("gap", [0, 5])
@pytest.mark.parametrize("m,n", [(6, 80), (50, 3000), (7, 33000)])
def test_rows(am, m, n, gap):
    g = rng(n)
    x, r = normal(g, m, n).to(BF16).cuda(), normal(g, m, n).to(BF16).cuda()
    y, _, total = am.wfst_am_norm(x, residual=r)
    b = Buffer(m, 4 * (n + gap), BF16, gap)
    so, xi, yo, ri = b.take(n), b.take(n, x), b.take(n), b.take(n, r)
    am.wfst_am_norm(xi, residual=ri, out=yo, sum_out=so)
    assert torch.equal(yo, y) and torch.equal(so, total) and torch.equal(xi, x) and torch.equal(ri, r)
    b.check()
    logits = x.float()
    idx, top = top_entries(g, m, n, 6)
    b = Buffer(m, 3 * (n + gap), F32, gap)
    li, xi, di = b.take(n), b.take(n, logits), b.take(n)
    am.wfst_am_loglikes(xi, out=li)
    am.wfst_am_distill(xi, idx.cuda(), top.cuda(), dlogits=di)
    assert torch.equal(li, am.wfst_am_loglikes(logits))
    assert torch.equal(di, am.wfst_am_distill(logits, idx.cuda(), top.cuda(), gradient=True)[2])
    b.check()


def test_slices_that_share_a_column(am):
    b = torch.zeros(6, 100, device="cuda")
    with pytest.raises(Exception, match="overlaps"):
        am.wfst_am_loglikes(b[:, :41], out=b[:, 40:81])
    am.wfst_am_loglikes(b[:, :40], out=b[:, 40:80])
    with pytest.raises(Exception, match="overlaps"):
        am.wfst_am_loglikes(b[:4, :40], out=b[2:, 39:79])
    am.wfst_am_loglikes(b[:4, :40], out=b[2:, 60:])
