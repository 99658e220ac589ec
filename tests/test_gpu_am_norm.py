"""Norms: 8-bit values at ties."""
import pytest

import am_reference as R
from test_gpu_am_operators import F8, F32

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
