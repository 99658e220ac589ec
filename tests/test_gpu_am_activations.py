"""gelu and its slope at every float16 from -16 to 16, in float32 outputs."""
import math

import pytest

import am_reference as R
from test_gpu_am_gradients import gradients
from test_gpu_am_operators import F16, F32

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def am():
    assert torch.cuda.is_available(), "no GPU"
    from paper_1808_00687_amd import acoustic
    return acoustic


def every(lo, hi):
    bits = torch.arange(-(1 << 15), 1 << 15, dtype=torch.int32).to(torch.int16)
    v = bits.view(F16)
    return v[(v >= lo) & (v <= hi)][:, None].contiguous()


def normal_error(z):
    """Of the normal distribution's function: the approximation (1.8e-8 / max(|z|, 1)) and its roundings relative to
    the tail: 6 x^2 from the exponent, 24 from a polynomial of six terms and three products; one of the result's."""
    tail = torch.special.ndtr(-z.abs())
    return 1.8e-8 / z.abs().clamp(min=1) + R.U32 * (tail * (3 * z * z + 24) + torch.special.ndtr(z))


def test_gelu(am):
    x = every(-16, 16)
    one = torch.ones(1, 1, dtype=F16).cuda()
    y = am.wfst_am_linear(x.cuda(), one, activation="gelu", out_dtype=F32)
    z = R.d(x)
    want = z * torch.special.ndtr(z)
    R.close(y, want, z.abs() * normal_error(z) + R.U32 * want.abs() + R.TINY[F32], "gelu")


def test_gelu_slope(am):
    x = every(-16, 16)
    one = torch.ones(1, 1, dtype=F16).cuda()
    dx, _, _ = gradients(am, torch.ones_like(x).cuda(), x.cuda(), one, "gelu", x.cuda())
    z = R.d(x)
    bell = z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    want = torch.special.ndtr(z) + bell
    # the bell: three roundings of its exponent z^2 / 2 and four more; dz in two 16-bit values
    err = normal_error(z) + R.U32 * ((1.5 * z * z + 6) * bell.abs() + 2 * want.abs()) + 2.0 ** -22 * want.abs() + 2.0 ** -35
    R.close(dx, want, err, "gelu's slope")
