"""Every tiled kernel of the gated layer in every type, result and epilogue against its definition in float64.  Inputs lie
among NaN, outputs among values that have to stay (test_gpu_am_operators.py)."""
import pytest

import am_reference as R
import am_reference_more as Q
from am_gated_tiles import SIZES
from test_gpu_am_operators import BF16, F8, F16, F32, Out, inside, normal, quantised, rng

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

KINDS = ["silu", "relu", "gelu", "none"]


@pytest.fixture(scope="module")
def am():
    assert torch.cuda.is_available(), "no GPU"
    from paper_1808_00687_amd import acoustic
    return acoustic


@pytest.mark.parametrize("dt", [BF16, F16, F8])
@pytest.mark.parametrize("m,k,n", list(SIZES))
def test_tiles(am, m, k, n, dt):
    g = rng(m + k)
    x, w = normal(g, m, k), normal(g, 2 * n, k, std=k ** -0.5)
    xs = ws = None
    if dt == F8:
        (x, xs), (w, ws) = quantised(x), quantised(w)
    else:
        x, w = x.to(dt), w.to(dt)
    b = normal(g, 2 * n, std=0.3)
    c = lambda t: None if t is None else t.cuda()  # noqa: E731
    xg, wg, xsg, wsg = inside(x), inside(w), c(xs), c(ws)
    first = (m + k + n) % 4
    for bias, kind, with_pre in ((b, KINDS[first], True), (None, KINDS[(first + 1) % 4], False)):
        y, z, e_z, e_y = Q.gated(x, w, bias, kind, xs, ws)
        for out in (F32, BF16, F16):
            yo = Out(m, n, out)
            po = Out(m, 2 * n, out) if with_pre else None
            am.wfst_am_gated(xg, wg, c(bias), activation=kind, x_scale=xsg, w_scale=wsg, pre=po.v if with_pre else None, out=yo.v)
            torch.cuda.synchronize()
            tag = "gated %s" % ((m, k, n, str(dt), kind, str(out), with_pre),)
            yo.check(tag)
            R.close(yo.v, y, e_y + R.U[out] * (y.abs() + e_y) + R.TINY[out], tag)
            if with_pre:
                R.close(po.v, z, e_z + R.U[out] * (z.abs() + e_z) + R.TINY[out], tag + " pre")
                po.check(tag)
