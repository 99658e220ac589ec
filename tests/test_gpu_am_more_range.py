"""The gated layer, the layer norm and the clipping at the ends of the types' ranges and of the sizes that they take."""
import pytest

import am_reference as R
import am_reference_more as Q
from test_gpu_am_operators import BF16, F32

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def am():
    assert torch.cuda.is_available(), "no GPU"
    from paper_1808_00687_amd import acoustic
    return acoustic


@pytest.mark.parametrize("kind", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("large", [(1e20, 1e20), (3e30, 1e12), (1e12, 3e30), (1e30, 1e-25), (1e-25, 1e30)])
def test_gradients_of_gates_whose_factors_are_far_from_one(am, kind, large):
    # dy value is no float32 where the slope makes dy value slope one, or 0.  A row a gate, so nothing is summed: dbias of a
    # row is its float32 dz, dw of x = 1 the dz as two bfloat16 values hold it
    size_dy, size_value = large
    for gate in (-100.0, -60.0, -20.0, -3.0, 0.0, 1.0):
        dy = torch.full((1, 1), size_dy).to(BF16)
        pre = torch.tensor([[gate, size_value]]).to(BF16)
        dz, slack = Q.gated_dz(dy, pre, kind)
        if not (dz.abs() < 3e38).all():
            continue
        one = torch.ones(1, 1, dtype=BF16).cuda()
        _, dw, db = am.wfst_am_gated_backward(dy.cuda(), pre.cuda(), one, torch.ones(2, 1, dtype=BF16).cuda(), activation=kind,
                                               weight_dtype=F32)
        err = slack + 2 * R.U32 * dz.abs()   # and the products' own roundings
        tag = "%s %s %g" % (kind, large, gate)
        R.close(db[None], dz, err, tag + " dbias")
        R.close(dw.t(), dz, err + 2.0 ** -16 * dz.abs() + R.TINY[BF16], tag + " dw")


def test_gradients_of_rows_of_2_to_the_27_columns(am):
    # their sums are joined by more workgroups than one launch takes
    width = (1 << 27) + 33
    g = torch.Generator("cuda").manual_seed(3)
    s, dy = (torch.randn(1, width, generator=g, device="cuda", dtype=BF16) for _ in range(2))
    dx, dg, db = am.wfst_am_layer_norm_backward(dy, s)
    assert torch.equal(db, dy[0].float())   # of one row
    del dx
    v = s[0].double()
    mean = v.mean()
    v -= mean
    r = float(1 / torch.sqrt((v * v).mean() + 1e-5))
    size = float(v.abs().mean())
    # am_reference_more.py's Moments: the mean, a difference, the reciprocal deviation
    e_mean = R.sum_bound(width, size * width) / width
    rel = (R.LAMBDA * width ** 0.5 + 8) * R.U32 / 2 + 6 * R.U32
    off = (dg.double() - v * r * dy[0].double()).abs_()
    bound = (v.abs_().mul_(r * (3 * R.U32 + rel + R.U32)).add_(r * e_mean)).mul_(dy[0].double().abs())
    assert bool((off <= bound).all()), float((off - bound).max())


def test_as_many_tensors_as_are_taken(am):
    # descriptions in 924 launches; sizes from 1 to 37 values, all of them 1 / 64, so sums and the factor are exact
    sizes = [1 + i * 7 % 37 for i in range(65536)]
    flat = torch.full((sum(sizes),), 1 / 64, device="cuda")
    out = torch.zeros_like(flat)
    want = (sum(sizes) / 4096) ** 0.5
    _, norm = am.wfst_am_clip(list(flat.split(sizes)), want / 8, out=list(out.split(sizes)))
    assert abs(float(norm) - want) <= R.U32 * want * 1.001
    assert float(out.min()) == float(out.max()) == 1 / 512
    with pytest.raises(Exception, match="65536"):
        am.wfst_am_clip([flat] + list(flat.split(sizes)), 1.0)


def test_norms_of_more_than_32_bits_of_values(am):
    # rows do not depend on one another; gradients of gain and bias are sums that float32 holds exactly
    m, width = (1 << 22) + 5, 1032
    x = torch.randn(m, width, device="cuda", dtype=BF16)
    assert x.numel() > 1 << 32
    tail = x[-9:].clone()
    y, scale, _ = am.wfst_am_layer_norm(x, out_dtype=torch.float8_e4m3fn)
    want, want_scale, _ = am.wfst_am_layer_norm(tail, out_dtype=torch.float8_e4m3fn)
    assert torch.equal(y[-9:].view(torch.uint8), want.view(torch.uint8)) and torch.equal(scale[-9:], want_scale)
    del y, scale
    dy = torch.ones_like(x)
    dx, _, db = am.wfst_am_layer_norm_backward(dy, x)
    assert torch.equal(db, torch.full_like(db, m))
    want, _, _ = am.wfst_am_layer_norm_backward(dy[-9:].clone(), tail)
    assert torch.equal(dx[-9:], want)
