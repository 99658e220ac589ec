"""The layer norm, the gated layer and the clipping together, as a training step and a
scoring in 8 bits use them: blocks of norm, gated layer and narrowing layer on a
residual stream, the loss against a teacher's top logits, gradients, their clipping."""
import math

import pytest

import am_reference as R
from test_gpu_am_operators import BF16, F8, F32, normal, quantised, rng

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

D, N, UNITS, BLOCKS, TOP = 136, 200, 80, 2, 5


@pytest.fixture(scope="module")
def am():
    assert torch.cuda.is_available(), "no GPU"
    from paper_1808_00687_amd import acoustic
    return acoustic


def parameters(seed):
    g = rng(seed)
    p = {}
    for i in range(BLOCKS):
        p["gain%d" % i], p["shift%d" % i] = 1 + normal(g, D, std=0.1), normal(g, D, std=0.1)
        p["gated%d" % i], p["gated_b%d" % i] = normal(g, 2 * N, D, std=D ** -0.5).to(BF16), normal(g, 2 * N, std=0.1)
        p["narrow%d" % i], p["narrow_b%d" % i] = normal(g, D, N, std=N ** -0.5).to(BF16), normal(g, D, std=0.1)
    p["gain"], p["shift"] = 1 + normal(g, D, std=0.1), normal(g, D, std=0.1)
    p["output"], p["output_b"] = normal(g, UNITS, D, std=D ** -0.5).to(BF16), normal(g, UNITS, std=0.1)
    return p


def batch(seed, m):
    g = rng(seed)
    x, teacher = normal(g, m, D).to(BF16), normal(g, m, UNITS, std=3.0)
    value, index = torch.topk(teacher, TOP, 1)
    return x, index.to(torch.int32), value


def step(am, p, x, index, top, max_norm):
    """Gradients by name, clipped in place, and their norm before that."""
    kept, stream, add = [], x, None
    for i in range(BLOCKS):
        y, _, total = am.wfst_am_layer_norm(stream, p["gain%d" % i], p["shift%d" % i], residual=add)
        stream = stream if total is None else total
        pre = torch.empty(x.shape[0], 2 * N, dtype=BF16, device=x.device)
        u = am.wfst_am_gated(y, p["gated%d" % i], p["gated_b%d" % i], pre=pre)
        add = am.wfst_am_linear(u, p["narrow%d" % i], p["narrow_b%d" % i])
        kept.append((stream, y, pre, u))
    y, _, stream = am.wfst_am_layer_norm(stream, p["gain"], p["shift"], residual=add)
    logits = am.wfst_am_linear(y, p["output"], p["output_b"], out_dtype=F32)
    weight = torch.full((x.shape[0],), 1.0 / x.shape[0], device=x.device)
    loss, _, dl = am.wfst_am_distill(logits, index, top, weight=weight, gradient=True)
    g = {}
    dy, g["output"], g["output_b"] = am.wfst_am_linear_backward((dl * SCALE).to(BF16), y, p["output"])
    d, g["gain"], g["shift"] = am.wfst_am_layer_norm_backward(dy, stream, p["gain"])
    for i in reversed(range(BLOCKS)):
        stream, y, pre, u = kept[i]
        du, g["narrow%d" % i], g["narrow_b%d" % i] = am.wfst_am_linear_backward(d, u, p["narrow%d" % i])
        dy, g["gated%d" % i], g["gated_b%d" % i] = am.wfst_am_gated_backward(du, pre, y, p["gated%d" % i])
        d, g["gain%d" % i], g["shift%d" % i] = am.wfst_am_layer_norm_backward(dy, stream, p["gain%d" % i], dsum=d)
    g["x"] = d
    names = [k for k in g if k != "x"]
    _, norm = am.wfst_am_clip([g[k] for k in names], max_norm)
    return loss, logits, g, norm


SCALE = 64.0   # of the loss, so that small gradients keep their bits


def reference(p, x, index, top):
    """The loss, the logits and the gradients in float64 by autograd."""
    p = {k: v.double().requires_grad_() for k, v in p.items()}
    x = x.double().requires_grad_()

    def norm(s, gain, shift):
        var, mean = torch.var_mean(s, 1, correction=0, keepdim=True)
        return (s - mean) / torch.sqrt(var + 1e-5) * gain + shift

    s = x
    for i in range(BLOCKS):
        z = norm(s, p["gain%d" % i], p["shift%d" % i]) @ p["gated%d" % i].t() + p["gated_b%d" % i]
        u = z[:, :N] * torch.sigmoid(z[:, :N]) * z[:, N:]
        s = s + u @ p["narrow%d" % i].t() + p["narrow_b%d" % i]
    logits = norm(s, p["gain"], p["shift"]) @ p["output"].t() + p["output_b"]
    q = torch.log_softmax(logits, 1).gather(1, index.long())
    t = torch.log_softmax(top.double(), 1)
    loss = (t.exp() * (t - q)).sum(1) / x.shape[0]
    (loss.sum() * SCALE).backward()
    return loss, logits, {**{k: v.grad for k, v in p.items()}, "x": x.grad}


def distance(a, b):
    a, b = R.d(a), R.d(b)
    return float((a - b).norm() / b.norm())


# Roundings to bf16 on the way of a gradient: y, pre, u and the stream twice over in the forward pass, dl, dy, d, du, dy, d,
# du, dy, d and the gradient itself backward, 20 with the last; each moves what follows relatively by at most u, as
# independent errors of all elements, and no step here enlarges relative errors of whole matrices more than twice.
ALLOWED = 2 * math.sqrt(20) * R.U[BF16]


@pytest.mark.parametrize("m", [1, 7, 300])
def test_training_step(am, m):
    p, (x, index, top) = parameters(1), batch(m, m)
    loss, logits, want = reference(p, x, index, top)
    loss, logits = loss.detach(), logits.detach()
    got = step(am, {k: v.cuda() for k, v in p.items()}, x.cuda(), index.cuda(), top.cuda(), math.inf)
    assert distance(got[1], logits) < ALLOWED
    assert abs(float(got[0].double().sum()) - float(loss.sum())) < ALLOWED * float(logits.abs().max())
    for k in want:
        assert distance(got[2][k], want[k]) < ALLOWED, k
    names = [k for k in want if k != "x"]
    norm = math.sqrt(sum(float((R.d(got[2][k]) ** 2).sum()) for k in names))
    assert abs(float(got[3]) - norm) < 1e-6 * norm
    # clipped: the same gradients, shorter
    again = step(am, {k: v.cuda() for k, v in p.items()}, x.cuda(), index.cuda(), top.cuda(), norm / 4)
    assert torch.equal(again[3], got[3])
    short = math.sqrt(sum(float((R.d(again[2][k]) ** 2).sum()) for k in names))
    assert abs(short - norm / 4) < R.U[BF16] * norm
    for k in names:
        assert distance(again[2][k] * 4, got[2][k]) < R.U[BF16], k
    assert torch.equal(again[2]["x"], got[2]["x"])


def test_step_in_a_graph(am):
    p = {k: v.cuda() for k, v in parameters(2).items()}
    x, index, top = (t.cuda() for t in batch(3, 90))
    step(am, p, x, index, top, 1.0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(am, p, x, index, top, 1.0)
    for seed in (4, 5, 6):
        for a, b in zip((x, index, top), batch(seed, 90)):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        want = step(am, p, x, index, top, 1.0)
        torch.cuda.synchronize()
        for a, b in ((got[0], want[0]), (got[1], want[1]), (got[3], want[3])):
            assert torch.equal(a, b)
        assert all(torch.equal(got[2][k], want[2][k]) for k in got[2])


def test_scoring_in_8_bits(am):
    # norm to 8 bits, gated layer in 8 bits, narrowing layer, rows of log-likelihoods: each call against its definition
    # on the values that the one before it gave
    import am_reference_more as Q
    p = parameters(5)
    x, _, _ = batch(6, 50)
    gain, shift = p["gain0"], p["shift0"]
    y, scale, _ = am.wfst_am_layer_norm(x.cuda(), gain.cuda(), shift.cuda(), out_dtype=F8)
    w8, ws = quantised(p["gated0"].float())
    u = am.wfst_am_gated(y, w8.cuda(), p["gated_b0"].cuda(), x_scale=scale, w_scale=ws.cuda())
    want, _, _, err = Q.gated(y.cpu(), w8, p["gated_b0"], "silu", scale.cpu(), ws)
    R.close(u, want, err + R.U[BF16] * (want.abs() + err), "gated")
    s = am.wfst_am_linear(u, p["narrow0"].cuda(), p["narrow_b0"].cuda(), residual=x.cuda())
    y, scale, _ = am.wfst_am_layer_norm(s, p["gain"].cuda(), p["shift"].cuda(), out_dtype=F8)
    o8, os_ = quantised(p["output"].float())
    logits = am.wfst_am_linear(y, o8.cuda(), p["output_b"].cuda(), x_scale=scale, w_scale=os_.cuda(), out_dtype=F32)
    rows = am.wfst_am_loglikes(logits, scale=0.5)
    want = R.loglikes(logits, None, 0.5)
    R.close(rows, want, 16 * R.U32 * (1 + R.d(logits).abs().max()), "rows")
    # and near the rows of the 16-bit layers: an e4m3 rounding is 2^-4 of a value at most, three of them one after the other
    # in relative terms of whole rows 2^-4 / sqrt(3) each
    y, _, _ = am.wfst_am_layer_norm(x.cuda(), gain.cuda(), shift.cuda())
    u = am.wfst_am_gated(y, p["gated0"].cuda(), p["gated_b0"].cuda())
    s = am.wfst_am_linear(u, p["narrow0"].cuda(), p["narrow_b0"].cuda(), residual=x.cuda())
    y, _, _ = am.wfst_am_layer_norm(s, p["gain"].cuda(), p["shift"].cuda())
    same = am.wfst_am_linear(y, p["output"].cuda(), p["output_b"].cuda(), out_dtype=F32)
    assert distance(logits, same) < 4 * 2.0 ** -4
