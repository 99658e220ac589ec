"""The acoustic-model operators together: training by distillation, serving in
8 bits and the search, as in examples/acoustic_model.py; the training step's
gradients against torch's in float64."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    assert torch.cuda.is_available(), "no GPU"
    spec = importlib.util.spec_from_file_location("acoustic_model", os.path.join(ROOT, "examples", "acoustic_model.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_train_score_decode(example):
    got = example.main(steps=25, say=lambda *_: None)
    losses = got["losses"]
    assert losses[-1] < 0.8 * losses[0], losses
    # e4m3 keeps 3 bits after the leading one: scores move by a few percent of their spread
    off = (got["rows"] - got["rows16"]).abs().mean()
    assert float(off) < 0.1 * float(got["rows16"].std())
    assert got["decoded"].status == got["decoded16"].status == 0
    assert got["decoded"].path_arcs.size > 0 and got["decoded"].lat_arc.size >= got["decoded"].path_arcs.size
    assert abs(got["decoded"].cost - got["decoded16"].cost) < 0.05 * abs(got["decoded16"].cost)


def test_gradients_of_the_whole_step(example):
    from paper_1808_00687_amd import acoustic as am
    g = torch.Generator().manual_seed(3)
    model = example.Model(24, 32, 50, 2, seed=5)
    for t in model.gains:
        t.copy_(1 + 0.1 * torch.randn(t.shape, generator=g))
    x = torch.randn(60, 24, generator=g).to(torch.bfloat16).cuda()
    idx = torch.stack([torch.randperm(50, generator=g)[:6] for _ in range(60)]).to(torch.int32).cuda()
    top = torch.randn(60, 6, generator=g).cuda()
    logits, saved = model.forward(x)
    _, _, dl = am.wfst_am_distill(logits, idx, top, temperature=2.0, gradient=True)
    got = {id(p): (p, d) for p, d in model.gradients(dl, saved)}

    leaf = {k: p.detach().cpu().double().requires_grad_() for k, (p, _) in got.items()}
    of = lambda t: leaf[id(t)]  # noqa: E731

    def norm(v, gain):
        return v / torch.sqrt((v * v).mean(1, keepdim=True) + 1e-6) * of(gain)

    h = x.cpu().double() @ of(model.input.w).t() + of(model.input.b)
    for wide, narrow, gain in zip(model.wide, model.narrow, model.gains):
        u = torch.nn.functional.gelu(norm(h, gain) @ of(wide.w).t() + of(wide.b))
        h = h + u @ of(narrow.w).t() + of(narrow.b)
    z = norm(h, model.gains[-1]) @ of(model.output.w).t() + of(model.output.b)
    p = torch.softmax(top.cpu().double() / 2, 1)
    log_q = torch.log_softmax(z / 2, 1).gather(1, idx.cpu().long())
    (4 * (p * (p.log() - log_q)).sum()).backward()
    # activations and their gradients pass a dozen roundings to bfloat16 (2^-9 relative each, as independent errors)
    for k, (param, grad) in got.items():
        want = leaf[k].grad
        rel = float((grad.cpu().double() - want).norm() / want.norm())
        assert rel < 4 * (12 ** 0.5) * 2.0 ** -9, (tuple(param.shape), rel)
