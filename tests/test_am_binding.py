"""The acoustic-model operators' binding, without a GPU: what it makes of its
arguments before it calls the library."""
import pytest

torch = pytest.importorskip("torch")


@pytest.fixture
def am():
    from paper_1808_00687_amd import acoustic
    return acoustic


class Gpu:
    """Stands in for a tensor on a GPU."""

    is_cuda = True

    def __init__(self, device):
        self.device = device

    def get_device(self):
        return self.device


def test_the_device_is_the_first_operands(am, monkeypatch):
    # by name and in any order, too: the calls below are not on the current device, 0
    entered = []

    class On:
        def __init__(self, device, stream):
            entered.append((device, stream))

        def __enter__(self):
            pass

        def __exit__(self, *exc):
            pass

    monkeypatch.setattr(am, "_On", On)
    monkeypatch.setattr(am, "_device", lambda t, name: t.get_device())
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(am.torch, "Tensor", Gpu)
    call = am._here(lambda x, w, *, activation="none": "done")
    assert call(Gpu(1), Gpu(1)) == "done" and entered == [(1, None)]
    assert call(activation="relu", w=Gpu(2), x=Gpu(3)) == "done" and entered[1:] == [(3, None)]
    assert call(w=Gpu(2), x=Gpu(3), stream=7) == "done" and entered[2:] == [(3, 7)]
    assert call(activation="relu", x=Gpu(0), w=Gpu(0)) == "done" and len(entered) == 3
    assert am.wfst_am_linear.__wrapped__.__code__.co_varnames[0] == "x"


def test_a_stream_with_operands_by_name(am):
    x = torch.zeros(2, 8)
    with pytest.raises(TypeError, match="x must be a torch tensor on a GPU"):
        am.wfst_am_linear(activation="relu", x=x, w=x, stream=0)
    with pytest.raises(TypeError, match="logits must be a torch tensor on a GPU"):
        am.wfst_am_loglikes(scale=2.0, logits=x, stream=0)


@pytest.fixture
def on_cpu(am, monkeypatch):
    """Calls go up to the library's, with tensors on the CPU; what it would be called with."""
    calls = []
    monkeypatch.setattr(am, "_device", lambda t, name: t.get_device())
    monkeypatch.setattr(am, "_raw_stream", lambda d: 0)
    monkeypatch.setattr(am, "_call", lambda name, packed, stream: calls.append(name))
    return calls


def test_entries_have_their_logits_shape(am, on_cpu):
    x, top, idx = torch.zeros(6, 20), torch.zeros(6, 3), torch.zeros(6, 3, dtype=torch.int32)
    lse = torch.zeros(6)
    both = (lambda i: am.wfst_am_distill.__wrapped__(x, i, top), lambda i: am.wfst_am_distill_backward.__wrapped__(x, i, top, lse))
    for call in both:
        call(idx)
        for other in (idx.t().contiguous(), idx.flatten(), idx.reshape(3, 6), idx.reshape(2, 9), idx[:, :2].contiguous()):
            with pytest.raises(ValueError, match="top_index must be .6 x 3."):
                call(other)
        for other in (idx.long(), torch.zeros(6, 4, dtype=torch.int32)[:, :3]):
            with pytest.raises(ValueError, match="top_index"):
                call(other)
    assert on_cpu == ["wfst_am_distill", "wfst_am_distill_backward"]


def calls_of(am):
    """Every operator with tensors on the CPU: {name: (call, operands, results' places)}."""
    f = lambda *shape: torch.zeros(*shape)  # noqa: E731
    h = lambda *shape: torch.zeros(*shape, dtype=torch.bfloat16)  # noqa: E731
    idx = torch.zeros(4, 3, dtype=torch.int32)
    linear = dict(x=h(4, 8), w=h(6, 8), bias=f(6), residual=h(4, 6))
    norm = dict(x=h(4, 8), gain=f(8), residual=h(4, 8))
    distill = dict(logits=f(4, 9), top_logit=f(4, 3), weight=f(4))
    return {
        "linear": (lambda **kw: am.wfst_am_linear.__wrapped__(**kw), linear, dict(out=h(4, 6), pre=h(4, 6))),
        "norm": (lambda **kw: am.wfst_am_norm.__wrapped__(**kw), norm, dict(out=h(4, 8), sum_out=h(4, 8))),
        "norm_backward": (lambda **kw: am.wfst_am_norm_backward.__wrapped__(gain_gradient=False, **kw),
                          dict(dy=h(4, 8), s=h(4, 8), gain=f(8), dsum=h(4, 8)), {}),
        "linear_backward": (lambda **kw: am.wfst_am_linear_backward.__wrapped__(activation="silu", bias_gradient=False, **kw),
                            dict(dy=h(4, 6), x=h(4, 8), w=h(6, 8), pre=h(4, 6)), {}),
        "distill": (lambda **kw: am.wfst_am_distill.__wrapped__(top_index=idx, **kw), distill, dict(dlogits=f(4, 9))),
        "distill_backward": (lambda **kw: am.wfst_am_distill_backward.__wrapped__(top_index=idx, **kw),
                             dict(distill, lse=f(4)), dict(dlogits=f(4, 9))),
        "loglikes": (lambda **kw: am.wfst_am_loglikes.__wrapped__(**kw), dict(logits=f(4, 9), log_prior=f(9)), dict(out=f(4, 9))),
    }


NAMES = ["linear", "linear_backward", "norm", "norm_backward", "distill", "distill_backward", "loglikes"]


@pytest.mark.parametrize("name", NAMES)
def test_operands_that_require_a_gradient(am, on_cpu, name, monkeypatch):
    monkeypatch.setattr(am, "_bytes_for", lambda *_: 0)
    call, operands, places = calls_of(am)[name]
    call(**operands, **places)
    for k in list(operands) + list(places):
        changed = {n: t.detach().requires_grad_() if n == k else t for n, t in {**operands, **places}.items()}
        with pytest.raises(ValueError, match="%s requires a gradient" % k):
            call(**changed)
        with torch.no_grad():
            call(**changed)
        with torch.inference_mode():
            call(**changed)


@pytest.mark.parametrize("name", [n for n in NAMES if not n.endswith("m_backward") and n != "linear_backward"])
def test_results_count_as_written(am, on_cpu, name):
    call, operands, places = calls_of(am)[name]
    at = {k: t._version for k, t in places.items()}
    call(**operands, **places)
    for k, t in places.items():
        assert t._version > at[k], k
    for k, t in operands.items():
        assert t._version == 0, k
    # a graph that kept a result's old value notices
    k, t = next(iter(places.items()))
    leaf = torch.ones_like(t).requires_grad_()
    loss = (leaf * t).sum()
    call(**operands, **places)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    with torch.inference_mode():
        call(**operands, **{k: torch.zeros_like(t) for k, t in places.items()})
