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
