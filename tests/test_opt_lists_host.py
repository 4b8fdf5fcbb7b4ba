"""Lists of the optimizer step that the binding refuses by their devices.  No GPU: tensors that only say where they lie."""
import pytest
import torch

from paper_2509_03047_gb300 import flashrec as fr


class On:
    """What the binding asks of a tensor of `n` fp32 elements on GPU `index` (-1: the host)."""
    dtype = torch.float32

    def __init__(self, index, n=8):
        self.index, self.n = index, n
        self.device = torch.device("cuda", index) if index >= 0 else torch.device("cpu")
        self.is_cuda, self.nbytes = index >= 0, 4 * n

    def get_device(self):
        return self.index

    def numel(self):
        return self.n

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 0x7F0000000000


class Library:
    """Takes every list, makes no plan (the handle stays null); counts the calls."""

    def __init__(self):
        self.calls = []

    def fr_opt_create(self, tensors, count, out):
        self.calls.append("create")
        return fr.FR_OK

    def fr_opt_info(self, *args):
        return fr.FR_OK

    def fr_grad_clip(self, *args):
        self.calls.append("clip")
        return fr.FR_OK

    def fr_adamw_step(self, *args):
        self.calls.append("step")
        return fr.FR_OK


@pytest.fixture
def library(monkeypatch):
    made = Library()
    monkeypatch.setattr(fr, "lib", made)
    monkeypatch.setattr(fr, "_stream", lambda stream: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    return made


def test_lists_on_the_current_device_are_taken(library):
    plan = fr.OptPlan([On(1)], [On(1)], [On(1)], [On(1)])
    assert plan.device == torch.device("cuda", 1)
    plan = fr.OptPlan(grads=[On(-1, 0), On(0, 0), On(1), On(2, 0)])  # those without elements may lie anywhere
    assert plan.device == torch.device("cuda", 1)
    assert fr.OptPlan(grads=[On(0, 0)]).device == torch.device("cuda", 1)
    assert library.calls == ["create"] * 3


@pytest.mark.parametrize("lists", [dict(grads=[On(1), On(0)]), dict(grads=[On(0), On(1)]), dict(weights=[On(1)], grads=[On(2)]),
                                   dict(m=[On(1), None, On(1)], v=[On(1), None, On(0)]), dict(weights=[On(0)], grads=[On(0)]),
                                   dict(grads=[On(1), On(-1)])])
def test_lists_on_other_devices_are_refused(library, lists):
    with pytest.raises(ValueError, match="device"):
        fr.OptPlan(**lists)
    assert library.calls == []


@pytest.mark.parametrize("index", [0, -1])
def test_a_record_on_another_device_is_refused(library, index):
    plan = fr.OptPlan([On(1)], [On(1)], [On(1)], [On(1)])
    del library.calls[:]
    with pytest.raises(ValueError):
        plan.clip(out=On(index))
    with pytest.raises(ValueError):
        plan.step(fr.fr_adamw(1e-3, 0.9, 0.99, 1e-8, 0.0, 1, 0, 0), On(index))
    assert library.calls == []
    plan.clip(out=On(1))
    plan.step(fr.fr_adamw(1e-3, 0.9, 0.99, 1e-8, 0.0, 1, 0, 0), On(1))
    plan.step(fr.fr_adamw(1e-3, 0.9, 0.99, 1e-8, 0.0, 1, 0, 0))
    assert library.calls == ["clip", "step", "step"]
