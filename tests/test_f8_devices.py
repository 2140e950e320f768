"""Tensors of another device than the current one, or of several, are refused by the binding: a kernel would run on the current device
with addresses of another.  Without a GPU: tensors that say where they lie, and a library that records what reaches it."""
import pytest
import torch

import paper_2204_08211_b200 as co3
from paper_2204_08211_b200 import binding


class On(torch.Tensor):
    """A host tensor that passes for one of device `self.at`."""
    is_cuda = property(lambda self: True)

    def get_device(self):
        return self.at


def on(device, *shape, dtype=torch.float32):
    t = torch.zeros(*shape, dtype=dtype).as_subclass(On)
    t.at = device
    return t


class Library:
    def __init__(self):
        self.calls = 0

    def __getattr__(self, name):
        def call(*_):
            self.calls += 1
            return co3.OK
        return call


@pytest.fixture
def library(monkeypatch):
    lib = Library()
    monkeypatch.setattr(binding, "_lib", lib)
    monkeypatch.setattr(binding, "_several_devices", True, raising=False)
    monkeypatch.setattr(binding, "_current_device", lambda: 0, raising=False)
    monkeypatch.setattr(binding, "_current_stream", lambda device: 0)
    return lib


F8 = dict(dtype=torch.uint8)
# name, the call, its tensors (shape, type)
CALLS = [
    ("pack", lambda t: co3.co3_f8_pack(*t), [((4, 8), {}), ((512,), F8)]),
    ("unpack", lambda t: co3.co3_f8_unpack(*t), [((512,), F8), ((4, 8), {})]),
    ("activation", lambda t: co3.co3_f8_activation(t[0], co3.ACT_RELU, *t[1:]), [((4, 8), {}), ((4, 8), {}), ((512,), F8), ((512,), F8)]),
    ("activation_backward", lambda t: co3.co3_f8_activation_backward(t[0], t[1], co3.ACT_RELU, t[2]), [((4, 8), {}), ((512,), F8), ((4, 8), {})]),
    ("linear", lambda t: co3.co3_f8_linear(*t[:5], res=t[5]), [((4, 8), {}), ((512,), F8), ((512,), F8), ((8,), {}), ((4, 8), {}), ((64,), F8)]),
    ("linear_of_blocks", lambda t: co3.co3_f8_linear(None, *t, cols=8), [((512,), F8), ((512,), F8), ((8,), {}), ((4, 8), {})]),
    ("weight_gradient", lambda t: co3.co3_f8_weight_gradient(t[0], t[1], 8, t[2], t[3], 1, 0, t[4], res=t[5]),
     [((4, 8), {}), ((512,), F8), ((64,), {}), ((8,), {}), ((512,), F8), ((64,), F8)]),
]


@pytest.mark.parametrize("name,call,tensors", CALLS, ids=[c[0] for c in CALLS])
def test_one_device_and_the_current_one(name, call, tensors, library):
    make = lambda devices: [on(d, *shape, **kind) for d, (shape, kind) in zip(devices, tensors)]
    n = len(tensors)
    assert call(make([0] * n)) == co3.OK and library.calls == 1
    for devices in [[1] * n] + [[int(k == i) for k in range(n)] for i in range(n)] + [[int(k != i) for k in range(n)] for i in range(n)]:
        with pytest.raises(ValueError):
            call(make(devices))
    assert library.calls == 1


def test_layer_norm_of_another_device(library):
    x, y = on(1, 4, 8), on(1, 4, 8)
    with pytest.raises(ValueError):
        co3.co3_layer_norm(x, None, None, y)
    with pytest.raises(ValueError):
        co3.co3_layer_norm(on(0, 4, 8), None, None, y)
    assert library.calls == 0
