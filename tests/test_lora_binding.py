"""What LoRAProjection and the wrappers of the lora_* calls check and pass on, with the library and CUDA faked; runs without
a GPU."""
import types

import pytest
import torch

import paper_2609_33252_b200 as cep
from paper_2609_33252_b200 import binding


def on_device(t, index):
    """A CPU tensor as a CUDA tensor of device `index` looks to the binding."""
    class Fake:
        is_cuda = True
        get_device = staticmethod(lambda: index)

        def __getattr__(self, name):
            return getattr(t, name)
    return Fake()


@pytest.fixture
def plans(monkeypatch):
    """No GPU, device 0 current; returns the list of (what, arguments) that reach the library."""
    made = []
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(binding, "lora_plan", lambda *a: made.append(("plan", a)) or 1)
    monkeypatch.setattr(binding, "lora_plan_destroy", lambda plan: None)
    return made


def test_a_weight_of_another_device_is_refused(plans):
    w = torch.zeros(16, 64, dtype=torch.bfloat16)
    with pytest.raises(cep.CepError, match="device"):
        cep.LoRAProjection(on_device(w, 1), 4)
    assert not plans
    cep.LoRAProjection(on_device(w, 0), 4)
    assert len(plans) == 1


def test_a_stream_of_another_device_is_refused(plans):
    stream = types.SimpleNamespace(cuda_stream=5, device=torch.device("cuda", 1))
    with pytest.raises(cep.CepError, match="device"):
        cep.LoRAProjection(on_device(torch.zeros(16, 64, dtype=torch.bfloat16), 0), 4, stream=stream)
    assert not plans
