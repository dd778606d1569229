"""What LoRAProjection and the wrappers of the lora_* calls check and pass on, with the library and CUDA faked; runs without
a GPU."""
import types

import pytest
import torch

import paper_2609_33252_b200 as cep
from paper_2609_33252_b200 import binding


def on_device(t, index):
    """A CPU tensor as a CUDA tensor of device `index` looks to the binding; `recorded`: the streams it was recorded on."""
    class Fake:
        is_cuda = True
        get_device = staticmethod(lambda: index)
        recorded = ()

        def record_stream(self, stream):
            self.recorded += (stream,)

        def __getattr__(self, name):
            return getattr(t, name)
    return Fake()


@pytest.fixture
def plans(monkeypatch):
    """No GPU, device 0 current; returns the list of (what, arguments) that reach the library."""
    made = []
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(binding, "lora_plan", lambda *a: made.append(("plan", a)))                # (no handle: nothing to destroy)
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


def test_run_records_its_tensors_on_the_stream_it_is_given(plans, monkeypatch):
    # the caller may drop them at once: their memory is not to be given away before the stream has used it
    monkeypatch.setattr(binding, "lora_project", lambda *a: plans.append(("project", a)))
    layer = cep.LoRAProjection(on_device(torch.zeros(16, 64, dtype=torch.bfloat16), 0), 4, 1, 8)
    x, ids = on_device(torch.zeros(4, 64, dtype=torch.bfloat16), 0), on_device(torch.zeros(4, dtype=torch.int32), 0)
    out = on_device(torch.zeros(4, 16, dtype=torch.bfloat16), 0)
    layer.run(x, ids, out)
    assert x.recorded == ids.recorded == out.recorded == ()                  # the current stream's order is torch's
    stream = types.SimpleNamespace(cuda_stream=5)
    layer.run(x, ids, out, stream=stream)
    assert x.recorded == ids.recorded == out.recorded == (stream,)
    layer.run(x, None, out, stream=stream)


def test_norm_records_its_tensors_on_the_stream_it_is_given(monkeypatch):
    monkeypatch.setattr(binding, "_lib", types.SimpleNamespace(moe_norm=lambda *a: 0))
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 0)
    t = dict(x=torch.zeros(3, 256, dtype=torch.bfloat16), weight=torch.zeros(256), residual=torch.zeros(3, 256),
             residual_out=torch.zeros(3, 256), y=torch.zeros(3, 256, dtype=torch.bfloat16),
             codes=torch.zeros(3, 256, dtype=torch.float8_e4m3fn), scales=torch.zeros(3, 2))
    t = {k: on_device(v, 0) for k, v in t.items()}
    cep.moe_norm(**t, dtype=cep.CEP_FP8_E4M3_BLOCK128)
    assert all(v.recorded == () for v in t.values())
    stream = types.SimpleNamespace(cuda_stream=5)
    cep.moe_norm(**t, dtype=cep.CEP_FP8_E4M3_BLOCK128, stream=stream)
    assert all(v.recorded == (stream,) for v in t.values())
    cep.moe_norm(t["x"], y=t["y"], stream=stream)


@pytest.mark.parametrize("at", range(9))
def test_the_first_norm_of_one_thread_does_not_disturb_anothers(monkeypatch, at):
    # another thread's first call in the middle of this one's: here where the first call looks up its `at`-th type
    monkeypatch.setattr(binding, "_lib", types.SimpleNamespace(moe_norm=lambda *a: 0))
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 0)
    fresh = dict(vars(binding))
    for name in ("_ELEM", "_NORM_DTYPES", "_norm_types"):
        if name in fresh:
            monkeypatch.setattr(binding, name, type(fresh[name])() if fresh[name] is not None else None)
    x, weight = on_device(torch.zeros(3, 256, dtype=torch.bfloat16), 0), on_device(torch.zeros(256), 0)
    y = on_device(torch.zeros(3, 256, dtype=torch.bfloat16), 0)
    calls = []

    class Torch:
        def __getattr__(self, name):
            if name != "_C":
                calls.append(name)
                if len(calls) == at + 1:
                    cep.moe_norm(x, weight, y=y)
            return getattr(torch, name)

    monkeypatch.setattr(binding, "_torch_module", Torch())
    cep.moe_norm(x, weight, y=y)
    assert len(calls) >= 5


def test_an_adapter_of_one_row_may_have_any_row_stride(plans, monkeypatch):
    # the stride of a dimension of one element means nothing; torch calls these tensors contiguous
    given = []
    monkeypatch.setattr(binding, "lib", lambda: types.SimpleNamespace(lora_load_adapter=lambda *a: given.append(a) or 0))
    down = torch.zeros(64, 1, dtype=torch.bfloat16).t()
    up = torch.zeros(16, 1, dtype=torch.bfloat16)
    assert down.is_contiguous() and down.stride(0) == 1
    binding.lora_load_adapter(7, 0, 1, 1.0, down, up, stream=5)
    assert given[0][5] >= 64 and given[0][7] >= 1
    up = torch.zeros(8, 1, dtype=torch.bfloat16).t()           # one output column
    assert up.stride(0) == 1
    binding.lora_load_adapter(7, 0, 8, 1.0, torch.zeros(8, 64, dtype=torch.bfloat16), up, stream=5)
    assert given[1][5] == 64 and given[1][7] >= 8
