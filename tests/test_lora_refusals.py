"""What the lora_* calls refuse before their first CUDA call, through the C ABI; runs without a GPU.  (Addresses are made
up; nothing dereferences them.)"""
import ctypes

import pytest

import paper_2609_33252_b200 as cep

P = 1 << 20
GOOD = dict(in_features=64, out_features=40, max_tokens=16, max_adapters=2, max_rank=8, out_elem=0)


def config(**kw):
    return cep.LoraConfig(**dict(GOOD, **kw))


@pytest.mark.parametrize("kw", [
    dict(in_features=0), dict(in_features=60), dict(out_features=0), dict(max_tokens=0), dict(max_adapters=-1), dict(max_adapters=4097),
    dict(max_rank=257), dict(max_rank=-1), dict(max_rank=0), dict(max_adapters=0), dict(out_elem=2)])
def test_configurations(kw):
    n = ctypes.c_size_t()
    assert cep.lib().lora_plan_workspace_bytes(ctypes.byref(config(**kw)), ctypes.byref(n)) == -1
    assert cep.lib().lora_bank_bytes(ctypes.byref(config(**kw)), ctypes.byref(n)) == -1
    assert "lora" in cep.cep_last_error()


def test_sizes():
    assert cep.lora_bank_bytes(config(max_adapters=0, max_rank=0)) == 0
    # 2 slots x 16 padded ranks x (64 + 40) bf16, and the slots' ranks and scales
    assert cep.lora_bank_bytes(config()) == 256 + 256 + 2 * 16 * 64 * 2 + 2 * 16 * 40 * 2
    small, large = cep.lora_plan_workspace_bytes(config()), cep.lora_plan_workspace_bytes(config(max_tokens=16384))
    assert 0 < small < large
    assert cep.lib().lora_plan_workspace_bytes(ctypes.byref(config()), None) == -1


@pytest.mark.parametrize("code,kw", [
    (-1, dict(weight=None)), (-1, dict(workspace=None)), (-1, dict(weight=P + 8)), (-1, dict(stride=56)), (-1, dict(stride=68)),
    (-3, dict(workspace_bytes=1024)), (-3, dict(workspace=P + 16)), (-3, dict(bank=None)), (-3, dict(bank_bytes=100)), (-3, dict(bank=P + 4))])
def test_plans(code, kw):
    a = dict(weight=P, stride=64, bank=P, bank_bytes=1 << 30, workspace=P, workspace_bytes=1 << 40)
    a.update(kw)
    h = ctypes.c_void_p()
    cfg = config()
    assert cep.lib().lora_plan(ctypes.byref(cfg), a["weight"], a["stride"], a["bank"], a["bank_bytes"], a["workspace"], a["workspace_bytes"],
                               None, ctypes.byref(h)) == code
    assert not h.value


def test_a_missing_plan_is_refused():
    L = cep.lib()
    assert L.lora_project(None, P, 64, 1, None, P, 40, None) == -1
    assert L.lora_load_adapter(None, 0, 1, 1.0, P, 64, P, 8, None) == -1
    assert L.lora_status(None) == -1
    assert L.lora_plan_destroy(None) == 0
    cfg = config()
    assert L.lora_plan(ctypes.byref(cfg), P, 64, P, 1 << 30, P, 1 << 40, None, None) == -1
