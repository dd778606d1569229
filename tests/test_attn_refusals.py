"""What attn_append and the attn_* calls refuse before their first CUDA call, through the C ABI, and what their Python wrappers
check; runs without a GPU.  (Addresses are made up; nothing dereferences them.)"""
import ctypes
import types

import pytest
import torch

import paper_2609_33252_b200 as cep
from paper_2609_33252_b200 import binding

from test_attn_schedule import config

P = 1 << 20


def append(q=None, k=P, v=P, positions=P, slots=P, inv_freq=P, q_out=None, k_cache=P, v_cache=P, k_scale=None, v_scale=None, status=None, **kw):
    d = dict(n_tokens=2, n_heads=0, n_kv_heads=2, head_dim=64, rotary_dim=64, interleaved=0, cache_elem=0, page_size=16, n_pages=4, q_token_stride=128,
             q_head_stride=64, q_out_token_stride=128, q_out_head_stride=64, k_token_stride=128, k_head_stride=64, v_token_stride=128, v_head_stride=64)
    d.update({n: x for n, x in kw.items() if n not in ("k_cache_stride", "v_cache_stride")})
    desc = cep.AppendDesc(**d)
    desc.k_cache_stride[:] = kw.get("k_cache_stride", (2048, 128, 64))
    desc.v_cache_stride[:] = kw.get("v_cache_stride", (2048, 128, 64))
    return cep.lib().attn_append(ctypes.byref(desc), q, k, v, positions, slots, inv_freq, q_out, k_cache, v_cache, k_scale, v_scale, status, None)


def test_an_append_of_no_tokens_does_nothing():
    assert append(n_tokens=0) == 0
    assert append(n_tokens=0, k=None, v=None, positions=None, slots=None, k_cache=None, v_cache=None) == 0


@pytest.mark.parametrize("code,kw", [
    (-1, dict(k=None)), (-1, dict(v=None)), (-1, dict(positions=None)), (-1, dict(slots=None)), (-1, dict(inv_freq=None)), (-1, dict(k_cache=None)),
    (-1, dict(n_tokens=-1)), (-1, dict(n_kv_heads=0)), (-1, dict(n_heads=-1)), (-1, dict(head_dim=63)), (-1, dict(head_dim=0)), (-1, dict(rotary_dim=66)),
    (-1, dict(rotary_dim=-2)), (-1, dict(rotary_dim=33)), (-9, dict(head_dim=1026)), (-9, dict(n_kv_heads=1 << 20)), (-1, dict(cache_elem=1)), (-1, dict(page_size=24)),
    (-1, dict(page_size=0)), (-1, dict(n_pages=0)), (-1, dict(n_pages=1 << 60)), (-1, dict(q=P)), (-1, dict(q=P, q_out=P)), (-1, dict(n_heads=2)), (-1, dict(n_heads=2, q=P)),
    (-1, dict(k_scale=P)), (-1, dict(v_scale=P)), (-1, dict(k_token_stride=60)), (-1, dict(v_head_stride=0)), (-1, dict(k_cache_stride=(2048, 128, 32))),
    (-1, dict(v_cache_stride=(0, 128, 64))), (-1, dict(n_heads=2, q=P, q_out=P, q_out_token_stride=8)), (-1, dict(k=P + 1)), (-1, dict(positions=P + 2)),
    (-1, dict(slots=P + 4)), (-1, dict(inv_freq=P + 2)), (-1, dict(status=P + 1)), (-1, dict(k_scale=P + 2, cache_elem=2))])
def test_appends_that_are_refused(code, kw):
    assert append(**kw) == code
    assert "append" in cep.cep_last_error()


def test_missing_things_are_refused():
    L, cfg, h = cep.lib(), config(16, 8, 64, 8, 1), ctypes.c_void_p()
    assert L.attn_append(None, *[P] * 12, None) == -1
    assert L.attn_prefix(None, *[P] * 10, None) == -1
    assert L.attn_status(None) == -1
    assert L.attn_plan_destroy(None) == 0
    assert L.attn_plan_workspace_bytes(ctypes.byref(cfg), None) == -1
    assert L.attn_plan_workspace_bytes(None, ctypes.byref(ctypes.c_size_t())) == -1
    assert L.attn_plan(ctypes.byref(cfg), P, P, None, None, P, 1 << 40, None, None) == -1
    for a in ((None, P, P), (P, None, P), (P, P, None), (P + 8, P, P)):
        assert L.attn_plan(ctypes.byref(cfg), a[0], a[1], None, None, a[2], 1 << 40, None, ctypes.byref(h)) == -1
    assert L.attn_plan(ctypes.byref(cfg), P, P, P + 2, None, P, 1 << 40, None, ctypes.byref(h)) == -1
    assert L.attn_plan(ctypes.byref(cfg), P, P, None, None, P, 1024, None, ctypes.byref(h)) == -3
    assert L.attn_plan(ctypes.byref(cfg), P, P, None, None, P + 16, 1 << 40, None, ctypes.byref(h)) == -3
    assert not h.value


def test_the_workspace_grows_with_what_it_holds():
    small, tokens, seqs = (cep.attn_plan_workspace_bytes(config(16, 8, *a)) for a in ((64, 8, 1), (4096, 8, 1), (4096, 512, 1)))
    assert 0 < small < tokens < seqs


def on_device(t, index=0):
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
def calls(monkeypatch):
    """No GPU, device 0 current; the list of what reaches the library."""
    made = []
    fake = lambda name: lambda *a: made.append((name, a)) or 0
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 0, raising=False)
    monkeypatch.setattr(binding, "_lib", types.SimpleNamespace(attn_append=fake("append"), attn_prefix=fake("prefix")))
    monkeypatch.setattr(binding, "attn_plan_workspace_bytes", lambda cfg: 16)
    monkeypatch.setattr(binding, "attn_plan", lambda *a: made.append(("plan", a)))                # (no handle: nothing to destroy)
    return made


def tensors(T=3, Hq=4, Hk=2, D=16, **kw):
    bf16 = torch.bfloat16
    t = dict(k=torch.zeros(T, Hk, D, dtype=bf16), v=torch.zeros(T, Hk, D, dtype=bf16), positions=torch.zeros(T, dtype=torch.int32), slots=torch.zeros(T, dtype=torch.int64),
             inv_freq=torch.zeros(D // 2), k_cache=torch.zeros(2, 16, Hk, D, dtype=bf16), v_cache=torch.zeros(2, 16, Hk, D, dtype=bf16),
             q=torch.zeros(T, Hq, D, dtype=bf16), q_out=torch.zeros(T, Hq, D, dtype=bf16))
    t.update(kw)
    return {n: None if x is None else x if hasattr(x, "recorded") else on_device(x) for n, x in t.items()}


def run_append(t, **kw):
    t = dict(t)
    first = [t.pop(n) for n in ("k", "v", "positions", "slots", "inv_freq", "k_cache", "v_cache")]
    return cep.attn_append(*first, **t, **kw)


@pytest.mark.parametrize("kw", [
    dict(k=torch.zeros(3, 2, 16)), dict(v=torch.zeros(3, 2, 18, dtype=torch.bfloat16)), dict(positions=torch.zeros(3, dtype=torch.int64)), dict(slots=torch.zeros(4, dtype=torch.int64)),
    dict(slots=torch.zeros(3, dtype=torch.int32)), dict(inv_freq=torch.zeros(8, dtype=torch.float64)), dict(q=torch.zeros(4, 4, 16, dtype=torch.bfloat16)), dict(q=None),
    dict(k_cache=torch.zeros(2, 16, 2, 16)), dict(v_cache=torch.zeros(3, 16, 2, 16, dtype=torch.bfloat16)), dict(q_out=torch.zeros(3, 4, 16)),
    dict(k=on_device(torch.zeros(3, 2, 16, dtype=torch.bfloat16), 1)), dict(v_cache=on_device(torch.zeros(2, 16, 2, 16, dtype=torch.bfloat16), 1)),
    dict(k=torch.zeros(3, 2, 32, dtype=torch.bfloat16)[..., ::2]), dict(status=torch.zeros(2, dtype=torch.int32)), dict(k_scale=torch.zeros(3)),
    dict(k=torch.zeros(3, 32, dtype=torch.bfloat16))])
def test_appends_that_the_binding_refuses(calls, kw):
    with pytest.raises(cep.CepError):
        run_append(tensors(**kw))
    assert not calls


def test_append_records_its_tensors_on_the_stream_it_is_given(calls):
    t = tensors(status=torch.zeros(1, dtype=torch.int32))
    assert run_append(t) is t["q_out"]
    assert all(x.recorded == () for x in t.values())                 # the current stream's order is torch's
    stream = types.SimpleNamespace(cuda_stream=5)
    run_append(t, stream=stream)
    assert all(x.recorded == (stream,) for x in t.values()) and len(calls) == 2


def plan(**kw):
    cache = lambda: on_device(torch.zeros(4, 16, 2, 16, dtype=torch.bfloat16))
    a = dict(k_cache=cache(), v_cache=cache(), n_heads=4, max_tokens=8, max_seqs=2)
    a.update(kw)
    return cep.PrefixAttention(**a)


@pytest.mark.parametrize("kw", [
    dict(k_cache=on_device(torch.zeros(4, 16, 2, 16))), dict(v_cache=on_device(torch.zeros(4, 16, 2, 32, dtype=torch.bfloat16))),
    dict(v_cache=on_device(torch.zeros(4, 16, 2, 16, dtype=torch.bfloat16), 1)), dict(k_scale=on_device(torch.zeros(2), 1)), dict(k_scale=on_device(torch.zeros(3))),
    dict(stream=types.SimpleNamespace(cuda_stream=5, device=torch.device("cuda", 1)))])
def test_plans_that_the_binding_refuses(calls, kw):
    with pytest.raises(cep.CepError):
        plan(**kw)
    assert not calls


def batch(**kw):
    i32 = lambda *n: torch.zeros(*n, dtype=torch.int32)
    t = dict(q=torch.zeros(3, 4, 16, dtype=torch.bfloat16), q_start=i32(3), kv_len=i32(2), page_table=i32(2, 5), prefix_len=i32(1), prefix_pages=i32(1, 7),
             out=torch.zeros(3, 4, 16, dtype=torch.bfloat16))
    t.update(kw)
    return {n: None if x is None else x if hasattr(x, "recorded") else on_device(x) for n, x in t.items()}


@pytest.mark.parametrize("kw", [
    dict(q=torch.zeros(3, 4, 16)), dict(q=torch.zeros(3, 5, 16, dtype=torch.bfloat16)), dict(q_start=torch.zeros(2, dtype=torch.int32)), dict(kv_len=torch.zeros(2, dtype=torch.int64)),
    dict(page_table=torch.zeros(3, 5, dtype=torch.int32)), dict(page_table=torch.zeros(2, 5, dtype=torch.int64)), dict(prefix_pages=None), dict(prefix_len=None),
    dict(prefix_pages=torch.zeros(2, 7, dtype=torch.int32)), dict(prefix_start=torch.zeros(1, dtype=torch.int32)), dict(out=torch.zeros(3, 4, 16)),
    dict(prefix_len=torch.zeros(2, dtype=torch.int32), prefix_pages=torch.zeros(2, 7, dtype=torch.int32)), dict(lse=torch.zeros(3, 5)), dict(lse=torch.zeros(3, 4, dtype=torch.float64)),
    dict(q=on_device(torch.zeros(3, 4, 16, dtype=torch.bfloat16), 1)), dict(q=torch.zeros(3, 4, 32, dtype=torch.bfloat16)[..., ::2])])
def test_batches_that_the_binding_refuses(calls, kw):
    layer = plan()
    with pytest.raises(cep.CepError):
        layer.run(**batch(**kw))
    assert [c[0] for c in calls] == ["plan"]


def test_run_records_its_tensors_on_the_stream_it_is_given(calls):
    layer, t = plan(), batch(lse=torch.zeros(3, 4), prefix_start=torch.zeros(2, dtype=torch.int32))
    assert layer.run(**t) is t["out"]
    assert all(x.recorded == () for x in t.values())
    stream = types.SimpleNamespace(cuda_stream=5)
    layer.run(**t, stream=stream)
    assert all(x.recorded == (stream,) for x in t.values())
