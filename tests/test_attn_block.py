"""What AttentionBlock hands to its steps and what it makes of their reports, with the steps and CUDA faked; runs without a GPU."""
import types

import pytest
import torch

from paper_2609_33252_b200 import block as blocks

HQ, HK, D, H = 4, 2, 16, 32


class Event:
    def __init__(self, log):
        self.log = log

    def record(self, stream=None):
        self.log.append("done")

    def synchronize(self):
        self.log.append("waited")


@pytest.fixture
def fake(monkeypatch):
    """The steps as a log of their names; `codes`: what the projection's and the attention's status() return; `fail`: a step that raises."""
    f = types.SimpleNamespace(log=[], codes={"projection": 0, "attention": 0}, appended=[], made=[], fail=None)

    def step(name):
        if f.fail == name:
            raise blocks.cep.CepError(-1, name)
        f.log.append(name)

    class Layer:
        def __init__(self, name, *a, **kw):
            self.name, self.k_scale, self.v_scale = name, None, None
            f.made.append((name, a, kw))
            if name == "attention":
                self.k_cache, self.v_cache = a[:2]

        def run(self, *a, **kw):
            step(self.name)

        def status(self):
            code, f.codes[self.name] = f.codes[self.name], 0
            return code
    stream = types.SimpleNamespace(wait_event=lambda e: f.log.append("wait"), synchronize=lambda: f.log.append("cleared"))
    monkeypatch.setattr(blocks.cep, "LoRAProjection", lambda *a, **kw: Layer("projection", *a, **kw))
    monkeypatch.setattr(blocks.cep, "PrefixAttention", lambda *a, **kw: Layer("attention", *a, **kw))
    monkeypatch.setattr(blocks.cep, "attn_append", lambda *a, **kw: (f.appended.append(kw), step("append")))
    monkeypatch.setattr(torch.cuda, "Event", lambda: Event(f.log))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: stream)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    return f


def make(**kw):
    cache = torch.zeros(4, 16, HK, D, dtype=torch.bfloat16)
    return blocks.AttentionBlock(torch.zeros((HQ + 2 * HK) * D, H, dtype=torch.bfloat16), cache, cache.clone(), HQ, torch.ones(D // 2), 8, 2, **kw)


def run(block, T=3):
    return block.run(torch.zeros(T, H, dtype=torch.bfloat16), torch.zeros(T, dtype=torch.int32), torch.zeros(T, dtype=torch.int64), {})


def test_slots_outside_the_cache_are_reported_once(fake):
    block = make()
    run(block)
    status = fake.appended[0]["status"]                              # (what the write into the cache sets)
    assert status.dtype is torch.int32 and status.shape == (1,) and int(status) == 0
    assert block.status() == 0
    status.fill_(1)
    assert block.status() == -6 and fake.log[-1] == "cleared" and int(status) == 0
    assert block.status() == 0


@pytest.mark.parametrize("codes,slot,want", [((-7, 0), 0, -7), ((0, -4), 0, -4), ((-6, -4), 1, -6), ((0, -4), 1, -4), ((0, 0), 1, -6)])
def test_the_first_report_is_returned_and_all_are_cleared(fake, codes, slot, want):
    block = make()
    run(block)
    fake.codes.update(projection=codes[0], attention=codes[1])
    fake.appended[0]["status"].fill_(slot)
    assert block.status() == want
    assert block.status() == 0


def test_what_a_refused_call_has_started_is_waited_for(fake):
    # the next call may come on another stream: it would write the buffers that the steps before the refusal still use
    block = make()
    fake.log.clear()
    fake.fail = "attention"
    with pytest.raises(blocks.cep.CepError):
        run(block)
    assert fake.log == ["wait", "projection", "append", "done"]


def test_what_a_refused_call_of_the_expert_block_has_started_is_waited_for(fake):
    def refuse():
        raise blocks.cep.CepError(-1, "refused")
    block = object.__new__(blocks.MoEBlock)
    block.H, block.done = H, torch.cuda.Event()
    block.steps = lambda *a: [("first", lambda: fake.log.append("first")), ("second", refuse)]
    with pytest.raises(blocks.cep.CepError):
        block.run(torch.zeros(3, H), torch.zeros(3, H))
    assert fake.log == ["wait", "first", "done"]


@pytest.mark.parametrize("kw,want", [({}, None), (dict(scale=0.03), 0.03)])
def test_the_scale_of_the_scores_reaches_the_attention(fake, kw, want):
    make(**kw)
    (name, args, options), = [m for m in fake.made if m[0] == "attention"]
    assert options == {} and args[8] == want                         # k_cache, v_cache, heads, tokens, seqs, prefixes, two scales, scale
