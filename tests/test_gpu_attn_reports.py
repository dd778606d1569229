"""What the attention operators report or refuse instead of a wrong result."""
import pytest
import torch

import paper_2609_33252_b200 as cep
from paper_2609_33252_b200.block import AttentionBlock

from test_gpu_attn import Batch, rand

pytestmark = pytest.mark.gpu


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("e4m3", [False, True])
def test_a_block_reports_slots_outside_the_cache(e4m3):
    pages, page, D = 3, 16, 64
    kv = [torch.zeros(pages, page, 2, D, device="cuda").to(torch.float8_e4m3fn if e4m3 else torch.bfloat16) for _ in range(2)]
    att = AttentionBlock(rand((10 * D, 128), 1, 128 ** -0.5), *kv, 6, torch.rand(D // 2, device="cuda"), 8, 4)
    x, positions = rand((4, 128), 2), i32([0, 1, 2, 0])
    batch = dict(q_start=i32([0, 3, 4]), kv_len=i32([3, 1]), page_table=i32([[0], [1]]))
    run = lambda slots: att.run(x, positions, torch.tensor(slots, device="cuda"), batch).clone()
    want = run([0, 1, 2, page])
    assert att.status() == 0
    raw = [c.view(torch.uint8).clone() for c in kv]
    for bad in (pages * page, -2, 1 << 40):
        run([0, 1, 2, bad])                                          # (the last token's place holds the values of the call before)
        assert att.status() == -6 and att.status() == 0
    assert all(torch.equal(c.view(torch.uint8), r) for c, r in zip(kv, raw))
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        run([pages * page, 1, 2, page])
    assert att.status() == -6
    assert torch.equal(run([0, 1, 2, -1]), want) and att.status() == 0     # -1 is no fault
    # the attention's own reports come through as well, and only once
    bad_batch = dict(batch, page_table=i32([[0], [pages]]))
    att.run(x, positions, torch.tensor([0, 1, 2, pages * page], device="cuda"), bad_batch)
    assert att.status() == -6 and att.status() == 0
    att.run(x, positions, torch.tensor([0, 1, 2, pages * page], device="cuda"), dict(batch, kv_len=i32([3, 100])))
    assert att.status() == -4 and att.status() == 0
    assert torch.equal(run([0, 1, 2, page]), want)
    att.close()


def test_an_output_that_overlaps_the_queries_is_refused():
    b = Batch([1, 30, 300, 2], [50, 30, 400, 2], 6, 2, 64, prefix=[200])
    want = b.check()
    T, meta = b.T, b.meta
    store = torch.zeros(T + 1, 13, 64, dtype=torch.bfloat16, device="cuda")
    store[:T, :6] = b.q
    q = store[:T, :6]
    turned = torch.zeros(6, 2 * T, 64, dtype=torch.bfloat16, device="cuda").transpose(0, 1)      # heads outside
    turned[:T] = b.q
    for x, out in ((b.q, b.q), (q, q), (q, store[:T, 5:11]), (q, store[1:, :6]), (q, store[1:, 3:9]), (turned[:T], turned[:T]), (turned[:T], turned[T - 1:2 * T - 1]),
                   (q, store.view(-1)[64:64 * (6 * T + 1)].view(T, 6, 64))):
        before = store.clone(), turned.clone()
        with pytest.raises(cep.CepError, match="overlaps"):
            b.layer.run(x, out=out, **meta)
        assert torch.equal(store, before[0]) and torch.equal(turned, before[1])
    # other columns, rows or heads of one buffer
    for x, out in ((q, store[:T, 6:12]), (q, store[:T, 7:13]), (turned[:T], turned[T:])):
        assert torch.equal(b.layer.run(x, out=out, **meta), want) and torch.equal(x, b.q)
    both = torch.stack((b.q, torch.zeros_like(b.q)), dim=2).view(T, 12, 64)                      # every other head
    assert torch.equal(b.layer.run(both[:, ::2], out=both[:, 1::2], **meta), want) and torch.equal(both[:, ::2], b.q)
    assert b.layer.status() == 0


def test_a_block_with_a_scale_of_its_own():
    D = 64
    kv = [torch.zeros(4, 16, 2, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    w, inv_freq = rand((10 * D, 128), 1, 128 ** -0.5), torch.rand(D // 2, device="cuda")
    x, positions, slots = rand((4, 128), 2), i32([0, 1, 2, 3]), torch.arange(4, device="cuda")
    batch = dict(q_start=i32([0, 4]), kv_len=i32([4]), page_table=i32([[0]]))
    outs = []
    for kw in ({}, dict(scale=D ** -0.5), dict(scale=0.7)):
        att = AttentionBlock(w, *kv, 6, inv_freq, 8, 1, **kw)
        outs.append(att.run(x, positions, slots, batch).clone())
        layer = cep.PrefixAttention(*kv, 6, 8, 1, **kw)
        assert torch.equal(layer.run(att.qkv[:4, :6], **batch).view(4, -1), outs[-1])
        assert att.status() == 0 and layer.status() == 0
        att.close()
        layer.close()
    assert torch.equal(outs[0], outs[1]) and not torch.equal(outs[0], outs[2])
