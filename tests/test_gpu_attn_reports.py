"""What the attention operators report or refuse instead of a wrong result."""
import pytest
import torch

import paper_2609_33252_b200 as cep
from paper_2609_33252_b200.block import AttentionBlock

from test_gpu_attn import rand

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
