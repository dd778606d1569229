"""PrefixAttention with page tables that have room for far more keys than the batch has (costs of the schedule are scaled down, from a shift of 2 to
one of 9): same batches, formula and tolerances as test_gpu_attn.py (Batch.check)."""
import pytest
import torch

from test_gpu_attn import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("width", [1 << 15, 1 << 19, (1 << 22) - 1])
@pytest.mark.parametrize("heads,kv_heads,q_len,kv_len", [(128, 1, [400, 1, 5], [600, 300, 5]), (16, 2, [1] * 40 + [300], [30 * i for i in range(1, 41)] + [700])])
def test_wide_page_tables(heads, kv_heads, q_len, kv_len, width, e4m3):
    if width > 1 << 20 and len(q_len) > 3:
        width = 1 << 20                                              # (a table of 41 rows)
    b = Batch(q_len, kv_len, heads, kv_heads, 64, page=256, prefix=[300], e4m3=e4m3)
    want = b.check()
    for name in ("page_table", "prefix_pages"):
        t = b.meta[name]
        wide = torch.full((t.shape[0], width), -7, dtype=torch.int32, device="cuda")
        wide[:, :t.shape[1]] = t
        b.meta[name] = wide
    got = b.check()
    assert torch.equal(b.check(), got)
    # how the keys are split, and with it the order of sums, may differ: the bounds are the same
    assert got.shape == want.shape
