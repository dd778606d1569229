"""The schedule of the attention behind shared prefixes (test_attn_schedule.py) where page tables have room for far more keys than the call has:
costs are scaled down so that their sum stays within 32 bits, which may not change how even the shares are; runs without a GPU.

The tables' room: that of a sequence without tokens, which has no work but a length."""
import random

import pytest

import paper_2609_33252_b200 as cep

from test_attn_schedule import check, config


def work_of_ctas(heads, kv_heads, q_len, kv_len, n_ctas, prefix=0):
    """Per CTA: 128 keys of two row tiles cost 512 units, an item 1200 beside them (a part of an item its part)."""
    starts = [0]
    for n in q_len:
        starts.append(starts[-1] + n)
    pre = dict(prefix_start=[0, len(q_len)], prefix_len=[prefix]) if prefix else {}
    parts, _ = cep.cep_debug_attn_schedule(config(heads, kv_heads, starts[-1], len(q_len), 1 if prefix else 0), starts, kv_len, causal=True, n_ctas=n_ctas, **pre)
    work = [0] * n_ctas
    for p in parts:
        work[p["cta"]] += (p["end"] - p["first"]) * (512 + 1200 / p["steps"])
    return work


@pytest.mark.parametrize("room", [1 << 14, 1 << 20, 1 << 24])
@pytest.mark.parametrize("heads,kv_heads,tokens", [(128, 1, 16384), (64, 1, 30000), (128, 2, 16384), (56, 8, 16384)])
def test_a_long_prompt_is_shared_evenly_whatever_the_tables_hold(heads, kv_heads, tokens, room):
    work = work_of_ctas(heads, kv_heads, [tokens, 0], [tokens, max(room, tokens)], 148)
    mean = sum(work) / 148
    # Shares are equal in estimated cost: 1200 + 4 keys an item, of which up to 512 are missing where a step is not full (512 / 1200: at most 43 %, in
    # the first items), and up to two units of 2^8 too much by the scaling (2^39 / 2e9), 1.5 % of a mean item's 34000; and a share ends on a step.
    assert max(work) <= 1.45 * mean + 2 * 1712, (max(work), mean)


@pytest.mark.parametrize("room", [1 << 20, 1 << 26, (1 << 30) - 256])
@pytest.mark.parametrize("heads,kv_heads", [(8, 8), (16, 2), (56, 8), (128, 1)])
def test_every_key_once_with_wide_tables(heads, kv_heads, room):
    rng = random.Random(room + heads)
    for _ in range(12):
        B = rng.choice([1, 2, 17])
        q_len = [rng.choice([1, 1, 5, 700, 3000]) for _ in range(B)] + [0]
        kv_len = [n + rng.choice([0, 0, rng.randint(0, 3000)]) for n in q_len[:-1]] + [room]
        check(heads, kv_heads, q_len, kv_len, [0, B + 1], [rng.choice([0, 129, rng.randint(1, 9000)])], rng.random() < 0.8, rng.choice([7, 148]))
