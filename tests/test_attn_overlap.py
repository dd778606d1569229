"""attn_append refuses a q_out that shares bytes with what other threads read, and nothing else: against the sets of bytes; runs without a
GPU.  (Every call here is refused, at the latest for a status that is not aligned; addresses are made up.)"""
import random

import pytest

import paper_2609_33252_b200 as cep

from test_attn_refusals import P, append


def touched(at, tokens, heads, token_stride, head_stride, dim):
    return {at + 2 * (t * token_stride + h * head_stride) + i for t in range(tokens) for h in range(heads) for i in range(2 * dim)}


def call(T, dim, q, q_out, k, v, heads=2, kv_heads=2):
    """Operands as (address, token stride, head stride); whether the call was refused for their overlap."""
    strides = {n + "_" + s + "_stride": x[i] for n, x in (("q", q), ("q_out", q_out), ("k", k), ("v", v)) for i, s in ((1, "token"), (2, "head"))}
    code = append(q=q[0], q_out=q_out[0], k=k[0], v=v[0], n_tokens=T, n_heads=heads, n_kv_heads=kv_heads, head_dim=dim, rotary_dim=dim, status=P + 1,
                  k_cache_stride=(1 << 12, 1 << 8, 64), v_cache_stride=(1 << 12, 1 << 8, 64), **strides)
    assert code == -1
    what = cep.cep_last_error()
    assert "overlaps" in what or "aligned" in what
    return "overlaps" in what


def test_in_place_and_side_by_side():
    D, W = 64, 8 * 64                                                # a token of one projection's output: 4 heads of q, 2 of k, 2 of v
    q, k, v = (P, W, D), (P + 2 * 4 * D, W, D), (P + 2 * 6 * D, W, D)
    far = (P + (1 << 20), 4 * D, D)
    for T in (1, 2, 300):
        args = dict(heads=4, kv_heads=2)
        assert not call(T, D, q, q, k, v, **args) and not call(T, D, q, far, k, v, **args)
        assert not call(T, D, (P, W, D), (P, W, D), k, v, **args)
        assert call(T, D, q, (P + 2 * D, W, D), k, v, **args)        # a head further
        assert call(T, D, q, k, k, v, **args) and call(T, D, far, (v[0] - 2, W, D), k, v, **args)
        assert call(T, D, q, (P + 2, W, D), k, v, **args)
        assert call(T, D, q, (P, W, 2 * D), k, v, **args)            # the same place, heads elsewhere
        assert call(T, D, q, (P + 2 * W, W, D), k, v, **args) == (T > 1)
        assert not call(T, D, q, (P + 2 * W * T, W, D), k, v, **args)


@pytest.mark.parametrize("seed", range(4))
def test_any_layout(seed):
    rng = random.Random(seed)
    seen = [0, 0]
    for _ in range(3000):
        T, heads, kv_heads, dim = rng.randint(1, 5), rng.randint(1, 4), rng.randint(1, 3), rng.choice([2, 4, 6])
        token_stride = dim + rng.randint(0, 60)
        operand = lambda: (P + 2 * rng.randint(-60, 60), token_stride, dim + rng.choice([0, 0, rng.randint(0, 20)]))
        q, q_out, k, v = operand(), operand(), operand(), operand()
        if rng.random() < 0.7:
            k, v = (k[0] + (1 << 19), *k[1:]), (v[0] + (1 << 20), *v[1:])
        if rng.random() < 0.2:
            q_out = q
        new = touched(*q_out[:1], T, heads, *q_out[1:], dim)
        meets = lambda x, n: bool(new & touched(x[0], T, n, *x[1:], dim))
        want = (q != q_out and meets(q, heads)) or meets(k, kv_heads) or meets(v, kv_heads)
        same = q[0] == q_out[0] and (heads == 1 or q[2] == q_out[2])     # (the stride of a single head means nothing)
        want = want and not (same and not meets(k, kv_heads) and not meets(v, kv_heads))
        assert call(T, dim, q, q_out, k, v, heads, kv_heads) == want
        seen[want] += 1
    assert min(seen) > 500
