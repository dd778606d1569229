"""Rows with one strong key among many weak ones: what the weak ones add.

The strong key's value is 0, the others' 1, so that the output is sum of the weak weights / sum of all.  With all weak scores d below the strong
one (in powers of two) a weak weight is 2^-d of the strong one.  Error: half a step of a weight (bf16 2^-8; fp16 2^-11, and 2^-32 of the strong
one below fp16's normal range), of the result (2^-8), and the exponents': scores are sums of at most 64 exact products (of ones: exact),
scale and its product with the maximum are each off by 2^-24 of d and the exponential by 2^-22, together less than 2^-17 of a weight here."""
import math

import pytest
import torch

import paper_2609_33252_b200 as cep

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("n", [2, 100, 1000])
@pytest.mark.parametrize("tokens,heads", [(1, 1), (3, 8), (200, 4)])
@pytest.mark.parametrize("d", [3.4, 7.9, 8.2, 13.6, 20.5, 24.6, 25.5, 28.4])
def test_weak_keys_beside_a_strong_one(d, tokens, heads, n, e4m3):
    page, D = 16, 64
    pages = -(-n // page)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    for at in (0, n // 2, n - 1):
        k, v = (torch.full((pages, page, 1, D), x, device="cuda") for x in (0.0, 1.0))
        k[at // page, at % page], v[at // page, at % page] = 1.0, 0.0
        kind = torch.float8_e4m3fn if e4m3 else torch.bfloat16
        layer = cep.PrefixAttention(k.to(kind), v.to(kind), heads, tokens, 1, scale=d * math.log(2) / D)
        lse = torch.zeros(tokens, heads, device="cuda")
        got = layer.run(torch.ones(tokens, heads, D, dtype=torch.bfloat16, device="cuda"), i32([0, tokens]), i32([n]), i32([list(range(pages))]), causal=False, lse=lse)
        assert layer.status() == 0
        scale = torch.tensor(d * math.log(2) / D, dtype=torch.float32).double()            # (as the plan holds it)
        weak = (n - 1) * float(torch.exp(-scale * D))
        want = weak / (1 + weak)
        near = want * (2.0 ** -8 + (2.0 ** -11 if e4m3 else 2.0 ** -8) + 2.0 ** -16) + (e4m3 and (n - 1) * 2.0 ** -32)
        assert float((got.double() - want).abs().max()) <= near
        assert float((lse.double() - float(scale * D) - math.log1p(weak)).abs().max()) <= 2.0 ** -17 + 2.0 ** -23 * d
        layer.close()
