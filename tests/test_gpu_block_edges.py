"""MoEBlock where calls meet: several streams, no tokens (the steps' formulas: test_gpu_block.py)."""
import pytest
import torch

import paper_2609_33252_b200 as cep

from test_gpu_block import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "mxfp4"])
def test_calls_on_different_streams(dtype):
    # one block's buffers between the steps are shared: the calls take turns
    cfg, host, w, block, ad, attention, residual, ids = make(dtype, 300)
    inputs = [(attention, residual, ids), (attention.flip(0).contiguous(), residual.flip(0).contiguous(), ids.flip(0).contiguous())]
    want = [(block.run(a, r1, i), r1) for a, r, i in inputs for r1 in [r.clone()]]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for n in range(12):
        a, r, i = inputs[n % 2]
        with torch.cuda.stream(streams[n % 2]):
            r1 = r.clone()
            got.append((block.run(a, r1, i, n_chunks=1 + n % 3), r1))
    torch.cuda.synchronize()
    assert cep.ffn_status(block.layer.plan) == 0 and block.projection.status() == 0
    for n, (out, r1) in enumerate(got):
        assert torch.equal(r1, want[n % 2][1]) and torch.equal(out, want[n % 2][0]), n
    block.close()


@pytest.mark.parametrize("dtype", ["bf16", "mxfp4"])
def test_no_tokens(dtype):
    # a rank without tokens in this step
    cfg, host, w, block, ad, attention, residual, ids = make(dtype, 40)
    want = block.run(attention, residual.clone(), ids)
    out = block.run(attention[:0], residual[:0], ids[:0])
    assert out.shape == (0, cfg.H) and out.dtype == torch.bfloat16
    assert block.run(attention[:0], residual[:0], n_chunks=3).shape == (0, cfg.H)
    assert torch.equal(block.run(attention, residual, ids), want)
    torch.cuda.synchronize()
    assert cep.ffn_status(block.layer.plan) == 0
    block.close()


def test_fewer_tokens_than_chunks():
    cfg, host, w, block, ad, attention, residual, ids = make("bf16", 2)
    want = block.run(attention, residual.clone(), ids)
    assert torch.equal(block.run(attention, residual, ids, n_chunks=3), want)
    torch.cuda.synchronize()
    assert cep.ffn_status(block.layer.plan) == 0
    block.close()
