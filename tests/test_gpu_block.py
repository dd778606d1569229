"""The operators in front of the expert layer, run together with it (block.MoEBlock), step by step against each step's
formula in 64 bits on the step's own inputs, and the expert layer against the oracle on what they produced."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_33252_b200 as cep
from paper_2609_33252_b200 import workloads as wl
from paper_2609_33252_b200.block import MoEBlock

from helpers import check_close

pytestmark = pytest.mark.gpu


def make(dtype, T, seed=3):
    base = wl.CONFIGS["mxfp4_tiny" if dtype == "mxfp4" else "tiny"]
    cfg = wl.scaled(base, T=T, chunks=(T,), dtype=dtype)
    host = wl.make_inputs(cfg)
    H, A = cfg.H, 384
    g = torch.Generator().manual_seed(seed)
    rand = lambda *shape, std=1.0: (torch.randn(shape, generator=g) * std).to(torch.bfloat16).cuda()
    w = dict(out=rand(H, A, std=A ** -0.5), norm=1 + rand(H, std=0.1), router=rand(cfg.E_global, H, std=4 * H ** -0.5))
    block = MoEBlock(w["out"], w["norm"], w["router"], cfg.I, cfg.E_local, cfg.k, T, max_chunks=3, dtype=cep.DTYPE_OF[dtype], max_adapters=2, max_rank=16)
    ad = [(rand(r, A, std=A ** -0.5), rand(H, r, std=r ** -0.5), s) for r, s in ((16, 0.5), (8, 2.0))]
    for i, (a, b, s) in enumerate(ad):
        block.projection.load_adapter(i, a, b, s)
    dev = lambda t: None if t is None else t.cuda()
    block.load_experts(dev(host.w_gate), dev(host.w_up), dev(host.w_down), dev(host.s_gate), dev(host.s_up), dev(host.s_down))
    attention, residual = rand(T, A), rand(T, H)
    ids = torch.randint(-1, 2, (T,), generator=g).to(torch.int32).cuda()
    return cfg, host, w, block, ad, attention, residual, ids


@pytest.mark.parametrize("n_chunks", [1, 3])
@pytest.mark.parametrize("T", [1, 96, 300])
@pytest.mark.parametrize("dtype", ["bf16", "fp8", "mxfp4"])
def test_block(dtype, T, n_chunks):
    cfg, host, w, block, ad, attention, residual, ids = make(dtype, T)
    before = residual.clone()
    out = block.run(attention, residual, ids, n_chunks=n_chunks if T > 1 else 1)
    torch.cuda.synchronize()
    assert cep.ffn_status(block.layer.plan) == 0 and block.projection.status() == 0
    # projection and adapters: half a unit of bf16, and the fp32 sums
    delta = attention.double() @ w["out"].double().t()
    for i, (a, b, s) in enumerate(ad):
        rows = ids.long() == i
        delta[rows] += s * (attention[rows].double() @ a.double().t()) @ b.double().t()
    got = block.delta[:T].double()
    assert (torch.abs(got - delta) <= 2 ** -8 * delta.abs() + 1e-4).all()
    # residual and norm, from the projection's output
    h = got + before.double()
    assert torch.equal(residual, (block.delta[:T].float() + before.float()).to(torch.bfloat16))
    y = h / torch.sqrt((h * h).mean(dim=1, keepdim=True) + block.eps) * w["norm"].double()
    assert (torch.abs(block.y[:T].double() - y) <= (2 ** -8 + 1e-5) * y.abs()).all()
    # the router, from the norm's output: logits, then exactly the selection its own logits give
    logits = block.y[:T].double() @ w["router"].double().t()
    assert ((block.logits[:T].double() - logits).norm() / logits.norm()).item() <= 1.3e-6
    want_ids, want_w = wl.route(block.logits[:T], cfg.k)
    assert torch.equal(block.ids[:T], want_ids) and torch.allclose(block.weights[:T], want_w, rtol=5e-6, atol=0)
    # the experts, from the codes and scales (or the bf16 rows) that the norm wrote
    import dataclasses
    x = block.y[:T] if dtype == "bf16" else block.codes[:T]
    xs = None if dtype == "bf16" else block.scales[:T].cpu()
    ref = oracle.from_inputs(dataclasses.replace(host, x=x.cpu(), x_scale=xs, topk_ids=block.ids[:T].cpu(), topk_w=block.weights[:T].cpu()))
    check_close(out, ref, "%s, %d tokens" % (dtype, T))
    block.close()


def test_command_runs(capsys):
    from paper_2609_33252_b200 import block
    block.main("mxfp4", 512)
    lines = capsys.readouterr().out.strip().splitlines()
    assert len(lines) == 5 and all(l.endswith("us") for l in lines)
