"""From an attention block's output to the expert layer's result, with the library's operators in the order a server
runs them: the output projection with per-request low-rank adapters, the residual's addition with the norm and the
expert layer's activation format, the router's logits and selection, the routed experts.

``python -m paper_2609_33252_b200.block [dtype] [tokens]`` runs it on random weights and prints the device time of every
step (dtype: bf16, fp8 or mxfp4).
"""
from __future__ import annotations

import sys

import torch

from . import binding as cep
from . import workloads as wl


class MoEBlock:
    """Owns the plans and the buffers between the steps.  All weights are the caller's tensors.

    w_out bf16 [H, A] (attention width A), norm_weight bf16 or fp32 [H], w_router bf16 [E_global, H]; ``load_experts``
    takes what ``MoELayer.load_weights`` takes.  ``run`` may be called on different streams: each call waits for the one
    before, as the buffers between the steps are shared (who runs ``steps`` orders them).
    """

    def __init__(self, w_out, norm_weight, w_router, inter, n_experts_local, top_k, max_tokens, max_chunks=1, dtype=cep.CEP_BF16,
                 max_adapters=0, max_rank=0, eps=1e-6, **layer_options):
        H, E = w_out.shape[0], w_router.shape[0]
        dev = w_out.device
        self.H, self.k, self.dtype, self.eps = H, top_k, dtype, eps
        self.norm_weight = norm_weight
        self.projection = cep.LoRAProjection(w_out, max_tokens, max_adapters, max_rank)
        self.router = cep.LoRAProjection(w_router, max_tokens, out_elem=cep.CEP_ELEM_FP32)
        self.layer = cep.MoELayer(H, inter, E, n_experts_local, top_k, max_tokens, max_chunks, dtype=dtype, device=dev, **layer_options)
        empty = lambda *shape, dtype: torch.empty(shape, dtype=dtype, device=dev)
        self.delta = empty(max_tokens, H, dtype=torch.bfloat16)
        self.y = empty(max_tokens, H, dtype=torch.bfloat16)
        self.logits = empty(max_tokens, E, dtype=torch.float32)
        self.ids = empty(max_tokens, top_k, dtype=torch.int32)
        self.weights = empty(max_tokens, top_k, dtype=torch.float32)
        self.done = torch.cuda.Event()                       # the end of the last call
        self.codes = self.scales = None
        if dtype != cep.CEP_BF16:
            self.codes = empty(max_tokens, H, dtype=torch.float8_e4m3fn)
            self.scales = (empty(max_tokens, H // 128, dtype=torch.float32) if dtype == cep.CEP_FP8_E4M3_BLOCK128 else
                           empty(max_tokens, H // 32, dtype=torch.uint8))

    def load_experts(self, *weights, **kw):
        self.layer.load_weights(*weights, **kw)

    def steps(self, attention, residual, adapter_ids, out, n_chunks=1):
        """The block as (name, call) pairs; running the calls in order runs the block.  residual [T,H] is updated in place."""
        T = attention.shape[0]
        delta, y, logits, ids, w = (t[:T] for t in (self.delta, self.y, self.logits, self.ids, self.weights))
        codes, scales = (None, None) if self.codes is None else (self.codes[:T], self.scales[:T])
        cuts = [T * c // n_chunks for c in range(n_chunks + 1)]
        x, xs = (y, None) if codes is None else (codes, scales)
        chunks = [(a, x[a:b], None if xs is None else xs[a:b], ids[a:b], w[a:b]) for a, b in zip(cuts, cuts[1:])]
        return [
            ("projection + adapters", lambda: self.projection.run(attention, adapter_ids, delta)),
            ("residual + norm + format", lambda: cep.moe_norm(delta, self.norm_weight, self.eps, residual=residual, residual_out=residual, y=y,
                                                              codes=codes, scales=scales, dtype=self.dtype)),
            ("router logits", lambda: self.router.run(y, None, logits)),
            ("router selection", lambda: cep.moe_route(logits, self.k, ids, w)),
            ("routed experts", lambda: self.layer.run(out, chunks)),
        ]

    def run(self, attention, residual, adapter_ids=None, out=None, n_chunks=1):
        """attention bf16 [T,A], residual bf16 or fp32 [T,H] (updated in place), adapter_ids int32 [T] or None.
        Returns the experts' output bf16 [T,H], to be added to the residual by the next layer's norm."""
        if out is None:
            out = torch.empty(attention.shape[0], self.H, dtype=torch.bfloat16, device=attention.device)
        if attention.shape[0] == 0:                          # (empty tensors have no address, which the layer's calls refuse)
            return out
        stream = torch.cuda.current_stream(attention.device)
        stream.wait_event(self.done)                         # (before the first call: nothing to wait for)
        for _, call in self.steps(attention, residual, adapter_ids, out, n_chunks):
            call()
        self.done.record(stream)
        return out

    def close(self):
        self.projection.close()
        self.router.close()
        self.layer.close()


def main(dtype="mxfp4", tokens=4096):
    cfg = wl.scaled(wl.CONFIGS["mid"], T=tokens, chunks=(tokens,), dtype=dtype)
    inp = wl.make_inputs(cfg, device="cuda")
    H, g = cfg.H, torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *shape, std=1.0: (torch.randn(shape, generator=g, device="cuda") * std).to(torch.bfloat16)
    block = MoEBlock(rand(H, H, std=H ** -0.5), 1 + rand(H, std=0.1), rand(cfg.E_global, H, std=H ** -0.5), cfg.I, cfg.E_local, cfg.k, tokens,
                     max_chunks=4, dtype=cep.DTYPE_OF[dtype], max_adapters=4, max_rank=32)
    for s in range(4):
        block.projection.load_adapter(s, rand(32, H, std=H ** -0.5), rand(H, 32, std=32 ** -0.5), 0.5)
    block.load_experts(inp.w_gate, inp.w_up, inp.w_down, inp.s_gate, inp.s_up, inp.s_down)
    attention, residual = rand(tokens, H), rand(tokens, H)
    adapters = (torch.arange(tokens, device="cuda") * 5 // tokens - 1).to(torch.int32)       # five requests, the first without
    out = torch.empty(tokens, H, dtype=torch.bfloat16, device="cuda")
    steps = block.steps(attention, residual, adapters, out, n_chunks=4)
    for _ in range(3):
        for _, call in steps:
            call()
    marks = [torch.cuda.Event(enable_timing=True) for _ in range(len(steps) + 1)]
    marks[0].record()
    for (_, call), m in zip(steps, marks[1:]):
        call()
        m.record()
    torch.cuda.synchronize()
    assert cep.ffn_status(block.layer.plan) == 0 and block.projection.status() == 0
    for (name, _), a, b in zip(steps, marks, marks[1:]):
        print("%-26s %8.1f us" % (name, 1e3 * a.elapsed_time(b)))
    block.close()


if __name__ == "__main__":
    main(*(sys.argv[1:2] or ["mxfp4"]), *[int(v) for v in sys.argv[2:3]])
