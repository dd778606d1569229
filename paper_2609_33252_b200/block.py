"""From an attention block's output to the expert layer's result, with the library's operators in the order a server
runs them: the output projection with per-request low-rank adapters, the residual's addition with the norm and the
expert layer's activation format, the router's logits and selection, the routed experts.

``AttentionBlock`` is what comes before: projection to q, k and v, rotation and the write into a paged cache, attention of
requests that share a prefix.

``python -m paper_2609_33252_b200.block [dtype] [tokens] [prefix]`` runs it on random weights and prints the device time of every
step (dtype: bf16, fp8 or mxfp4); with a prefix, the attention block too, requests of 64 tokens behind that many shared keys.
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
        try:
            for _, call in self.steps(attention, residual, adapter_ids, out, n_chunks):
                call()
        finally:                                             # (a step that is refused leaves those before it at work)
            self.done.record(stream)
        return out

    def close(self):
        self.projection.close()
        self.router.close()
        self.layer.close()


class AttentionBlock:
    """From a layer's normed input to its attention output (what ``MoEBlock`` takes), over the layer's paged cache.

    w_qkv bf16 [(Hq + 2 Hkv) D, H]: rows of all query heads, then the key heads, then the value heads; k_cache, v_cache
    [pages, page_size, Hkv, D] bf16 or float8_e4m3fn (with k_scale, v_scale fp32 [Hkv]); inv_freq fp32 [R/2]; scale of the scores, 1/sqrt(D)
    by default.  All are the caller's tensors.  ``run`` may be called on different streams: each call waits for the one before, as the buffers between the
    steps are shared (who runs ``steps`` orders them, and who captures ``run`` into a graph its replays).
    """

    def __init__(self, w_qkv, k_cache, v_cache, n_heads, inv_freq, max_tokens, max_seqs, max_prefixes=1, k_scale=None, v_scale=None, interleaved=False,
                 max_adapters=0, max_rank=0, scale=None):
        Hk, D = k_cache.shape[2:]
        self.heads = (n_heads, Hk, D)
        if w_qkv.shape[0] != (n_heads + 2 * Hk) * D:
            raise cep.CepError(-1, "w_qkv must have (%d + 2 * %d) * %d rows" % (n_heads, Hk, D))
        self.inv_freq, self.interleaved = inv_freq, interleaved
        self.bad_slots = torch.zeros(1, dtype=torch.int32, device=w_qkv.device)      # set by the write into the cache
        self.projection = cep.LoRAProjection(w_qkv, max_tokens, max_adapters, max_rank)
        self.attention = cep.PrefixAttention(k_cache, v_cache, n_heads, max_tokens, max_seqs, max_prefixes, k_scale, v_scale, scale)
        self.qkv = torch.empty(max_tokens, n_heads + 2 * Hk, D, dtype=torch.bfloat16, device=w_qkv.device)
        self.out = torch.empty(max_tokens, n_heads, D, dtype=torch.bfloat16, device=w_qkv.device)
        self.done = torch.cuda.Event()                       # the end of the last call
        self.done.record(torch.cuda.current_stream(w_qkv.device))    # (before the first: of the clearing above)

    def steps(self, x, positions, slots, batch, adapter_ids=None, causal=True):
        """The block as (name, call) pairs.  x bf16 [T,H]; positions int32 [T]; slots int64 [T]; batch: the lengths and page
        tables of ``PrefixAttention.run`` as a dict, kv_len with the new tokens.  The result is ``out`` [T,Hq,D]."""
        T, (Hq, Hk, D) = x.shape[0], self.heads
        if T > self.out.shape[0]:
            raise cep.CepError(-4, "%d tokens, the block was made for %d" % (T, self.out.shape[0]))
        qkv, out, att = self.qkv[:T], self.out[:T], self.attention
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]
        return [
            ("projection to q, k, v", lambda: self.projection.run(x, adapter_ids, qkv.view(T, -1))),
            ("rotation + cache", lambda: cep.attn_append(k, v, positions, slots, self.inv_freq, att.k_cache, att.v_cache, q=q, q_out=q,
                                                         interleaved=self.interleaved, k_scale=att.k_scale, v_scale=att.v_scale,
                                                         status=self.bad_slots)),
            ("attention", lambda: att.run(q, causal=causal, out=out, **batch)),
        ]

    def run(self, x, positions, slots, batch, adapter_ids=None, causal=True):
        """Returns the attention output [T, Hq D], a view of the block's buffer (valid until the next call)."""
        T, (Hq, _, D) = x.shape[0], self.heads
        stream = torch.cuda.current_stream(x.device)
        capturing = torch.cuda.is_current_stream_capturing()            # (a graph cannot wait for what is not in it)
        if not capturing:
            stream.wait_event(self.done)
        try:
            if T:                                            # (empty tensors have no address)
                for _, call in self.steps(x, positions, slots, batch, adapter_ids, causal):
                    call()
        finally:                                             # (a step that is refused leaves those before it at work)
            if not capturing:
                self.done.record(stream)
        return self.out[:T].view(T, Hq * D)

    def status(self) -> int:
        """Waits for the block's work and returns what its steps reported since the last call: 0, or the projection's status, the
        attention's, or -6 (CEP_ERR_BAD_ROUTING) where a slot other than -1 lay outside the cache, whose token's key and value were not
        written; the first of them, and all are cleared.  (Replays of a graph are the caller's to wait for.)"""
        codes = [self.projection.status(), self.attention.status()]
        self.done.synchronize()
        if int(self.bad_slots):
            self.bad_slots.zero_()
            torch.cuda.current_stream(self.bad_slots.device).synchronize()           # (the next call may come on another stream)
            codes.append(-6)
        return next((c for c in codes if c), 0)

    def close(self):
        self.projection.close()
        self.attention.close()


def _requests(tokens, prefix, page, per_request=64):
    """Lengths, tables, positions and slots of requests of up to 64 new tokens each behind one prefix; (batch, positions, slots, pages)."""
    n = [per_request] * (tokens // per_request) + ([tokens % per_request] if tokens % per_request else [])
    ahead, each = -(-prefix // page), -(-per_request // page)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    first = torch.tensor([0] + n).cumsum(0).tolist()
    table = [[ahead + b * each + i for i in range(each)] for b in range(len(n))]
    batch = dict(q_start=i32(first), kv_len=i32(n), page_table=i32(table), prefix_len=i32([prefix]), prefix_pages=i32([list(range(ahead))]))
    positions = i32([prefix + i for m in n for i in range(m)])
    slots = torch.tensor([table[b][i // page] * page + i % page for b, m in enumerate(n) for i in range(m)], device="cuda")
    return batch, positions, slots, ahead + each * len(n)


def main(dtype="mxfp4", tokens=4096, prefix=0):
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
    before = None
    if prefix:
        heads, kv_heads, dim, page = H // 128, max(1, H // 512), 128, 64
        batch, positions, slots, pages = _requests(tokens, prefix, page)
        cache = [rand(pages, page, kv_heads, dim) for _ in range(2)]
        inv_freq = (10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim)).float().cuda()
        before = AttentionBlock(rand((heads + 2 * kv_heads) * dim, H, std=H ** -0.5), *cache, heads, inv_freq, tokens, batch["kv_len"].numel())
        attention = before.out[:tokens].view(tokens, -1)
    adapters = (torch.arange(tokens, device="cuda") * 5 // tokens - 1).to(torch.int32)       # five requests, the first without
    out = torch.empty(tokens, H, dtype=torch.bfloat16, device="cuda")
    steps = block.steps(attention, residual, adapters, out, n_chunks=4)
    if before:
        steps = before.steps(rand(tokens, H), positions, slots, batch) + steps
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
    assert not before or before.status() == 0
    for (name, _), a, b in zip(steps, marks, marks[1:]):
        print("%-26s %8.1f us" % (name, 1e3 * a.elapsed_time(b)))
    block.close()
    if before:
        before.close()


if __name__ == "__main__":
    main(*(sys.argv[1:2] or ["mxfp4"]), *[int(v) for v in sys.argv[2:4]])
