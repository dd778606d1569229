"""What the pre-expert operators are timed on: the step from an attention block's output to the expert layer's input.

Two operators, each in its plain form (elementary torch operations in 32 bits) and, where ``own`` is set, as a user
of this package calls it:

* ``project``  y = x W^T + scale_a (x A_a^T) B_a^T: a projection shared by all requests with one low-rank adapter per
  request beside it (``LoRAProjection``); without adapters and with 32-bit output it is the router's logits.
* ``norm``     h = x + residual, y = h / rms(h) * weight, and y as the expert layer takes it: bf16, e4m3 with a 32-bit
  scale per 128 columns, or e4m3 with a power-of-two scale per 32 columns (``moe_norm``).
"""
import math

import torch

own = False

EPS = 1e-6
E4M3_MAX = 448.0


# ---------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one decoded token on its way into a block-scaled fp8 expert layer
        dict(name="norm_token_fp8", op="norm", tokens=1, hidden=7168, fmt="fp8", residual="bf16", copy=False, pad=0),
        # a decode batch into a microscaling expert layer; the bf16 copy feeds the router and the shared expert
        dict(name="norm_decode_mx", op="norm", tokens=61, hidden=7168, fmt="mx", residual="bf16", copy=True, pad=0),
        # a ragged mid-sized batch: x is a column slice of a wider buffer, and the last scale block is short
        dict(name="norm_ragged_fp8", op="norm", tokens=4097, hidden=2120, fmt="fp8", residual="bf16", copy=False, pad=64),
        # an odd width, which rules out wide loads
        dict(name="norm_odd_bf16", op="norm", tokens=1531, hidden=2047, fmt="bf16", residual="none", copy=True, pad=0),
        # prefill of the EP-shard layer in fp8, with the bf16 copy
        dict(name="norm_prefill_fp8", op="norm", tokens=16384, hidden=7168, fmt="fp8", residual="bf16", copy=True, pad=0),
        # prefill of the microscaling layer with a 32-bit residual stream
        dict(name="norm_prefill_mx", op="norm", tokens=16384, hidden=7168, fmt="mx", residual="fp32", copy=False, pad=0),
        # one decoded token, one adapter: reads the whole weight once
        dict(name="project_token", op="project", tokens=1, inputs=7168, outputs=7168, requests=1, adapters=8, rank=16, mix="decode", out="bf16"),
        # a decode batch in arrival order: 64 requests over 24 adapters of ranks 16 to 64, some requests without one
        dict(name="project_decode", op="project", tokens=64, inputs=7168, outputs=7168, requests=64, adapters=24, rank=64, mix="decode", out="bf16"),
        # chunked prefill beside decoding requests, on the mid-sized layer's width
        dict(name="project_mixed", op="project", tokens=519, inputs=2048, outputs=2048, requests=40, adapters=9, rank=32, mix="mixed", out="bf16"),
        # prefill of a few long requests, non-square
        dict(name="project_prefill_mid", op="project", tokens=4096, inputs=2048, outputs=7168, requests=6, adapters=4, rank=32, mix="prefill", out="bf16"),
        # a full prefill batch of the EP-shard layer
        dict(name="project_prefill", op="project", tokens=16384, inputs=7168, outputs=7168, requests=40, adapters=32, rank=64, mix="prefill", out="bf16"),
        # the router's logits of that batch
        dict(name="router_logits", op="project", tokens=16384, inputs=7168, outputs=256, requests=0, adapters=0, rank=0, mix="prefill", out="fp32"),
    ]


def _log_int(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return n + (n == 3072)


def draw(rng):
    if rng.random() < 0.5:
        hidden = _log_int(rng, 512, 7168)
        shape = rng.random()
        if shape < 0.6:
            hidden = max(512, hidden // 256 * 256)      # what the expert layer takes
        elif shape < 0.85:
            hidden = hidden // 8 * 8                    # a short last scale block
        if hidden == 3072:
            hidden += 256
        fmt = rng.choice(["bf16", "fp8", "mx"])
        return dict(op="norm", tokens=_log_int(rng, 1, 16384), hidden=hidden, fmt=fmt, residual=rng.choice(["none", "bf16", "fp32"]),
                    copy=fmt == "bf16" or rng.random() < 0.5, pad=rng.choice([0, 0, 64]))
    tokens = _log_int(rng, 1, 16384)
    size = lambda: _log_int(rng, 512, 7168) // 8 * 8
    inputs, outputs = size(), size()
    if rng.random() < 0.5:
        inputs, outputs = inputs // 128 * 128, outputs // 128 * 128
    inputs, outputs = inputs + 128 * (inputs == 3072), outputs + 128 * (outputs == 3072)
    if rng.random() < 0.15:
        return dict(op="project", tokens=tokens, inputs=inputs, outputs=rng.choice([8, 64, 100, 256, 384]), requests=0, adapters=0, rank=0,
                    mix="prefill", out="fp32")
    mix = rng.choice(["decode", "mixed", "prefill"])
    if mix == "decode":
        tokens = max(1, min(tokens, 256))
    requests = tokens if mix == "decode" else max(1, min(tokens, _log_int(rng, 1, 64)))
    return dict(op="project", tokens=tokens, inputs=inputs, outputs=outputs, requests=requests, adapters=_log_int(rng, 1, 32),
                rank=rng.choice([8, 16, 32, 64]), mix=mix, out="bf16")


def _rank(case, slot):
    """Adapters of one deployment differ in rank: full, half and quarter, at least 8."""
    return max(min(8, case["rank"]), case["rank"] >> (slot % 3))


def work(case):
    T = case["tokens"]
    if case["op"] == "norm":
        H = case["hidden"]
        res = {"none": 0, "bf16": 2, "fp32": 4}[case["residual"]]
        per_row = 2 * H + 2 * res * H + (2 * H if case["copy"] else 0)
        per_row += {"bf16": 0, "fp8": H + 4 * -(-H // 128), "mx": H + -(-H // 32)}[case["fmt"]]
        return {"bytes": T * per_row + 4 * H, "flops": 6 * T * H}
    K, N = case["inputs"], case["outputs"]
    used = min(case["adapters"], case["requests"])
    ranks = sum(_rank(case, s) for s in range(used))
    mean_rank = ranks / used if used else 0
    return {"bytes": 2 * T * K + 2 * N * K + 2 * ranks * (K + N) + T * N * (4 if case["out"] == "fp32" else 2) + 4 * T * (used > 0),
            "flops": 2 * T * K * N + 2 * T * mean_rank * (K + N) * (used / (used + 1) if used > 1 else 1)}


# ---------------------------------------------------------------------------------------------------- inputs
def _gen(seed, k):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 16 + k)
    return g


def _normal(shape, std, seed, k):
    return torch.randn(shape, generator=_gen(seed, k), device="cuda") * std


def _lengths(case, seed):
    """Tokens of each request, in batch order (on the host, as a scheduler has them)."""
    T, R = case["tokens"], case["requests"]
    g = torch.Generator()
    g.manual_seed(seed)
    if case["mix"] == "decode" or R <= 1:
        return [1] * R if case["mix"] == "decode" else [T]
    single = R // 2 if case["mix"] == "mixed" else 0
    long = R - single
    left = T - single
    cuts = torch.sort(torch.randperm(left - 1, generator=g)[:long - 1] + 1).values.tolist() if long > 1 else []
    ends = cuts + [left]
    return [1] * single + [b - a for a, b in zip([0] + cuts, ends)]


def _norm_inputs(case, seed):
    T, H, pad = case["tokens"], case["hidden"], case["pad"]
    wide = _normal((T, H + pad), 1.0, seed, 0)
    hot = torch.randperm(H, generator=_gen(seed, 1), device="cuda")[:max(1, H // 256)]
    wide[:, hot] *= 12.0                                             # outlier channels, as residual streams have
    x = wide.to(torch.bfloat16)[:, :H]
    weight = (1.0 + _normal((H,), 0.1, seed, 2)).to(torch.bfloat16)
    residual = None
    if case["residual"] != "none":
        residual = _normal((T, H), 2.0, seed, 3).to(torch.bfloat16 if case["residual"] == "bf16" else torch.float32)
    return x, weight, residual


def _project_inputs(case, seed):
    T, K, N, S = case["tokens"], case["inputs"], case["outputs"], case["adapters"]
    x = _normal((T, K), 1.0, seed, 0).to(torch.bfloat16)
    weight = _normal((N, K), K ** -0.5, seed, 1).to(torch.bfloat16)
    if not S:
        return dict(x=x, weight=weight, ids=None, down=None, up=None, scale=None, ranks=[])
    lengths = _lengths(case, seed)
    slots = [r % (S + 1) for r in range(case["requests"])]
    slots = [-1 if s == S else s for s in slots]                     # one request in S+1 has no adapter
    ids = torch.repeat_interleave(torch.tensor(slots, dtype=torch.int32), torch.tensor(lengths))
    if case["mix"] == "decode":
        g = torch.Generator()
        g.manual_seed(seed + 1)
        ids = ids[torch.randperm(ids.numel(), generator=g)]          # arrival order, not adapter order
    ranks = [_rank(case, s) for s in range(S)]
    down = _normal((S, case["rank"], K), K ** -0.5, seed, 4)
    up = _normal((S, N, case["rank"]), case["rank"] ** -0.5, seed, 5)
    keep = torch.arange(case["rank"], device="cuda")[None, :] < torch.tensor(ranks, device="cuda")[:, None]
    down = (down * keep[:, :, None]).to(torch.bfloat16)
    up = (up * keep[:, None, :]).to(torch.bfloat16)
    scale = 0.5 + torch.rand(S, generator=_gen(seed, 6), device="cuda")
    return dict(x=x, weight=weight, ids=ids.cuda(), down=down, up=up, scale=scale, ranks=ranks)


def prepare(case, seed):
    T = case["tokens"]
    if case["op"] == "norm":
        x, weight, residual = _norm_inputs(case, seed)
        H = case["hidden"]
        state = dict(case=case, x=x, weight=weight, residual=residual)
        if own:
            empty = lambda shape, dtype: torch.empty(shape, dtype=dtype, device="cuda")
            state["residual_out"] = None if residual is None else torch.empty_like(residual)
            state["y"] = empty((T, H), torch.bfloat16) if case["copy"] else None
            state["codes"] = empty((T, H), torch.float8_e4m3fn) if case["fmt"] != "bf16" else None
            state["scales"] = {"bf16": None, "fp8": ((T, -(-H // 128)), torch.float32), "mx": ((T, -(-H // 32)), torch.uint8)}[case["fmt"]]
            if state["scales"]:
                state["scales"] = empty(*state["scales"])
        return state
    d = _project_inputs(case, seed)
    state = dict(case=case, **d)
    if own:
        import paper_2609_33252_b200 as cep
        elem = cep.CEP_ELEM_FP32 if case["out"] == "fp32" else cep.CEP_ELEM_BF16
        layer = cep.LoRAProjection(d["weight"], max_tokens=T, max_adapters=case["adapters"], max_rank=case["rank"], out_elem=elem)
        for slot, rank in enumerate(d["ranks"]):
            layer.load_adapter(slot, d["down"][slot, :rank], d["up"][slot, :, :rank], float(d["scale"][slot]))
        state["layer"] = layer
        state["out"] = torch.empty((T, case["outputs"]), dtype=torch.float32 if case["out"] == "fp32" else torch.bfloat16, device="cuda")
    return state


# ---------------------------------------------------------------------------------------------------- one pass
def _plain_norm(state):
    case, x = state["case"], state["x"].float()
    T, H = x.shape
    out = {}
    h = x
    if state["residual"] is not None:
        h = x + state["residual"].float()
        out["residual"] = h.to(state["residual"].dtype)
    y = h * torch.rsqrt((h * h).mean(dim=1, keepdim=True) + EPS) * state["weight"].float()
    if case["copy"]:
        out["y"] = y.to(torch.bfloat16)
    if case["fmt"] != "bf16":
        block = 128 if case["fmt"] == "fp8" else 32
        n = -(-H // block)
        b = torch.nn.functional.pad(y, (0, n * block - H)).view(T, n, block)
        amax = b.abs().amax(dim=2)
        if case["fmt"] == "fp8":
            scale = torch.where(amax == 0, torch.ones_like(amax), amax / E4M3_MAX)
            out["scales"] = scale
        else:
            # the smallest power of two s with amax <= 448 s (448 = 1.75 * 2^8)
            m, e = torch.frexp(amax)
            p = torch.where(amax == 0, torch.zeros_like(e), e - 9 + (m > 0.875).to(e.dtype)).clamp(-127, 127)
            scale = torch.ldexp(torch.ones_like(amax), p)
            out["scales"] = (p + 127).to(torch.uint8).view(torch.float8_e8m0fnu)
        q = (b / scale[:, :, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
        out["codes"] = q.view(T, n * block)[:, :H].contiguous()
    return out


def _plain_project(state):
    x = state["x"].float()
    y = x @ state["weight"].float().t()
    if state["ids"] is not None:
        S, R, K = state["down"].shape
        mine = state["ids"][:, None] == torch.arange(S, dtype=torch.int32, device=x.device)[None, :]      # [T,S], no row for -1
        low = (x @ state["down"].float().view(S * R, K).t()).view(-1, S, R) * (mine * state["scale"])[:, :, None]
        y = y + low.view(-1, S * R) @ state["up"].float().permute(0, 2, 1).reshape(S * R, -1)
    return {"y": y if state["case"]["out"] == "fp32" else y.to(torch.bfloat16)}


def run(state):
    if not own:
        return _plain_norm(state) if state["case"]["op"] == "norm" else _plain_project(state)
    import paper_2609_33252_b200 as cep
    case = state["case"]
    if case["op"] == "project":
        return {"y": state["layer"].run(state["x"], state["ids"], state["out"])}
    dtype = {"bf16": cep.CEP_BF16, "fp8": cep.CEP_FP8_E4M3_BLOCK128, "mx": cep.CEP_MXFP4_E4M3}[case["fmt"]]
    cep.moe_norm(state["x"], state["weight"], EPS, residual=state["residual"], residual_out=state["residual_out"], y=state["y"],
                 codes=state["codes"], scales=state["scales"], dtype=dtype)
    out = {}
    if state["residual"] is not None:
        out["residual"] = state["residual_out"]
    if case["copy"]:
        out["y"] = state["y"]
    if case["fmt"] != "bf16":
        out["scales"] = state["scales"] if case["fmt"] == "fp8" else state["scales"].view(torch.float8_e8m0fnu)
        out["codes"] = state["codes"]
    return out


# ---------------------------------------------------------------------------------------------------- the definition, in 64 bits
def exact(case, seed):
    if case["op"] == "project":
        d = _project_inputs(case, seed)
        y = torch.matmul(d["x"].double(), d["weight"].double().t())
        if d["ids"] is not None:
            ids = d["ids"].long()
            for slot, rank in enumerate(d["ranks"]):
                rows = torch.nonzero(ids == slot).flatten()
                if rows.numel():
                    low = torch.matmul(d["x"][rows].double(), d["down"][slot, :rank].double().t())
                    y[rows] += float(d["scale"][slot]) * torch.matmul(low, d["up"][slot, :, :rank].double().t())
        return {"y": y}
    x, weight, residual = _norm_inputs(case, seed)
    T, H = x.shape
    block = {"bf16": H, "fp8": 128, "mx": 32}[case["fmt"]]
    n = -(-H // block)
    parts = {}
    for r0 in range(0, T, 2048):                                     # slabs, to bound the memory in use
        rows = slice(r0, min(T, r0 + 2048))
        h = x[rows].double()
        if residual is not None:
            h = h + residual[rows].double()
            parts.setdefault("residual", []).append(h)
        y = h / torch.sqrt(torch.sum(h ** 2, dim=1, keepdim=True) / H + EPS) * weight.double()
        if case["copy"]:
            parts.setdefault("y", []).append(y)
        if case["fmt"] != "bf16":
            padded = torch.zeros(h.shape[0], n * block, dtype=torch.float64, device=h.device)
            padded[:, :H] = y
            b = padded.view(-1, n, block)
            amax = b.abs().max(dim=2).values
            if case["fmt"] == "fp8":
                scale = amax / E4M3_MAX
            else:
                scale = torch.exp2(torch.ceil(torch.log2(amax / E4M3_MAX)).clamp(-127, 127))
            scale = torch.where(amax == 0, torch.ones_like(scale), scale)
            q = (b / scale[:, :, None]).float().to(torch.float8_e4m3fn).double()
            parts.setdefault("scales", []).append(scale)
            parts.setdefault("codes", []).append(q.view(-1, n * block)[:, :H])
    return {k: torch.cat(v) for k, v in parts.items()}
