"""What the attention operators in front of the expert layer are timed on: a paged cache and the attention that reads it.

Two operators, each in its plain form (elementary torch operations in 32 bits, angles in 64) and, where ``own`` is set, as
a user of this package calls it:

* ``append``  rotates the heads of q and k by their tokens' positions and writes k and v into the pages of a cache, in bf16
  or e4m3 with a scale per head (``attn_append``).
* ``attend``  softmax(scale q k^T) v of a batch of requests that share a long prefix: every token sees its group's prefix
  and its own request's keys up to itself (``PrefixAttention``).
"""
import math
import random

import torch

own = False

THETA = 1000000.0
E4M3_MAX = 448.0


# ---------------------------------------------------------------------------------------------------- cases
def _append(name, **kw):
    case = dict(name=name, op="append", tokens=1, pad=0, heads=16, kv_heads=4, dim=128, rotary=128, interleaved=False, cache="bf16", page=64, fused=True)
    case.update(kw)
    return case


def _attend(name, **kw):
    case = dict(name=name, op="attend", mode="decode", seqs=1, tokens=0, heads=16, kv_heads=4, dim=128, page=64, cache="bf16", prefix=0, prefixes=1, own=64,
                empty=False, lse=False)
    case.update(kw)
    return case


def listed():
    return [
        # one decoded token of a 2048-wide model
        _append("append_token"),
        # a decode batch of a 7168-wide model, its last rows padding of the batch's captured size, into an 8-bit cache
        _append("append_decode_e4m3", tokens=64, pad=3, heads=56, kv_heads=8, cache="e4m3", page=32),
        # chunked prefill with a partial, interleaved rotation of odd-sized heads, q, k and v in buffers of their own
        _append("append_ragged", tokens=1531, heads=12, kv_heads=12, dim=80, rotary=32, interleaved=True, page=16, fused=False),
        # a full prefill batch of the 7168-wide model
        _append("append_prefill", tokens=16384, heads=56, kv_heads=8),
        # one request's decode step behind a short tool description
        _attend("attend_token", prefix=777, own=33),
        # a small decode batch behind one system prompt; the sums' logarithms go to a caller that merges further keys
        _attend("attend_decode_small", seqs=8, prefix=2048, own=300, lse=True),
        # a decode batch of agents behind a long tool prompt: the shared part is read once for all
        _attend("attend_decode", seqs=64, heads=56, kv_heads=8, prefix=8192, own=2000),
        # the same in an 8-bit cache with two different prompts
        _attend("attend_decode_e4m3", seqs=128, heads=64, kv_heads=8, page=32, cache="e4m3", prefix=5000, prefixes=2, own=1500),
        # the largest decode batch: mostly the requests' own keys
        _attend("attend_decode_large", seqs=256, heads=56, kv_heads=8, prefix=32768, own=4096),
        # a few drafted tokens per request, verified at once; heads of 64, short pages, three prompts, rows that see nothing
        _attend("attend_verify_odd", mode="verify", seqs=33, heads=16, kv_heads=16, dim=64, page=16, prefix=1001, prefixes=3, own=517, empty=True),
        # prompts of new requests beside decoding ones, mid-sized model
        _attend("attend_mixed", mode="mixed", seqs=40, tokens=4096, prefix=2048, own=700),
        # a full prefill batch behind the long tool prompt
        _attend("attend_prefill", mode="prefill", seqs=24, tokens=16384, heads=56, kv_heads=8, page=128, prefix=8192, own=0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    dim = rng.choice([64, 128, 128, 128, 80, 96, 112, 32])
    kv_heads, group = rng.choice([(1, 8), (2, 8), (4, 4), (8, 7), (8, 8), (8, 1), (4, 1), (12, 1), (2, 16), (8, 4), (3, 5)])
    cache = rng.choice(["bf16", "bf16", "e4m3"])
    page = rng.choice([16, 32, 64, 128, 256])
    heads = kv_heads * group
    if rng.random() < 0.3:
        tokens = _log_int(rng, 1, 16384)
        rotary = dim if rng.random() < 0.7 else dim // 2
        return dict(op="append", tokens=tokens, pad=rng.choice([0, 0, tokens // 5]), heads=heads, kv_heads=kv_heads, dim=dim, rotary=rotary,
                    interleaved=rng.random() < 0.4, cache=cache, page=page, fused=rng.random() < 0.6)
    mode = rng.choice(["decode", "decode", "verify", "mixed", "prefill"])
    prefix = 0 if rng.random() < 0.1 else _log_int(rng, 16, 32768)
    prefixes = rng.choice([1, 1, 1, 2, 4])
    empty = rng.random() < 0.2
    case = dict(op="attend", mode=mode, tokens=0, heads=heads, kv_heads=kv_heads, dim=dim, page=page, cache=cache, prefix=prefix, prefixes=prefixes, empty=empty,
                lse=not empty and rng.random() < 0.3)
    if mode in ("decode", "verify"):
        seqs = _log_int(rng, 1, 256 if mode == "decode" else 64)
        return dict(case, seqs=seqs, own=_log_int(rng, 8, 4096))
    tokens = _log_int(rng, 32, 16384)
    most = max(64, 7340032 // heads * 8192 // tokens // 10)           # keys a token may see at the cost of the largest case
    case["prefix"] = min(prefix, most)
    return dict(case, seqs=min(tokens, _log_int(rng, 1, 48)), tokens=tokens, own=0 if mode == "prefill" else _log_int(rng, 8, 1024))


def _lengths(case):
    """Per request: new tokens, own keys (the new ones among them) and the group whose prefix it sees (-1: none); and the
    groups' prefix lengths.  What a scheduler has on the host; requests of a group lie together."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    B, G = case["seqs"], min(case["prefixes"], case["seqs"])
    if case["mode"] == "decode":
        q_len = [1] * B
    elif case["mode"] == "verify":
        q_len = [rng.randint(1, 8) for _ in range(B)]
    else:
        decoding = B // 2 if case["mode"] == "mixed" else 0
        decoding = min(decoding, max(0, case["tokens"] - 1))
        left, n = case["tokens"] - decoding, B - decoding
        cuts = sorted(rng.sample(range(1, left), n - 1)) if 1 < n <= left else []
        q_len = [1] * decoding + [b - a for a, b in zip([0] + cuts, cuts + [left])]
        B = len(q_len)
        rng.shuffle(q_len)
    kv_len = [n + (rng.randint(0, case["own"]) if case["own"] else 0) for n in q_len]
    group = [b * G // B for b in range(B)]
    prefix = [max(0, case["prefix"] - rng.randint(0, case["prefix"] // 3) * (g > 0)) for g in range(G)]
    if case["empty"]:
        q_len[0], group[-1], kv_len[-1] = 0, -1, 0                    # nothing asked; nothing to see
        if B > 2:
            group[-2], kv_len[-2] = -1, (q_len[-2] + 1) // 2          # fewer keys than tokens: the first tokens see nothing
    return q_len, kv_len, group, prefix


def work(case):
    T, Hq, Hk, D = case["tokens"], case["heads"], case["kv_heads"], case["dim"]
    elem = 1 if case["cache"] == "e4m3" else 2
    if case["op"] == "append":
        return {"bytes": T * (2 * Hq * D * 2 + 2 * Hk * D * 2 + 12) + (T - case["pad"]) * 2 * Hk * D * elem,
                "flops": 3 * T * (Hq + Hk) * case["rotary"]}
    q_len, kv_len, group, prefix = _lengths(case)
    pairs = sum(n * (prefix[g] if g >= 0 else 0) + sum(max(0, l - n + i + 1) for i in range(n)) for n, l, g in zip(q_len, kv_len, group))
    keys = sum(kv_len) + sum(prefix[g] for g in set(group) if g >= 0)
    T = sum(q_len)
    return {"bytes": T * Hq * D * 4 + 2 * keys * Hk * D * elem + T * Hq * 4 * case["lse"] + 4 * (keys // case["page"]), "flops": 4 * D * Hq * pairs}


# ---------------------------------------------------------------------------------------------------- inputs
def _gen(seed, k):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 16 + k)
    return g


def _normal(shape, std, seed, k):
    return (torch.randn(shape, generator=_gen(seed, k), device="cuda", dtype=torch.bfloat16) * std)


def _caches(case, pages, seed):
    """k and v [pages, page, kv_heads, dim]; in e4m3 with a scale per head."""
    shape = (pages, case["page"], case["kv_heads"], case["dim"])
    k, v = _normal(shape, 1.0, seed, 0), _normal(shape, 1.0, seed, 1)
    if case["cache"] == "bf16":
        return k, v, None, None
    scale = lambda i: (0.5 + torch.rand(case["kv_heads"], generator=_gen(seed, i), device="cuda")) * 0.03
    k_scale, v_scale = scale(2), scale(3)
    code = lambda t, s: (t.float() / s[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    return code(k, k_scale), code(v, v_scale), k_scale, v_scale


def _append_inputs(case, seed):
    T, Hq, Hk, D, page = case["tokens"], case["heads"], case["kv_heads"], case["dim"], case["page"]
    if case["fused"]:                                                  # the columns of one projection's output
        qkv = _normal((T, Hq + 2 * Hk, D), 1.0, seed, 4)
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]
    else:
        q, k, v = (_normal((T, h, D), 1.0, seed, 4 + i) for i, h in enumerate((Hq, Hk, Hk)))
    pages = -(-T // page) + max(4, 2048 // page)
    k_cache, v_cache, k_scale, v_scale = _caches(case, pages, seed)
    rng = random.Random(seed)
    real = T - case["pad"]
    slots, positions, order = [], [], rng.sample(range(pages), pages)
    if T <= 256:                                                       # decoding: every token in a page of some request
        slots = rng.sample(range(pages * page), real)
        positions = [rng.randrange(0, 131072) for _ in range(real)]
    else:                                                              # prompts: runs of positions over whole pages
        at = rng.randrange(0, 100000)
        for i in range(real):
            if rng.random() < 0.002:
                at = rng.randrange(0, 100000)
            positions.append(at + i)
            slots.append(order[i // page] * page + i % page)
    slots += [-1] * case["pad"]
    positions += [0] * case["pad"]
    inv_freq = (THETA ** (-torch.arange(0, case["rotary"], 2, dtype=torch.float64) / case["rotary"])).float().cuda()
    return dict(q=q, k=k, v=v, k_cache=k_cache, v_cache=v_cache, k_scale=k_scale, v_scale=v_scale, real=real, inv_freq=inv_freq,
                slots=torch.tensor(slots, dtype=torch.int64).cuda(), positions=torch.tensor(positions, dtype=torch.int32).cuda())


def _attend_inputs(case, seed):
    q_len, kv_len, group, prefix = _lengths(case)
    page, B, G = case["page"], len(q_len), len(prefix)
    count = lambda n: -(-n // page)
    total = sum(map(count, kv_len)) + sum(map(count, prefix)) + 2
    order = list(range(total))
    random.Random(seed).shuffle(order)
    take = lambda n: [order.pop() for _ in range(count(n))]
    own_pages, prefix_pages = [take(n) for n in kv_len], [take(n) for n in prefix]
    k_cache, v_cache, k_scale, v_scale = _caches(case, total, seed)
    q = _normal((sum(q_len), case["heads"], case["dim"]), 2.0, seed, 4)
    return dict(q=q, k_cache=k_cache, v_cache=v_cache, k_scale=k_scale, v_scale=v_scale, q_len=q_len, kv_len=kv_len, group=group, prefix=prefix,
                own_pages=own_pages, prefix_pages=prefix_pages)


def _table(rows):
    """Page lists as one rectangular int32 tensor."""
    width = max(1, max((len(r) for r in rows), default=1))
    return torch.tensor([r + [-1] * (width - len(r)) for r in rows], dtype=torch.int32).view(-1, width).cuda()


def prepare(case, seed):
    if case["op"] == "append":
        state = dict(case=case, **_append_inputs(case, seed))
        state["q_out"] = torch.empty((case["tokens"], case["heads"], case["dim"]), dtype=torch.bfloat16, device="cuda")
        return state
    d = _attend_inputs(case, seed)
    state = dict(case=case, **d)
    ints = lambda values: torch.tensor(values, dtype=torch.int32).cuda()
    state["own_pages"] = [torch.tensor(p, dtype=torch.int64).cuda() for p in d["own_pages"]]
    state["prefix_pages"] = [torch.tensor(p, dtype=torch.int64).cuda() for p in d["prefix_pages"]]
    if own:
        import paper_2609_33252_b200 as cep
        B, G, T = len(d["q_len"]), len(d["prefix"]), d["q"].shape[0]
        starts = [0]
        for n in d["q_len"]:
            starts.append(starts[-1] + n)
        inside = [[b for b in range(B) if d["group"][b] == g] for g in range(G)]
        first = [i[0] if i else B for i in inside] + [1 + max((b for b in range(B) if d["group"][b] >= 0), default=-1)]
        for g in reversed(range(G)):
            first[g] = min(first[g], first[g + 1])                     # a group without requests
        state["meta"] = dict(q_start=ints(starts), kv_len=ints(d["kv_len"]), page_table=_table(d["own_pages"]), prefix_start=ints(first),
                             prefix_len=ints(d["prefix"]), prefix_pages=_table(d["prefix_pages"]))
        state["layer"] = cep.PrefixAttention(d["k_cache"], d["v_cache"], case["heads"], max_tokens=max(T, 1), max_seqs=B, max_prefixes=G, k_scale=d["k_scale"],
                                             v_scale=d["v_scale"])
        state["out"] = torch.empty_like(d["q"])
        state["lse"] = torch.empty((T, case["heads"]), dtype=torch.float32, device="cuda") if case["lse"] else None
    return state


# ---------------------------------------------------------------------------------------------------- one pass
def _plain_rotate(x, cos, sin, case):
    x, R = x.float(), case["rotary"]
    if case["interleaved"]:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        turned = torch.stack((a * cos - b * sin, a * sin + b * cos), dim=-1).flatten(-2)
    else:
        a, b = x[..., :R // 2], x[..., R // 2:R]
        turned = torch.cat((a * cos - b * sin, a * sin + b * cos), dim=-1)
    return torch.cat((turned, x[..., R:]), dim=-1)


def _plain_append(state):
    case, n = state["case"], state["real"]
    angle = state["positions"].double()[:, None] * state["inv_freq"].double()
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    state["q_out"].copy_(_plain_rotate(state["q"], cos, sin, case))
    k, v = _plain_rotate(state["k"], cos, sin, case)[:n], state["v"][:n].float()
    for new, name in ((k, "k"), (v, "v")):
        cache = state[name + "_cache"]
        if case["cache"] == "e4m3":
            new = (new / state[name + "_scale"][:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
            cache = cache.view(torch.uint8)
        cache.view(-1, *cache.shape[2:])[state["slots"][:n]] = new.to(cache.dtype)
    return {"q": state["q_out"], "k": state["k_cache"], "v": state["v_cache"]}


def _plain_gather(cache, scale, pages, length):
    if scale is None:
        return cache[pages].flatten(0, 1)[:length].float()
    codes = cache.view(torch.uint8)[pages].view(torch.float8_e4m3fn)
    return codes.flatten(0, 1)[:length].float() * scale[:, None]


def _plain_attend(state):
    case = state["case"]
    Hq, Hk, D = case["heads"], case["kv_heads"], case["dim"]
    out = torch.empty_like(state["q"])
    lse = torch.empty(out.shape[:2], dtype=torch.float32, device=out.device)
    shared = [[_plain_gather(state[c + "_cache"], state[c + "_scale"], p, n) for c in "kv"] for p, n in zip(state["prefix_pages"], state["prefix"])]
    t = 0
    for n, length, g, pages in zip(state["q_len"], state["kv_len"], state["group"], state["own_pages"]):
        k, v = (_plain_gather(state[c + "_cache"], state[c + "_scale"], pages, length) for c in "kv")
        ahead = 0
        if g >= 0:
            ahead = state["prefix"][g]
            k, v = torch.cat((shared[g][0], k)), torch.cat((shared[g][1], v))
        k, v = k.permute(1, 2, 0), v.permute(1, 0, 2)                  # [Hk,D,L], [Hk,L,D]
        slab = max(1, (1 << 29) // max(1, Hq * k.shape[2]))            # tokens at once, to bound the memory in use
        for i0 in range(0, n, slab):
            m = min(slab, n - i0)
            q = state["q"][t + i0:t + i0 + m].float().view(m, Hk, Hq // Hk, D).permute(1, 0, 2, 3).reshape(Hk, -1, D)
            s = (q @ k).view(Hk, m, Hq // Hk, -1) * D ** -0.5
            last = ahead + length - n + i0 + torch.arange(m, device=out.device)
            hidden = torch.arange(k.shape[2], device=out.device)[None, :] > last[:, None]
            s = s.masked_fill(hidden[:, None, :], -math.inf)
            top = s.amax(dim=3, keepdim=True) if k.shape[2] else s.new_full((Hk, m, Hq // Hk, 1), -math.inf)
            p = torch.exp(s - top.clamp(min=-1e30))
            total = p.sum(dim=3, keepdim=True)
            o = (p.view(Hk, m * (Hq // Hk), -1 if k.shape[2] else 0) @ v).view(Hk, m, Hq // Hk, D) / total.clamp(min=1e-30)
            out[t + i0:t + i0 + m] = o.permute(1, 0, 2, 3).reshape(m, Hq, D).to(out.dtype)
            lse[t + i0:t + i0 + m] = (top + torch.log(total)).permute(1, 0, 2, 3).reshape(m, Hq)
        t += n
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}


def run(state):
    case = state["case"]
    if not own:
        return _plain_append(state) if case["op"] == "append" else _plain_attend(state)
    import paper_2609_33252_b200 as cep
    if case["op"] == "append":
        cep.attn_append(state["k"], state["v"], state["positions"], state["slots"], state["inv_freq"], state["k_cache"], state["v_cache"], q=state["q"],
                        q_out=state["q_out"], interleaved=case["interleaved"], k_scale=state["k_scale"], v_scale=state["v_scale"])
        return {"q": state["q_out"], "k": state["k_cache"], "v": state["v_cache"]}
    state["layer"].run(state["q"], out=state["out"], lse=state["lse"], **state["meta"])
    return {"out": state["out"], "lse": state["lse"]} if case["lse"] else {"out": state["out"]}


# ---------------------------------------------------------------------------------------------------- the definition, in 64 bits
def _exact_append(case, seed):
    d = _append_inputs(case, seed)
    R, n = case["rotary"], d["real"]
    first = torch.arange(R // 2, device="cuda") * (2 if case["interleaved"] else 1)
    second = first + (1 if case["interleaved"] else R // 2)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), d["positions"].double()[:, None, None] * d["inv_freq"].double())

    def rotated(x):
        y = x.double()
        z = torch.complex(y[..., first], y[..., second]) * turn
        y[..., first], y[..., second] = z.real, z.imag
        return y
    out = {"q": rotated(d["q"])}
    for name, new in (("k", rotated(d["k"])), ("v", d["v"].double())):
        cache, scale = d[name + "_cache"].double(), d[name + "_scale"]
        if scale is not None:
            new = (new / scale.double()[:, None]).clamp(-E4M3_MAX, E4M3_MAX).float().to(torch.float8_e4m3fn).double()
        cache.view(-1, *cache.shape[2:])[d["slots"][:n]] = new[:n]
        out[name] = cache
    return out


def _exact_attend(case, seed):
    d = _attend_inputs(case, seed)
    Hq, Hk, D, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    if work(case)["flops"] > 2.5e13:
        return None
    out = torch.zeros(d["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(d["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    flat = {c: d[c + "_cache"].view(-1, Hk, D) for c in "kv"}

    def keys(c, where):
        rows = flat[c].view(torch.uint8)[where].view(torch.float8_e4m3fn) if d["k_scale"] is not None else flat[c][where]
        rows = rows.double()
        return rows if d["k_scale"] is None else rows * d[c + "_scale"].double()[:, None]
    places = lambda pages, n: torch.tensor([pages[j // page] * page + j % page for j in range(n)], dtype=torch.int64).cuda()
    shared = [places(p, n) for p, n in zip(d["prefix_pages"], d["prefix"])]
    t = 0
    for n, length, g, pages in zip(d["q_len"], d["kv_len"], d["group"], d["own_pages"]):
        ahead = d["prefix"][g] if g >= 0 else 0
        where = torch.cat(([shared[g]] if g >= 0 else []) + [places(pages, length)])
        K, V = keys("k", where), keys("v", where)
        for i in range(0, n, 1024):
            rows = range(i, min(n, i + 1024))
            seen = torch.tensor([ahead + length - n + r + 1 for r in rows], device="cuda").clamp(min=ahead)
            if int(seen.max()) <= 0:
                continue
            mask = torch.arange(K.shape[0], device="cuda") < seen[:, None]
            for h in range(Hq):
                s = torch.matmul(d["q"][t + i:t + i + len(rows), h].double(), K[:, h * Hk // Hq].t()) / math.sqrt(D)
                s = torch.where(mask, s, torch.full_like(s, -math.inf))
                z = torch.logsumexp(s, dim=1)
                p = torch.exp(s - torch.where(torch.isinf(z), torch.zeros_like(z), z)[:, None])
                out[t + i:t + i + len(rows), h] = torch.matmul(p, V[:, h * Hk // Hq])
                lse[t + i:t + i + len(rows), h] = z
        t += n
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}


def exact(case, seed):
    return _exact_append(case, seed) if case["op"] == "append" else _exact_attend(case, seed)
