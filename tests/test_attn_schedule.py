"""How the attention behind shared prefixes cuts a batch into work (cep_debug_attn_schedule, the arithmetic that the kernels use):
every key of every token in exactly one part, partial results in places of their own, shares of even cost; runs without a GPU."""
import random

import pytest

import paper_2609_33252_b200 as cep


def config(heads, kv_heads, max_tokens, max_seqs, max_prefixes, **kw):
    a = dict(n_heads=heads, n_kv_heads=kv_heads, head_dim=64, page_size=16, n_pages=4, cache_elem=0, max_tokens=max_tokens, max_seqs=max_seqs,
             max_prefixes=max_prefixes, scale=1.0)
    a.update(kw)
    cfg = cep.AttnConfig(**a)
    cfg.k_stride[:] = cfg.v_stride[:] = (16 * kv_heads * 64, kv_heads * 64, 64)
    return cfg


def check(heads, kv_heads, q_len, kv_len, prefix_start, prefix_len, causal, n_ctas):
    B, G, Gh = len(q_len), len(prefix_len), heads // kv_heads
    starts = [0]
    for n in q_len:
        starts.append(starts[-1] + n)
    cfg = config(heads, kv_heads, max(1, starts[-1]), B, G)
    if starts[-1] == 0:
        return
    parts, rows = cep.cep_debug_attn_schedule(cfg, starts, kv_len, prefix_start, prefix_len, causal, n_ctas)
    tile = 2 * (128 // Gh)
    group = [-1] * B
    for g in range(G):
        for b in range(prefix_start[g], prefix_start[g + 1]):
            group[b] = g
    items, places, cost = {}, [], {}
    for p in parts:
        key = (p["kind"], p["seq"], p["group"] if p["kind"] == 0 else 0, p["head"], p["token"])
        items.setdefault(key, []).append(p)
        assert 0 < p["tokens"] <= tile and 0 <= p["head"] < kv_heads
        if p["row"] >= 0:
            places.append((p["row"], p["row"] + p["results"] * p["tokens"] * Gh))
            assert p["results"] in (1, 2) and p["results"] * p["tokens"] <= tile
        else:
            assert p["kind"] == 2
        cost[p["cta"]] = cost.get(p["cta"], 0) + p["cost"] * (p["end"] - p["first"]) / p["steps"]
    places.sort()
    assert all(a[1] <= b[0] for a, b in zip(places, places[1:]))
    assert not places or (places[0][0] >= 0 and places[-1][1] <= rows)
    short_of = {g: 0 for g in range(G)}
    up = lambda n: -(-n // 128)
    want = {}
    for b in range(B):
        g, n = group[b], q_len[b]
        ahead = prefix_len[g] if g >= 0 else 0
        members = prefix_start[g + 1] - prefix_start[g] if g >= 0 else 0
        if n and ahead and n <= tile and members >= 2:
            short_of[g] += n
            if kv_len[b]:
                for h in range(kv_heads):
                    want[(1, b, 0, h, 0)] = (n, up(kv_len[b]))
        else:
            for t in range(0, n, tile):
                m = min(tile, n - t)
                seen = max(0, min(kv_len[b], kv_len[b] - n + t + m)) if causal else kv_len[b]
                for h in range(kv_heads):
                    want[(2, b, 0, h, t)] = (m, max(1, up(ahead) + up(seen)))
    for g in range(G):
        for t in range(0, short_of[g], tile):
            for h in range(kv_heads):
                want[(0, -1, g, h, t)] = (min(tile, short_of[g] - t), up(prefix_len[g]))
    assert set(want) == set(items)
    for key, ps in items.items():
        ps.sort(key=lambda p: p["first"])
        assert all(p["tokens"] == want[key][0] and p["steps"] == want[key][1] for p in ps)
        assert ps[0]["first"] == 0 and ps[-1]["end"] == want[key][1]
        assert all(a["end"] == b["first"] and a["cta"] < b["cta"] for a, b in zip(ps, ps[1:]))
        assert (len(ps) == 1 and key[0] == 2 and ps[0]["results"] == 1) == (ps[0]["row"] < 0)
    return cost


@pytest.mark.parametrize("heads,kv_heads", [(8, 8), (16, 2), (56, 8), (15, 3), (128, 1), (96, 1), (130, 2), (4, 4)])
@pytest.mark.parametrize("n_ctas", [1, 7, 148])
def test_every_key_once(heads, kv_heads, n_ctas):
    rng = random.Random(heads * 1000 + n_ctas)
    for _ in range(40):
        B = rng.choice([1, 2, 3, 17, 60])
        G = rng.choice([0, 1, 1, 2, 5])
        style = rng.choice(["decode", "verify", "mixed", "prefill"])
        q_len = [{"decode": 1, "verify": rng.randint(0, 9), "mixed": rng.choice([1, 1, 700]), "prefill": rng.randint(1, 900)}[style] for _ in range(B)]
        kv_len = [max(0, n + rng.choice([0, 0, -n // 2, rng.randint(0, 3000), -n])) for n in q_len]
        cuts = sorted(rng.randint(0, B) for _ in range(G + 1)) if G else [0]
        check(heads, kv_heads, q_len, kv_len, cuts, [rng.choice([0, 1, 127, 128, 129, rng.randint(1, 9000)]) for _ in range(G)], rng.random() < 0.7, n_ctas)


def test_shares_are_even():
    cost = check(56, 8, [1] * 256, [2048 + 16 * (b % 7) for b in range(256)], [0, 256], [32768], True, 148)
    assert len(cost) == 148 and max(cost.values()) < 1.1 * sum(cost.values()) / 148


def test_largest_batch():
    check(8, 8, [16] * 1024, [16 + b for b in range(1024)], [4 * g for g in range(257)], [1 + 7 * g for g in range(256)], True, 148)


@pytest.mark.parametrize("code,kw", [(-1, dict(n_heads=10)), (-9, dict(n_heads=129, n_kv_heads=1)), (-9, dict(head_dim=60)), (-9, dict(head_dim=136)),
                                     (-9, dict(page_size=24)), (-9, dict(page_size=8)), (-1, dict(n_pages=0)), (-1, dict(cache_elem=1)), (-1, dict(max_tokens=0)),
                                     (-1, dict(max_tokens=1 << 30)), (-1, dict(max_seqs=1025)), (-1, dict(max_prefixes=257)), (-1, dict(scale=0.0)),
                                     (-1, dict(scale=float("nan"))), (-9, dict(cache_elem=2, head_dim=72))])
def test_configurations_that_are_refused(code, kw):
    cfg = config(16, 8, 64, 8, 1)
    for k, v in kw.items():
        setattr(cfg, k, v)
    with pytest.raises(cep.CepError) as e:
        cep.attn_plan_workspace_bytes(cfg)
    assert e.value.code == code


def test_strides_that_are_refused():
    for i, bad in ((0, 8), (1, 60), (1, 516), (2, 36)):
        cfg = config(16, 8, 64, 8, 1)
        cfg.v_stride[i] = bad
        with pytest.raises(cep.CepError):
            cep.attn_plan_workspace_bytes(cfg)
