"""PrefixAttention against the formula in 64 bits.

Per output: the weights enter the product with V as bf16 (each off by at most 2^-8 of itself), the result is rounded once (2^-8):
|error| <= 2^-8 (A + |out|) + small, A = sum p |v| / sum p.  Roundings are independent, so over many outputs the root mean square
of the error stays below 2^-8 (rms(B) + rms(out)), B = sqrt(sum p^2 v^2) / sum p; a key left out or counted twice shows there.
`small`: the scores' own error d (fp32 sums of exact products over D columns, truncated: at most D/4 + 1 steps of 2^-23 of
sum |q k|; the exponent's rounding, 2^-24 of its size; 2^-22 of the exponential) is a relative error of a weight: A * 2 d."""
import math
import random

import pytest
import torch

import paper_2609_33252_b200 as cep

pytestmark = pytest.mark.gpu


def rand(shape, seed, std=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * std).to(torch.bfloat16)


class Batch:
    """A paged cache with `spoil` in every place that no sequence owns, and a plan over it."""

    def __init__(self, q_len, kv_len, heads, kv_heads, dim, page=16, prefix=(), start=None, e4m3=False, seed=1, spoil=float("nan"), layout="page", q_std=1.5,
                 tail_rows=0, extra_tokens=0):
        self.q_len, self.kv_len, self.heads, self.kv_heads, self.dim, self.page = q_len, kv_len, heads, kv_heads, dim, page
        self.prefix, self.start = list(prefix), ([0, len(q_len)] if start is None and len(prefix) else start)
        B, G = len(q_len), len(self.prefix)
        count = lambda n: -(-n // page)
        need = sum(map(count, kv_len)) + sum(map(count, self.prefix)) + 3
        order = list(range(need))
        random.Random(seed).shuffle(order)
        self.own = [[order.pop() for _ in range(count(n))] for n in kv_len]
        self.ahead = [[order.pop() for _ in range(count(n))] for n in self.prefix]
        used = torch.zeros(need, page, dtype=torch.bool)
        for pages, n in list(zip(self.own, kv_len)) + list(zip(self.ahead, self.prefix)):
            for j in range(n):
                used[pages[j // page], j % page] = True
        used = used.cuda()[:, :, None, None]
        self.scales = [None, None]
        caches = []
        for i in range(2):
            x = rand((need, page, kv_heads, dim), seed * 10 + i).float()
            if e4m3:
                self.scales[i] = (0.4 + torch.rand(kv_heads, device="cuda")) * 0.05
                x = x / self.scales[i][:, None]
            x = torch.where(used, x, torch.full_like(x, spoil)).to(torch.float8_e4m3fn if e4m3 else torch.bfloat16)
            if layout == "head":                          # [pages, heads, page, D] in memory
                x = x.transpose(1, 2).contiguous().transpose(1, 2)
            elif layout == "pad":                         # heads padded, k and v in one buffer
                wide = torch.zeros(need, page, kv_heads, dim + 16, dtype=torch.uint8 if e4m3 else torch.bfloat16, device="cuda").view(x.dtype)
                wide[..., :dim].copy_(x)
                x = wide[..., :dim]
            caches.append(x)
        self.k_cache, self.v_cache = caches
        self.T = sum(q_len) + tail_rows
        q = rand((self.T + extra_tokens, heads, dim + 8), seed * 10 + 2, q_std)
        self.q = q[extra_tokens:, :, :dim] if layout == "pad" else q[extra_tokens:, :, :dim].contiguous()
        ints = lambda v: torch.tensor(v, dtype=torch.int32).cuda()
        table = lambda rows: ints([r + [-7] * (max(1, max(map(len, rows))) - len(r)) for r in rows])
        starts = [0]
        for n in q_len:
            starts.append(starts[-1] + n)
        self.meta = dict(q_start=ints(starts), kv_len=ints(kv_len), page_table=table(self.own))
        if G:
            self.meta.update(prefix_start=ints(self.start), prefix_len=ints(self.prefix), prefix_pages=table(self.ahead))
        self.layer = cep.PrefixAttention(self.k_cache, self.v_cache, heads, max_tokens=self.T, max_seqs=B, max_prefixes=G, k_scale=self.scales[0],
                                         v_scale=self.scales[1])

    def keys(self, i, pages, n):
        cache = (self.k_cache, self.v_cache)[i]
        rows = [cache[p].double() for p in pages]
        x = torch.cat(rows)[:n] if rows else torch.zeros(0, self.kv_heads, self.dim, dtype=torch.float64, device="cuda")
        return x if self.scales[i] is None else x * self.scales[i].double()[:, None]

    def want(self, causal=True, scale=None):
        """out, lse and the bounds of the errors: per output, lse, and the terms of the root mean square."""
        scale = self.dim ** -0.5 if scale is None else scale
        T = sum(self.q_len)
        out = torch.zeros(T, self.heads, self.dim, dtype=torch.float64, device="cuda")
        lse = torch.full((T, self.heads), -math.inf, dtype=torch.float64, device="cuda")
        near, spread, lse_near = torch.zeros_like(out), torch.zeros_like(out), torch.zeros_like(lse)
        t = 0
        for b, (n, length) in enumerate(zip(self.q_len, self.kv_len)):
            K, V = self.keys(0, self.own[b], length), self.keys(1, self.own[b], length)
            ahead = 0
            for g in range(len(self.prefix)):
                if self.start[g] <= b < self.start[g + 1]:
                    ahead = self.prefix[g]
                    K, V = torch.cat((self.keys(0, self.ahead[g], ahead), K)), torch.cat((self.keys(1, self.ahead[g], ahead), V))
            if n == 0 or K.shape[0] == 0:
                t += n
                continue
            K, V = (x.repeat_interleave(self.heads // self.kv_heads, dim=1).permute(1, 0, 2) for x in (K, V))
            q = self.q[t:t + n].double().permute(1, 0, 2)
            s = q @ K.transpose(1, 2) * scale
            size = q.abs() @ K.abs().transpose(1, 2) * scale
            last = torch.arange(n, device="cuda") + ahead + length - n if causal else torch.full((n,), K.shape[1], device="cuda")
            hidden = torch.arange(K.shape[1], device="cuda") > last[:, None].clamp(min=ahead - 1)
            s = s.masked_fill(hidden, -math.inf)
            z = torch.logsumexp(s, dim=2)
            p = torch.exp(s - z[..., None].clamp(min=-1e300))
            off = ((self.dim / 4 + 1) * 2.0 ** -23 * size + 2.0 ** -24 * (s.abs() + z.abs()[..., None]).clamp(max=1e4) * 1.5 + 2.0 ** -21).masked_fill(hidden, 0)
            o = p @ V
            out[t:t + n], lse[t:t + n] = o.permute(1, 0, 2), z.permute(1, 0)
            A = p @ V.abs()
            d = (off.amax(dim=2) * 2)[..., None]
            near[t:t + n] = (2.0 ** -8 * (A + o.abs()) * 1.01 + A * d).permute(1, 0, 2)
            spread[t:t + n] = ((p * p) @ (V * V)).sqrt().permute(1, 0, 2)
            lse_near[t:t + n] = (d[..., 0] + 1e-6 + 2.0 ** -23 * z.abs().clamp(max=1e9)).permute(1, 0)
            t += n
        return out, lse, near, spread, lse_near

    def check(self, causal=True, with_lse=True, out=None):
        T = sum(self.q_len)
        lse = torch.full((self.T, self.heads), 7.0, device="cuda") if with_lse else None
        if out is None:
            out = torch.full((self.T, self.heads, self.dim), 5.0, dtype=torch.bfloat16, device="cuda")
        got = self.layer.run(self.q, causal=causal, out=out, lse=lse, **self.meta)
        assert self.layer.status() == 0
        o, z, near, spread, lse_near = self.want(causal)
        err = (got[:T].double() - o).abs()
        assert torch.isfinite(err).all()
        assert (err <= near).all(), float((err - near).max())
        rms = lambda x: float(x.square().mean().sqrt())
        assert rms(err) <= 2.0 ** -8 * (rms(spread) + rms(o)) + 1e-12, (rms(err), rms(spread), rms(o))
        assert (got[T:] == 5).all()                        # rows behind the last sequence stay
        if with_lse:
            empty = torch.isinf(z)
            assert torch.equal(torch.isinf(lse[:T]), empty)
            assert ((lse[:T].double() - z).abs().masked_fill(empty, 0) <= lse_near).all()
            assert (lse[T:] == 7).all()
        return got


def test_one_token_one_key():
    Batch([1], [1], 1, 1, 64).check()


@pytest.mark.parametrize("dim", [64, 128, 8, 40, 72, 96, 120])
def test_one_sequence(dim):
    Batch([1], [200], 4, 2, dim, prefix=[130]).check()


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("n", [1, 15, 127, 128, 129, 300, 1000])
def test_lengths_and_pages(page, n):
    Batch([1, 1, 1], [n, n + 1, 2], 8, 2, 128, page=page, prefix=[n]).check()


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (5, 1), (14, 2), (8, 8), (128, 1), (96, 1), (65, 1), (56, 8)])
def test_heads(heads, kv_heads):
    Batch([1, 3, 2, 1], [70, 140, 2, 33], heads, kv_heads, 64, prefix=[300]).check()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("q_len", [[1, 300, 17, 1, 64], [513], [129, 1, 1, 1], [40, 33, 32, 31]])
def test_prompts(q_len, causal):
    Batch(q_len, [n + 90 * (i % 2) for i, n in enumerate(q_len)], 8, 2, 128, page=32, prefix=[257]).check(causal)


def test_rows_that_see_nothing():
    b = Batch([0, 4, 2, 40, 1, 300], [0, 2, 0, 10, 0, 100], 16, 2, 64, tail_rows=3)
    got = b.check()
    assert (got[:2] == 0).all() and (got[4:6] == 0).all()
    Batch([2, 4, 2], [0, 2, 5], 16, 2, 64, prefix=[0]).check()
    Batch([2, 4, 2, 3], [0, 2, 5, 0], 16, 2, 64, prefix=[33, 40], start=[0, 2, 3]).check()


def test_groups():
    Batch([1] * 12 + [9, 40], [30 * i for i in range(1, 13)] + [9, 55], 14, 2, 128, prefix=[500, 0, 128, 77], start=[1, 5, 7, 7, 13], tail_rows=2).check()


@pytest.mark.parametrize("layout", ["head", "pad"])
@pytest.mark.parametrize("dim", [64, 128, 80])
def test_strides(layout, dim):
    Batch([1, 2, 60, 1], [50, 2, 160, 1], 6, 2, dim, prefix=[200], layout=layout, extra_tokens=1).check()


def test_many_decoding():
    Batch([1] * 200, [1 + 37 * i % 400 for i in range(200)], 16, 4, 128, page=64, prefix=[1500]).check()


def test_large_scores():
    # sharp rows: the running maximum rises often, weights underflow
    Batch([1, 2, 200], [900, 400, 500], 8, 2, 128, prefix=[1000], q_std=40.0).check()


@pytest.mark.parametrize("dim", [64, 128, 16, 48, 80, 112])
@pytest.mark.parametrize("page", [16, 64, 256])
def test_e4m3_caches(dim, page):
    Batch([1, 1, 3, 90], [200, 1, 129, 400], 8, 2, dim, page=page, prefix=[333], e4m3=True).check()


def test_e4m3_layouts_and_batches():
    Batch([1, 2, 60, 1], [50, 2, 160, 1], 6, 2, 80, prefix=[200], e4m3=True, layout="head").check()
    Batch([1, 2, 60, 1], [50, 2, 160, 1], 6, 2, 96, prefix=[200], e4m3=True, layout="pad").check()
    Batch([1] * 700, [1 + 37 * i % 150 for i in range(700)], 8, 2, 128, page=32, prefix=[400, 129], start=[0, 300, 650], e4m3=True).check()
    Batch([700, 1, 300], [900, 40, 300], 14, 2, 128, page=128, prefix=[600], e4m3=True).check()


def test_every_e4m3_code():
    # one key, weight 1: the output is the value, whatever its code (NaN too)
    codes = torch.arange(256, dtype=torch.uint8).cuda().view(torch.float8_e4m3fn)
    v = torch.zeros(4, 16, 1, 64, device="cuda").to(torch.float8_e4m3fn)
    v.view(torch.uint8)[:, 0, 0] = codes.view(torch.uint8).view(4, 64)
    layer = cep.PrefixAttention(torch.zeros_like(v), v, 1, max_tokens=4, max_seqs=4, max_prefixes=0)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    got = layer.run(rand((4, 1, 64), 1), i32([0, 1, 2, 3, 4]), i32([1, 1, 1, 1]), i32([[0], [1], [2], [3]])).view(256)
    want = codes.float()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got.float().nan_to_num(), want.nan_to_num())
