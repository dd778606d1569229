"""Cache, attention and expert layer as a server runs them (block.AttentionBlock, block.MoEBlock): a prompt that becomes the shared
prefix, requests behind it in chunks, decode steps; the cache and each attention output against the formula in 64 bits on the
step's own inputs (tolerances of test_gpu_append.py and test_gpu_attn.py)."""
import math

import pytest
import torch

import paper_2609_33252_b200 as cep
from paper_2609_33252_b200.block import AttentionBlock, MoEBlock

from test_gpu_append import rotated
from test_gpu_attn import rand

pytestmark = pytest.mark.gpu

H, HQ, HK, D, PAGE = 256, 12, 3, 64, 16


class Server:
    def __init__(self, e4m3, seqs, prefix, interleaved=False):
        pages = 200
        self.scales = [0.01 + 0.02 * torch.rand(HK, device="cuda") for _ in range(2)] if e4m3 else [None, None]
        self.cache = [torch.full((pages, PAGE, HK, D), float("nan"), device="cuda").to(torch.float8_e4m3fn if e4m3 else torch.bfloat16) for _ in range(2)]
        self.inv_freq = (10000.0 ** (-torch.arange(0, D // 2, 2, dtype=torch.float64) / (D // 2))).float().cuda()
        self.interleaved, self.prefix = interleaved, prefix
        self.w = rand(((HQ + 2 * HK) * D, H), 1, 1.5 * H ** -0.5)
        self.block = AttentionBlock(self.w, *self.cache, HQ, self.inv_freq, 600, seqs + 1, 1, *self.scales, interleaved=interleaved)
        g = torch.Generator().manual_seed(5)
        self.free = torch.randperm(pages, generator=g).tolist()
        self.pages = [[] for _ in range(seqs)]
        self.len = [0] * seqs
        self.ahead = []
        self.keys = [[[], []] for _ in range(seqs + 1)]                # of every sequence, the prefix last: k, v as the cache holds them

    def step(self, new, seed, onto_prefix=False):
        """`new` tokens for each sequence (or for the prefix itself); checks everything and returns the output."""
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
        if onto_prefix:
            places, start, group = [self.ahead], [0], False
            lens = [new[0]]
        else:
            places, start, group = self.pages, self.len, True
            lens = [a + b for a, b in zip(self.len, new)]
        slots, positions = [], []
        for p, a, n, total in zip(places, start, new, lens):
            while len(p) * PAGE < total:
                p.append(self.free.pop())
            slots += [p[i // PAGE] * PAGE + i % PAGE for i in range(a, a + n)]
            positions += [i + (self.prefix if group else 0) for i in range(a, a + n)]
        width = max(1, max(map(len, places)))
        first = torch.tensor([0] + new).cumsum(0).tolist()
        batch = dict(q_start=i32(first), kv_len=i32(lens), page_table=i32([p + [0] * (width - len(p)) for p in places]))
        if group:
            batch.update(prefix_len=i32([self.prefix]), prefix_pages=i32([self.ahead]))
        x = rand((sum(new), H), seed)
        got = self.block.run(x, i32(positions), torch.tensor(slots, device="cuda"), batch)
        assert self.block.attention.status() == 0
        T = sum(new)
        # the projection's k and v are still in the block's buffer, q has been rotated in place: formula from x for q
        proj = (x.double() @ self.w.double().t()).view(T, HQ + 2 * HK, D)
        q_want, size = rotated(proj[:, :HQ].to(torch.bfloat16), i32(positions), self.inv_freq, self.interleaved)
        q = self.block.qkv[:T, :HQ]
        # The projection's bf16 here and there are roundings of sums 1e-4 apart at most (test_gpu_block.py): equal or one step, 2^-7 of the
        # value, apart, and 1e-4 where it is small; a rotated value has both of its pair's, a copied one (size 0) its own.
        x_of = torch.where(size > 0, size, q_want.abs())
        assert ((q.double() - q_want).abs() <= 2.0 ** -8 * q_want.abs() + 2.0 ** -7 * x_of + 2e-4).all()
        for c in range(2):
            source = self.block.qkv[:T, HQ + c * HK:HQ + (c + 1) * HK]
            want, size = rotated(source, i32(positions), self.inv_freq, self.interleaved) if c == 0 else (source.double(), 0 * source.double())
            held = self.cache[c].float().view(-1, HK, D)[torch.tensor(slots, device="cuda")].double()
            s = self.scales[c]
            if s is None:
                assert ((held - want).abs() <= 2.0 ** -8 * want.abs() + 1.01 * 2.0 ** -21 * size).all()
            else:
                want, size = (want / s.double()[:, None]).clamp(-448, 448), size / s.double()[:, None]
                assert ((held - want).abs() <= torch.clamp(2.0 ** -4 * want.abs(), min=2.0 ** -10) + 2.0 ** -20 * (size + want.abs())).all()
                held = held * s.double()[:, None]
            t = 0
            for b, n in enumerate(new):
                self.keys[-1 if onto_prefix else b][c].append(held[t:t + n])
                t += n
        if not onto_prefix:
            self.len = lens
        # attention over what the cache holds
        t = 0
        for b, n in enumerate(new):
            mine = self.keys[-1 if onto_prefix else b]
            K, V = (torch.cat((self.keys[-1][c] if not onto_prefix else []) + mine[c]).repeat_interleave(HQ // HK, dim=1).permute(1, 0, 2) for c in range(2))
            s = q[t:t + n].double().permute(1, 0, 2) @ K.transpose(1, 2) * D ** -0.5
            hidden = torch.arange(K.shape[1], device="cuda") > (torch.arange(n, device="cuda") + K.shape[1] - n)[:, None]
            p = torch.softmax(s.masked_fill(hidden, -math.inf), dim=2)
            o, A = p @ V, p @ V.abs()
            out = got[t:t + n].double().view(n, HQ, D).permute(1, 0, 2)
            assert ((out - o).abs() <= 2.0 ** -8 * (A + o.abs()) * 1.01 + 1e-4 * A).all()
            t += n
        return got


@pytest.mark.parametrize("e4m3,interleaved", [(False, False), (True, False), (False, True)])
def test_prefix_then_requests_then_decoding(e4m3, interleaved):
    s = Server(e4m3, 5, 100, interleaved)
    s.step([100], 1, onto_prefix=True)
    s.step([37, 1, 0, 200, 64], 2)
    s.step([40, 16, 5, 1, 1], 3)                                     # the next chunks
    for i in range(4):
        s.step([1, 1, 1, 1, 1], 10 + i)
    s.step([0, 1, 3, 0, 2], 20)                                      # some have finished, some verify drafts
    s.block.close()


def test_a_layer_of_attention_and_experts():
    from test_gpu_block import make
    cfg, host, w, block, ad, _, residual, ids = make("bf16", 96)     # the out projection takes 384 columns: 6 heads of 64
    kv = [torch.zeros(20, PAGE, 2, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    inv_freq = torch.rand(D // 2, device="cuda")
    att = AttentionBlock(rand((10 * D, cfg.H), 3, cfg.H ** -0.5), *kv, 6, inv_freq, 96, 4)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    x = rand((96, cfg.H), 4)
    batch = dict(q_start=i32([0, 24, 48, 72, 96]), kv_len=i32([24] * 4), page_table=i32([[2 * b, 2 * b + 1] for b in range(4)]), prefix_len=i32([33]),
                 prefix_pages=i32([[10, 11, 12]]))
    slots = torch.cat([torch.arange(24) + 32 * b for b in range(4)]).cuda()
    positions = (torch.arange(96) % 24 + 33).to(torch.int32).cuda()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    out = []
    for stream in (torch.cuda.current_stream(), side, torch.cuda.current_stream()):
        with torch.cuda.stream(stream):
            r = residual.clone()
            out.append(block.run(att.run(x, positions, slots, batch).contiguous(), r, ids))
    torch.cuda.synchronize()
    assert torch.isfinite(out[0].float()).all() and (out[0] != 0).any()
    assert torch.equal(out[0], out[1]) and torch.equal(out[0], out[2])
    att.close()
    block.close()


def test_the_command_with_a_prefix(capsys):
    from paper_2609_33252_b200 import block
    block.main("bf16", 300, 1000)
    lines = capsys.readouterr().out.strip().splitlines()
    assert len(lines) == 8 and all(l.endswith("us") for l in lines)


def test_a_projection_of_the_wrong_height_is_refused():
    kv = torch.zeros(2, PAGE, 2, D, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(cep.CepError, match="rows"):
        AttentionBlock(rand((9 * D, 64), 1), kv, kv.clone(), 6, torch.rand(32, device="cuda"), 8, 1)


def test_a_captured_block_replays_between_eager_calls():
    kv = [torch.zeros(8, PAGE, 2, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    att = AttentionBlock(rand((10 * D, 128), 1, 128 ** -0.5), *kv, 6, torch.rand(D // 2, device="cuda"), 8, 4)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    x, positions, slots = rand((4, 128), 2), i32([0, 1, 2, 0]), torch.tensor([0, 1, 2, PAGE], device="cuda")
    batch = dict(q_start=i32([0, 3, 4]), kv_len=i32([3, 1]), page_table=i32([[0], [1]]))
    want = att.run(x, positions, slots, batch).clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = att.run(x, positions, slots, batch)
    for _ in range(2):
        out.zero_()
        graph.replay()
        assert torch.equal(out, want)
        assert torch.equal(att.run(x, positions, slots, batch), want)
    torch.cuda.synchronize()
    assert att.attention.status() == 0
    del graph
    att.close()


def test_more_tokens_than_the_block_was_made_for_are_refused():
    kv = [torch.zeros(2, PAGE, 2, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    att = AttentionBlock(rand((10 * D, 64), 1), *kv, 6, torch.rand(32, device="cuda"), 8, 1)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    for T in (9, 16):
        with pytest.raises(cep.CepError, match="made for 8"):
            att.run(rand((T, 64), 2), i32([0] * T), torch.zeros(T, dtype=torch.int64, device="cuda"), dict(q_start=i32([0, T]), kv_len=i32([T]), page_table=i32([[0]])))
    att.close()
