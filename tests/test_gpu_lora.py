"""The projection with per-request low-rank adapters against its formula in 64 bits:
y[t] = W x[t] + scale_a B_a (A_a x[t]).

Tolerance, from the arithmetic, element by element: with M = sum_k |x_k W_k| and L = |scale| * sum_r |B_r| sum_k |A_rk x_k|,
  fp32 accumulation in steps of 16 products  (K/16 + R/8 + 8) * 2^-23 * (M + L)   (a unit in the last place per step)
  the adapter's inner sums, same steps       (K/16 + 8) * 2^-23 * L
  s as two bf16 terms                        2^-16 * L
  a bf16 output                              2^-8 * |y|
"""
import pytest
import torch

import paper_2609_33252_b200 as cep

pytestmark = pytest.mark.gpu


def rand(shape, seed, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * std).to(torch.bfloat16)


class Case:
    """Weight, adapters (ranks[slot], 0: not loaded) and the plan."""

    def __init__(self, K, N, ranks=(), max_tokens=256, max_rank=None, out="bf16", seed=1, weight=None):
        self.K, self.N, self.ranks = K, N, list(ranks)
        self.w = rand((N, K), seed, K ** -0.5) if weight is None else weight
        self.R = max_rank or max(list(ranks) + [0])
        self.out = out
        self.layer = cep.LoRAProjection(self.w, max_tokens, len(self.ranks), self.R,
                                        cep.CEP_ELEM_FP32 if out == "fp32" else cep.CEP_ELEM_BF16)
        self.a = [rand((r, K), seed + 100 + s, K ** -0.5) for s, r in enumerate(self.ranks)]
        self.b = [rand((N, r), seed + 200 + s, max(r, 1) ** -0.5) for s, r in enumerate(self.ranks)]
        self.scale = [0.5 + 0.25 * s for s in range(len(self.ranks))]
        for s, r in enumerate(self.ranks):
            if r:
                self.layer.load_adapter(s, self.a[s], self.b[s], self.scale[s])

    def reference(self, x, ids):
        xd, wd = x.double(), self.w.double()
        y, mag = xd @ wd.t(), xd.abs() @ wd.abs().t()
        tol = (self.K / 16 + self.R / 8 + 8) * 2.0 ** -23 * mag
        if ids is not None:
            for s, r in enumerate(self.ranks):
                rows = torch.nonzero(ids.long() == s).flatten()
                if r and rows.numel():
                    a, b = self.a[s].double(), self.b[s].double()
                    y[rows] += self.scale[s] * (xd[rows] @ a.t()) @ b.t()
                    low = abs(self.scale[s]) * (xd[rows].abs() @ a.abs().t()) @ b.abs().t()
                    tol[rows] += low * ((2 * self.K / 16 + self.R / 8 + 16) * 2.0 ** -23 + 2.0 ** -16)
        if self.out == "bf16":
            tol = tol + 2.0 ** -8 * y.abs()
        return y, tol

    def check(self, x, ids, status=0, out=None, what=""):
        T = x.shape[0]
        if out is None:
            out = torch.full((T, self.N), float("nan"), dtype=self.layer.out_dtype, device="cuda")
        got = self.layer.run(x, ids, out)
        assert self.layer.status() == status
        y, tol = self.reference(x, ids)
        bad = ~(torch.abs(got.double() - y) <= tol)
        assert not bad.any(), "%s: %d of %d off, first at %s" % (what, int(bad.sum()), bad.numel(), torch.nonzero(bad)[0].tolist())
        return got


def ids_of(T, n, seed, runs=False):
    """Slots -1..n-1 per token: at random, or in runs of requests."""
    g = torch.Generator().manual_seed(seed)
    if runs:
        cuts = torch.sort(torch.randint(0, T + 1, (max(1, T // 40),), generator=g)).values
        which = torch.bucketize(torch.arange(T), cuts, right=True)
        ids = torch.randint(-1, n, (int(which.max()) + 1,), generator=g)[which]
    else:
        ids = torch.randint(-1, n, (T,), generator=g)
    return ids.to(torch.int32).cuda()


TOKENS = [1, 2, 15, 16, 17, 64, 100, 127, 128, 129, 255, 256, 257, 300, 511, 513, 1000]


@pytest.mark.parametrize("out", ["bf16", "fp32"])
@pytest.mark.parametrize("T", TOKENS)
def test_plain_projection(T, out):
    c = Case(512, 384, max_tokens=1024, out=out)
    c.check(rand((T, 512), 7), None)


@pytest.mark.parametrize("K,N", [(8, 1), (64, 7), (72, 128), (128, 129), (200, 255), (1024, 256), (520, 1000), (2048, 64), (7168, 96), (64, 4099)])
@pytest.mark.parametrize("T", [1, 33, 200, 400])
def test_odd_sizes(K, N, T):
    for out in ("bf16", "fp32"):
        c = Case(K, N, ranks=(8, 16), max_tokens=400, out=out)
        x = rand((T, K), 8)
        c.check(x, None, what="plain")
        c.check(x, ids_of(T, 2, 9), what="adapters")


@pytest.mark.parametrize("T", TOKENS)
@pytest.mark.parametrize("runs", [False, True])
def test_adapters_over_lengths(T, runs):
    c = Case(576, 640, ranks=(16, 8, 64, 33), max_tokens=1024)
    c.check(rand((T, 576), 11), ids_of(T, 4, T, runs))


@pytest.mark.parametrize("rank", [1, 5, 15, 16, 17, 31, 32, 33, 48, 64, 65, 100, 128, 200, 256])
def test_ranks(rank):
    for T in (3, 150, 290):
        c = Case(256, 320, ranks=(rank, 0, 7), max_tokens=300)
        ids = ids_of(T, 3, rank)
        ids[ids == 1] = -1
        c.check(rand((T, 256), rank), ids, what="T=%d" % T)


@pytest.mark.parametrize("T", [64, 128, 200, 256, 600])
def test_many_adapters_in_one_batch(T):
    # as many adapters as tokens in a tile, in arrival order
    n = min(T, 256)
    c = Case(320, 256, ranks=[4 + (s * 7) % 29 for s in range(n)], max_tokens=T)
    ids = (torch.randperm(T, generator=torch.Generator().manual_seed(3)) % n).to(torch.int32).cuda()
    c.check(rand((T, 320), 5), ids)


@pytest.mark.parametrize("T", [5, 130, 700])
def test_no_token_or_every_token_has_an_adapter(T):
    c = Case(384, 512, ranks=(32, 16), max_tokens=T)
    x = rand((T, 384), 4)
    none = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    assert torch.equal(c.check(x, none), c.check(x, None))
    c.check(x, torch.ones(T, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("T", [9, 140, 520])
def test_strided_rows(T):
    K, N = 264, 200
    w = rand((N, K + 24), 1, K ** -0.5)[:, :K]
    c = Case(K, N, ranks=(12,), max_tokens=T, weight=w)
    wide = torch.full((T, N + 13), float("nan"), dtype=torch.bfloat16, device="cuda")
    out = wide[:, 3:3 + N]
    c.check(rand((T, K + 40), 2)[:, 16:16 + K], ids_of(T, 1, 1), out=out)
    assert torch.isnan(wide[:, :3]).all() and torch.isnan(wide[:, 3 + N:]).all()         # nothing beside the rows is touched


def test_adapter_slices_of_a_padded_bank():
    # adapters as views of a bank padded to the largest rank, with NaN in the padding
    K, N = 320, 256
    c = Case(K, N, ranks=(10, 20), max_tokens=200, max_rank=40)
    for s, r in enumerate(c.ranks):
        down = torch.full((40, K), float("nan"), dtype=torch.bfloat16, device="cuda")
        up = torch.full((N, 40), float("nan"), dtype=torch.bfloat16, device="cuda")
        down[:r], up[:, :r] = c.a[s], c.b[s]
        c.layer.load_adapter(s, down[:r], up[:, :r], c.scale[s])
    for T in (1, 60, 200):
        c.check(rand((T, K), 6), ids_of(T, 2, T))


@pytest.mark.parametrize("T", [40, 300])
def test_a_token_without_an_adapter_is_not_touched_by_its_neighbours(T):
    # one adapter's B holds infinities, one token's x holds NaN: only their own rows show it
    c = Case(256, 256, ranks=(16, 16), max_tokens=T)
    c.layer.load_adapter(1, c.a[1], torch.full_like(c.b[1], float("inf")), 1.0)
    ids = torch.zeros(T, dtype=torch.int32, device="cuda")
    x = rand((T, 256), 3)
    x[5] = float("nan")
    ids[6] = -1
    got = c.layer.run(x, ids)
    assert torch.isnan(got[5]).all()
    keep = torch.arange(T, device="cuda") != 5
    y, tol = c.reference(x, ids)
    assert (torch.abs(got.double() - y)[keep] <= tol[keep]).all()


@pytest.mark.parametrize("T", [33, 150, 600])
@pytest.mark.parametrize("value", [float("inf"), float("nan"), -float("inf")])
def test_an_adapter_that_is_not_finite_reaches_nobody_else(T, value):
    # one value of one adapter's B; tokens of both adapters share every tile
    c = Case(256, 320, ranks=(16, 20), max_tokens=T)
    bad = c.b[1].clone()
    bad[100, 3] = value
    c.layer.load_adapter(1, c.a[1], bad, 1.0)
    assert c.layer.status() == -1
    x, ids = rand((T, 256), 3), ids_of(T, 2, 5)
    c.ranks[1] = 0                                           # the slot is empty: its tokens get the shared projection alone
    c.check(x, ids, status=-6)
    c.layer.load_adapter(1, c.a[1], c.b[1], c.scale[1])      # and takes an adapter again
    c.ranks[1] = 20
    c.check(x, ids)


def test_infinite_products_stay_with_their_token():
    # values of x and A whose product overflows fp32: the token's own row, and no other
    c = Case(256, 256, ranks=(16,), max_tokens=200)
    a = c.a[0].clone()
    a[0] = 3e38
    c.layer.load_adapter(0, a, c.b[0], 1.0)
    x, ids = rand((200, 256), 3), torch.full((200,), -1, dtype=torch.int32, device="cuda")
    x[7] = 1e30
    ids[7] = 0
    got = c.layer.run(x, ids)
    assert not torch.isfinite(got[7]).any()
    keep = torch.arange(200, device="cuda") != 7
    y, tol = c.reference(x, None)
    assert (torch.abs(got.double() - y)[keep] <= tol[keep]).all()


def test_the_most_slots():
    c = cep.LoRAProjection(rand((48, 64), 1), 300, 4096, 16)
    slots = [0, 5, 4095]
    ad = {s: (rand((3 + s % 7, 64), 10 + s, 0.1), rand((48, 3 + s % 7), 20 + s)) for s in slots}
    for s, (a, b) in ad.items():
        c.load_adapter(s, a, b, 2.0)
    x = rand((300, 64), 2)
    ids = torch.tensor(slots + [-1], dtype=torch.int32, device="cuda")[torch.arange(300, device="cuda") % 4].contiguous()
    for T in (1, 3, 130, 300):
        y = x[:T].double() @ c.weight.double().t()
        for s, (a, b) in ad.items():
            m = (ids[:T] == s).double()[:, None]
            y += m * 2.0 * (x[:T].double() @ a.double().t()) @ b.double().t()
        got = c.run(x[:T], ids[:T])
        assert c.status() == 0
        assert (torch.abs(got.double() - y) <= 2 ** -8 * y.abs() + 1e-3).all()


@pytest.mark.parametrize("T", [20, 400])
def test_ids_that_name_nothing_are_reported_and_skipped(T):
    c = Case(256, 192, ranks=(16, 0, 16), max_tokens=T)
    x = rand((T, 256), 3)
    ids = ids_of(T, 1, 2)
    want = c.check(x, ids)
    for wrong in (1, 3, -2, 1 << 30):
        bad = ids.clone()
        bad[T - 1] = wrong
        ref = ids.clone()
        ref[T - 1] = -1
        got = c.layer.run(x, bad)
        assert c.layer.status() == -6
        y, tol = c.reference(x, ref)
        assert (torch.abs(got.double() - y) <= tol).all()
    assert torch.equal(c.check(x, ids), want)


def test_replacing_and_dropping_an_adapter():
    c = Case(256, 256, ranks=(16, 32), max_tokens=64)
    x, ids = rand((64, 256), 1), ids_of(64, 2, 1)
    c.check(x, ids)
    c.ranks[0], c.a[0], c.b[0], c.scale[0] = 8, rand((8, 256), 50, 0.06), rand((256, 8), 51, 0.3), -2.0
    c.layer.load_adapter(0, c.a[0], c.b[0], c.scale[0])
    c.check(x, ids)
    c.layer.drop_adapter(0)
    c.ranks[0] = 0
    c.check(x, ids, status=-6)


@pytest.mark.parametrize("T", [1, 64, 200, 900])
def test_repeats_bit_for_bit_and_over_streams(T):
    c = Case(2048, 1024, ranks=(16, 64, 32), max_tokens=T)
    x, ids = rand((T, 2048), 1), ids_of(T, 3, 4)
    want = c.check(x, ids)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    outs = [torch.empty_like(want) for _ in range(24)]
    for i, o in enumerate(outs):
        c.layer.run(x, ids, o, stream=streams[i % 3])       # one plan: the calls share its workspace
    torch.cuda.synchronize()
    assert c.layer.status() == 0
    for o in outs:
        assert torch.equal(o, want)


def test_different_lengths_in_turn_on_one_plan():
    c = Case(704, 512, ranks=(16, 48), max_tokens=1500)
    for T in (1, 1500, 3, 257, 256, 64, 1024, 1):
        c.check(rand((T, 704), T), ids_of(T, 2, T, runs=T > 300))
        c.check(rand((T, 704), T + 1), None)


@pytest.mark.parametrize("T", [2, 64, 600])
def test_graph_replay(T):
    c = Case(1024, 768, ranks=(16, 32), max_tokens=T)
    x, ids, out = rand((T, 1024), 1), ids_of(T, 2, 1), torch.empty(T, 768, dtype=torch.bfloat16, device="cuda")
    c.layer.run(x, ids, out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.layer.run(x, ids, out)
    x2, ids2 = rand((T, 1024), 2), ids_of(T, 2, 5)
    x.copy_(x2), ids.copy_(ids2)
    for _ in range(3):
        out.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        y, tol = c.reference(x2, ids2)
        assert (torch.abs(out.double() - y) <= tol).all()
    assert c.layer.status() == 0


@pytest.mark.parametrize("T,K,N", [(64, 7168, 7168), (1, 7168, 7168), (2048, 7168, 2048), (1531, 2048, 7168)])
def test_wide_layers(T, K, N):
    c = Case(K, N, ranks=(16, 64, 32), max_tokens=T)
    c.check(rand((T, K), 1), ids_of(T, 3, 1, runs=T > 300))


@pytest.mark.parametrize("T,N", [(1, 256), (64, 256), (100, 64), (256, 7168), (300, 256), (2048, 384)])
def test_fp32_outputs_keep_fp32_accuracy(T, N):
    # The matrix unit's additions truncate, so one chain over K drifts by about half a unit of 2^-23 per 16 products.  fp32
    # outputs are summed from chains of at most 1024 products (64 additions): 2^-23 * 64 / 2 = 3.8e-6 at the very worst,
    # and as a drift that grows with the partial sum (its mean size is half the final one) below a third of it.
    c = Case(7168, N, max_tokens=T, out="fp32")
    x = rand((T, 7168), 2)
    got, y = c.check(x, None).double(), c.reference(x, None)[0]
    assert ((got - y).norm() / y.norm()).item() <= 1.3e-6


@pytest.mark.parametrize("T,K,N,ranks,out", [(1, 64, 7, (8,), "bf16"), (77, 328, 520, (16, 33), "bf16"), (128, 512, 256, (4,) * 40, "fp32"),
                                             (513, 264, 300, (64, 8), "bf16"), (1030, 128, 100, (256, 1), "fp32")])
def test_nothing_is_written_past_the_buffers(T, K, N, ranks, out):
    # workspace, bank and output inside larger buffers filled with a pattern
    cfg = cep.LoraConfig(K, N, T, len(ranks), max(ranks), cep.CEP_ELEM_FP32 if out == "fp32" else cep.CEP_ELEM_BF16)
    big = {n: torch.full((size + 8192,), 0xA5, dtype=torch.uint8, device="cuda")
           for n, size in (("ws", cep.lora_plan_workspace_bytes(cfg)), ("bank", cep.lora_bank_bytes(cfg)))}
    w, x = rand((N, K), 1, K ** -0.5), rand((T, K), 2)
    plan = cep.lora_plan(cfg, w, big["bank"][:-8192], big["ws"][:-8192])
    for s, r in enumerate(ranks):
        cep.lora_load_adapter(plan, s, r, 1.0, rand((r, K), 10 + s, K ** -0.5), rand((N, r), 50 + s))
    dtype = torch.float32 if out == "fp32" else torch.bfloat16
    y = torch.full((T + 64, N), -77.0, dtype=dtype, device="cuda")
    for ids in (ids_of(T, len(ranks), 3), None):
        cep.lora_project(plan, x, ids, y[:T])
        assert cep.lora_status(plan) == 0
        assert (y[T:] == -77.0).all() and torch.isfinite(y[:T]).all()
        assert all((b[-8192:] == 0xA5).all() for b in big.values())
    cep.lora_plan_destroy(plan)


def test_python_refusals():
    c = Case(64, 64, ranks=(8,), max_tokens=16)
    x = rand((4, 64), 1)
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    bad = [lambda: c.layer.run(x.float(), ids), lambda: c.layer.run(x[:, :32], ids), lambda: c.layer.run(x, ids[:3]),
           lambda: c.layer.run(x, ids.long()), lambda: c.layer.run(rand((17, 64), 1), None), lambda: c.layer.run(x, ids, torch.empty(4, 64, device="cuda")),
           lambda: c.layer.run(x[:1].expand(4, 64), ids), lambda: c.layer.run(rand((4, 65), 1)[:, 1:], ids), lambda: c.layer.load_adapter(1, c.a[0], c.b[0]),
           lambda: c.layer.load_adapter(0, rand((9, 64), 1), rand((64, 9), 1)), lambda: c.layer.load_adapter(0, c.a[0], c.b[0].t()),
           lambda: c.layer.load_adapter(0, c.a[0], c.b[0], float("inf")), lambda: cep.LoRAProjection(c.w.float(), 4), lambda: cep.LoRAProjection(c.w[:, :60], 4)]
    for f in bad:
        with pytest.raises(cep.CepError):
            f()
    plain = cep.LoRAProjection(c.w, 16)
    with pytest.raises(cep.CepError):
        plain.run(x, ids)
    c.check(x, ids)


def test_no_tokens():
    c = Case(64, 64, ranks=(8,), max_tokens=16)
    assert c.layer.run(rand((0, 64), 1), torch.empty(0, dtype=torch.int32, device="cuda")).shape == (0, 64)


@pytest.mark.parametrize("T", [64, 300])
def test_outputs_and_adapters_of_another_stream(T):
    # the stream that computes is not the one the tensors' memory comes from, and that one is busy and reuses what it frees
    c = Case(512, 2048, ranks=(16, 32), max_tokens=T)
    x, ids = rand((T, 512), 1), ids_of(T, 2, 1)
    want = c.check(x, ids)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for handle in (side, side.cuda_stream):
        layer = cep.LoRAProjection(c.w, T, 2, 32, stream=handle)
        for s in range(2):
            layer.load_adapter(s, c.a[s].clone(), c.b[s].clone(), c.scale[s], stream=handle)     # dropped at once
            for r in (16, 32):
                torch.full((r, 512), 9.0, dtype=torch.bfloat16, device="cuda"), torch.full((2048, r), 9.0, dtype=torch.bfloat16, device="cuda")
        side.wait_stream(torch.cuda.current_stream())
        outs = []
        for _ in range(8):
            junk = torch.empty((T, 2048), dtype=torch.bfloat16, device="cuda")
            for _ in range(20):
                junk.fill_(3.0)
            del junk
            outs.append(layer.run(x, ids, stream=handle))
        torch.cuda.synchronize()
        assert layer.status() == 0
        for o in outs:
            assert torch.equal(o, want)
