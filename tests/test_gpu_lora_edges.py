"""The projection with adapters where shares, chains, devices and streams end: complements test_gpu_lora.py, same cases and
tolerances (Case.check)."""
import pytest
import torch

import paper_2609_33252_b200 as cep

from test_gpu_lora import Case, ids_of, rand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("out", ["bf16", "fp32"])
@pytest.mark.parametrize("T,K,N", [(13, 1024, 7168), (14, 1024, 7168), (27, 1024, 7100), (61, 1024, 7168), (63, 1024, 7042), (125, 1024, 7168),
                                   (300, 2048, 2148), (519, 2048, 2148), (385, 2048, 2304), (700, 2048, 1794), (257, 2048, 4164)])
def test_ragged_shares_of_the_exchange(T, K, N, out):
    # K split over two or more CTAs (or pairs) whose shares of the rows do not fill a round of a warp's reads, and column
    # blocks that end inside a half: only rows and columns that exist are read from the other CTAs
    c = Case(K, N, ranks=(16,), max_tokens=T, out=out)
    x = rand((T, K), 5)
    want = c.check(x, None)
    c.check(x, ids_of(T, 1, 6))
    for _ in range(20):
        assert torch.equal(c.layer.run(x), want)
    assert c.layer.status() == 0


def test_a_plan_is_not_made_inside_a_capture():
    # the clearing of its slots and counters would only be recorded
    w, x = rand((64, 64), 1), rand((4, 64), 2)
    g, y = torch.cuda.CUDAGraph(), torch.zeros(8, device="cuda")
    with torch.cuda.graph(g):
        with pytest.raises(cep.CepError, match="captured"):
            cep.LoRAProjection(w, 16, 2, 8)
        y += 1                                               # the capture goes on
    g.replay()
    torch.cuda.synchronize()
    assert (y == 1).all()
    layer = cep.LoRAProjection(w, 16, 2, 8)
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    layer.run(x, ids)
    assert layer.status() == -6                              # every slot is empty


def test_a_report_is_not_cleared_with_the_one_before():
    # reports in turn, each call enqueued as soon as the status of the one before has been read and cleared, on a stream that
    # does not wait for the default one
    c = Case(64, 64, ranks=(8,), max_tokens=4)
    x, out = rand((4, 64), 1), torch.empty(4, 64, dtype=torch.bfloat16, device="cuda")
    good = torch.zeros(4, dtype=torch.int32, device="cuda")
    bad = good + 1
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for i in range(300):
        c.layer.run(x, bad, out, stream=side)
        assert c.layer.status() == -6, i
        if i % 3 == 0:
            c.layer.run(x, good, out, stream=side)
            assert c.layer.status() == 0, i


@pytest.mark.parametrize("T", [64, 300])
def test_inputs_dropped_while_another_stream_uses_them(T):
    c = Case(512, 2048, ranks=(16, 32), max_tokens=T)
    x, ids = rand((T, 512), 1), ids_of(T, 2, 1)
    want = c.check(x, ids)
    h, w = rand((T, 2048), 4), rand((2048,), 3)
    normed = torch.empty_like(h)
    cep.moe_norm(h, w, y=normed)
    side = torch.cuda.Stream()
    busy = torch.empty(1 << 26, device="cuda")
    for stream in (side, side.cuda_stream):
        for _ in range(4):
            y = torch.empty_like(h)
            x1, ids1, h1, w1 = x.clone(), ids.clone(), h.clone(), w.clone()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                busy.fill_(1.0)                              # the calls begin after the memory could have been given away
            got = c.layer.run(x1, ids1, stream=stream)
            cep.moe_norm(h1, w1, y=y, stream=stream)
            del x1, ids1, h1, w1
            for like in (x, ids, h, w):
                for _ in range(3):
                    torch.empty_like(like).fill_(1)
            torch.cuda.synchronize()
            assert torch.equal(got, want) and torch.equal(y, normed)
    assert c.layer.status() == 0


# An fp32 output is as exact as a 32-bit evaluation.  By norm: the matrix unit's additions truncate, so a chain of n of them
# drifts by n/2 units of 2^-23 of its end at the worst, and below a third of that as a drift that grows with the sum
# (test_fp32_outputs_keep_fp32_accuracy).  Chains hold at most 1024 products (64 additions): 1.3e-6 for W x and for s = A x.
# The up projection adds 3R/16 products to one chain (R = 64: 12 additions, 2.4e-7); s as three bf16 terms and the scale's
# product are below 2^-23.
EXACT, EXACT_ADAPTERS = 1.3e-6, 1.3e-6 + 2.4e-7 + 1.2e-7


@pytest.mark.parametrize("T,K,N", [(1, 7168, 128), (40, 7168, 128), (64, 7168, 1024), (100, 7168, 128), (300, 7168, 128), (700, 7168, 512),
                                   (2048, 7168, 128)])
def test_fp32_outputs_keep_fp32_accuracy_with_adapters(T, K, N):
    # without the shared projection's part, so that nothing hides the adapters'
    c = Case(K, N, ranks=(64, 64), max_tokens=T, out="fp32", weight=torch.zeros(N, K, dtype=torch.bfloat16, device="cuda"))
    x, ids = rand((T, K), 2), (torch.arange(T, device="cuda") % 2).to(torch.int32)
    got, y = c.check(x, ids).double(), c.reference(x, ids)[0]
    assert ((got - y).norm() / y.norm()).item() <= EXACT_ADAPTERS
    # and with it
    c = Case(K, N, ranks=(64, 64), max_tokens=T, out="fp32")
    got, y = c.check(x, ids).double(), c.reference(x, ids)[0]
    assert ((got - y).norm() / y.norm()).item() <= EXACT + EXACT_ADAPTERS


@pytest.mark.parametrize("T,K,N", [(16384, 7168, 128), (3000, 16384, 256), (20000, 7168, 64), (33, 32768, 128), (600, 49152, 128)])
def test_fp32_accuracy_of_long_sums_in_the_down_projection(T, K, N):
    # few K parts a tile, or a K that is long even in eight: more accumulation chains, not longer ones
    c = Case(K, N, ranks=(64, 40), max_tokens=T, out="fp32", weight=torch.zeros(N, K, dtype=torch.bfloat16, device="cuda"))
    x, ids = rand((T, K), 2), (torch.arange(T, device="cuda") % 2).to(torch.int32)
    got, y = c.check(x, ids).double(), c.reference(x, ids)[0]
    assert ((got - y).norm() / y.norm()).item() <= EXACT_ADAPTERS


@pytest.mark.parametrize("T,K,N", [(64, 7168, 18944), (64, 16384, 18944), (40, 12288, 18944), (128, 16384, 9472), (64, 32768, 9472), (17, 57344, 9472), (64, 81920, 256)])
def test_fp32_accuracy_of_long_sums_over_wide_outputs(T, K, N):
    # as many column blocks as SMs, so that K is not split, or a K that is long even when it is: more accumulation chains than
    # accumulators
    c = Case(K, N, max_tokens=T, out="fp32")
    x = rand((T, K), 2)
    got, y = c.check(x, None).double(), c.reference(x, None)[0]
    assert ((got - y).norm() / y.norm()).item() <= EXACT


def test_fp32_long_sums_with_adapters_over_wide_outputs():
    c = Case(16384, 9472, ranks=(64, 20), max_tokens=64, out="fp32")
    for T in (3, 64):
        x, ids = rand((T, 16384), 2), ids_of(T, 2, 3)
        got, y = c.check(x, ids).double(), c.reference(x, ids)[0]
        assert ((got - y).norm() / y.norm()).item() <= EXACT + EXACT_ADAPTERS
        for _ in range(5):
            assert torch.equal(c.layer.run(x, ids).double(), got)


@pytest.mark.parametrize("pair", [(0, 1), (0, 2), (1, 3), (2, 3), (1, 2), (0, 1, 2, 3)])
def test_plans_side_by_side(pair):
    # several plans on a stream each: blocks of different plans share SMs, shared and tensor memory; every result is the one
    # the plan gives alone
    shapes = [(64, 2048, 4096, (64, 16, 32) * 4, "bf16"), (100, 2048, 1024, (16,) * 8, "fp32"), (600, 1024, 2048, (32,) * 6, "bf16"),
              (2048, 1024, 1024, (64, 8), "fp32")]
    plans = []
    for i in pair:
        T, K, N, ranks, out = shapes[i]
        c = Case(K, N, ranks=ranks, max_tokens=T, out=out, seed=10 * i)
        x, ids = rand((T, K), i), ids_of(T, len(ranks), i)
        plans.append((c, x, ids, c.check(x, ids), torch.cuda.Stream(), []))
    torch.cuda.synchronize()
    for _ in range(30):
        for c, x, ids, want, stream, got in plans:
            got.append(c.layer.run(x, ids, stream=stream))
    torch.cuda.synchronize()
    for c, x, ids, want, stream, got in plans:
        assert c.layer.status() == 0
        for y in got:
            assert torch.equal(y, want)


def test_streams_that_come_and_go():
    # the driver may give a new stream the handle of one that was destroyed with work under way: still another stream
    import ctypes
    cudart = ctypes.CDLL(next(l.split()[-1] for l in open("/proc/self/maps") if "libcudart" in l))
    c = Case(2048, 2048, ranks=(16, 32), max_tokens=600)
    x, ids = [rand((600, 2048), s) for s in (1, 2)], [ids_of(600, 2, s) for s in (3, 4)]
    want = [c.check(x[i], ids[i]) for i in range(2)]
    outs = [torch.empty_like(want[0]) for _ in range(40)]
    torch.cuda.synchronize()
    seen = set()
    for i, out in enumerate(outs):
        handle = ctypes.c_void_p()
        assert cudart.cudaStreamCreateWithFlags(ctypes.byref(handle), 1) == 0
        seen.add(handle.value)
        cep.lora_project(c.layer.plan, x[i % 2], ids[i % 2], out, stream=handle.value)
        assert cudart.cudaStreamDestroy(handle) == 0
    torch.cuda.synchronize()
    assert c.layer.status() == 0
    for i, out in enumerate(outs):
        assert torch.equal(out, want[i % 2]), (i, len(seen))
    print("%d handles" % len(seen))
