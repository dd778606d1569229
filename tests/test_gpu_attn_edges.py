"""PrefixAttention and attn_append where streams, graphs, bad tables, far offsets and large batches end; same batches, formula and
tolerances as test_gpu_attn.py (Batch.check)."""
import pytest
import torch

import paper_2609_33252_b200 as cep

from test_gpu_attn import Batch, rand

pytestmark = pytest.mark.gpu


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("e4m3", [False, True])
def test_the_same_bits_every_time(e4m3):
    # items split over many blocks, both warpgroups, partial pages: nothing may depend on when a tile arrives
    b = Batch([1] * 60 + [50, 300], [1 + 61 * i % 1900 for i in range(60)] + [80, 900], 56, 8, 128, page=64, prefix=[3000], e4m3=e4m3)
    want = b.check()
    out = torch.empty_like(want)
    for _ in range(60):
        out.zero_()
        b.layer.run(b.q, out=out, **b.meta)
        assert torch.equal(out, want)
    assert b.layer.status() == 0


def test_largest_tables():
    Batch([1] * 1024, [1 + i % 40 for i in range(1024)], 8, 1, 64, prefix=[3 + i % 50 for i in range(256)], start=[4 * i for i in range(257)]).check()
    Batch([2] * 1024, [2 + i % 20 for i in range(1024)], 2, 2, 64, prefix=[300]).check()


def test_a_long_context():
    Batch([1], [100001], 8, 1, 128, page=256).check()
    Batch([5, 1], [40000, 3], 4, 4, 64, page=128, prefix=[50001], e4m3=True).check()


def test_many_more_heads_than_a_row_tile_divides():
    Batch([9, 30, 1, 200], [100, 30, 500, 260], 100, 1, 64, prefix=[140]).check()
    Batch([9, 30, 1, 200], [100, 30, 500, 260], 43, 1, 128, prefix=[140]).check()


def test_every_short_length_around_a_row_tile():
    # groups of 4 heads: row tiles of 32 tokens; sequences of one tile, two tiles and just more
    for n in (31, 32, 33, 63, 64, 65):
        Batch([n, 1, n, 2], [n, 7, n + 130, 2], 8, 2, 64, prefix=[260]).check()


def test_nothing_to_do():
    b = Batch([1, 2], [3, 4], 4, 2, 64, prefix=[20])
    empty = torch.zeros(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    assert b.layer.run(empty, **b.meta).shape == (0, 4, 64)
    out = torch.full_like(b.q, 3.0)
    b.layer.run(b.q, i32([0]), i32([]), torch.zeros(0, 1, dtype=torch.int32, device="cuda"), out=out)
    assert (out == 3).all()
    cep.attn_append(empty[:, :2], empty[:, :2], i32([]), torch.zeros(0, dtype=torch.int64, device="cuda"), torch.ones(32, device="cuda"), b.k_cache, b.v_cache)
    assert b.layer.status() == 0
    b.check()


def test_streams_take_turns():
    b = Batch([1] * 40, [200 + i for i in range(40)], 16, 4, 128, prefix=[1000])
    want = b.check()
    side = [torch.cuda.Stream() for _ in range(3)]
    outs = [torch.zeros_like(want) for _ in range(30)]
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        if i % 2:
            b.layer.run(b.q, out=o, stream=side[i % 3], **b.meta)
        else:
            with torch.cuda.stream(side[i % 3]):
                b.layer.run(b.q, out=o, **b.meta)
    assert b.layer.status() == 0
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    with torch.cuda.stream(side[0]):
        got = b.layer.run(b.q, stream=side[1], **b.meta)             # allocated for the stream it is made on
    side[1].synchronize()
    assert torch.equal(got, want)


def test_two_plans_at_once():
    a = Batch([1] * 40, [200 + i for i in range(40)], 16, 4, 128, prefix=[1000])
    c = Batch([300, 20], [400, 20], 8, 2, 64, prefix=[700], e4m3=True, seed=2)
    wants = a.check(), c.check()
    s = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = []
    for _ in range(20):
        for b, st in zip((a, c), s):
            with torch.cuda.stream(st):
                outs.append(b.layer.run(b.q, **b.meta))
    torch.cuda.synchronize()
    assert all(torch.equal(o, wants[i % 2]) for i, o in enumerate(outs))
    assert a.layer.status() == 0 and c.layer.status() == 0


def test_a_captured_call_replays_with_other_lengths():
    b = Batch([1, 1, 1, 1], [500, 40, 3, 129], 8, 2, 64, prefix=[300, 77], start=[0, 2, 4])
    b.check()
    out, lse = torch.zeros_like(b.q), torch.zeros(b.T, 8, device="cuda")
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(g, stream=s):
        b.layer.run(b.q, out=out, lse=lse, **b.meta)
        b.layer.run(b.q, out=out, lse=lse, **b.meta)                 # twice in a graph
    for kv, pre in (([1, 2, 3, 4], [5, 6]), ([500, 40, 3, 129], [300, 77]), ([0, 40, 0, 128], [0, 77])):
        b.kv_len, b.prefix = kv, pre
        b.meta["kv_len"].copy_(i32(kv))
        b.meta["prefix_len"].copy_(i32(pre))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert b.layer.status() == 0
        o, z, near, _, lse_near = b.want()
        assert ((out.double() - o).abs() <= near).all()
        seen = ~torch.isinf(z)
        assert torch.equal(torch.isinf(lse), ~seen) and ((lse.double() - z).abs()[seen] <= lse_near[seen]).all()


def test_captured_appends_replay():
    k, cache = rand((3, 2, 64), 1), torch.zeros(2, 16, 2, 64, dtype=torch.bfloat16, device="cuda")
    v_cache, slots, positions = cache.clone(), torch.tensor([0, 5, -1], device="cuda"), i32([0, 0, 0])
    inv_freq, q_out = torch.ones(32, device="cuda"), torch.zeros(3, 2, 64, dtype=torch.bfloat16, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cep.attn_append(k, k, positions, slots, inv_freq, cache, v_cache, q=k, q_out=q_out)
    slots.copy_(torch.tensor([31, -1, 7], device="cuda"))
    g.replay()
    torch.cuda.synchronize()
    flat = v_cache.view(32, 2, 64)
    assert torch.equal(flat[31], k[0]) and torch.equal(flat[7], k[2]) and (flat[[0, 5]] == 0).all() and torch.equal(q_out, k)


def test_what_does_not_fit_is_cut_and_reported():
    b = Batch([2, 3, 1], [20, 30, 16], 4, 2, 64, prefix=[40])
    want = b.check()
    run = lambda **kw: b.layer.run(b.q, **dict(b.meta, **kw))
    for kw in (dict(kv_len=i32([20, 1000, 16])), dict(kv_len=i32([20, 30, -5])), dict(prefix_len=i32([49])), dict(prefix_len=i32([-1])), dict(q_start=i32([0, 2, 1, 6])),
               dict(q_start=i32([0, 2, 5, 100])), dict(q_start=i32([-3, 2, 5, 6])), dict(prefix_start=i32([2, 1])), dict(prefix_start=i32([0, 9]))):
        run(**kw)
        assert b.layer.status() == -4, kw
        assert b.layer.status() == 0
    bad = b.meta["page_table"].clone()
    for page in (-1, 1 << 20, b.k_cache.shape[0], -2**31, 2**31 - 1):
        bad[1, 0] = page
        got = run(page_table=bad)
        assert b.layer.status() == -6
        assert torch.equal(got[:2], want[:2]) and torch.equal(got[5:], want[5:]) and torch.isfinite(got.float()).all()
    got = run(prefix_pages=torch.full_like(b.meta["prefix_pages"], -1))
    assert b.layer.status() == -6 and torch.isfinite(got.float()).all()
    assert torch.equal(run(), want) and b.layer.status() == 0


def test_calls_beyond_the_plan_are_refused():
    b = Batch([1, 1], [3, 4], 4, 2, 64, prefix=[20])
    more = torch.zeros(3, 4, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(cep.CepError) as e:
        b.layer.run(more, **b.meta)
    assert e.value.code == -4
    with pytest.raises(cep.CepError) as e:
        b.layer.run(b.q, i32([0, 1, 2, 2]), i32([3, 4, 0]), i32([[0]] * 3))
    assert e.value.code == -4
    with pytest.raises(cep.CepError):                                # rows that do not start on 16 bytes
        b.layer.run(rand((2, 4, 68), 1)[:, :, :64], **b.meta)
    with pytest.raises(cep.CepError):
        b.layer.run(rand((2 * 256 + 1,), 1)[1:].view(2, 4, 64), **b.meta)
    b.check()


def test_a_plan_is_not_made_inside_a_capture():
    kv = torch.zeros(2, 16, 1, 64, dtype=torch.bfloat16, device="cuda")
    g, y = torch.cuda.CUDAGraph(), torch.zeros(8, device="cuda")
    with torch.cuda.graph(g):
        with pytest.raises(cep.CepError, match="captured"):
            cep.PrefixAttention(kv, kv, 1, 1, 1)
        y += 1                                                       # the capture goes on
    g.replay()
    torch.cuda.synchronize()
    assert (y == 1).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("which", [0, 1])
@pytest.mark.parametrize("e4m3", [False, True])
def test_values_that_are_not_finite_reach_those_who_see_them(which, bad, e4m3):
    if e4m3 and bad == bad:
        pytest.skip("the type has no infinity")
    b = Batch([1, 1, 1, 1, 40], [90, 300, 20, 140, 150], 8, 2, 64, prefix=[200, 33], start=[0, 2, 5], e4m3=e4m3)
    want = b.check()
    cache = (b.k_cache, b.v_cache)[which]
    raw = cache.view(torch.uint8) if e4m3 else cache
    value = 0x7f if e4m3 else bad

    def others(place, sees, head, column=None):
        page, at = place
        keep = raw[page, at, head].clone()
        raw[page, at, head, 3] = value
        got = b.layer.run(b.q, **b.meta)
        raw[page, at, head] = keep
        heads = torch.zeros(8, dtype=torch.bool, device="cuda")
        heads[4 * head:4 * head + 4] = True
        touched = torch.zeros(b.T, dtype=torch.bool, device="cuda")
        touched[sees] = True
        touched = touched[:, None] & heads
        assert torch.equal(got[~touched], want[~touched])
        if which == 1:                                               # a value: its column, in every row whose weight for it is not 0
            assert not torch.isfinite(got[touched][:, 3].float()).all()
            assert torch.equal(got[touched][:, 4:], want[touched][:, 4:])
        elif bad != bad:
            assert torch.isnan(got[touched].float()).all()
        else:                                                        # a key: q . k is infinite or the row is as if it were not there
            f = got[touched].float()
            assert (torch.isnan(f).all(dim=1) | torch.isfinite(f).all(dim=1)).all()
    others((b.own[1][17], 5), [1], 1)                                # one sequence's own key
    others((b.ahead[0][3], 2), [0, 1], 0)                            # a shared key: its group
    others((b.ahead[1][0], 0), list(range(2, 44)), 1)
    # the first key of a prompt's chunk: all its tokens see it
    others((b.own[4][0], 1), list(range(4, 44)), 0)
    # a place behind the last key: nobody (Batch has NaN there already)
    assert torch.equal(b.layer.run(b.q, **b.meta), want) and b.layer.status() == 0


def test_queries_that_are_not_finite_stay_alone():
    for e4m3 in (False, True):
        b = Batch([1, 1, 3, 40], [90, 300, 20, 150], 8, 2, 64, prefix=[200], e4m3=e4m3)
        want = b.check()
        q = b.q.clone()
        q[1, 3, 5], q[4, 0, 0], q[20, 7, 63] = float("nan"), float("inf"), -float("inf")
        got = b.layer.run(q, **b.meta)
        bad = torch.zeros(b.T, 8, dtype=torch.bool, device="cuda")
        bad[1, 3] = bad[4, 0] = bad[20, 7] = True
        assert torch.equal(got[~bad], want[~bad])
        assert torch.isnan(got[1, 3].float()).all()


def test_queries_of_any_size():
    # fp16 operands of an e4m3 cache's kernel: rows far above and below fp16's range
    for scale in (1e-30, 1e-6, 1e4, 1e20):
        b = Batch([1, 2, 30], [50, 20, 40], 4, 2, 64, prefix=[100], e4m3=True, q_std=1.0)
        b.q.mul_(scale)
        layer = cep.PrefixAttention(b.k_cache, b.v_cache, 4, b.T, 3, 1, *b.scales, scale=0.125 / scale)
        got = layer.run(b.q, **b.meta)
        o, _, near, _, _ = b.want(scale=0.125 / scale)
        assert ((got.double() - o).abs() <= near).all(), scale


def test_far_places_of_a_large_cache():
    # pages 2^31 elements apart: offsets pass 32 bits
    far = 1 << 31
    store = torch.zeros(2 * far + 4096, dtype=torch.bfloat16, device="cuda")
    k = store.as_strided((3, 16, 1, 64), (far, 64, 64, 1))
    v = store.as_strided((3, 16, 1, 64), (far, 64, 64, 1), 2048)
    new = rand((48, 2, 64), 1)
    slots = torch.arange(48, device="cuda")
    cep.attn_append(new[:, :1], new[:, 1:], torch.zeros(48, dtype=torch.int32, device="cuda"), slots, torch.ones(32, device="cuda"), k, v)
    assert torch.equal(torch.cat([k[i] for i in range(3)]), new[:, :1]) and torch.equal(torch.cat([v[i] for i in range(3)]), new[:, 1:])
    layer = cep.PrefixAttention(k, v, 1, 4, 1)
    q = rand((1, 1, 64), 2)
    got = layer.run(q, i32([0, 1]), i32([48]), i32([[0, 1, 2]]))
    p = torch.softmax(q[0].double() @ new[:, 0].double().t() / 8, dim=1)
    want, A = p @ new[:, 1].double(), p @ new[:, 1].double().abs()
    assert ((got[0].double() - want).abs() <= 2.0 ** -8 * (A + want.abs()) * 1.01).all()
    del store


def test_outputs_and_inputs_with_strides():
    b = Batch([1, 30, 300, 2], [50, 30, 400, 2], 6, 2, 80, prefix=[200])
    want = b.check()
    wide = torch.full((b.T, 7, 96), 9.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((b.T, 11), 9.0, device="cuda")
    b.layer.run(b.q, out=wide[:, :6, :80], lse=lse[:, :6], **b.meta)
    assert torch.equal(wide[:, :6, :80], want) and (wide[:, 6:] == 9).all() and (wide[:, :, 80:] == 9).all() and (lse[:, 6:] == 9).all()
    table = torch.zeros(4, 100, dtype=torch.int32, device="cuda") - 3
    n = b.meta["page_table"].shape[1]
    table[:, :n] = b.meta["page_table"]
    q = torch.stack([b.q] * 3, dim=1)                                # tokens three apart
    assert torch.equal(b.layer.run(q[:, 1], **dict(b.meta, page_table=table[:, :n])), want)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("page", [16, 128])
def test_long_and_short_requests_side_by_side(page, e4m3):
    """Items of one tile between items of many: the warpgroups' turns, the ring's places and the items' queue in every order."""
    for seed in range(6):
        g = torch.Generator().manual_seed(seed)
        q_len = [[1, 1, 2, 40, 1, 300][int(i)] for i in torch.randint(0, 6, (24,), generator=g)]
        kv_len = [n + [0, 3, 130, 1500][int(i)] for n, i in zip(q_len, torch.randint(0, 4, (24,), generator=g))]
        Batch(q_len, kv_len, 8, 2, 128, page=page, prefix=[257], e4m3=e4m3).check(causal=bool(seed & 1))
