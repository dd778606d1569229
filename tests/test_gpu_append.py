"""attn_append against the formula in 64 bits.

A rotated value is a c - b s (or a s + b c) in fp32: cosine and sine are off by at most 2^-22 (the angle's fraction, rounded to
fp32, below half a turn: 2^-24 of pi, and 2 units in the last place of sincospif), products and sum by 2^-24 each of their size;
so |error| <= 2^-21 (|a| + |b|) before the one rounding, 2^-8 of the value to bf16, 2^-4 to e4m3 (2^-10 below its normal range)."""
import pytest
import torch

import paper_2609_33252_b200 as cep

pytestmark = pytest.mark.gpu


def rand(shape, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


def rotated(x, positions, inv_freq, interleaved):
    """The formula, and |a| + |b| of each value's pair (0 where it is copied)."""
    R = 2 * inv_freq.numel()
    y, size = x.double(), torch.zeros(x.shape, dtype=torch.float64, device=x.device)
    i = torch.arange(R // 2, device=x.device)
    first, second = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
    angle = positions.double()[:, None, None] * inv_freq.double()
    a, b = x[..., first].double(), x[..., second].double()
    y[..., first], y[..., second] = a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()
    size[..., first] = size[..., second] = a.abs() + b.abs()
    return y, size


def case(T, heads, kv_heads, dim, rotary, interleaved=False, e4m3=False, page=16, pages=None, wide=0, seed=1, far=200000, layout="page", in_place=False):
    qkv = rand((T, heads + 2 * kv_heads, dim + wide), seed)[..., :dim]
    q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:]
    g = torch.Generator().manual_seed(seed)
    pages = pages or -(-T // page) + 3
    slots = torch.randperm(pages * page, generator=g)[:T]
    slots[torch.rand(T, generator=g) < 0.1] = -1
    positions = torch.randint(0, far, (T,), generator=g, dtype=torch.int32).cuda()
    slots = slots.cuda()
    inv_freq = (10000.0 ** (-torch.arange(0, rotary, 2, dtype=torch.float64) / max(rotary, 1))).float().cuda()
    caches, scales = [], [None, None]
    for i in range(2):
        c = rand((pages, page, kv_heads, dim + wide), seed + 5 + i)
        if e4m3:
            c = c.to(torch.float8_e4m3fn)
            scales[i] = 0.003 + 0.02 * torch.rand(kv_heads, device="cuda")
        if layout == "head":
            c = c.view(torch.uint8 if e4m3 else c.dtype).transpose(1, 2).contiguous().transpose(1, 2).view(c.dtype) if not wide else c
        caches.append(c[..., :dim])
    before = [c.clone() for c in caches]
    source = q.clone()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = cep.attn_append(k, v, positions, slots, inv_freq, *caches, q=q if heads else None, q_out=q if in_place else None, interleaved=interleaved,
                          k_scale=scales[0], v_scale=scales[1], status=status)
    if heads:
        want, size = rotated(source, positions, inv_freq, interleaved)
        assert ((got.double() - want).abs() <= 2.0 ** -8 * want.abs() + 1.01 * 2.0 ** -21 * size).all()
        if not in_place:
            assert torch.equal(q, source)
    for cache, old, scale, (want, size) in zip(caches, before, scales, (rotated(k, positions, inv_freq, interleaved), (v.double(), 0 * v.double()))):
        flat = lambda c: c.float().reshape(-1, kv_heads, dim).double()
        untouched = torch.ones(pages * page, dtype=torch.bool, device="cuda")
        untouched[slots[slots >= 0]] = False
        assert torch.equal(flat(cache)[untouched], flat(old)[untouched])
        new, want, size = flat(cache)[slots[slots >= 0]], want[slots >= 0], size[slots >= 0]
        if scale is None:
            assert ((new - want).abs() <= 2.0 ** -8 * want.abs() + 1.01 * 2.0 ** -21 * size).all()
        else:
            s = scale.double()[:, None]
            want, size = (want / s).clamp(-448, 448), size / s
            assert ((new - want).abs() <= torch.clamp(2.0 ** -4 * want.abs(), min=2.0 ** -10) + 1.01 * 2.0 ** -21 * size + 2.0 ** -24 * want.abs()).all()
    assert int(status) == 0
    return got


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,rotary", [(64, 64), (128, 128), (80, 32), (128, 64), (96, 96), (72, 64), (2, 2), (6, 4), (66, 32), (40, 24), (16, 0), (1024, 1024)])
def test_dims(dim, rotary, interleaved):
    case(37, 3, 2, dim, rotary, interleaved)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("T", [1, 2, 61, 295, 296, 297, 1531, 9000])
def test_tokens(T, e4m3):
    case(T, 7, 1, 128, 128, e4m3=e4m3, page=64)
    case(T, 2, 2, 32, 16, interleaved=True, e4m3=e4m3, page=1)


@pytest.mark.parametrize("layout,wide", [("head", 0), ("page", 8), ("page", 3), ("page", 16)])
@pytest.mark.parametrize("e4m3", [False, True])
def test_strides(layout, wide, e4m3):
    case(50, 4, 2, 64, 64, e4m3=e4m3, wide=wide, layout=layout)
    case(50, 0, 2, 64, 48, e4m3=e4m3, wide=wide, layout=layout, interleaved=True)


@pytest.mark.parametrize("T", [1, 300])
def test_in_place(T):
    case(T, 5, 1, 128, 64, in_place=True)
    case(T, 5, 1, 64, 64, in_place=True, interleaved=True, wide=1)


def test_far_positions():
    case(64, 2, 1, 128, 128, far=2**31 - 1)
    k = rand((4, 1, 64), 1)
    cache = torch.zeros(1, 4, 1, 64, dtype=torch.bfloat16, device="cuda")
    positions = torch.tensor([-5, -2**31, 2**31 - 1, 0], dtype=torch.int32, device="cuda")
    inv_freq = torch.rand(32, device="cuda")
    cep.attn_append(k, k, positions, torch.arange(4, device="cuda"), inv_freq, cache, cache.clone())
    want, size = rotated(k, positions, inv_freq, False)
    assert ((cache[0].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -20 * size).all()     # (2^31 turns: the fraction's fp64 error, 2^-20 of a turn at most)


def test_slots_outside_are_reported_and_skipped():
    k, cache = rand((5, 2, 64), 1), torch.zeros(3, 4, 2, 64, dtype=torch.bfloat16, device="cuda")
    v_cache, status = cache.clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
    slots = torch.tensor([0, 12, -2, 1 << 40, 11], device="cuda")
    args = (k, k, torch.zeros(5, dtype=torch.int32, device="cuda"), slots, torch.ones(32, device="cuda"), cache, v_cache)
    cep.attn_append(*args, status=status)
    assert int(status) == 1
    cep.attn_append(*args)
    assert torch.equal(cache.view(12, 2, 64)[[0, 11]], k[[0, 4]]) and int((v_cache != 0).any(dim=3).any(dim=2).sum()) == 2


def test_values_that_are_not_finite_stay_with_their_pair():
    k = rand((3, 1, 64), 1)
    k[1, 0, 5], k[1, 0, 6] = float("nan"), float("inf")
    for dtype in (torch.bfloat16, torch.float8_e4m3fn):
        cache = torch.zeros(1, 4, 1, 64, device="cuda").to(dtype)
        cep.attn_append(k, k, torch.zeros(3, dtype=torch.int32, device="cuda"), torch.arange(3, device="cuda"), torch.ones(32, device="cuda"), cache, cache.clone())
        bad = ~torch.isfinite(cache.float()[0, :3, 0])
        assert bad[1, [5, 37]].all() and not bad[0].any() and not bad[2].any() and int(bad[1].sum()) <= 4
