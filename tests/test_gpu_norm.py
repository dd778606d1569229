"""moe_norm against the formula in 64 bits: h = x + residual, y = h / sqrt(mean(h^2) + eps) * weight, y also as e4m3 codes
with fp32 1x128 or ue8m0 1x32 scales.

Tolerances, from the arithmetic: fp32 throughout, so before rounding a value is off by the rounding of the sum of squares
(every term positive, at most a few hundred roundings per thread and six in each of the two shuffles: below 64 * 2^-24
relative for any width here), of the mean, the reciprocal root (2 ulp) and three products: REL32 = 1e-5 is above all of it.
  bf16 output      half a unit in the last place, 2^-8 relative, + REL32
  fp8 scale        REL32 relative
  ue8m0 scale      amax <= 448 s and amax > 224 s, both up to REL32
  codes            half a step of e4m3: 2^-4 |v| for normal values, 2^-10 for subnormal ones (v in units of the scale), + REL32
"""
import numpy as np
import pytest
import torch

import paper_2609_33252_b200 as cep

pytestmark = pytest.mark.gpu
REL32 = 1e-5
FMT = {"bf16": cep.CEP_BF16, "fp8": cep.CEP_FP8_E4M3_BLOCK128, "mx": cep.CEP_MXFP4_E4M3}
BLOCK = {"fp8": 128, "mx": 32}


def draw(T, H, seed, dtype=torch.bfloat16, pad=0, std=1.0, offset=0):
    g = torch.Generator().manual_seed(seed)
    wide = (torch.randn(T, H + pad, generator=g) * std)
    flat = torch.zeros(wide.numel() + offset, dtype=dtype)
    flat[offset:] = wide.to(dtype).flatten()
    return flat.cuda()[offset:].view(T, H + pad)[:, :H]


def run(x, weight=None, eps=1e-6, residual=None, fmt="bf16", y=True, inplace=False, stream=None):
    T, H = x.shape
    out = {}
    if residual is not None:
        out["residual"] = residual if inplace else torch.full_like(residual, float("nan"), memory_format=torch.contiguous_format)
    if y:
        out["y"] = torch.full((T, H), float("nan"), dtype=torch.bfloat16, device="cuda")
    if fmt != "bf16":
        out["codes"] = torch.full((T, H), 0x55, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
        n = -(-H // BLOCK[fmt])
        out["scales"] = (torch.full((T, n), float("nan"), device="cuda") if fmt == "fp8" else
                         torch.full((T, n), 255, dtype=torch.uint8, device="cuda"))
    cep.moe_norm(x, weight, eps, residual=residual, residual_out=out.get("residual"), y=out.get("y"), codes=out.get("codes"),
                 scales=out.get("scales"), dtype=FMT[fmt], stream=stream)
    torch.cuda.synchronize()
    return out


def formula(x, weight, eps, residual):
    h = x.double().cpu()
    if residual is not None:
        h = h + residual.double().cpu()
    y = h / torch.sqrt((h * h).mean(dim=1, keepdim=True) + eps)
    return h, y if weight is None else y * weight.double().cpu()


def check(out, x, weight, eps, residual, fmt):
    h, y = formula(x, weight, eps, residual)
    if residual is not None:
        s = x.float() + residual.float()
        assert torch.equal(out["residual"].cpu(), s.to(residual.dtype).cpu())       # one fp32 addition, one rounding
    if "y" in out:
        got = out["y"].double().cpu()
        assert (torch.abs(got - y) <= (2 ** -8 + REL32) * y.abs() + 1e-38).all()
    if fmt == "bf16":
        return
    T, H = y.shape
    b = BLOCK[fmt]
    n = -(-H // b)
    yb = torch.zeros(T, n * b, dtype=torch.float64)
    yb[:, :H] = y
    yb = yb.view(T, n, b)
    amax = yb.abs().amax(dim=2)
    if fmt == "fp8":
        s = out["scales"].double().cpu()
        want = torch.where(amax == 0, torch.ones_like(amax), amax / 448)
        assert (torch.abs(s - want) <= REL32 * want).all()
    else:
        s = torch.exp2(out["scales"].double().cpu() - 127)
        live = amax > 0
        assert (amax <= 448 * s * (1 + REL32)).all() and (amax[live] > 224 * s[live] * (1 - REL32)).all()
        assert (out["scales"].cpu()[~live] == 127).all()
    c = torch.zeros(T, n * b, dtype=torch.float64)
    c[:, :H] = out["codes"].float().double().cpu()
    c = c.view(T, n, b)
    v = (yb / s[:, :, None]).clamp(-448, 448)
    half = torch.maximum(v.abs() * 2 ** -4, torch.full_like(v, 2.0 ** -10))
    assert (torch.abs(c - v) <= half + REL32 * v.abs()).all()


SHAPES = [(1, 7168, 0), (3, 512, 0), (5, 2120, 64), (129, 256, 8), (2, 8, 0), (7, 1, 0), (4, 31, 0), (6, 2047, 0), (3, 130, 3),
          (2, 4104, 0), (1, 32768, 0), (2, 32767, 0), (1100, 768, 0), (5, 5000, 0)]


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "mx"])
@pytest.mark.parametrize("T,H,pad", SHAPES)
def test_shapes_and_formats(T, H, pad, fmt):
    x = draw(T, H, 1, pad=pad)
    w = draw(1, H, 2)[0].contiguous()
    r = draw(T, H, 3, std=2.0)
    check(run(x, w, residual=r, fmt=fmt), x, w, 1e-6, r, fmt)


@pytest.mark.parametrize("xdt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rdt", [None, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("wdt", [None, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H", [1024, 77])
def test_every_combination_of_types(xdt, rdt, wdt, H):
    for k, fmt in enumerate(("bf16", "fp8", "mx")):
        x = draw(9, H, 10 + k, xdt, pad=16)
        r = None if rdt is None else draw(9, H, 20 + k, rdt, pad=24)
        w = None if wdt is None else draw(1, H, 30 + k, wdt)[0].contiguous()
        check(run(x, w, 1e-5, r, fmt), x, w, 1e-5, r, fmt)


@pytest.mark.parametrize("fmt", ["fp8", "mx"])
def test_wide_and_element_paths_agree(fmt):
    # the same rows at an address that rules out 16-byte loads: scales and codes may differ only where a rounding is near
    x, r, w = draw(37, 1160, 4), draw(37, 1160, 5), draw(1, 1160, 6)[0].contiguous()
    x1 = draw(37, 1160, 4, offset=1)
    assert x1.data_ptr() % 16 != 0 and torch.equal(x, x1)
    a, b = run(x, w, residual=r, fmt=fmt), run(x1, w, residual=r, fmt=fmt)
    check(b, x, w, 1e-6, r, fmt)
    assert torch.equal(a["residual"], b["residual"])
    assert (a["codes"].view(torch.uint8) != b["codes"].view(torch.uint8)).float().mean() < 1e-3


@pytest.mark.parametrize("H", [2048, 333])
def test_residual_updated_in_place_and_norm_in_place(H):
    x, r, w = draw(41, H, 7), draw(41, H, 8), draw(1, H, 9)[0].contiguous()
    want = run(x, w, residual=r.clone(), fmt="mx")
    r2 = r.clone()
    got = run(x, w, residual=r2, fmt="mx", inplace=True)
    for k in want:
        assert torch.equal(want[k].view(torch.uint8), got[k].view(torch.uint8)), k
    x2 = x.clone()
    cep.moe_norm(x2, w, 1e-6, residual=r, y=x2)
    torch.cuda.synchronize()
    assert torch.equal(x2, want["y"])


@pytest.mark.parametrize("H", [512, 515])
@pytest.mark.parametrize("fmt", ["bf16", "fp8", "mx"])
def test_special_rows(H, fmt):
    x = draw(6, H, 11).clone()
    x[0] = 0                       # nothing in the row
    x[1, 3] = float("nan")
    x[2, 5] = float("inf")
    x[3] = 1e-30                   # the sum of squares underflows: eps decides
    x[4, H // 2:] = 0              # whole blocks of zeros beside live ones
    out = run(x, None, 1e-6, fmt=fmt)
    y = out["y"].float().cpu()
    assert (y[0] == 0).all()
    assert torch.isnan(y[1]).all()
    assert torch.isnan(y[2, 5]) and (torch.cat([y[2, :5], y[2, 6:]]) == 0).all()
    check({k: v[3:] for k, v in out.items()}, x[3:], None, 1e-6, None, fmt)
    if fmt != "bf16":
        c = out["codes"].float().cpu()
        assert (c[0] == 0).all() and torch.isnan(c[1]).all() and torch.isnan(c[2, 5])
        assert (out["scales"][0].float() == (1.0 if fmt == "fp8" else 127.0)).all()
    # a row of zeros without eps is 0/0
    assert torch.isnan(run(x[:1], None, 0.0)["y"]).all()


def test_tiny_values_stay_in_range():
    # blocks whose scale is subnormal, or underflows to zero: codes and scales stay finite
    H = 256
    x = torch.ones(2, H)
    w = torch.full((H,), 2.0 ** -126)
    w[128:] = 2.0 ** -149
    for fmt in ("fp8", "mx"):
        out = run(x.cuda(), w.cuda(), 0.0, fmt=fmt)
        c, s = out["codes"].float().cpu(), out["scales"].cpu()
        assert torch.isfinite(c).all()
        if fmt == "fp8":
            assert torch.isfinite(s).all() and (s > 0).all()
            # the first block's scale is the subnormal nearest to 2^-126/448 (2^-149 steps), its codes that many steps
            v = c[:, :128].double() * s[:, :1].double()
            assert (torch.abs(v - 2.0 ** -126) <= 2.0 ** -126 * 2 ** -4 + 448 * 2.0 ** -150).all()
        else:
            assert (s[:, :4] == 0).all() and (c[:, :128] == 2.0).all()


def test_another_stream_and_repeatability():
    x, r, w = draw(2000, 2048, 12), draw(2000, 2048, 13), draw(1, 2048, 14)[0].contiguous()
    want = run(x, w, residual=r, fmt="fp8")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = run(x, w, residual=r, fmt="fp8", stream=s)
    for k in want:
        assert torch.equal(want[k].view(torch.uint8), got[k].view(torch.uint8)), k


def test_no_rows():
    x = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    cep.moe_norm(x, None, y=torch.empty_like(x))


def test_feeds_the_layer_formats_as_the_input_generator_does():
    # fed the generator's own fp32 rows without a norm's effect (weight that undoes it), the codes and scales are what
    # the plans already take: same block layout, same scale rule
    from paper_2609_33252_b200 import workloads as wl
    g = torch.Generator().manual_seed(5)
    x = torch.randn(64, 512, generator=g)
    x = x / torch.sqrt((x.double() ** 2).mean(dim=1, keepdim=True)).float()
    q8, s8 = wl.quantize_rows_1x128(x)
    out = run(x.cuda(), None, 0.0, fmt="fp8", y=False)
    assert torch.allclose(out["scales"].cpu(), s8, rtol=REL32, atol=0)
    assert (out["codes"].cpu().view(torch.uint8) != q8.view(torch.uint8)).float().mean() < 1e-3
    qm, sm = wl.quantize_mx(x, "e4m3", 1)
    out = run(x.cuda(), None, 0.0, fmt="mx", y=False)
    assert (out["scales"].cpu() != sm).float().mean() < 1e-3
    assert (out["codes"].cpu().view(torch.uint8) != qm.view(torch.uint8)).float().mean() < 2e-3


def test_python_refusals():
    x = draw(4, 64, 1)
    y = torch.empty(4, 64, dtype=torch.bfloat16, device="cuda")
    bad = [dict(x=x.half()), dict(x=x.t()), dict(x=x.cpu()), dict(y=y[:3]), dict(weight=torch.ones(63, device="cuda")),
           dict(dtype=cep.CEP_FP8_E4M3_BLOCK128), dict(residual_out=y), dict(eps=-1.0), dict(x=x[:1].expand(4, 64)),
           dict(residual=x, residual_out=torch.empty(4, 64, device="cuda")), dict(y=None),
           dict(dtype=cep.CEP_MXFP4_E4M3, codes=torch.empty(4, 64, dtype=torch.uint8, device="cuda"),
                scales=torch.empty(4, 2, dtype=torch.float32, device="cuda"))]
    for kw in bad:
        a = dict(x=x, weight=None, y=y)
        a.update(kw)
        with pytest.raises(cep.CepError):
            cep.moe_norm(a.pop("x"), a.pop("weight"), a.pop("eps", 1e-6), **a)
