"""What moe_norm refuses, through the C ABI: every check precedes the first CUDA call, so this runs without a GPU.
(Addresses are made up; nothing dereferences them.)"""
import ctypes

import pytest

import paper_2609_33252_b200 as cep

P = 1 << 20


def call(desc=None, x=P, residual=None, weight=None, residual_out=None, y=P, codes=None, scales=None, **kw):
    d = dict(n_tokens=1, hidden=64, dtype=cep.CEP_BF16, x_elem=0, residual_elem=0, weight_elem=0, x_stride=64, residual_stride=64,
             residual_out_stride=64, y_stride=64, eps=1e-6)
    d.update(kw)
    return cep.lib().moe_norm(ctypes.byref(cep.NormDesc(**d)), x, residual, weight, residual_out, y, codes, scales, None)


def test_a_valid_call_without_rows_does_nothing():
    assert call(n_tokens=0) == 0
    assert call(n_tokens=0, x=None, y=None) == 0                   # an empty tensor may have no address


@pytest.mark.parametrize("code,kw", [
    (-1, dict(x=None)), (-1, dict(dtype=7)), (-1, dict(x_elem=2)), (-1, dict(residual_elem=-1)), (-1, dict(n_tokens=-1)),
    (-1, dict(hidden=0)), (-9, dict(hidden=32769, x_stride=40000, y_stride=40000)), (-1, dict(eps=-1.0)),
    (-1, dict(eps=float("nan"))), (-1, dict(eps=float("inf"))), (-1, dict(codes=P)), (-1, dict(scales=P)),
    (-1, dict(dtype=cep.CEP_MXFP4_E4M3)), (-1, dict(dtype=cep.CEP_MXFP4_E4M3, codes=P)), (-1, dict(residual_out=P)),
    (-1, dict(y=None)), (-1, dict(x_stride=63)), (-1, dict(y_stride=0)), (-1, dict(residual=P, residual_stride=8)),
    (-1, dict(residual=P, residual_out=P, residual_out_stride=8)), (-1, dict(x=P + 1)), (-1, dict(weight=P + 2, weight_elem=1)),
    (-1, dict(dtype=cep.CEP_FP8_E4M3_BLOCK128, codes=P, scales=P + 2))])
def test_refusals(code, kw):
    assert call(**kw) == code
    assert "norm" in cep.cep_last_error()


def test_a_missing_description_is_refused():
    assert cep.lib().moe_norm(None, P, None, None, None, P, None, None, None) == -1
