"""ctypes binding of include/cascade_ffn.h: same names, argument marshalling only.

Every step of the path runs inside the library's CUDA kernels.  torch is used for
device memory and streams.  If the library cannot be loaded the import of a symbol
raises: there is no CPU or PyTorch fallback.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import List, Optional, Sequence

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libcascade_ffn.so")

CEP_BF16, CEP_FP8_E4M3_BLOCK128, CEP_MXFP4_E4M3 = 0, 1, 2
DTYPE_OF = {"bf16": CEP_BF16, "fp8": CEP_FP8_E4M3_BLOCK128, "mxfp4": CEP_MXFP4_E4M3}   # workload dtype names
CEP_ELEM_BF16, CEP_ELEM_FP32, CEP_ELEM_E4M3 = 0, 1, 2
CEP_MODE_SYNC, CEP_MODE_ASYNC, CEP_MODE_STREAMFFN = 0, 1, 2
CEP_GEMM_TCGEN05, CEP_GEMM_SIMT, CEP_GEMM_TCGEN05_1CTA = 0, 1, 2
STATUS_NAMES = {0: "CEP_OK", -1: "CEP_ERR_ARG", -2: "CEP_ERR_STATE", -3: "CEP_ERR_WORKSPACE",
                -4: "CEP_ERR_CAPACITY", -5: "CEP_ERR_INCOMPLETE", -6: "CEP_ERR_BAD_ROUTING",
                -7: "CEP_ERR_DEVICE_TIMEOUT", -8: "CEP_ERR_CUDA", -9: "CEP_ERR_UNSUPPORTED"}

EXPORTS = ["moe_plan_workspace_bytes", "moe_packed_weight_bytes", "moe_plan", "moe_load_weights",
           "ffn_begin", "ffn_submit_chunk", "ffn_flush", "combine", "ffn_status", "ffn_num_invocations",
           "ffn_query", "ffn_debug_export", "cep_kernel_launches", "moe_plan_destroy", "cep_last_error",
           "cep_debug_decode_tile", "cep_debug_schedule", "layout_indices_noalloc", "cep_debug_wait_timeout", "ffn_set_addend", "moe_route", "cep_debug_check_guards", "ffn_wait_invocation",
           "ffn_set_active_streams", "cep_calibrate", "ffn_query_call", "cep_calibrate_routed", "moe_norm",
           "lora_plan_workspace_bytes", "lora_bank_bytes", "lora_plan", "lora_load_adapter", "lora_project", "lora_status",
           "lora_plan_destroy", "attn_append", "attn_plan_workspace_bytes", "attn_plan", "attn_prefix", "attn_status", "attn_plan_destroy",
           "cep_debug_attn_schedule"]


class CepConfig(ctypes.Structure):
    _fields_ = [("hidden", ctypes.c_int32), ("inter", ctypes.c_int32),
                ("n_experts_global", ctypes.c_int32), ("n_experts_local", ctypes.c_int32),
                ("top_k", ctypes.c_int32), ("max_tokens", ctypes.c_int32), ("max_chunks", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("mode", ctypes.c_int32), ("n_streams", ctypes.c_int32),
                ("threshold_pairs", ctypes.c_int64), ("gemm_impl", ctypes.c_int32),
                ("debug_checks", ctypes.c_int32), ("profile_kernels", ctypes.c_int32),
                ("defer_while_busy", ctypes.c_int32), ("gather_a", ctypes.c_int32)]


class NormDesc(ctypes.Structure):
    _fields_ = [("n_tokens", ctypes.c_int32), ("hidden", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("x_elem", ctypes.c_int32), ("residual_elem", ctypes.c_int32), ("weight_elem", ctypes.c_int32),
                ("x_stride", ctypes.c_int64), ("residual_stride", ctypes.c_int64),
                ("residual_out_stride", ctypes.c_int64), ("y_stride", ctypes.c_int64), ("eps", ctypes.c_float)]


class LoraConfig(ctypes.Structure):
    _fields_ = [("in_features", ctypes.c_int32), ("out_features", ctypes.c_int32), ("max_tokens", ctypes.c_int32),
                ("max_adapters", ctypes.c_int32), ("max_rank", ctypes.c_int32), ("out_elem", ctypes.c_int32)]


class AppendDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_tokens", "n_heads", "n_kv_heads", "head_dim", "rotary_dim", "interleaved", "cache_elem", "page_size")] + \
               [(n, ctypes.c_int64) for n in ("n_pages", "q_token_stride", "q_head_stride", "q_out_token_stride", "q_out_head_stride", "k_token_stride",
                                              "k_head_stride", "v_token_stride", "v_head_stride")] + \
               [("k_cache_stride", ctypes.c_int64 * 3), ("v_cache_stride", ctypes.c_int64 * 3)]


class AttnConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_heads", "n_kv_heads", "head_dim", "page_size", "n_pages", "cache_elem", "max_tokens", "max_seqs",
                                              "max_prefixes")] + \
               [("scale", ctypes.c_float), ("k_stride", ctypes.c_int64 * 3), ("v_stride", ctypes.c_int64 * 3)]


class AttnBatch(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_tokens", "n_seqs", "n_prefixes", "causal", "table_width", "prefix_width")] + \
               [(n, ctypes.c_int64) for n in ("table_stride", "prefix_stride", "q_token_stride", "q_head_stride", "out_token_stride", "out_head_stride",
                                              "lse_token_stride")]


class InvocationInfo(ctypes.Structure):
    _fields_ = [("n_chunks", ctypes.c_int32), ("first_chunk_pos", ctypes.c_int32),
                ("stream_index", ctypes.c_int32), ("n_tokens", ctypes.c_int32),
                ("pairs_bound", ctypes.c_int64), ("elapsed_ms", ctypes.c_float),
                ("layout_ms", ctypes.c_float), ("gemm1_ms", ctypes.c_float), ("gemm2_ms", ctypes.c_float),
                ("combine_ms", ctypes.c_float), ("index_ms", ctypes.c_float), ("scatter_ms", ctypes.c_float)]


class ProfilePoint(ctypes.Structure):
    _fields_ = [("rows_per_expert", ctypes.c_int32), ("n_tokens", ctypes.c_int32), ("expert_tokens", ctypes.c_int64),
                ("ffn_ms", ctypes.c_float), ("layer_ms", ctypes.c_float), ("tflops", ctypes.c_float),
                ("eta", ctypes.c_float)]


class Calibration(ctypes.Structure):
    _fields_ = [("rho", ctypes.c_float), ("peak_tflops", ctypes.c_float), ("theta_pairs", ctypes.c_int64),
                ("theta_rows_per_expert", ctypes.c_int32), ("best_streams", ctypes.c_int32),
                ("probe_invocations", ctypes.c_int32), ("stream_ms", ctypes.c_float * 16)]


class CepError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__("%s: %s" % (STATUS_NAMES.get(code, str(code)), msg))
        self.code = code


_lib = None


def load_library(build_if_missing: bool = True):
    """dlopen the C-ABI library (building it with nvcc first if it is absent or stale)."""
    global _lib
    if _lib is not None:
        return _lib
    if build_if_missing:
        from .build import build
        try:
            build()
        except Exception:
            if not os.path.exists(LIB_PATH):
                raise
    if not os.path.exists(LIB_PATH):
        raise RuntimeError("libcascade_ffn.so is missing: build it with `python -m paper_2609_33252_b200.build`")
    L = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    cfgp = ctypes.POINTER(CepConfig)
    sig = {
        "moe_plan_workspace_bytes": (ctypes.c_int, [cfgp, ctypes.POINTER(sz)]),
        "moe_packed_weight_bytes": (ctypes.c_int, [cfgp, ctypes.POINTER(sz)]),
        "moe_plan": (ctypes.c_int, [cfgp, vp, sz, ctypes.POINTER(vp)]),
        "moe_load_weights": (ctypes.c_int, [vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]),
        "ffn_begin": (ctypes.c_int, [vp, vp, i32, i32]),
        "ffn_submit_chunk": (ctypes.c_int, [vp, i32, i32, i32, vp, vp, vp, vp, i64, vp]),
        "ffn_flush": (ctypes.c_int, [vp]),
        "combine": (ctypes.c_int, [vp, vp]),
        "ffn_status": (ctypes.c_int, [vp]),
        "ffn_num_invocations": (ctypes.c_int, [vp]),
        "ffn_wait_invocation": (ctypes.c_int, [vp, i32, vp]),
        "ffn_query": (ctypes.c_int, [vp, i32, ctypes.POINTER(InvocationInfo)]),
        "ffn_query_call": (ctypes.c_int, [vp, i32, i32, ctypes.POINTER(InvocationInfo)]),
        "ffn_debug_export": (ctypes.c_int, [vp, i32, vp, vp, vp, vp, vp]),
        "cep_kernel_launches": (i64, [vp]),
        "moe_plan_destroy": (ctypes.c_int, [vp]),
        "cep_last_error": (ctypes.c_char_p, [vp]),
        "cep_debug_decode_tile": (ctypes.c_int, [vp, i32, i32, i32, i32] + [ctypes.POINTER(i32)] * 3),
        "cep_debug_schedule": (ctypes.c_int, [vp, i32, i32, i64, vp]),
        "cep_debug_wait_timeout": (ctypes.c_int, [vp, i32, vp]),
        "ffn_set_addend": (ctypes.c_int, [vp, vp]),
        "cep_debug_check_guards": (ctypes.c_int, [vp, ctypes.POINTER(i32)]),
        "moe_route": (ctypes.c_int, [vp, i32, i32, i32, vp, vp, vp]),
        "ffn_set_active_streams": (ctypes.c_int, [vp, i32]),
        "cep_calibrate": (ctypes.c_int, [vp, ctypes.c_float, vp, i32, i32, vp, vp, vp, vp, vp,
                                         ctypes.POINTER(ProfilePoint), ctypes.POINTER(Calibration)]),
        "cep_calibrate_routed": (ctypes.c_int, [vp, ctypes.c_float, vp, i32, i32, vp, vp, vp, vp, vp,
                                                ctypes.POINTER(ProfilePoint), ctypes.POINTER(Calibration)]),
        "moe_norm": (ctypes.c_int, [vp, vp, vp, vp, vp, vp, vp, vp, vp]),
        "lora_plan_workspace_bytes": (ctypes.c_int, [vp, ctypes.POINTER(sz)]),
        "lora_bank_bytes": (ctypes.c_int, [vp, ctypes.POINTER(sz)]),
        "lora_plan": (ctypes.c_int, [vp, vp, i64, vp, sz, vp, sz, vp, ctypes.POINTER(vp)]),
        "lora_load_adapter": (ctypes.c_int, [vp, i32, i32, ctypes.c_float, vp, i64, vp, i64, vp]),
        "lora_project": (ctypes.c_int, [vp, vp, i64, i32, vp, vp, i64, vp]),
        "lora_status": (ctypes.c_int, [vp]),
        "lora_plan_destroy": (ctypes.c_int, [vp]),
        "attn_append": (ctypes.c_int, [vp] * 14),
        "attn_plan_workspace_bytes": (ctypes.c_int, [vp, ctypes.POINTER(sz)]),
        "attn_plan": (ctypes.c_int, [vp, vp, vp, vp, vp, vp, sz, vp, ctypes.POINTER(vp)]),
        "attn_prefix": (ctypes.c_int, [vp] * 12),
        "attn_status": (ctypes.c_int, [vp]),
        "attn_plan_destroy": (ctypes.c_int, [vp]),
        "cep_debug_attn_schedule": (ctypes.c_int, [vp, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, i32, vp]),
        "layout_indices_noalloc": (ctypes.c_int, [vp, i32, i32, i32, i32, vp, vp, vp, vp, vp, i32, vp, vp]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(L, name)
        fn.restype, fn.argtypes = res, args
    _lib = L
    return L


def lib():
    return load_library()


def _check(rc: int, plan=None, allow: Sequence[int] = ()):
    if rc != 0 and rc not in allow:
        msg = lib().cep_last_error(plan)
        raise CepError(rc, msg.decode() if msg else "")
    return rc


def _dptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream_handle(stream) -> int:
    import torch
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _stream_object(stream):
    import torch
    return stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(int(stream))


def _record(stream, *tensors):
    """Tells torch's allocator that `stream` uses the tensors (those that are given): the caller may drop them at once."""
    s = _stream_object(stream)
    for t in tensors:
        if t is not None:
            t.record_stream(s)


def _allocating_on(stream):
    """Context in which torch allocates for use on `stream` (memory from another stream's pool may still be in use there)."""
    import torch
    return torch.cuda.stream(None if stream is None else _stream_object(stream))


def _current_stream() -> int:
    """Handle of the current stream of the current device, without a Python stream object around it."""
    return _torch()._C._cuda_getCurrentRawStream(_torch()._C._cuda_getDevice())


_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


# ---------------------------------------------------------------- same-named wrappers
def moe_plan_workspace_bytes(cfg: CepConfig) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().moe_plan_workspace_bytes(ctypes.byref(cfg), ctypes.byref(n)))
    return n.value


def moe_packed_weight_bytes(cfg: CepConfig) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().moe_packed_weight_bytes(ctypes.byref(cfg), ctypes.byref(n)))
    return n.value


def moe_plan(cfg: CepConfig, workspace) -> int:
    """workspace: torch uint8 CUDA tensor.  Returns the plan handle."""
    h = ctypes.c_void_p()
    _check(lib().moe_plan(ctypes.byref(cfg), workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                          ctypes.byref(h)))
    return h.value


def moe_load_weights(plan, w_gate, w_up, w_down, s_gate, s_up, s_down, packed, stream=None):
    _check(lib().moe_load_weights(plan, _dptr(w_gate), _dptr(w_up), _dptr(w_down), _dptr(s_gate), _dptr(s_up),
                                  _dptr(s_down), packed.data_ptr(), packed.numel() * packed.element_size(),
                                  _stream_handle(stream)), plan)


def ffn_begin(plan, out, n_tokens_total: int, n_chunks_expected: int):
    _check(lib().ffn_begin(plan, out.data_ptr(), n_tokens_total, n_chunks_expected), plan)


def ffn_set_addend(plan, addend):
    _check(lib().ffn_set_addend(plan, _dptr(addend)), plan)


def moe_route(logits, top_k: int, topk_ids, topk_weights, stream=None):
    n_tokens, n_experts_global = logits.shape
    _check(lib().moe_route(logits.data_ptr(), n_tokens, n_experts_global, top_k, topk_ids.data_ptr(),
                           topk_weights.data_ptr(), _stream_handle(stream)))


_NORM_DESC = struct.Struct("6i4qf4x")                  # NormDesc, packed in one call
_ELEM = {}                                             # torch dtype -> CEP_ELEM_*, filled with the first call
_NORM_DTYPES = []                                      # of weight, codes, ue8m0 scales, fp32 scales


def _norm_rows(t, name, shape, dev):
    """(element type, row stride) of a [T,H] tensor on device `dev` with contiguous rows; raises for what the call cannot take."""
    elem = _ELEM.get(t.dtype)
    if elem is None:
        raise CepError(-1, "%s has dtype %s" % (name, t.dtype))
    if t.shape != shape or t.get_device() != dev:
        raise CepError(-1, "%s must be a %s CUDA tensor on the current device" % (name, list(shape)))
    stride, inner = t.stride()
    if inner != 1 and shape[1] > 1:
        raise CepError(-1, "the rows of %s must be contiguous" % name)
    return elem, stride


def _norm_dense(t, name, shape, dtypes, dev):
    if t.dtype not in dtypes or t.shape != shape or t.get_device() != dev or not t.is_contiguous():
        raise CepError(-1, "%s must be a contiguous CUDA tensor of %s %s on the current device" % (name, list(shape), dtypes[0]))
    return t.data_ptr()


def moe_norm(x, weight=None, eps: float = 1e-6, residual=None, residual_out=None, y=None, codes=None, scales=None,
             dtype: int = CEP_BF16, stream=None):
    """Residual addition, root-mean-square norm and the expert layer's activation format in one pass (see the header).

    x [T,H] bf16 or fp32; residual / residual_out [T,H] bf16 or fp32 (one type); weight [H] bf16 or fp32; y bf16 [T,H];
    codes float8_e4m3fn [T,H] and scales fp32 [T,ceil(H/128)] (CEP_FP8_E4M3_BLOCK128) or uint8 [T,ceil(H/32)]
    (CEP_MXFP4_E4M3).  Rows of x, residual, residual_out and y may be strided.  Tensors are recorded on a `stream` that is given."""
    torch = _torch_module or _torch()
    if not _ELEM:                                      # (another thread's first call may come at any point: the marker last)
        dtypes = ((torch.bfloat16, torch.float32), (torch.float8_e4m3fn, torch.uint8), (torch.uint8,), (torch.float32,))
        elem = {torch.bfloat16: CEP_ELEM_BF16, torch.float32: CEP_ELEM_FP32}
        _NORM_DTYPES[:] = dtypes
        _ELEM.update(elem)
    shape = x.shape
    if len(shape) != 2 or not x.is_cuda:
        raise CepError(-1, "x must be a [T, H] CUDA tensor")
    T, H = shape
    dev = torch._C._cuda_getDevice()
    xe, xs = _norm_rows(x, "x", shape, dev)
    re = we = rs = os_ = ys = 0
    rp = op = yp = wp = cp = sp = None
    if residual is not None:
        re, rs = _norm_rows(residual, "residual", shape, dev)
        rp = residual.data_ptr()
    if residual_out is not None:
        oe, os_ = _norm_rows(residual_out, "residual_out", shape, dev)
        if rp is not None and oe != re:
            raise CepError(-1, "residual_out has dtype %s" % residual_out.dtype)
        op = residual_out.data_ptr()
    if y is not None:
        ye, ys = _norm_rows(y, "y", shape, dev)
        if ye != CEP_ELEM_BF16:
            raise CepError(-1, "y has dtype %s" % y.dtype)
        yp = y.data_ptr()
    if T <= 1:                                         # the stride of a single row means nothing
        xs = rs = os_ = ys = H
    if weight is not None:
        wp = _norm_dense(weight, "weight", (H,), _NORM_DTYPES[0], dev)
        we = _ELEM[weight.dtype]
    if codes is not None:
        cp = _norm_dense(codes, "codes", shape, _NORM_DTYPES[1], dev)
    if scales is not None:
        if dtype == CEP_MXFP4_E4M3:
            sp = _norm_dense(scales, "scales", (T, (H + 31) // 32), _NORM_DTYPES[2], dev)
        else:
            sp = _norm_dense(scales, "scales", (T, (H + 127) // 128), _NORM_DTYPES[3], dev)
    rc = (_lib or lib()).moe_norm(_NORM_DESC.pack(T, H, dtype, xe, re, we, xs, rs, os_, ys, eps), x.data_ptr(), rp, wp, op, yp, cp, sp,
                                  torch._C._cuda_getCurrentRawStream(dev) if stream is None else _stream_handle(stream))
    if rc:
        _check(rc)
    if stream is not None:
        _record(stream, x, weight, residual, residual_out, y, codes, scales)


def lora_plan_workspace_bytes(cfg: LoraConfig) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().lora_plan_workspace_bytes(ctypes.byref(cfg), ctypes.byref(n)))
    return n.value


def lora_bank_bytes(cfg: LoraConfig) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().lora_bank_bytes(ctypes.byref(cfg), ctypes.byref(n)))
    return n.value


def lora_plan(cfg: LoraConfig, weight, bank, workspace, stream=None) -> int:
    """weight: bf16 [N,K] CUDA tensor; bank, workspace: torch uint8 CUDA tensors.  Returns the plan handle."""
    h = ctypes.c_void_p()
    _check(lib().lora_plan(ctypes.byref(cfg), weight.data_ptr(), weight.stride(0) if weight.shape[0] > 1 else weight.shape[1], _dptr(bank), 0 if bank is None else bank.numel(),
                           workspace.data_ptr(), workspace.numel(), _stream_handle(stream), ctypes.byref(h)))
    return h.value


def lora_load_adapter(plan, slot: int, rank: int, scale: float, down, up, stream=None):
    stride = lambda t: 0 if t is None else t.stride(0) if t.shape[0] > 1 else t.shape[1]     # (that of a single row means nothing)
    _check(lib().lora_load_adapter(plan, slot, rank, scale, _dptr(down), stride(down), _dptr(up), stride(up), _stream_handle(stream)))


def lora_project(plan, x, adapter_ids, y, stream=None):
    T = x.shape[0]                                        # (the stride of a single row means nothing)
    rc = (_lib or lib()).lora_project(plan, x.data_ptr(), x.stride(0) if T > 1 else x.shape[1], T,
                                      None if adapter_ids is None else adapter_ids.data_ptr(), y.data_ptr(),
                                      y.stride(0) if T > 1 else y.shape[1], _current_stream() if stream is None else _stream_handle(stream))
    if rc:
        _check(rc)


def lora_status(plan) -> int:
    return lib().lora_status(plan)


def lora_plan_destroy(plan):
    _check(lib().lora_plan_destroy(plan))


_APPEND_DESC = struct.Struct("8i15q")                  # AppendDesc, packed in one call
_ATTN_BATCH = struct.Struct("6i7q")                    # AttnBatch


def _heads(t, name, shape, dtype, dev):
    """(token stride, head stride) of a [T, heads, D] tensor on device `dev` with contiguous heads."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev:
        raise CepError(-1, "%s must be a %s CUDA tensor %s on the current device" % (name, dtype, list(shape)))
    st = t.stride()
    if st[2] != 1:
        raise CepError(-1, "the heads of %s must be contiguous" % name)
    return st


def _vector(t, name, n, dtype, dev):
    if t.dtype is not dtype or t.shape != (n,) or t.get_device() != dev or not t.is_contiguous():
        raise CepError(-1, "%s must be a contiguous CUDA tensor [%d] of %s on the current device" % (name, n, dtype))
    return t.data_ptr()


def _page_rows(t, name, n, dtype, dev):
    """(width, row stride) of an int32 [n, width] page table."""
    if t.dtype is not dtype or t.dim() != 2 or t.shape[0] != n or t.get_device() != dev or (t.shape[1] > 1 and t.stride(1) != 1):
        raise CepError(-1, "%s must be an int32 CUDA tensor [%d, width] on the current device with contiguous rows" % (name, n))
    return t.shape[1], t.stride(0)


def attn_append(k, v, positions, slots, inv_freq, k_cache, v_cache, q=None, q_out=None, interleaved: bool = False, k_scale=None, v_scale=None,
                status=None, stream=None):
    """Rotates the heads of q and k by their tokens' positions and writes k and v to their slots of a paged cache (see the header).

    k, v bf16 [T,Hkv,D]; q bf16 [T,Hq,D] or None; positions int32 [T]; slots int64 [T] (-1: not written); inv_freq fp32 [R/2];
    k_cache, v_cache bf16 or float8_e4m3fn [pages, page_size, Hkv, D], any strides with contiguous heads; k_scale, v_scale fp32 [Hkv]
    (e4m3); status int32 [1], set to 1 where a slot lies outside the cache.  Returns the rotated q in q_out (allocated if not given;
    may be q, but not overlap k, v or a part of q).  Tensors are recorded on a `stream` that is given."""
    torch = _torch_module or _torch()
    dev = torch._C._cuda_getDevice()
    bf16 = torch.bfloat16
    if k.dim() != 3 or k_cache.dim() != 4:
        raise CepError(-1, "k must be [T, heads, D], k_cache [pages, page_size, heads, D]")
    T, Hk, D = k.shape
    ks, vs = _heads(k, "k", k.shape, bf16, dev), _heads(v, "v", k.shape, bf16, dev)
    Hq, qp, op, qs, os_ = 0, None, None, (0, 0), (0, 0)
    if q is not None:
        Hq = q.shape[1] if q.dim() == 3 else -1
        qs = _heads(q, "q", (T, Hq, D), bf16, dev)
        if q_out is None:
            if stream is None:
                q_out = torch.empty((T, Hq, D), dtype=bf16, device=q.device)
            else:
                with _allocating_on(stream):
                    q_out = torch.empty((T, Hq, D), dtype=bf16, device=q.device)
        os_ = qs if q_out is q else _heads(q_out, "q_out", (T, Hq, D), bf16, dev)
        qp, op = q.data_ptr(), q_out.data_ptr()
    elif q_out is not None:
        raise CepError(-1, "q_out without q")
    shape = k_cache.shape
    e4m3 = k_cache.dtype is torch.float8_e4m3fn
    if not e4m3 and k_cache.dtype is not bf16:
        raise CepError(-1, "k_cache has dtype %s" % k_cache.dtype)
    kcs, vcs = k_cache.stride(), v_cache.stride()
    if (v_cache.dtype is not k_cache.dtype or v_cache.shape != shape or shape[2] != Hk or shape[3] != D or k_cache.get_device() != dev or
            v_cache.get_device() != dev or kcs[3] != 1 or vcs[3] != 1):
        raise CepError(-1, "k_cache and v_cache must be CUDA tensors [pages, page_size, %d, %d] of one type on the current device, with contiguous heads" % (Hk, D))
    pp, sp = _vector(positions, "positions", T, torch.int32, dev), _vector(slots, "slots", T, torch.int64, dev)
    fp = _vector(inv_freq, "inv_freq", inv_freq.numel(), torch.float32, dev)
    kp = None if k_scale is None else _vector(k_scale, "k_scale", Hk, torch.float32, dev)
    vp = None if v_scale is None else _vector(v_scale, "v_scale", Hk, torch.float32, dev)
    tp = None if status is None else _vector(status, "status", 1, torch.int32, dev)
    rc = (_lib or lib()).attn_append(
        _APPEND_DESC.pack(T, Hq, Hk, D, 2 * inv_freq.shape[0], 1 if interleaved else 0, CEP_ELEM_E4M3 if e4m3 else CEP_ELEM_BF16, shape[1], shape[0], qs[0], qs[1],
                          os_[0], os_[1], ks[0], ks[1], vs[0], vs[1], kcs[0], kcs[1], kcs[2], vcs[0], vcs[1], vcs[2]),
        qp, k.data_ptr(), v.data_ptr(), pp, sp, fp, op, k_cache.data_ptr(), v_cache.data_ptr(), kp, vp, tp,
        torch._C._cuda_getCurrentRawStream(dev) if stream is None else _stream_handle(stream))
    if rc:
        _check(rc)
    if stream is not None:
        _record(stream, q, k, v, positions, slots, inv_freq, q_out, k_cache, v_cache, k_scale, v_scale, status)
    return q_out


def attn_plan_workspace_bytes(cfg: AttnConfig) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().attn_plan_workspace_bytes(ctypes.byref(cfg), ctypes.byref(n)))
    return n.value


def attn_plan(cfg: AttnConfig, k_cache, v_cache, k_scale, v_scale, workspace, stream=None) -> int:
    """All tensors CUDA; workspace torch uint8.  Returns the plan handle."""
    h = ctypes.c_void_p()
    _check(lib().attn_plan(ctypes.byref(cfg), k_cache.data_ptr(), v_cache.data_ptr(), _dptr(k_scale), _dptr(v_scale), workspace.data_ptr(), workspace.numel(),
                           _stream_handle(stream), ctypes.byref(h)))
    return h.value


def attn_prefix(plan, batch: bytes, q, q_start, kv_len, page_table, prefix_start, prefix_len, prefix_pages, out, lse, stream=None):
    """batch: an AttnBatch or its bytes; the others CUDA tensors (see the header)."""
    rc = (_lib or lib()).attn_prefix(plan, batch if isinstance(batch, bytes) else ctypes.addressof(batch), q.data_ptr(), q_start.data_ptr(), kv_len.data_ptr(),
                                     page_table.data_ptr(), _dptr(prefix_start), _dptr(prefix_len), _dptr(prefix_pages), out.data_ptr(), _dptr(lse),
                                     _current_stream() if stream is None else _stream_handle(stream))
    if rc:
        _check(rc)


def attn_status(plan) -> int:
    return lib().attn_status(plan)


def attn_plan_destroy(plan):
    _check(lib().attn_plan_destroy(plan))


def cep_debug_attn_schedule(cfg: AttnConfig, q_start, kv_len, prefix_start=None, prefix_len=(), causal: bool = True, n_ctas: int = 148):
    """(parts as dicts, partial rows that the workspace has) of a batch with these host lengths (see the header)."""
    import numpy as np
    ints = lambda v: np.ascontiguousarray(v, dtype=np.int32)
    qs, kl, pl = ints(q_start), ints(kv_len), ints(prefix_len)
    ps = None if prefix_start is None else ints(prefix_start)
    ptr = lambda a: None if a is None else a.ctypes.data
    rows = ctypes.c_int64()
    call = lambda parts, n: lib().cep_debug_attn_schedule(ctypes.byref(cfg), int(qs[-1]), len(kl), len(pl), int(causal), n_ctas, ptr(qs), ptr(kl), ptr(ps), ptr(pl),
                                                          parts.ctypes.data, n, ctypes.addressof(rows))
    n = call(np.zeros((1, 13), np.int64), 0)
    if n < 0:
        _check(n)
    parts = np.zeros((max(n, 1), 13), np.int64)
    call(parts, n)
    names = ("cta", "kind", "seq", "group", "head", "token", "tokens", "first", "end", "steps", "row", "cost", "results")
    return [dict(zip(names, map(int, r))) for r in parts[:n]], rows.value


def ffn_submit_chunk(plan, chunk_id: int, token_offset: int, n_tokens: int, tokens, token_scales, topk_ids,
                     topk_weights, n_local_pairs: int = -1, stream=None):
    _check(lib().ffn_submit_chunk(plan, chunk_id, token_offset, n_tokens, _dptr(tokens), _dptr(token_scales),
                                  _dptr(topk_ids), _dptr(topk_weights), n_local_pairs, _stream_handle(stream)),
           plan)


def ffn_flush(plan, allow_incomplete: bool = False) -> int:
    return _check(lib().ffn_flush(plan), plan, allow=(-5,) if allow_incomplete else ())


def combine(plan, stream=None, allow_incomplete: bool = False) -> int:
    return _check(lib().combine(plan, _stream_handle(stream)), plan, allow=(-5,) if allow_incomplete else ())


def ffn_status(plan) -> int:
    return lib().ffn_status(plan)


def ffn_wait_invocation(plan, inv: int, stream=None):
    _check(lib().ffn_wait_invocation(plan, inv, _stream_handle(stream)), plan)


def ffn_num_invocations(plan) -> int:
    return lib().ffn_num_invocations(plan)


def ffn_query(plan, inv: int) -> InvocationInfo:
    info = InvocationInfo()
    _check(lib().ffn_query(plan, inv, ctypes.byref(info)), plan)
    return info


def ffn_query_call(plan, calls_back: int, inv: int) -> InvocationInfo:
    info = InvocationInfo()
    _check(lib().ffn_query_call(plan, calls_back, inv, ctypes.byref(info)), plan)
    return info


def ffn_debug_export(plan, inv: int, n_experts_local: int, n_pairs: int):
    """Returns dict of numpy int32 arrays: counts, offsets, padded_offsets, row_of_pair, pair_of_row."""
    import numpy as np
    E = n_experts_local
    counts = np.zeros(E, np.int32)
    offsets = np.zeros(E + 1, np.int32)
    padded = np.zeros(E + 1, np.int32)
    rop = np.full(max(n_pairs, 1), -1, np.int32)
    p = lambda a: a.ctypes.data_as(ctypes.c_void_p)
    _check(lib().ffn_debug_export(plan, inv, p(counts), p(offsets), p(padded), p(rop), None), plan)
    por = np.full(max(int(padded[E]), 1), -1, np.int32)
    _check(lib().ffn_debug_export(plan, inv, None, None, None, None, p(por)), plan)
    return dict(counts=counts, offsets=offsets, padded_offsets=padded, row_of_pair=rop[:n_pairs],
                pair_of_row=por[:int(padded[E])])


def ffn_set_active_streams(plan, n: int):
    _check(lib().ffn_set_active_streams(plan, n), plan)


def cep_calibrate(plan, rho: float, rows_per_expert: Sequence[int], reps: int, tokens, token_scales, ids, weights, out):
    """Returns (list of profile-point dicts, calibration dict); the tensors are device scratch (see the header)."""
    n = len(rows_per_expert)
    rows = (ctypes.c_int32 * n)(*[int(r) for r in rows_per_expert])
    pts = (ProfilePoint * n)()
    cal = Calibration()
    _check(lib().cep_calibrate(plan, float(rho), ctypes.cast(rows, ctypes.c_void_p), n, reps, _dptr(tokens),
                               _dptr(token_scales), _dptr(ids), _dptr(weights), _dptr(out), pts, ctypes.byref(cal)), plan)
    points = [{f: getattr(p, f) for f, _ in ProfilePoint._fields_} for p in pts]
    result = {f: getattr(cal, f) for f, _ in Calibration._fields_ if f != "stream_ms"}
    result["stream_ms"] = [v for v in cal.stream_ms if v >= 0]
    return points, result


def cep_calibrate_routed(plan, rho: float, n_tokens: Sequence[int], reps: int, tokens, token_scales, ids, weights, out):
    """Calibration on the caller's routing: profile on growing prefixes of one real batch (see the header)."""
    n = len(n_tokens)
    nt = (ctypes.c_int32 * n)(*[int(v) for v in n_tokens])
    pts = (ProfilePoint * n)()
    cal = Calibration()
    _check(lib().cep_calibrate_routed(plan, float(rho), ctypes.cast(nt, ctypes.c_void_p), n, reps, _dptr(tokens),
                                      _dptr(token_scales), _dptr(ids), _dptr(weights), _dptr(out), pts, ctypes.byref(cal)), plan)
    points = [{f: getattr(p, f) for f, _ in ProfilePoint._fields_} for p in pts]
    result = {f: getattr(cal, f) for f, _ in Calibration._fields_ if f != "stream_ms"}
    return points, result


def cep_kernel_launches(plan) -> int:
    return lib().cep_kernel_launches(plan)


def moe_plan_destroy(plan):
    _check(lib().moe_plan_destroy(plan))


def cep_last_error(plan=None) -> str:
    m = lib().cep_last_error(plan)
    return m.decode() if m else ""


def cep_debug_check_guards(plan) -> int:
    """Number of damaged guard gaps of a plan made with debug_checks (0 = no overrun)."""
    n = ctypes.c_int32(-1)
    _check(lib().cep_debug_check_guards(plan, ctypes.byref(n)), plan)
    return n.value


def cep_debug_wait_timeout(plan, limit_ms: int, stream=None):
    _check(lib().cep_debug_wait_timeout(plan, limit_ms, _stream_handle(stream)), plan)


def cep_debug_decode_tile(tile_prefix, n_blocks_n: int, tile: int, n_group: int = 0):
    import numpy as np
    tp = np.ascontiguousarray(tile_prefix, dtype=np.int32)
    e, m, n = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int32()
    rc = lib().cep_debug_decode_tile(tp.ctypes.data_as(ctypes.c_void_p), tp.shape[0] - 1, n_blocks_n,
                                     n_group if n_group > 0 else n_blocks_n, tile,
                                     ctypes.byref(e), ctypes.byref(m), ctypes.byref(n))
    return None if rc else (e.value, m.value, n.value)


def cep_debug_schedule(pairs: Sequence[int], mode: int, theta: int) -> List[int]:
    import numpy as np
    pr = np.ascontiguousarray(pairs, dtype=np.int64)
    out = np.zeros(max(len(pr), 1), np.int32)
    n = lib().cep_debug_schedule(pr.ctypes.data_as(ctypes.c_void_p), len(pr), mode, theta,
                                 out.ctypes.data_as(ctypes.c_void_p))
    if n < 0:
        raise CepError(n, "cep_debug_schedule")
    return out[:len(pr)].tolist()


def layout_indices_noalloc(topk_ids, n_experts_local: int, n_experts_global: int, counts, offsets,
                           padded_offsets, row_of_pair, pair_of_row, status=None, stream=None) -> int:
    """Index half of the layout transform with no workspace (all arguments are CUDA tensors the
    caller allocated beforehand).  Returns the library's status code instead of raising, so a caller
    can test the size limit."""
    n_tokens, top_k = topk_ids.shape
    return lib().layout_indices_noalloc(topk_ids.data_ptr(), n_tokens, top_k, n_experts_local, n_experts_global,
                                        counts.data_ptr(), offsets.data_ptr(), padded_offsets.data_ptr(),
                                        row_of_pair.data_ptr(), pair_of_row.data_ptr(), pair_of_row.numel(),
                                        _dptr(status), _stream_handle(stream))


# ---------------------------------------------------------------- convenience owner of the buffers
class MoELayer:
    """Owns the torch-allocated workspace and packed weights of one plan.

    Plumbing only: allocation and pointer passing.  ``run`` submits the chunks of one
    layer call in the given order on the given streams and joins on ``stream``.
    """

    def __init__(self, hidden, inter, n_experts_global, n_experts_local, top_k, max_tokens, max_chunks,
                 dtype=CEP_BF16, mode=CEP_MODE_STREAMFFN, n_streams=2, threshold_pairs=0,
                 gemm_impl=CEP_GEMM_TCGEN05, debug_checks=0, profile_kernels=0, defer_while_busy=0, gather_a=0,
                 device="cuda"):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("the streamFFN library needs a CUDA device; there is no CPU path")
        self.cfg = CepConfig(hidden, inter, n_experts_global, n_experts_local, top_k, max_tokens, max_chunks,
                             dtype, mode, n_streams, threshold_pairs, gemm_impl, debug_checks, profile_kernels,
                             defer_while_busy, gather_a)
        self.device = torch.device(device)
        self.workspace = torch.empty(moe_plan_workspace_bytes(self.cfg), dtype=torch.uint8, device=self.device)
        self.packed = torch.empty(moe_packed_weight_bytes(self.cfg), dtype=torch.uint8, device=self.device)
        self.plan = moe_plan(self.cfg, self.workspace)

    def load_weights(self, w_gate, w_up, w_down, s_gate=None, s_up=None, s_down=None, stream=None):
        moe_load_weights(self.plan, w_gate, w_up, w_down, s_gate, s_up, s_down, self.packed, stream)

    def run(self, out, chunks, order=None, streams=None, stream=None, n_local_pairs=None, addend=None):
        """chunks: list of (token_offset, x, x_scale, ids, w).  Returns the number of invocations."""
        n_tok = sum(c[1].shape[0] for c in chunks)
        ffn_begin(self.plan, out, n_tok, len(chunks))
        if addend is not None:
            ffn_set_addend(self.plan, addend)
        order = list(range(len(chunks))) if order is None else order
        for c in order:
            off, x, xs, ids, w = chunks[c]
            ffn_submit_chunk(self.plan, c, off, x.shape[0], x, xs, ids, w,
                             -1 if n_local_pairs is None else n_local_pairs[c],
                             None if streams is None else streams[c])
        ffn_flush(self.plan)
        combine(self.plan, stream)
        return ffn_num_invocations(self.plan)

    def close(self):
        if getattr(self, "plan", None):
            moe_plan_destroy(self.plan)
            self.plan = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class LoRAProjection:
    """A projection shared by all requests with one low-rank adapter per request beside it: owns the torch-allocated
    workspace and adapter bank of one plan, and keeps the weight alive.

    weight bf16 [N,K] (the layout of a linear layer's weight), used in place.  ``load_adapter`` fills a slot; ``run``
    takes the slot of every token.  The weight's device has to be the current one, here and in every call.  max_adapters = 0
    gives the plain projection (with out_elem=CEP_ELEM_FP32 the
    router's logits).
    """

    def __init__(self, weight, max_tokens, max_adapters=0, max_rank=0, out_elem=CEP_ELEM_BF16, stream=None):
        import torch
        if not weight.is_cuda or weight.dtype != torch.bfloat16 or weight.dim() != 2 or weight.stride(1) != 1:
            raise CepError(-1, "weight must be a bf16 CUDA tensor [out, in] with contiguous rows")
        dev = torch.cuda.current_device()                # the plan is made for this one
        if weight.get_device() != dev:
            raise CepError(-1, "the weight is on device %d, device %d is current" % (weight.get_device(), dev))
        if getattr(stream, "device", None) is not None and stream.device.index != dev:
            raise CepError(-1, "the stream is of device %s, device %d is current" % (stream.device.index, dev))
        self.weight = weight
        self.out_dtype = torch.float32 if out_elem == CEP_ELEM_FP32 else torch.bfloat16
        self.out_features, self.in_features = weight.shape
        self.cfg = LoraConfig(self.in_features, self.out_features, max_tokens, max_adapters, max_rank, out_elem)
        self.device_index = dev
        nb = lora_bank_bytes(self.cfg)
        with _allocating_on(stream):                     # (lora_plan clears both on `stream`)
            self.workspace = torch.empty(lora_plan_workspace_bytes(self.cfg), dtype=torch.uint8, device=weight.device)
            self.bank = torch.empty(nb, dtype=torch.uint8, device=weight.device) if nb else None
        self.plan = lora_plan(self.cfg, weight, self.bank, self.workspace, stream)

    def load_adapter(self, slot, down, up, scale=1.0, stream=None):
        """down = A [rank, in], up = B [out, rank], bf16, rows may be strided; replaces what the slot held."""
        import torch
        rank = down.shape[0]
        for t, name, shape in ((down, "down", (rank, self.cfg.in_features)), (up, "up", (self.cfg.out_features, rank))):
            if t.dtype != torch.bfloat16 or t.get_device() != self.device_index or tuple(t.shape) != shape or (shape[1] > 1 and t.stride(1) != 1):
                raise CepError(-1, "%s must be a bf16 tensor [%d, %d] on the weight's device with contiguous rows" % ((name,) + shape))
        lora_load_adapter(self.plan, slot, rank, scale, down, up, stream)
        if stream is not None:
            _record(stream, down, up)

    def drop_adapter(self, slot, stream=None):
        """Empties a slot: its id then names no adapter."""
        lora_load_adapter(self.plan, slot, 0, 0.0, None, None, stream)

    def run(self, x, adapter_ids=None, out=None, stream=None):
        """x bf16 [T,in], adapter_ids int32 [T] (-1: none) or None; returns out [T,out] (allocated if not given).  Tensors are
        recorded on a `stream` that is given."""
        torch = _torch()
        dev = self.device_index
        if x.dim() != 2 or x.dtype is not torch.bfloat16 or x.get_device() != dev or x.shape[1] != self.in_features or x.stride(1) != 1:
            raise CepError(-1, "x must be a bf16 tensor [T, %d] on the weight's device with contiguous rows" % self.in_features)
        T, N = x.shape[0], self.out_features
        if adapter_ids is not None and (adapter_ids.dtype is not torch.int32 or adapter_ids.shape != (T,) or
                                        not adapter_ids.is_contiguous() or adapter_ids.get_device() != dev):
            raise CepError(-1, "adapter_ids must be a contiguous int32 tensor [%d] on the weight's device" % T)
        if out is None:
            if stream is None:
                out = torch.empty((T, N), dtype=self.out_dtype, device=x.device)
            else:
                with _allocating_on(stream):
                    out = torch.empty((T, N), dtype=self.out_dtype, device=x.device)
        elif out.dtype is not self.out_dtype or out.shape != (T, N) or out.get_device() != dev or (N > 1 and out.stride(1) != 1):
            raise CepError(-1, "out must be a %s tensor [%d, %d] on the weight's device with contiguous rows" % (self.out_dtype, T, N))
        lora_project(self.plan, x, adapter_ids, out, stream)
        if stream is not None:
            _record(stream, x, adapter_ids, out)
        return out

    def status(self) -> int:
        return lora_status(self.plan)

    def close(self):
        if getattr(self, "plan", None):
            lora_plan_destroy(self.plan)
            self.plan = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class PrefixAttention:
    """Attention of batches whose sequences share prefixes, over a paged cache of keys and values that it keeps alive: owns the
    torch-allocated workspace of one plan.

    k_cache, v_cache bf16 or float8_e4m3fn [pages, page_size, Hkv, D] (any strides with contiguous heads), used in place; k_scale,
    v_scale fp32 [Hkv] or None (all ones): a key is its stored value times its head's scale; scale: of the scores, 1/sqrt(D) by
    default.  The caches' device has to be the current one, here and in every call.
    """

    def __init__(self, k_cache, v_cache, n_heads, max_tokens, max_seqs, max_prefixes=1, k_scale=None, v_scale=None, scale=None, stream=None):
        import torch
        dev = torch.cuda.current_device()                # the plan is made for this one
        shape = k_cache.shape
        elem = {torch.bfloat16: CEP_ELEM_BF16, torch.float8_e4m3fn: CEP_ELEM_E4M3}.get(k_cache.dtype)
        if (len(shape) != 4 or elem is None or not k_cache.is_cuda or v_cache.shape != shape or v_cache.dtype != k_cache.dtype or k_cache.stride(3) != 1 or
                v_cache.stride(3) != 1):
            raise CepError(-1, "k_cache and v_cache must be bf16 or float8_e4m3fn CUDA tensors [pages, page_size, heads, D] of one shape with contiguous heads")
        for t, name in ((k_cache, "k_cache"), (v_cache, "v_cache"), (k_scale, "k_scale"), (v_scale, "v_scale")):
            if t is not None and t.get_device() != dev:
                raise CepError(-1, "%s is on device %d, device %d is current" % (name, t.get_device(), dev))
        if getattr(stream, "device", None) is not None and stream.device.index != dev:
            raise CepError(-1, "the stream is of device %s, device %d is current" % (stream.device.index, dev))
        pages, page_size, Hk, D = shape
        for t, name in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            if t is not None:
                _vector(t, name, Hk, torch.float32, dev)
        self.k_cache, self.v_cache, self.k_scale, self.v_scale = k_cache, v_cache, k_scale, v_scale
        self.n_heads, self.head_dim, self.device_index = n_heads, D, dev
        self.cfg = AttnConfig(n_heads, Hk, D, page_size, pages, elem, max_tokens, max_seqs, max_prefixes, D ** -0.5 if scale is None else scale,
                              (ctypes.c_int64 * 3)(*k_cache.stride()[:3]), (ctypes.c_int64 * 3)(*v_cache.stride()[:3]))
        nb = attn_plan_workspace_bytes(self.cfg)
        with _allocating_on(stream):                     # (attn_plan clears the status word on `stream`)
            self.workspace = torch.empty(nb, dtype=torch.uint8, device=k_cache.device)
        self.plan = attn_plan(self.cfg, k_cache, v_cache, k_scale, v_scale, self.workspace, stream)

    def run(self, q, q_start, kv_len, page_table, prefix_start=None, prefix_len=None, prefix_pages=None, causal=True, out=None, lse=None, stream=None):
        """q bf16 [T,Hq,D] (heads may be strided), q_start int32 [B+1], kv_len int32 [B], page_table int32 [B,W]; prefixes: prefix_len
        int32 [G], prefix_pages int32 [G,Wp], prefix_start int32 [G+1] first sequence of each group (None: one group of all).  Returns out
        [T,Hq,D] (allocated if not given; it may not overlap q); lse fp32 [T,Hq] is filled if given.  Tensors are recorded on a `stream` that is given."""
        torch = _torch()
        dev, i32 = self.device_index, torch.int32
        T = q.shape[0]
        shape = (T, self.n_heads, self.head_dim)
        qs = _heads(q, "q", shape, torch.bfloat16, dev)
        B = kv_len.shape[0] if kv_len.dim() == 1 else -1
        _vector(q_start, "q_start", B + 1, i32, dev)
        _vector(kv_len, "kv_len", B, i32, dev)
        G = W2 = s2 = 0
        if prefix_len is not None:
            G = prefix_len.numel()
            _vector(prefix_len, "prefix_len", G, i32, dev)
            if prefix_pages is None:
                raise CepError(-1, "prefix_len without prefix_pages")
            W2, s2 = _page_rows(prefix_pages, "prefix_pages", G, i32, dev)
            if prefix_start is not None:
                _vector(prefix_start, "prefix_start", G + 1, i32, dev)
            elif G > 1:
                raise CepError(-1, "%d prefixes need prefix_start" % G)
        elif prefix_start is not None or prefix_pages is not None:
            raise CepError(-1, "prefix_start or prefix_pages without prefix_len")
        W, s1 = _page_rows(page_table, "page_table", B, i32, dev)
        if out is None:
            if stream is None:
                out = torch.empty(shape, dtype=torch.bfloat16, device=q.device)
            else:
                with _allocating_on(stream):
                    out = torch.empty(shape, dtype=torch.bfloat16, device=q.device)
        os_ = _heads(out, "out", shape, torch.bfloat16, dev)
        ls = 0
        if lse is not None:
            if lse.dtype is not torch.float32 or lse.shape != shape[:2] or lse.get_device() != dev or (self.n_heads > 1 and lse.stride(1) != 1):
                raise CepError(-1, "lse must be a float32 tensor %s on the caches' device with contiguous rows" % list(shape[:2]))
            ls = lse.stride(0)
        attn_prefix(self.plan, _ATTN_BATCH.pack(T, B, G, 1 if causal else 0, W, W2, s1, s2, qs[0], qs[1], os_[0], os_[1], ls), q, q_start, kv_len, page_table,
                    prefix_start, prefix_len, prefix_pages, out, lse, stream)
        if stream is not None:
            _record(stream, q, q_start, kv_len, page_table, prefix_start, prefix_len, prefix_pages, out, lse)
        return out

    def status(self) -> int:
        return attn_status(self.plan)

    def close(self):
        if getattr(self, "plan", None):
            attn_plan_destroy(self.plan)
            self.plan = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
