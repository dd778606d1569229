// RMS norm in front of the expert layer: h = x + residual, y = h / sqrt(mean(h^2) + eps) * weight, and y written in
// the activation format a plan takes: e4m3 codes with one fp32 scale per 1x128 block, or with one ue8m0 scale per 1x32
// block, and / or bf16.  The residual stream (h) is written back in its own type.
//
// Every input is read once and every output written once: the row is kept in registers between the sum of squares and
// the scaling.  All arithmetic is fp32 from the loads on: h, the sum of squares, the normalised values and the block
// maxima; each output is rounded once, from the unrounded value.  The kernel is bound by memory.
#include <cuda_bf16.h>

#include <type_traits>

#include "cep_common.h"

namespace cep {
namespace {

constexpr int kMaxWarps = 32;

__device__ __forceinline__ uint32_t pack2_bf16(float lo, float hi) {
  __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack2_e4m3(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}

// Two fp32 values in one 64-bit register pair: one instruction adds, multiplies or accumulates both.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair(float lo, float hi) { f32x2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi)); return r; }
__device__ __forceinline__ float lo(f32x2 v) { float a, b; asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); return a; }
__device__ __forceinline__ float hi(f32x2 v) { float a, b; asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); return b; }
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) { f32x2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) { f32x2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) { f32x2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ float max_abs3(float a, float b, float c) { float r; asm("max.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c)); return r; }

// Eight consecutive elements as they are loaded: one 16-byte register quad of bf16, two of fp32; and as four pairs.
template <typename T> struct Vec8;
template <> struct Vec8<__nv_bfloat16> {
  uint4 a;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { a = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void get(f32x2 (&f)[4]) const {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = pair(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
  }
  static __device__ __forceinline__ void store(__nv_bfloat16* p, const f32x2 (&f)[4]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack2_bf16(lo(f[0]), hi(f[0])), pack2_bf16(lo(f[1]), hi(f[1])), pack2_bf16(lo(f[2]), hi(f[2])),
                                              pack2_bf16(lo(f[3]), hi(f[3])));
  }
};
template <> struct Vec8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) { a = reinterpret_cast<const float4*>(p)[0]; b = reinterpret_cast<const float4*>(p)[1]; }
  __device__ __forceinline__ void get(f32x2 (&f)[4]) const { f[0] = pair(a.x, a.y); f[1] = pair(a.z, a.w); f[2] = pair(b.x, b.y); f[3] = pair(b.z, b.w); }
  static __device__ __forceinline__ void store(float* p, const f32x2 (&f)[4]) {
    reinterpret_cast<float4*>(p)[0] = make_float4(lo(f[0]), hi(f[0]), lo(f[1]), hi(f[1]));
    reinterpret_cast<float4*>(p)[1] = make_float4(lo(f[2]), hi(f[2]), lo(f[3]), hi(f[3]));
  }
};
struct NoResidual {};

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// The block scale from the block's largest magnitude: the factor the values are multiplied with, and the stored scale.
// fp8: scale = amax/448, as a product with 1/448 (1 ulp); the factor is its reciprocal (1 ulp), so a value on a rounding edge
// may land on either side.  A scale so small that its reciprocal overflows (or that underflows to zero: 1 is stored) takes the
// reciprocal of the scale times 2^64 first.
struct Fp8Scale { float scale, factor; };
__device__ __forceinline__ Fp8Scale fp8_scale(float amax) {
  Fp8Scale r;
  r.scale = amax * (1.f / 448.f);
  if (r.scale == 0.f) r.scale = 1.f;
  r.factor = __fdividef(1.f, r.scale);
  return r;
}
__device__ __forceinline__ bool fp8_tiny(float scale) { return scale < 1.17549435e-38f; }
// ue8m0: code of the smallest power of two s with amax <= 448 s (448 = 1.75 * 2^8), from the exponent and fraction bits
__device__ __forceinline__ int mx_code(float amax) {
  const uint32_t u = __float_as_uint(amax);
  int c = (int)((u >> 23) & 0xff) - 8 + ((u & 0x7fffff) > 0x600000 ? 1 : 0);
  c = c < 0 ? 0 : c > 254 ? 254 : c;
  return amax == 0.f ? 127 : c;
}
__device__ __forceinline__ float mx_factor(int code) {       // 2^(127 - code); code 254 gives the subnormal 2^-127
  return code == 254 ? __uint_as_float(0x00400000u) : __uint_as_float((uint32_t)(254 - code) << 23);
}

__device__ __forceinline__ float block_sum(float v, float* part) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = blockDim.x >> 5;
  if (lane == 0) part[warp] = v;
  __syncthreads();
  v = lane < n ? part[lane] : 0.f;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

struct NormArgs {
  const void* x; const void* residual; const void* weight;
  void* residual_out; __nv_bfloat16* y; uint8_t* codes; void* scales;
  int64_t x_stride, residual_stride, residual_out_stride, y_stride;
  int hidden, weight_fp32, n_scales;
  float eps;
};

// One block per row, eight elements per thread and step, kVec steps.  Threads of a group of 16 (fp8) or 4 (mx)
// consecutive lanes hold one scale block, so the block maximum is a shuffle inside the group.  The weight is multiplied in
// before the row's sum is known (y = (h * weight) * inv), so that after it only the maximum and one product per output are
// left; arithmetic is on pairs.
template <typename XT, typename RT, int kFmt, int kVec>
__global__ void __launch_bounds__(1024)
norm_kernel(const NormArgs a) {
  __shared__ float part[kMaxWarps];
  pdl_enter();
  const size_t row = blockIdx.x;
  const int n_vec = a.hidden >> 3;
  constexpr bool kRes = !std::is_same<RT, NoResidual>::value;
  using RL = typename std::conditional<kRes, RT, float>::type;
  const XT* x = static_cast<const XT*>(a.x) + row * a.x_stride;
  const RL* res = static_cast<const RL*>(a.residual) + (kRes ? row * a.residual_stride : 0);
  Vec8<XT> xv[kVec];
  Vec8<RL> rv[kVec];
#pragma unroll
  for (int v = 0; v < kVec; ++v) {
    const int i = v * blockDim.x + threadIdx.x;
    if (i < n_vec) {
      xv[v].load(x + 8 * i);
      if (kRes) rv[v].load(res + 8 * i);
    }
  }
  f32x2 h[kVec][4];
  f32x2 ss = pair(0.f, 0.f);
#pragma unroll
  for (int v = 0; v < kVec; ++v) {
    const int i = v * blockDim.x + threadIdx.x;
    if (i < n_vec) {
      f32x2 w[4];
      if (a.weight) {
        if (a.weight_fp32) { Vec8<float> q; q.load(static_cast<const float*>(a.weight) + 8 * i); q.get(w); }
        else { Vec8<__nv_bfloat16> q; q.load(static_cast<const __nv_bfloat16*>(a.weight) + 8 * i); q.get(w); }
      }
      xv[v].get(h[v]);
      if (kRes) {
        f32x2 r[4];
        rv[v].get(r);
#pragma unroll
        for (int j = 0; j < 4; ++j) h[v][j] = add2(h[v][j], r[j]);
        if (a.residual_out) Vec8<RL>::store(static_cast<RL*>(a.residual_out) + row * a.residual_out_stride + 8 * i, h[v]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) ss = fma2(h[v][j], h[v][j], ss);
      if (a.weight) {
#pragma unroll
        for (int j = 0; j < 4; ++j) h[v][j] = mul2(h[v][j], w[j]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) h[v][j] = pair(0.f, 0.f);
    }
  }
  const float inv = rsqrtf(block_sum(lo(ss) + hi(ss), part) / (float)a.hidden + a.eps);
  const f32x2 inv2 = pair(inv, inv);
#pragma unroll
  for (int v = 0; v < kVec; ++v) {
    const int i = v * blockDim.x + threadIdx.x;
    const bool in = i < n_vec;
    f32x2 y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = mul2(h[v][j], inv2);
    if (in && a.y) Vec8<__nv_bfloat16>::store(a.y + row * a.y_stride + 8 * i, y);
    if (kFmt == CEP_BF16) continue;
    constexpr int kGroup = kFmt == CEP_FP8_E4M3_BLOCK128 ? 16 : 4;
    float amax = max_abs3(lo(y[0]), hi(y[0]), lo(y[1]));
    amax = max_abs3(amax, hi(y[1]), lo(y[2]));
    amax = max_abs3(amax, hi(y[2]), lo(y[3]));
    amax = max_abs3(amax, hi(y[3]), 0.f);
    if (!in) amax = 0.f;                               // (a row whose sum is zero or infinite has inv infinite or zero: 0 * inf)
#pragma unroll
    for (int o = kGroup / 2; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
    if (!in) continue;
    float factor;
    if (kFmt == CEP_FP8_E4M3_BLOCK128) {
      const Fp8Scale s = fp8_scale(amax);
      factor = s.factor;
      if (fp8_tiny(s.scale)) {                         // y to the normal range first
        const f32x2 up = pair(18446744073709551616.f, 18446744073709551616.f);
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = mul2(y[j], up);
        factor = __fdividef(1.f, s.scale * 18446744073709551616.f);
      }
      if (threadIdx.x % kGroup == 0) static_cast<float*>(a.scales)[row * a.n_scales + i / kGroup] = s.scale;
    } else {
      const int code = mx_code(amax);
      factor = mx_factor(code);
      if (threadIdx.x % kGroup == 0) static_cast<uint8_t*>(a.scales)[row * a.n_scales + i / kGroup] = (uint8_t)code;
    }
    const f32x2 f2 = pair(factor, factor);
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = mul2(y[j], f2);
    uint2 c;
    c.x = pack2_e4m3(lo(y[0]), hi(y[0])) | (pack2_e4m3(lo(y[1]), hi(y[1])) << 16);
    c.y = pack2_e4m3(lo(y[2]), hi(y[2])) | (pack2_e4m3(lo(y[3]), hi(y[3])) << 16);
    *reinterpret_cast<uint2*>(a.codes + row * a.hidden + 8 * i) = c;
  }
}

// Widths, strides or addresses that rule out 16-byte accesses: element loads, the row kept in shared memory, one warp
// per scale block.
template <typename XT, typename RT, int kFmt>
__global__ void __launch_bounds__(256)
norm_any_kernel(const NormArgs a) {
  extern __shared__ float hs[];
  __shared__ float part[kMaxWarps];
  pdl_enter();
  const size_t row = blockIdx.x;
  constexpr bool kRes = !std::is_same<RT, NoResidual>::value;
  using RL = typename std::conditional<kRes, RT, float>::type;
  const XT* x = static_cast<const XT*>(a.x) + row * a.x_stride;
  const RL* res = static_cast<const RL*>(a.residual) + (kRes ? row * a.residual_stride : 0);
  RL* rout = static_cast<RL*>(a.residual_out) + (kRes && a.residual_out ? row * a.residual_out_stride : 0);
  float ss = 0.f;
  constexpr int kU = 4;                                 // loads in flight per thread
  for (int i0 = threadIdx.x; i0 < a.hidden; i0 += kU * blockDim.x) {
    XT xe[kU];
    RL re[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int i = i0 + u * blockDim.x;
      if (i < a.hidden) {
        xe[u] = x[i];
        if (kRes) re[u] = res[i];
      }
    }
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int i = i0 + u * blockDim.x;
      if (i < a.hidden) {
        float h = to_f32(xe[u]);
        if (kRes) {
          h += to_f32(re[u]);
          if (a.residual_out) put(rout + i, h);
        }
        hs[i] = h;
        ss = fmaf(h, h, ss);
      }
    }
  }
  const float inv = rsqrtf(block_sum(ss, part) / (float)a.hidden + a.eps);     // (also orders the writes to hs)
  constexpr int kBlock = kFmt == CEP_MXFP4_E4M3 ? 32 : 128;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n_warps = blockDim.x >> 5;
  for (int b = warp; b * kBlock < a.hidden; b += n_warps) {
    float y[kBlock / 32], amax = 0.f;
#pragma unroll
    for (int j = 0; j < kBlock / 32; ++j) {
      const int i = b * kBlock + j * 32 + lane;
      y[j] = 0.f;
      if (i < a.hidden) {
        const float w = !a.weight ? 1.f : a.weight_fp32 ? static_cast<const float*>(a.weight)[i]
                                                        : __bfloat162float(static_cast<const __nv_bfloat16*>(a.weight)[i]);
        y[j] = hs[i] * w * inv;
        if (a.y) a.y[row * a.y_stride + i] = __float2bfloat16_rn(y[j]);
      }
      amax = fmaxf(amax, fabsf(y[j]));
    }
    if (kFmt == CEP_BF16) continue;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
    Fp8Scale s = fp8_scale(amax);
    const int code = mx_code(amax);
    if (kFmt == CEP_MXFP4_E4M3) {
      s.factor = mx_factor(code);
    } else if (fp8_tiny(s.scale)) {
#pragma unroll
      for (int j = 0; j < kBlock / 32; ++j) y[j] *= 18446744073709551616.f;
      s.factor = __fdividef(1.f, s.scale * 18446744073709551616.f);
    }
    if (lane == 0) {
      if (kFmt == CEP_MXFP4_E4M3) static_cast<uint8_t*>(a.scales)[row * a.n_scales + b] = (uint8_t)code;
      else static_cast<float*>(a.scales)[row * a.n_scales + b] = s.scale;
    }
#pragma unroll
    for (int j = 0; j < kBlock / 32; ++j) {
      const int i = b * kBlock + j * 32 + lane;
      if (i < a.hidden) a.codes[row * a.hidden + i] = (uint8_t)pack2_e4m3(y[j] * s.factor, 0.f);
    }
  }
}

template <typename XT, typename RT, int kFmt>
cudaError_t launch_fmt(const NormArgs& a, int n_tokens, bool wide, cudaStream_t s) {
  if (!wide) {
    const size_t smem = (size_t)a.hidden * 4;
    cudaError_t e = cudaFuncSetAttribute(norm_any_kernel<XT, RT, kFmt>, cudaFuncAttributeMaxDynamicSharedMemorySize, kNormMaxHidden * 4);
    if (e != cudaSuccess) return e;
    return launch_pdl(norm_any_kernel<XT, RT, kFmt>, dim3(n_tokens), dim3(256), smem, s, 1, a);
  }
  const int n_vec = a.hidden / 8;
  // Steps per thread.  Few rows: one step, the row's latency is what counts (7168 fp8, 128 rows: 3.0 us against 3.2 and 4.2
  // with two and four steps; 1024 rows 15.0 against 15.6 and 15.8).  Many rows: more steps keep more bytes in flight per
  // thread (16384 rows of 7168 fp8: 159 us with four, 177 with one or two; of 2048: 38 with two, 40 with one or four; of 512:
  // 13.0 with one, 13.8 with two), but with an fp32 tensor four steps do not fit the registers (194 us with two, 220 with four).
  const bool fp32 = sizeof(XT) == 4 || std::is_same<RT, float>::value;
  const int kv = n_vec > 2048 ? 4 : n_vec <= 64 || (n_tokens <= 1024 && n_vec <= 1024) ? 1 : n_vec <= 512 || fp32 ? 2 : 4;
  const int threads = ((n_vec + kv - 1) / kv + 31) / 32 * 32;
  return launch_pdl(kv == 1 ? norm_kernel<XT, RT, kFmt, 1> : kv == 2 ? norm_kernel<XT, RT, kFmt, 2> : norm_kernel<XT, RT, kFmt, 4>, dim3(n_tokens),
                    dim3(threads), 0, s, 1, a);
}

template <typename XT, typename RT>
cudaError_t launch_types(const NormArgs& a, int dtype, int n_tokens, bool wide, cudaStream_t s) {
  if (dtype == CEP_FP8_E4M3_BLOCK128) return launch_fmt<XT, RT, CEP_FP8_E4M3_BLOCK128>(a, n_tokens, wide, s);
  if (dtype == CEP_MXFP4_E4M3) return launch_fmt<XT, RT, CEP_MXFP4_E4M3>(a, n_tokens, wide, s);
  return launch_fmt<XT, RT, CEP_BF16>(a, n_tokens, wide, s);
}

template <typename XT>
cudaError_t launch_x(const NormArgs& a, const cep_norm_desc& d, bool wide, cudaStream_t s) {
  if (!a.residual) return launch_types<XT, NoResidual>(a, d.dtype, d.n_tokens, wide, s);
  if (d.residual_elem == CEP_ELEM_FP32) return launch_types<XT, float>(a, d.dtype, d.n_tokens, wide, s);
  return launch_types<XT, __nv_bfloat16>(a, d.dtype, d.n_tokens, wide, s);
}

bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

}  // namespace
}  // namespace cep

using namespace cep;

extern "C" int moe_norm(const cep_norm_desc* d, const void* x, const void* residual, const void* weight, void* residual_out,
                        void* y, void* codes, void* scales, void* stream) {
  if (!d) return record_error(CEP_ERR_ARG, "norm: the description is NULL");
  if (d->dtype != CEP_BF16 && d->dtype != CEP_FP8_E4M3_BLOCK128 && d->dtype != CEP_MXFP4_E4M3)
    return record_error(CEP_ERR_ARG, "norm: unknown dtype %d", d->dtype);
  const int elems[3] = {d->x_elem, d->residual_elem, d->weight_elem};
  for (int e : elems)
    if (e != CEP_ELEM_BF16 && e != CEP_ELEM_FP32) return record_error(CEP_ERR_ARG, "norm: unknown element type %d", e);
  if (d->n_tokens < 0 || d->hidden <= 0) return record_error(CEP_ERR_ARG, "norm: need n_tokens >= 0 and hidden > 0");
  if (d->hidden > kNormMaxHidden) return record_error(CEP_ERR_UNSUPPORTED, "norm: hidden %d is above %d", d->hidden, kNormMaxHidden);
  if (!(d->eps >= 0.f) || d->eps > 3.402823466e38f) return record_error(CEP_ERR_ARG, "norm: eps must be finite and not negative");
  if (d->n_tokens == 0) return CEP_OK;                        // nothing to do: empty tensors may have no address
  if (!x) return record_error(CEP_ERR_ARG, "norm: x is NULL");
  const bool quant = d->dtype != CEP_BF16;
  if (quant && (!codes || !scales)) return record_error(CEP_ERR_ARG, "norm: this dtype needs codes and scales");
  if (!quant && (codes || scales)) return record_error(CEP_ERR_ARG, "norm: CEP_BF16 writes no codes or scales");
  if (residual_out && !residual) return record_error(CEP_ERR_ARG, "norm: residual_out without a residual");
  if (!quant && !y && !residual_out) return record_error(CEP_ERR_ARG, "norm: no output given");
  const int64_t H = d->hidden;
  if (d->x_stride < H || (residual && d->residual_stride < H) || (residual_out && d->residual_out_stride < H) || (y && d->y_stride < H))
    return record_error(CEP_ERR_ARG, "norm: a row stride is smaller than hidden");
  const size_t xb = d->x_elem == CEP_ELEM_FP32 ? 4 : 2, rb = d->residual_elem == CEP_ELEM_FP32 ? 4 : 2, wb = d->weight_elem == CEP_ELEM_FP32 ? 4 : 2;
  if (!aligned(x, xb) || !aligned(residual, rb) || !aligned(residual_out, rb) || !aligned(weight, wb) || !aligned(y, 2) ||
      (d->dtype == CEP_FP8_E4M3_BLOCK128 && !aligned(scales, 4)))
    return record_error(CEP_ERR_ARG, "norm: a pointer is not aligned to its element type");
  // 16-byte accesses need every row of every tensor to start on 16 bytes (8 for the codes) and whole vectors
  auto wide_rows = [](const void* p, int64_t stride, size_t bytes, size_t align) {
    return !p || (aligned(p, align) && (size_t)stride * bytes % align == 0);
  };
  const bool wide = H % 8 == 0 && wide_rows(x, d->x_stride, xb, 16) && wide_rows(residual, d->residual_stride, rb, 16) &&
                    wide_rows(residual_out, d->residual_out_stride, rb, 16) && wide_rows(y, d->y_stride, 2, 16) &&
                    aligned(weight, 16) && wide_rows(codes, H, 1, 8);
  NormArgs a{x, residual, weight, residual_out, static_cast<__nv_bfloat16*>(y), static_cast<uint8_t*>(codes), scales,
             d->x_stride, d->residual_stride, d->residual_out_stride, d->y_stride, d->hidden, d->weight_elem == CEP_ELEM_FP32,
             quant ? (int)((H + (d->dtype == CEP_MXFP4_E4M3 ? 31 : 127)) / (d->dtype == CEP_MXFP4_E4M3 ? 32 : 128)) : 0, d->eps};
  const cudaError_t e = d->x_elem == CEP_ELEM_FP32 ? launch_x<float>(a, *d, wide, static_cast<cudaStream_t>(stream))
                                                   : launch_x<__nv_bfloat16>(a, *d, wide, static_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) return record_error(CEP_ERR_CUDA, "norm launch failed: %s", cudaGetErrorString(e));
  return CEP_OK;
}
