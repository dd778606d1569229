// What the two projection kernels share: operand descriptors, rows of s as operands, the lists of the down projection.
#pragma once
#include <cuda_bf16.h>

#include "lora.h"
#include "lora_ptx.cuh"

namespace cep {

using ptx::pack_bf16;

constexpr int kKBytes = 128;                          // bytes of K per stage: one 128-byte swizzle span, 64 bf16
constexpr int kUpBytes = 128 * 32;                    // 128 columns x one chunk of 16 ranks, 32-byte rows
constexpr int kSlabSteps = 12;                        // K steps (of 64) per accumulation chain of an fp32 output
// The up projection's steps.  A step covers kChunks chunks of 16 ranks and takes a stage of the ring: the adapter's columns of
// B (by TMA) where the K steps have W, and the tokens' rows of s (by the s-row warps) where they have x.  The loading thread
// tells those warps that the stage is free (ready); they tell the MMA thread that the rows are written (sfull).  The fence
// between their stores and the MMA costs as much as the stores, so a few steps share one (kBatch in either kernel).
// s is fp32 and enters as the sum of kTerms bf16 terms: two leave 2^-17 of it, which a bf16 output does not see; an fp32
// output takes three (2^-25), of which a 128-byte row holds one chunk instead of two.
template <typename OT>
struct UpStep {
  static constexpr int kTerms = sizeof(OT) == 4 ? 3 : 2, kChunks = sizeof(OT) == 4 ? 1 : 2;
};

// Waits for the end of the launch before this one / lets the next one be scheduled (it waits for this one's end in turn).
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void pdl_release() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
// K-major operand with rows of 32 bytes (16 ranks), 32-byte swizzle, 8-row groups 256 bytes apart
__device__ __forceinline__ uint64_t make_smem_desc_32b(uint32_t saddr) {
  uint64_t d = 0;
  d |= (uint64_t)((saddr & 0x3FFFFu) >> 4);
  d |= (uint64_t)1 << 16;
  d |= (uint64_t)(256 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)6 << 61;
  return d;
}

// The lists and s as the kernels read them; has == 0: no adapters in this call.  The lists are read past the L1: they are
// rewritten by every call.
struct LoraArgs {
  int has, rank_pad;
  const int32_t* ids; const int32_t* n_chunks; const int32_t* chunks;
  const float* s;
};

// A chunk (16 ranks) of a token is 32 bytes of operand row per term, [value | remainder | remainder of that].
template <int kTerms>
struct SChunk {
  uint32_t w[8 * kTerms];
  __device__ __forceinline__ void fetch(const float* __restrict__ s) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float4 v = __ldcg(reinterpret_cast<const float4*>(s) + q);
#pragma unroll
      for (int t = 0; t < kTerms; ++t) {
        const uint32_t h0 = pack_bf16(v.x, v.y), h1 = pack_bf16(v.z, v.w);
        w[8 * t + 2 * q] = h0; w[8 * t + 2 * q + 1] = h1;
        v.x -= __uint_as_float(h0 << 16); v.y -= __uint_as_float(h0 & 0xffff0000u);
        v.z -= __uint_as_float(h1 << 16); v.w -= __uint_as_float(h1 & 0xffff0000u);
      }
    }
  }
  // Writes the h-th chunk of row r of a 128-byte-swizzled tile (zeros when the token has another adapter).
  __device__ __forceinline__ void put(uint8_t* tile, int r, int h, bool mine) const {
#pragma unroll
    for (int j = 0; j < 2 * kTerms; ++j) {
      uint4 v = make_uint4(0, 0, 0, 0);
      if (mine) v = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
      *reinterpret_cast<uint4*>(tile + r * 128 + (((h * 2 * kTerms + j) ^ (r & 7)) << 4)) = v;
    }
  }
};

// The first kAhead chunks of a token's own adapter, fetched before its steps come up; the others when they do.
template <int kAhead, int kTerms>
struct SRow {
  const float* s;
  int my;                                              // the token's adapter, -1: none
  SChunk<kTerms> chunk[kAhead > 0 ? kAhead : 1];
  // t: the token, or negative where there is none
  __device__ __forceinline__ void fetch(const LoraArgs& la, int t) {
    s = la.s + (size_t)(t >= 0 ? t : 0) * la.rank_pad;
#pragma unroll
    for (int c = 0; c < kAhead; ++c)
      if (t >= 0 && c * kLoraChunk < la.rank_pad) chunk[c].fetch(s + c * kLoraChunk);      // (of use only if my >= 0)
    my = t >= 0 ? __ldcg(la.ids + t) : -1;
  }
  // Writes entry v of the list as the h-th chunk of row r.
  __device__ __forceinline__ void put(uint8_t* tile, int r, int h, int v) const {
    const int c = v % kLoraMaxChunks;
    const bool mine = my == v / kLoraMaxChunks;
    if (kAhead == 0 || c >= kAhead) {
      SChunk<kTerms> far;
      if (mine) far.fetch(s + c * kLoraChunk);
      far.put(tile, r, h, mine);
    } else {
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        if (c == k) chunk[k].put(tile, r, h, mine);
    }
  }
};

template <typename OT> __device__ __forceinline__ void put_out(OT* p, float v);
template <> __device__ __forceinline__ void put_out<float>(float* p, float v) { *p = v; }
template <> __device__ __forceinline__ void put_out<__nv_bfloat16>(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// The list entries of a step (one or two, -1 past the end).  They are read whether there are that many or not, so that the
// reads do not wait for the list's length; `cap` entries exist, an even number.
template <int kChunks>
__device__ __forceinline__ int2 list_step(const int32_t* list, int c, int cap) {
  if (kChunks == 1) return make_int2(c < cap ? __ldcg(list + c) : -1, -1);
  return c + 1 < cap ? __ldcg(reinterpret_cast<const int2*>(list + c)) : make_int2(-1, -1);
}
__device__ __forceinline__ int2 up_to(int2 e, int c, int total) { return make_int2(c < total ? e.x : -1, c + 1 < total ? e.y : -1); }
constexpr int kLookAhead = 8;                          // steps whose entries the loading thread reads at once

// Index of a chunk's [N][16] block in the up bank.
__device__ __forceinline__ int up_block(int v, int rank_pad) { return v / kLoraMaxChunks * (rank_pad / kLoraChunk) + v % kLoraMaxChunks; }

inline LoraArgs lora_args(const ProjectArgs& a) {
  LoraArgs la{};
  if (!a.bank) return la;
  la.has = 1; la.rank_pad = a.bank->rank_pad;
  la.ids = a.step.ids; la.n_chunks = a.step.n_chunks; la.chunks = a.step.chunks; la.s = a.step.s;
  return la;
}

}  // namespace cep
