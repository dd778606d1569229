// The shared projection with the adapters' up projection inside its accumulator:
//
//   y[t,n] = sum_k x[t,k] W[n,k] + sum_r s[t,r] B_a[n,r],   a = adapter of token t, s = scale_a * x A_a^T (lora_shrink.cu)
//
// The adapters are further K steps of the same matrix product: for every adapter present in a token tile one more step per
// 32 ranks multiplies the tile's rows of s (rows of other adapters: zeros) with that adapter's rows of B.  So the up
// projection adds neither a pass over y nor a rounding of it.  s is fp32; the tensor core takes it as the sum of two bf16
// terms (value and remainder, 2^-17 relative), two MMAs against the same B columns.
//
// The tensor core's fp32 additions truncate: one chain over K = 7168 ends 8e-6 low on average (measured), which a bf16
// output does not see and an fp32 output does.  fp32 outputs are therefore summed from chains of about 768 products, added
// with rounding: the small kernel keeps several accumulators, the large one adds each slab to y.
//
// Two kernels, both warp-specialised, TMA-fed, fp32 accumulators in tensor memory, every wait bounded (status word):
//   large   CTA pairs on 256 tokens x 256 columns, tokens on the MMA's M side, persistent with a tile counter
//   small   the weight on the M side (128 columns of y), up to 128 tokens on the N side, K split over the CTAs of a cluster so
//           that the weight streams through as many SMs as there are; the CTAs exchange partial sums through shared memory,
//           each adds a share of the tokens in split order
#include <cuda.h>
#include <cuda_bf16.h>

#include "lora.h"
#include "lora_ptx.cuh"

namespace cep {
namespace {

using namespace ptx;

constexpr int kSlabSteps = 12;                        // K steps (of 64) per accumulation chain of an fp32 output
constexpr int kKBytes = 128;                          // bytes of K per stage: one 128-byte swizzle span, 64 bf16
constexpr int kUpBytes = 128 * 32;                    // 128 columns x one chunk of 16 ranks, 32-byte rows

__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
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

// ------------------------------------------------------------------ the up projection's steps
// A step covers kStep chunks of 16 ranks and takes a stage of the ring: the adapter's columns of B (by TMA) where the K steps
// have W, and the tokens' rows of s (by the s-row warps) where they have x.  The loading thread tells those warps that the
// stage is free (ready); they tell the MMA thread that the rows are written (sfull).
constexpr int kStep = 2;

// A chunk (16 ranks) of a token is 64 bytes of operand row, [value | remainder]; a 128-byte row holds two chunks.
struct SChunk {
  uint32_t w[16];
  __device__ __forceinline__ void fetch(const float* __restrict__ s) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float4 v = __ldcg(reinterpret_cast<const float4*>(s) + q);
      const uint32_t h0 = pack_bf16(v.x, v.y), h1 = pack_bf16(v.z, v.w);
      w[2 * q] = h0; w[2 * q + 1] = h1;
      w[8 + 2 * q] = pack_bf16(v.x - __uint_as_float(h0 << 16), v.y - __uint_as_float(h0 & 0xffff0000u));
      w[8 + 2 * q + 1] = pack_bf16(v.z - __uint_as_float(h1 << 16), v.w - __uint_as_float(h1 & 0xffff0000u));
    }
  }
  // Writes half h of row r of a 128-byte-swizzled tile (zeros when the token has another adapter).
  __device__ __forceinline__ void put(uint8_t* tile, int r, int h, bool mine) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint4 v = make_uint4(0, 0, 0, 0);
      if (mine) v = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
      *reinterpret_cast<uint4*>(tile + r * 128 + (((h * 4 + j) ^ (r & 7)) << 4)) = v;
    }
  }
};

template <typename OT> __device__ __forceinline__ void put_out(OT* p, float v);
template <> __device__ __forceinline__ void put_out<float>(float* p, float v) { *p = v; }
template <> __device__ __forceinline__ void put_out<__nv_bfloat16>(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// Index of a chunk's [N][16] block in the up bank.
__device__ __forceinline__ int up_block(int v, int rank_pad) { return v / kLoraMaxChunks * (rank_pad / kLoraChunk) + v % kLoraMaxChunks; }

struct LoraArgs {                                      // bank == nullptr on the host: has == 0
  int has, rank_pad;
  const int32_t* ids; const int32_t* n_chunks; const int32_t* chunks;
  const float* s;
};

// ------------------------------------------------------------------ small kernel
constexpr int kSmallThreads = 192;
constexpr int kSmallMaxStages = 12;
constexpr int kMaxSplits = 8;                          // CTAs of a portable cluster

constexpr int kWStage = 128 * kKBytes;                 // 16 KiB of weight
#ifndef CEP_LORA_SMALL_RING
#define CEP_LORA_SMALL_RING (200 * 1024)
#endif
constexpr int kSmallRing = CEP_LORA_SMALL_RING;       // ring + s tiles
constexpr int kSharedRing = 136 * 1024;               // the same beside a block of the down projection
struct __align__(8) SmallBarriers {
  uint64_t full[kSmallMaxStages], empty[kSmallMaxStages], ready[kSmallMaxStages], sfull[kSmallMaxStages], acc_full;
  uint32_t tmem_base;
  int abort_flag;
};
static_assert(sizeof(SmallBarriers) <= 512, "barrier block");

// Grid (column tiles, K splits, token tiles of `tok`).  npad: token columns of the MMA, a multiple of 16.  n_acc: accumulators
// (npad columns each) that share the CTA's K steps.
template <typename OT>
__global__ void __launch_bounds__(kSmallThreads, 1)
project_small_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_x,
                     const __grid_constant__ CUtensorMap tm_up, int T, int N, int num_kb, int tok, int npad, int stages, int n_acc, const LoraArgs la,
                     OT* __restrict__ y, int64_t y_stride, int vec_ok, int32_t* __restrict__ status) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const int x_stage = npad * kKBytes, stage_bytes = kWStage + x_stage;
  SmallBarriers* bars = reinterpret_cast<SmallBarriers*>(smem + stages * stage_bytes);
  volatile int* abort_flag = &bars->abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int n0 = blockIdx.x * 128, t0 = blockIdx.z * tok;
  const int split = blockIdx.y, splits = gridDim.y;
  constexpr int kCols = sizeof(OT) == 4 ? 512 : kSmallTok;           // tensor-memory columns
  const int kb0 = (int)((long long)num_kb * split / splits), kb1 = (int)((long long)num_kb * (split + 1) / splits);

  // The K steps of x and W do not depend on the down projection: they start before it has finished.
  auto load_k_step = [&](int kb, int stage) {
    const uint32_t full = smem_u32(&bars->full[stage]);
    uint8_t* st = smem + stage * stage_bytes;
    mbar_expect_tx(full, stage_bytes);
    tma_load_2d(smem_u32(st), &tm_w, kb * (kKBytes / 2), n0, full);
    tma_load_2d(smem_u32(st + kWStage), &tm_x, kb * (kKBytes / 2), t0, full);
  };
  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) {
      mbar_init(smem_u32(&bars->full[s]), 1); mbar_init(smem_u32(&bars->empty[s]), 1);
      mbar_init(smem_u32(&bars->ready[s]), 1); mbar_init(smem_u32(&bars->sfull[s]), 4);
    }
    mbar_init(smem_u32(&bars->acc_full), 1);
    bars->abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    // the ring is empty: its first loads go out before the rest of the block is set up
    for (int s = 0; s < stages && kb0 + s < kb1; ++s) load_k_step(kb0 + s, s);
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32(&bars->tmem_base)), "n"(kCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bars->tmem_base;

  if (warp == 0) {
    if (lane == 0) {
      const int ahead = min(stages, kb1 - kb0);        // loaded above
      int stage = ahead % stages; uint32_t phase = ahead == stages;
      bool ok = true;
      for (int kb = kb0 + ahead; kb < kb1; ++kb) {
        if (!mbar_wait(smem_u32(&bars->empty[stage]), phase ^ 1u, abort_flag, status)) { ok = false; break; }
        load_k_step(kb, stage);
        if (++stage == stages) { stage = 0; phase ^= 1u; }
      }
      if (la.has && ok) {
        pdl_wait();
        const int total = la.n_chunks[blockIdx.z];
        const int32_t* list = la.chunks + (size_t)t0 * kLoraMaxChunks;
        for (int c0 = split * kStep; c0 < total; c0 += splits * kStep) {
          if (!mbar_wait(smem_u32(&bars->empty[stage]), phase ^ 1u, abort_flag, status)) break;
          const uint32_t full = smem_u32(&bars->full[stage]);
          uint8_t* st = smem + stage * stage_bytes;
          const int n = min(kStep, total - c0);
          mbar_expect_tx(full, n * kUpBytes);
          mbar_arrive(smem_u32(&bars->ready[stage]));
          for (int i = 0; i < n; ++i) tma_load_3d(smem_u32(st + i * kUpBytes), &tm_up, 0, n0, up_block(list[c0 + i], la.rank_pad), full);
          if (++stage == stages) { stage = 0; phase ^= 1u; }
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t idesc = make_idesc_bf16(128, npad);
      int stage = 0; uint32_t phase = 0;
      bool ok = true;
      int slab = 0, slab_end = kb0 + (kb1 - kb0) / n_acc;           // chain `slab` ends before K step slab_end
      uint32_t first = 1;
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!mbar_wait(smem_u32(&bars->full[stage]), phase, abort_flag, status)) { ok = false; break; }
        tc_fence_after();
        if (kb == slab_end) { ++slab; slab_end = kb0 + (int)((long long)(kb1 - kb0) * (slab + 1) / n_acc); first = 1; }
        const uint32_t d = tmem + (uint32_t)(slab * npad);
        const uint64_t wdesc = make_smem_desc(smem_u32(smem + stage * stage_bytes));
        const uint64_t xdesc = make_smem_desc(smem_u32(smem + stage * stage_bytes + kWStage));
#pragma unroll
        for (int k4 = 0; k4 < 4; ++k4)
          tc_mma_f16(d, wdesc + (uint64_t)(k4 * 2), xdesc + (uint64_t)(k4 * 2), idesc, k4 != 0 ? 1u : first ^ 1u);
        first = 0;
        tc_commit(smem_u32(&bars->empty[stage]));
        if (++stage == stages) { stage = 0; phase ^= 1u; }
      }
      if (la.has && ok) {
        pdl_wait();
        const int total = la.n_chunks[blockIdx.z];
        const uint32_t last_acc = tmem + (uint32_t)(slab * npad);
        uint32_t sphase = 0;                             // one parity bit per stage
        for (int c0 = split * kStep; c0 < total; c0 += splits * kStep) {
          if (!mbar_wait(smem_u32(&bars->full[stage]), phase, abort_flag, status) ||
              !mbar_wait(smem_u32(&bars->sfull[stage]), (sphase >> stage) & 1u, abort_flag, status)) { ok = false; break; }
          sphase ^= 1u << stage;
          tc_fence_after();
          const uint32_t up = smem_u32(smem + stage * stage_bytes);
          const int n = min(kStep, total - c0);
          for (int i = 0; i < n; ++i) {
            const uint64_t udesc = make_smem_desc_32b(up + i * kUpBytes);
            const uint64_t sdesc = make_smem_desc(up + kWStage) + (uint64_t)(i * 4);
            tc_mma_f16(last_acc, udesc, sdesc, idesc, 1u);
            tc_mma_f16(last_acc, udesc, sdesc + 2, idesc, 1u);
          }
          tc_commit(smem_u32(&bars->empty[stage]));
          if (++stage == stages) { stage = 0; phase ^= 1u; }
        }
      }
      if (ok) tc_commit(smem_u32(&bars->acc_full));
    }
  } else {
    // ---------------------------------------------------------------- warps 2..5: rows of s, then the epilogue
    const int lane_grp = warp & 3, tid = threadIdx.x - 64;
    bool ok = true;
    if (la.has) {
      pdl_wait();
      const int t = t0 + tid;
      const int my = tid < npad && t < T ? la.ids[t] : -1;
      const float* srow = la.s + (size_t)(my >= 0 ? t : 0) * la.rank_pad;
      constexpr int kAhead = 4;
      SChunk row[kAhead];                              // the first 64 ranks of this thread's token, fetched ahead
#pragma unroll
      for (int c = 0; c < kAhead; ++c)
        if (my >= 0 && c * kLoraChunk < la.rank_pad) row[c].fetch(srow + c * kLoraChunk);
      const int total = la.n_chunks[blockIdx.z];
      const int32_t* list = la.chunks + (size_t)t0 * kLoraMaxChunks;
      int stage = (kb1 - kb0) % stages;                // where the K steps end
      uint32_t phase = 0;                              // one parity bit per stage
      for (int c0 = split * kStep; c0 < total; c0 += splits * kStep) {
        int v[kStep];
#pragma unroll
        for (int i = 0; i < kStep; ++i) v[i] = c0 + i < total ? list[c0 + i] : -1;
        ok = mbar_wait(smem_u32(&bars->ready[stage]), (phase >> stage) & 1u, abort_flag, status);
        if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
        phase ^= 1u << stage;
        uint8_t* rows = smem + stage * stage_bytes + kWStage;
        if (tid < npad) {
#pragma unroll
          for (int i = 0; i < kStep; ++i) {
            if (v[i] < 0) break;
            const int c = v[i] % kLoraMaxChunks;
            const bool mine = my == v[i] / kLoraMaxChunks;
            if (c >= kAhead) {
              SChunk r;
              if (mine) r.fetch(srow + c * kLoraChunk);
              r.put(rows, tid, i, mine);
            } else {
#pragma unroll
              for (int k = 0; k < kAhead; ++k)
                if (c == k) row[k].put(rows, tid, i, mine);
            }
          }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bars->sfull[stage]));
        if (++stage == stages) stage = 0;
      }
    }
    const bool got = ok && mbar_wait_relaxed(smem_u32(&bars->acc_full), 0u, abort_flag, status);
    const bool all = __all_sync(0xffffffffu, got);
    const int n = n0 + lane_grp * 32 + lane;
    const int cols = min(tok, T - t0);                 // token columns that exist
    const uint32_t taddr = tmem + ((uint32_t)(lane_grp * 32) << 16);
    float* mine = reinterpret_cast<float*>(smem);      // [token][128] partial sums, in the ring: every load has been consumed
    if (all) {
      tc_fence_after();
      for (int c = 0; c < cols; c += 16) {
        __syncwarp();                                  // the load is warp-collective
        uint32_t d[16];
        tc_ld16(taddr + c, d);
        tc_wait_ld();
        for (int s = 1; s < n_acc; ++s) {
          uint32_t e[16];
          tc_ld16(taddr + s * npad + c, e);
          tc_wait_ld();
#pragma unroll
          for (int i = 0; i < 16; ++i) d[i] = __float_as_uint(__uint_as_float(d[i]) + __uint_as_float(e[i]));
        }
        if (splits == 1) {
          if (n < N) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (c + i < cols) put_out(y + (size_t)(t0 + c + i) * y_stride + n, __uint_as_float(d[i]));
          }
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (c + i < cols) mine[(c + i) * 128 + lane_grp * 32 + lane] = __uint_as_float(d[i]);
        }
      }
    }
  }
  if (splits > 1) {
    // (a CTA that gave up still takes both barriers; its sums are then meaningless and the status word says so)
    cluster_sync_all();
    const int cols = min(tok, T - t0);
    const int c0 = cols * split / splits, c1 = cols * (split + 1) / splits;
    const uint32_t base = smem_u32(smem);
    // four columns of y per lane, a token per warp
    for (int c = c0 + warp; c < c1; c += kSmallThreads / 32) {
      float4 v[kMaxSplits];
#pragma unroll
      for (int s = 0; s < kMaxSplits; ++s)
        if (s < splits) v[s] = ld_cluster_f4(mapa(base + (uint32_t)((c * 128 + lane * 4) * 4), (uint32_t)s));
      float4 o = v[0];
#pragma unroll
      for (int s = 1; s < kMaxSplits; ++s)
        if (s < splits) { o.x += v[s].x; o.y += v[s].y; o.z += v[s].z; o.w += v[s].w; }
      OT* row = y + (size_t)(t0 + c) * y_stride + n0 + lane * 4;
      const int left = N - n0 - lane * 4;
      if (left >= 4 && vec_ok) {
        if (sizeof(OT) == 2) *reinterpret_cast<uint2*>(row) = make_uint2(pack_bf16(o.x, o.y), pack_bf16(o.z, o.w));
        else *reinterpret_cast<float4*>(row) = o;
      } else {
        if (left > 0) put_out(row, o.x);
        if (left > 1) put_out(row + 1, o.y);
        if (left > 2) put_out(row + 2, o.z);
        if (left > 3) put_out(row + 3, o.w);
      }
    }
    cluster_sync_reads();                              // no CTA leaves while another reads its sums
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(kCols) : "memory");
  }
}

// ------------------------------------------------------------------ large kernel
#ifndef CEP_LORA_LARGE_STAGES
#define CEP_LORA_LARGE_STAGES 6
#endif
constexpr int kLargeStages = CEP_LORA_LARGE_STAGES;
constexpr int kHalf = 128 * kKBytes;                   // one CTA's 128 rows of either operand: 16 KiB
constexpr int kRing = 4;                               // tile ids in flight
constexpr int kPoison = -2;
constexpr int kLargeThreads = 352;                     // warp 0 loads, 1 MMA, 2-5 epilogue, 6 tile ids, 7-10 rows of s
constexpr int kReaders = 19;                           // leader: loads, MMA, 4 epilogue, 4 s-row warps; peer: loads, 4, 4
struct __align__(8) LargeBarriers {
  uint64_t full[kLargeStages], empty[kLargeStages], ready[kLargeStages], sfull[kLargeStages], acc_full[2], acc_empty[2];
  uint64_t ring_full[kRing], ring_empty[kRing];
  int32_t ring_tile[kRing];
  uint32_t tmem_base;
  int abort_flag;
};
static_assert(sizeof(LargeBarriers) <= 512, "barrier block");
constexpr int kLargeSmem = kLargeStages * 2 * kHalf + 512 + 1024;
static_assert(kLargeSmem <= 227 * 1024, "shared memory");

// Reader side of the ring of tile ids (written by the leader's warp 6, into both CTAs); -1 ends the kernel.
struct RingReader {
  int slot = 0; uint32_t phase = 0;
  __device__ __forceinline__ int next(LargeBarriers* bars, bool is_peer, volatile int* abort_flag, int32_t* status) {
    const uint32_t bar = smem_u32(&bars->ring_full[slot]);
    const bool ok = is_peer ? mbar_wait_acq_cluster(bar, phase, abort_flag, status) : mbar_wait_relaxed(bar, phase, abort_flag, status);
    if (!ok) return -1;
    const int t = *reinterpret_cast<volatile int32_t*>(&bars->ring_tile[slot]);
    if (t < -1) { atomicExch(&status[kStTimeout], 1); *abort_flag = 1; return -1; }
    return t;
  }
  __device__ __forceinline__ void done(LargeBarriers* bars, bool signal) {
    if (signal) mbar_arrive_cluster(mapa(smem_u32(&bars->ring_empty[slot]), 0));
    if (++slot == kRing) { slot = 0; phase ^= 1u; }
  }
};

// Linear tile -> (token tile, column block): column blocks in groups whose weight panel stays in the L2, each group swept
// over all token tiles with the column block as the fast index.
__device__ __forceinline__ void large_tile(int tile, int m_tiles, int n_blocks, int n_group, int* m, int* nb) {
  const int g = tile / (m_tiles * n_group);
  const int rem = tile - g * m_tiles * n_group;
  const int gn = min(n_group, n_blocks - g * n_group);
  *m = rem / gn;
  *nb = g * n_group + rem % gn;
}

template <typename OT>
__global__ void __launch_bounds__(kLargeThreads, 1)
project_large_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_x,
                     const __grid_constant__ CUtensorMap tm_up, int T, int N, int num_kb, int slab_steps, int m_tiles, int n_blocks, int n_group,
                     const LoraArgs la, OT* __restrict__ y, int64_t y_stride, int vec_ok, int32_t* __restrict__ tile_counter,
                     int32_t* __restrict__ status) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* smem_x = smem;
  uint8_t* smem_w = smem + kLargeStages * kHalf;
  LargeBarriers* bars = reinterpret_cast<LargeBarriers*>(smem_w + kLargeStages * kHalf);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const bool is_peer = rank != 0;
  volatile int* abort_flag = &bars->abort_flag;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kLargeStages; ++s) {
      mbar_init(smem_u32(&bars->full[s]), 1); mbar_init(smem_u32(&bars->empty[s]), 1);
      mbar_init(smem_u32(&bars->ready[s]), 1); mbar_init(smem_u32(&bars->sfull[s]), 8);
    }
    for (int s = 0; s < 2; ++s) { mbar_init(smem_u32(&bars->acc_full[s]), 1); mbar_init(smem_u32(&bars->acc_empty[s]), 8); }
    for (int s = 0; s < kRing; ++s) {
      mbar_init(smem_u32(&bars->ring_full[s]), 1); mbar_init(smem_u32(&bars->ring_empty[s]), kReaders);
      bars->ring_tile[s] = kPoison;
    }
    bars->abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32(&bars->tmem_base)), "n"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem = bars->tmem_base;
  const int total = m_tiles * n_blocks;
  pdl_wait();

  if (warp == 0) {
    // ---------------------------------------------------------------- TMA loads (both CTAs)
    if (lane == 0) {
      int stage = 0; uint32_t phase = 0;
      bool ok = true;
      RingReader rd;
      while (ok) {
        const int tile = rd.next(bars, is_peer, abort_flag, status);
        rd.done(bars, true);
        if (tile < 0) break;
        int m, nb;
        large_tile(tile, m_tiles, n_blocks, n_group, &m, &nb);
        const int t0 = m * kLargeTok + (int)rank * 128, n0 = nb * 256 + (int)rank * 128;
        for (int kb = 0; kb < num_kb; ++kb) {
          if (!mbar_wait(smem_u32(&bars->empty[stage]), phase ^ 1u, abort_flag, status)) { ok = false; break; }
          const uint32_t full = mapa(smem_u32(&bars->full[stage]), 0);
          if (rank == 0) mbar_expect_tx(smem_u32(&bars->full[stage]), 4 * kHalf);      // both CTAs' bytes
          tma_load_2d_pair(smem_u32(smem_x + stage * kHalf), &tm_x, kb * (kKBytes / 2), t0, full);
          tma_load_2d_pair(smem_u32(smem_w + stage * kHalf), &tm_w, kb * (kKBytes / 2), n0, full);
          if (++stage == kLargeStages) { stage = 0; phase ^= 1u; }
        }
        const int total = la.has ? la.n_chunks[m] : 0;
        const int32_t* list = la.chunks + (size_t)m * kLargeTok * kLoraMaxChunks;
        for (int c0 = 0; ok && c0 < total; c0 += kStep) {
          if (!mbar_wait(smem_u32(&bars->empty[stage]), phase ^ 1u, abort_flag, status)) { ok = false; break; }
          const uint32_t full = mapa(smem_u32(&bars->full[stage]), 0);
          const int n = min(kStep, total - c0);
          if (rank == 0) mbar_expect_tx(smem_u32(&bars->full[stage]), 2 * n * kUpBytes);
          mbar_arrive(smem_u32(&bars->ready[stage]));
          for (int i = 0; i < n; ++i)
            tma_load_3d_pair(smem_u32(smem_w + stage * kHalf + i * kUpBytes), &tm_up, 0, n0, up_block(list[c0 + i], la.rank_pad), full);
          if (++stage == kLargeStages) { stage = 0; phase ^= 1u; }
        }
      }
    }
  } else if (warp == 1) {
    // ---------------------------------------------------------------- MMA issuer (leader only)
    if (lane == 0 && rank == 0) {
      constexpr uint32_t idesc = make_idesc_bf16(256, 256);
      int stage = 0; uint32_t phase = 0;
      int acc = 0; uint32_t acc_phase = 0;
      uint32_t sphase = 0;                               // one parity bit per stage
      bool ok = true;
      RingReader rd;
      while (ok) {
        const int tile = rd.next(bars, false, abort_flag, status);
        rd.done(bars, true);
        if (tile < 0) break;
        if (!mbar_wait(smem_u32(&bars->acc_empty[acc]), acc_phase ^ 1u, abort_flag, status)) break;
        tc_fence_after();
        uint32_t d = tmem + (uint32_t)(acc * 256);
        uint32_t more = 0;                               // 0: the accumulator starts with this step
        for (int kb = 0, left = slab_steps; kb < num_kb; ++kb, --left) {
          if (left == 0) {                               // this chain is complete: the epilogue adds it to y
            tc_commit_pair_both(smem_u32(&bars->acc_full[acc]), 3);
            if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
            if (!mbar_wait(smem_u32(&bars->acc_empty[acc]), acc_phase ^ 1u, abort_flag, status)) { ok = false; break; }
            tc_fence_after();
            d = tmem + (uint32_t)(acc * 256);
            more = 0; left = slab_steps;
          }
          if (!mbar_wait(smem_u32(&bars->full[stage]), phase, abort_flag, status)) { ok = false; break; }
          tc_fence_after();
          const uint64_t xdesc = make_smem_desc(smem_u32(smem_x + stage * kHalf));
          const uint64_t wdesc = make_smem_desc(smem_u32(smem_w + stage * kHalf));
#pragma unroll
          for (int k4 = 0; k4 < 4; ++k4)
            tc_mma_f16_pair(d, xdesc + (uint64_t)(k4 * 2), wdesc + (uint64_t)(k4 * 2), idesc, k4 != 0 ? 1u : more);
          more = 1;
          tc_commit_pair_both(smem_u32(&bars->empty[stage]), 3);
          if (++stage == kLargeStages) { stage = 0; phase ^= 1u; }
        }
        if (ok && la.has) {
          int m, nb;
          large_tile(tile, m_tiles, n_blocks, n_group, &m, &nb);
          const int total = la.n_chunks[m];
          for (int c0 = 0; c0 < total; c0 += kStep) {
            if (!mbar_wait(smem_u32(&bars->full[stage]), phase, abort_flag, status) ||
                !mbar_wait_acq_cluster(smem_u32(&bars->sfull[stage]), (sphase >> stage) & 1u, abort_flag, status)) { ok = false; break; }
            sphase ^= 1u << stage;
            tc_fence_after();
            const uint64_t sdesc = make_smem_desc(smem_u32(smem_x + stage * kHalf));
            const int n = min(kStep, total - c0);
            for (int i = 0; i < n; ++i) {
              const uint64_t udesc = make_smem_desc_32b(smem_u32(smem_w + stage * kHalf) + i * kUpBytes);
              tc_mma_f16_pair(d, sdesc + (uint64_t)(i * 4), udesc, idesc, 1u);
              tc_mma_f16_pair(d, sdesc + (uint64_t)(i * 4 + 2), udesc, idesc, 1u);
            }
            tc_commit_pair_both(smem_u32(&bars->empty[stage]), 3);
            if (++stage == kLargeStages) { stage = 0; phase ^= 1u; }
          }
        }
        if (!ok) break;
        tc_commit_pair_both(smem_u32(&bars->acc_full[acc]), 3);
        if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
      }
    }
  } else if (warp == 6) {
    // ---------------------------------------------------------------- tile ids (leader only)
    if (lane == 0 && !is_peer) {
      int slot = 0; uint32_t phase = 0;
      for (;;) {
        if (!mbar_wait_relaxed(smem_u32(&bars->ring_empty[slot]), phase ^ 1u, abort_flag, status)) break;
        int t = atomicAdd(tile_counter, 1);
        if (t >= total) t = -1;
        bars->ring_tile[slot] = t;
        st_shared_cluster_u32(mapa(smem_u32(&bars->ring_tile[slot]), 1), (uint32_t)t);
        mbar_arrive(smem_u32(&bars->ring_full[slot]));
        mbar_arrive_release_cluster(mapa(smem_u32(&bars->ring_full[slot]), 1));
        if (t < 0) break;
        if (++slot == kRing) { slot = 0; phase ^= 1u; }
      }
    }
  } else if (warp >= 7) {
    // ---------------------------------------------------------------- rows of s (both CTAs, one token per thread)
    const int r = threadIdx.x - 7 * 32;
    int stage = 0; uint32_t phase = 0;                   // phase: one parity bit per stage
    bool ok = true;
    RingReader rd;
    while (ok) {
      const int tile = rd.next(bars, is_peer, abort_flag, status);
      __syncwarp();
      rd.done(bars, lane == 0);
      if (!__all_sync(0xffffffffu, tile >= 0)) break;
      if (!la.has) continue;
      int m, nb;
      large_tile(tile, m_tiles, n_blocks, n_group, &m, &nb);
      const int t = m * kLargeTok + (int)rank * 128 + r;
      const int my = t < T ? la.ids[t] : -1;
      const float* srow = la.s + (size_t)(my >= 0 ? t : 0) * la.rank_pad;
      const int total = la.n_chunks[m];
      const int32_t* list = la.chunks + (size_t)m * kLargeTok * kLoraMaxChunks;
      stage = (stage + num_kb) % kLargeStages;           // past the tile's K steps
      for (int c0 = 0; c0 < total; c0 += kStep) {
        SChunk row[kStep];
        bool mine[kStep];
        const int n = min(kStep, total - c0);
#pragma unroll
        for (int i = 0; i < kStep; ++i) {
          const int v = i < n ? list[c0 + i] : -1;
          mine[i] = v >= 0 && my == v / kLoraMaxChunks;
          if (mine[i]) row[i].fetch(srow + v % kLoraMaxChunks * kLoraChunk);
        }
        ok = mbar_wait(smem_u32(&bars->ready[stage]), (phase >> stage) & 1u, abort_flag, status);
        if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
        phase ^= 1u << stage;
#pragma unroll
        for (int i = 0; i < kStep; ++i) if (i < n) row[i].put(smem_x + stage * kHalf, r, i, mine[i]);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive_release_cluster(mapa(smem_u32(&bars->sfull[stage]), 0));
        if (++stage == kLargeStages) stage = 0;
      }
    }
  } else {
    // ---------------------------------------------------------------- epilogue (warps 2..5, both CTAs)
    const int lane_grp = warp & 3;
    int acc = 0; uint32_t acc_phase = 0;
    RingReader rd;
    for (;;) {
      const int tile = rd.next(bars, is_peer, abort_flag, status);
      __syncwarp();
      rd.done(bars, lane == 0);
      if (!__all_sync(0xffffffffu, tile >= 0)) break;
      int m, nb;
      large_tile(tile, m_tiles, n_blocks, n_group, &m, &nb);
      bool got = true;
      for (int kb = 0; kb < num_kb; kb += slab_steps) {  // one accumulation chain after the other
        got = mbar_wait_relaxed(smem_u32(&bars->acc_full[acc]), acc_phase, abort_flag, status);
        got = __all_sync(0xffffffffu, got);
        if (!got) break;
        tc_fence_after();
        const int t = m * kLargeTok + (int)rank * 128 + lane_grp * 32 + lane;
        OT* row = y + (size_t)t * y_stride + nb * 256;
        const uint32_t taddr = tmem + ((uint32_t)(lane_grp * 32) << 16) + (uint32_t)(acc * 256);
        const int left = N - nb * 256;                   // columns of this block that exist
#pragma unroll 1
        for (int c = 0; c < 256 && c < left; c += 32) {
          __syncwarp();                                  // the loads are warp-collective
          uint32_t d[32];
          tc_ld32(taddr + c, d);
          tc_wait_ld();
          if (t >= T) {
          } else if (vec_ok && c + 32 <= left) {
            if (sizeof(OT) == 2) {
              uint4* dst = reinterpret_cast<uint4*>(row + c);
#pragma unroll
              for (int q = 0; q < 4; ++q)
                dst[q] = make_uint4(pack_bf16(__uint_as_float(d[8 * q]), __uint_as_float(d[8 * q + 1])),
                                    pack_bf16(__uint_as_float(d[8 * q + 2]), __uint_as_float(d[8 * q + 3])),
                                    pack_bf16(__uint_as_float(d[8 * q + 4]), __uint_as_float(d[8 * q + 5])),
                                    pack_bf16(__uint_as_float(d[8 * q + 6]), __uint_as_float(d[8 * q + 7])));
            } else {
              float4* dst = reinterpret_cast<float4*>(row + c);
              float4 v[8];
#pragma unroll
              for (int q = 0; q < 8; ++q)
                v[q] = make_float4(__uint_as_float(d[4 * q]), __uint_as_float(d[4 * q + 1]), __uint_as_float(d[4 * q + 2]), __uint_as_float(d[4 * q + 3]));
              if (kb != 0) {
#pragma unroll
                for (int q = 0; q < 8; ++q) { const float4 o = dst[q]; v[q].x += o.x; v[q].y += o.y; v[q].z += o.z; v[q].w += o.w; }
              }
#pragma unroll
              for (int q = 0; q < 8; ++q) dst[q] = v[q];
            }
          } else {
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (c + i < left) put_out(row + c + i, __uint_as_float(d[i]) + (sizeof(OT) == 4 && kb != 0 ? (float)row[c + i] : 0.f));
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(mapa(smem_u32(&bars->acc_empty[acc]), 0));
        if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
      }
      if (!got) break;
    }
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(512) : "memory");
  }
}

// ------------------------------------------------------------------ host side
constexpr int kMaxDevices = 64;
int g_large_clusters[kMaxDevices];                     // co-resident CTA pairs + 1 (0: not set up)
int g_small_clusters[kMaxDevices][kMaxSplits + 1];     // co-resident clusters by size; [0]: set up

cudaError_t device_slot(int* dev) {
  cudaError_t e = cudaGetDevice(dev);
  if (e != cudaSuccess) return e;
  return (*dev < 0 || *dev >= kMaxDevices) ? cudaErrorInvalidDevice : cudaSuccess;
}

LoraArgs lora_args(const ProjectArgs& a) {
  LoraArgs la{};
  if (!a.bank) return la;
  la.has = 1; la.rank_pad = a.bank->rank_pad;
  la.ids = a.step.ids; la.n_chunks = a.step.n_chunks; la.chunks = a.step.chunks; la.s = a.step.s;
  return la;
}

}  // namespace

#ifndef CEP_LORA_SMALL_TOKENS
#define CEP_LORA_SMALL_TOKENS 256
#endif
bool project_is_small(int T, int N) { (void)N; return T <= CEP_LORA_SMALL_TOKENS; }
int project_small_tile(int out_f32) { return out_f32 ? 64 : kSmallTok; }       // (8 accumulators of 64 columns fill the tensor memory)
int project_small_tokens(int T, int out_f32) { return T >= project_small_tile(out_f32) ? project_small_tile(out_f32) : (T + 15) / 16 * 16; }

int make_tile_map(GemmTensorMap* out, const void* base, long long cols, long long rows, long long row_stride, long long depth,
                  long long depth_stride, int box_cols, int box_rows, int swizzle_bytes) {
  typedef CUresult (*Encode)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                             const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static Encode enc = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    const bool ok = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess;
    return ok ? reinterpret_cast<Encode>(p) : nullptr;
  }();
  if (!enc) return -1;
  cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)depth};
  cuuint64_t strides[2] = {(cuuint64_t)row_stride, (cuuint64_t)depth_stride};
  cuuint32_t box[3] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, 1}, es[3] = {1, 1, 1};
  const CUresult r = enc(reinterpret_cast<CUtensorMap*>(out), CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, depth > 0 ? 3 : 2, const_cast<void*>(base), dims,
                         strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle_bytes == 32 ? CU_TENSOR_MAP_SWIZZLE_32B : CU_TENSOR_MAP_SWIZZLE_128B,
                         CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? 0 : -2;
}

cudaError_t launch_project_small(const ProjectArgs& a, const GemmTensorMap& tm_w, const GemmTensorMap& tm_x, const GemmTensorMap& tm_up,
                                 cudaStream_t s) {
  int dev = 0;
  cudaError_t e = device_slot(&dev);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 1; attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.blockDim = dim3(kSmallThreads, 1, 1); cfg.stream = s; cfg.attrs = attr;
  int* clusters = g_small_clusters[dev];
  if (clusters[0] == 0) {
    e = cudaFuncSetAttribute(project_small_kernel<__nv_bfloat16>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmallRing + 2048);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(project_small_kernel<float>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmallRing + 2048);
    if (e != cudaSuccess) return e;
    for (int c = 1; c <= kMaxSplits; ++c) {
      attr[0].val.clusterDim.y = (unsigned)c;
      cfg.gridDim = dim3(kSms, c, 1); cfg.dynamicSmemBytes = kSmallRing + 2048; cfg.numAttrs = 1;
      e = cudaOccupancyMaxActiveClusters(&clusters[c], project_small_kernel<__nv_bfloat16>, &cfg);
      if (e != cudaSuccess) return e;
    }
    clusters[0] = 1;
  }
  const int npad = project_small_tokens(a.T, a.out_f32), tok = project_small_tile(a.out_f32);
  const int n_tiles = (a.N + 127) / 128, t_tiles = (a.T + tok - 1) / tok, num_kb = (a.K + 63) / 64;
  const long long tiles = (long long)n_tiles * t_tiles;
  // The cluster size with the least work for the busiest SM, in K steps: a cluster needs that many free SMs in one GPC,
  // so fewer SMs are usable for some sizes.  kExchange: what the exchange of partial sums costs (2 us).
  constexpr long long kExchange = 6;
  int splits = 1;
  long long best = 1ll << 60;
  for (int c = 1; c <= kMaxSplits && c <= num_kb; ++c) {
    if (clusters[c] < 1) continue;
    const long long cost = (tiles + clusters[c] - 1) / clusters[c] * ((num_kb + c - 1) / c) + (c > 1 ? kExchange : 0);
    if (cost < best) { best = cost; splits = c; }
  }
  const int steps = num_kb / splits;                   // K steps a CTA has at least
  int n_acc = a.out_f32 ? (steps + kSlabSteps - 1) / kSlabSteps : 1;
  if (n_acc > 512 / npad) n_acc = 512 / npad;
  if (n_acc < 1) n_acc = 1;
  const int stage = kWStage + npad * kKBytes;
  // With adapters and few tokens the ring leaves room for a block of the down projection, so that both run at once.
  const int ring = a.bank && lora_beside(a.T) ? kSharedRing : kSmallRing;
  int stages = ring / stage;
  if (stages > kSmallMaxStages) stages = kSmallMaxStages;
  const size_t smem = 1024 + (size_t)stages * stage + 512;
  const size_t elt = a.out_f32 ? 4 : 2;
  const int vec_ok = reinterpret_cast<uintptr_t>(a.y) % (4 * elt) == 0 && a.y_stride % 4 == 0;
  attr[0].val.clusterDim.y = (unsigned)splits;
  cfg.gridDim = dim3(n_tiles, splits, t_tiles); cfg.dynamicSmemBytes = smem;
  cfg.numAttrs = a.bank ? 2 : 1;                       // only ever overlaps this call's own down projection
  const CUtensorMap& w = reinterpret_cast<const CUtensorMap&>(tm_w);
  const CUtensorMap& x = reinterpret_cast<const CUtensorMap&>(tm_x);
  const CUtensorMap& u = reinterpret_cast<const CUtensorMap&>(tm_up);
  const LoraArgs la = lora_args(a);
  if (a.out_f32)
    return cudaLaunchKernelEx(&cfg, project_small_kernel<float>, w, x, u, a.T, a.N, num_kb, tok, npad, stages, n_acc, la, (float*)a.y, a.y_stride, vec_ok,
                              a.status);
  return cudaLaunchKernelEx(&cfg, project_small_kernel<__nv_bfloat16>, w, x, u, a.T, a.N, num_kb, tok, npad, stages, n_acc, la, (__nv_bfloat16*)a.y, a.y_stride,
                            vec_ok, a.status);
}

cudaError_t launch_project_large(const ProjectArgs& a, const GemmTensorMap& tm_w, const GemmTensorMap& tm_x, const GemmTensorMap& tm_up,
                                 int n_sms, cudaStream_t s) {
  int dev = 0;
  cudaError_t e = device_slot(&dev);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.blockDim = dim3(kLargeThreads, 1, 1); cfg.dynamicSmemBytes = kLargeSmem; cfg.stream = s; cfg.attrs = attr;
  if (g_large_clusters[dev] == 0) {
    e = cudaFuncSetAttribute(project_large_kernel<__nv_bfloat16>, cudaFuncAttributeMaxDynamicSharedMemorySize, kLargeSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(project_large_kernel<float>, cudaFuncAttributeMaxDynamicSharedMemorySize, kLargeSmem);
    if (e != cudaSuccess) return e;
    cfg.gridDim = dim3(n_sms & ~1, 1, 1); cfg.numAttrs = 1;
    int n = 0;
    e = cudaOccupancyMaxActiveClusters(&n, project_large_kernel<__nv_bfloat16>, &cfg);
    if (e != cudaSuccess) return e;
    g_large_clusters[dev] = n + 1;
  }
  const int resident = g_large_clusters[dev] - 1;
  if (resident < 1) return cudaErrorNotSupported;
  const int m_tiles = (a.T + kLargeTok - 1) / kLargeTok, n_blocks = (a.N + 255) / 256, num_kb = (a.K + 63) / 64;
  const long long total = (long long)m_tiles * n_blocks;
  if (total > (1ll << 30)) return cudaErrorInvalidValue;
  if (!a.bank) {                                       // (the down projection zeroes the counter)
    e = cudaMemsetAsync(a.tile_counter, 0, sizeof(int32_t), s);
    if (e != cudaSuccess) return e;
  }
  cfg.gridDim = dim3(2 * (unsigned)(total < resident ? total : resident), 1, 1);
  cfg.numAttrs = a.bank ? 2 : 1;
  const int n_group = n_group_for(n_blocks, 256, a.K, 2);
  const size_t elt = a.out_f32 ? 4 : 2;
  const int vec_ok = reinterpret_cast<uintptr_t>(a.y) % 16 == 0 && (size_t)a.y_stride * elt % 16 == 0;
  const CUtensorMap& w = reinterpret_cast<const CUtensorMap&>(tm_w);
  const CUtensorMap& x = reinterpret_cast<const CUtensorMap&>(tm_x);
  const CUtensorMap& u = reinterpret_cast<const CUtensorMap&>(tm_up);
  const LoraArgs la = lora_args(a);
  const int slab_steps = a.out_f32 ? kSlabSteps : num_kb;
  if (a.out_f32)
    return cudaLaunchKernelEx(&cfg, project_large_kernel<float>, w, x, u, a.T, a.N, num_kb, slab_steps, m_tiles, n_blocks, n_group, la, (float*)a.y, a.y_stride,
                              vec_ok, a.tile_counter, a.status);
  return cudaLaunchKernelEx(&cfg, project_large_kernel<__nv_bfloat16>, w, x, u, a.T, a.N, num_kb, slab_steps, m_tiles, n_blocks, n_group, la, (__nv_bfloat16*)a.y,
                            a.y_stride, vec_ok, a.tile_counter, a.status);
}

}  // namespace cep
