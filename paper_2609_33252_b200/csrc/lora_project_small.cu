// The shared projection with the adapters' up projection inside its accumulator, for short batches (for long ones:
// lora_project_large.cu):
//
//   y[t,n] = sum_k x[t,k] W[n,k] + sum_r s[t,r] B_a[n,r],   a = adapter of token t, s = scale_a * A_a x (lora_shrink.cu)
//
// The adapters are further K steps of the same matrix product: for every 32 ranks of the adapters present among the tokens
// one more step multiplies the tokens' rows of s (rows of other adapters: zeros) with the adapter's columns of B.  So the up
// projection adds neither a pass over y nor a rounding of it.  s is fp32; the tensor core takes it as the sum of two bf16
// terms (value and remainder, 2^-17 relative), two MMAs against the same columns of B.  An fp32 output takes three terms
// (2^-25) and a step per 16 ranks: the same error as without adapters, for 1000 tokens of 7168 -> 7168 with 24 adapters in
// every tile 240 us instead of 194, for 519 of 2048 -> 2048 with nine 26.9 instead of 26.2.
//
// A short batch is bound by reading W once.  W is the M side of the MMA (128 columns of y), up to 128 tokens the N side, so a
// token costs a column of the accumulator and not a row of 128; K is split over the CTAs of a cluster so that W streams
// through as many SMs as there are, and the CTAs exchange their partial sums through shared memory, each adding a share of
// the tokens in split order (the result does not depend on timing).  Warp-specialised, TMA-fed, fp32 accumulators in tensor
// memory, every wait bounded (status word).
//
// The tensor core's fp32 additions truncate: one chain over K = 7168 ends 8e-6 low on average (measured), which a bf16
// output does not see and an fp32 output does.  fp32 outputs are summed from several accumulators of about 768 products,
// at most 1024; where K needs more chains than there are accumulators, the epilogue's warps empty them on the way.
#include <cuda.h>
#include <cuda_bf16.h>

#include "lora_device.cuh"

namespace cep {
namespace {

using namespace ptx;

constexpr int kSmallThreads = 192;
constexpr int kSmallMaxStages = 12;
constexpr int kBatch = 2;                              // (64 tokens, 24 adapters: 36.3 us with two, 37.2 with four)
constexpr int kMaxSplits = 8;                          // CTAs of a portable cluster
constexpr int kMostF32 = 64;                           // token columns of a tile with fp32 outputs
constexpr int kLongestChain = 16;                      // K steps of a chain of an fp32 output
constexpr int kWStage = 128 * kKBytes;                 // 16 KiB of weight
constexpr int kSmallRing = 200 * 1024;
constexpr int kSharedRing = 136 * 1024;               // the same beside a block of the down projection
constexpr int stage_bytes_for(int npad) { return kWStage + npad * kKBytes; }
constexpr int stages_for(int ring, int npad) { return ring / stage_bytes_for(npad) < kSmallMaxStages ? ring / stage_bytes_for(npad) : kSmallMaxStages; }
constexpr int smem_for(int ring, int npad) { return 1024 + stages_for(ring, npad) * stage_bytes_for(npad) + 512; }
constexpr int least_smem(int ring) {
  int least = smem_for(ring, 16);
  for (int npad = 32; npad <= kSmallTok; npad += 16) least = smem_for(ring, npad) < least ? smem_for(ring, npad) : least;
  return least;
}
// With adapters and few tokens the ring leaves room for a block of the down projection, so that both run at once, and takes
// half of the tensor memory; a block that needs more of that takes the whole of the SM's shared memory instead.
constexpr int kSharedColumns = kSmTmemColumns / 2;
static_assert(least_smem(kSharedRing) >= kLeastTmemBlock && alone_on_its_sm(least_smem(kSmallRing)), "blocks that share an SM");
struct __align__(8) SmallBarriers {
  uint64_t full[kSmallMaxStages], empty[kSmallMaxStages], ready[kSmallMaxStages], sfull[kSmallMaxStages], acc_full, acc_empty;
  uint32_t tmem_base;
  int abort_flag;
};
static_assert(sizeof(SmallBarriers) <= 512, "barrier block");

// A warp's share of the tokens first, first + kWarps, ...: adds the cluster's sums in split order and stores, four columns of y
// per lane.  kTogether tokens are read at once, as a remote read takes 0.3 us whatever it brings.  Only what is used is read:
// the barrier behind this does not wait for a read whose value nothing needs, and the CTA read from could be gone by then.
template <int kSplits, int kTogether, typename OT>
__device__ __forceinline__ void add_splits(uint32_t base, int splits, int first, int end, int t0, int n0, int N, OT* __restrict__ y,
                                           int64_t y_stride, int vec_ok) {
  constexpr int kWarps = kSmallThreads / 32;
  const int lane = threadIdx.x & 31, left = N - n0 - lane * 4;
  for (int c = first; c < end; c += kTogether * kWarps) {
    float4 v[kTogether][kSplits];
#pragma unroll
    for (int u = 0; u < kTogether; ++u)
#pragma unroll
      for (int s = 0; s < kSplits; ++s)
        if (s < splits && c + u * kWarps < end && left > 0) v[u][s] = ld_cluster_f4(mapa(base + (uint32_t)(((c + u * kWarps) * 128 + lane * 4) * 4), (uint32_t)s));
#pragma unroll
    for (int u = 0; u < kTogether; ++u) {
      if (c + u * kWarps >= end || left <= 0) break;
      float4 o = v[u][0];
#pragma unroll
      for (int s = 1; s < kSplits; ++s)
        if (s < splits) { o.x += v[u][s].x; o.y += v[u][s].y; o.z += v[u][s].z; o.w += v[u][s].w; }
      OT* row = y + (size_t)(t0 + c + u * kWarps) * y_stride + n0 + lane * 4;
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
  }
}

// Grid (column tiles, K splits, token tiles of `tok`).  npad: token columns of the MMA, a multiple of 16.  chains: accumulation
// chains that share the CTA's K steps, in turn in n_acc accumulators of npad columns.  kEmpty: more chains than accumulators;
// the epilogue's warps then carry sums beside their rows of s, and with those registers the block would leave no room for one of
// the down projection (128 tokens of 7168 -> 2048 with eight adapters 30.7 us, without 25.0), so that is a kernel of its own.
template <typename OT, bool kEmpty>
__global__ void __launch_bounds__(kSmallThreads, 1)
project_small_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_x,
                     const __grid_constant__ CUtensorMap tm_up, int T, int N, int num_kb, int tok, int npad, int stages, int n_acc, int chains, int tmem_cols, const LoraArgs la,
                     OT* __restrict__ y, int64_t y_stride, int vec_ok, int32_t* __restrict__ status) {
  constexpr int kStep = UpStep<OT>::kChunks, kTerms = UpStep<OT>::kTerms;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const int x_stage = npad * kKBytes, stage_bytes = kWStage + x_stage;
  SmallBarriers* bars = reinterpret_cast<SmallBarriers*>(smem + stages * stage_bytes);
  volatile int* abort_flag = &bars->abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int n0 = blockIdx.x * 128, t0 = blockIdx.z * tok;
  const int split = blockIdx.y, splits = gridDim.y;
  const int kb0 = (int)((long long)num_kb * split / splits), kb1 = (int)((long long)num_kb * (split + 1) / splits);

  // The K steps of x and W do not depend on the down projection: they start before it has finished.  Without one the launch
  // before this is whatever wrote x.
  if (!la.has) pdl_wait();
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
    mbar_init(smem_u32(&bars->acc_full), 1); mbar_init(smem_u32(&bars->acc_empty), 4);
    bars->abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    // the ring is empty: its first loads go out before the rest of the block is set up
    for (int s = 0; s < stages && kb0 + s < kb1; ++s) load_k_step(kb0 + s, s);
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32(&bars->tmem_base)), "r"(tmem_cols) : "memory");
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
        const int32_t* list = la.chunks + (size_t)t0 * kLoraMaxChunks;
        const int cap = tok * kLoraMaxChunks;
        int total = cap;                               // (until it is read)
        for (int c0 = split * kStep; ok && c0 < total;) {
          int2 e[kLookAhead];
#pragma unroll
          for (int j = 0; j < kLookAhead; ++j) e[j] = list_step<kStep>(list, c0 + j * splits * kStep, cap);
          total = __ldcg(la.n_chunks + blockIdx.z);
#pragma unroll
          for (int j = 0; j < kLookAhead; ++j) e[j] = up_to(e[j], c0 + j * splits * kStep, total);
#pragma unroll
          for (int j = 0; j < kLookAhead; ++j) {
            if (e[j].x < 0) break;
            if (!mbar_wait(smem_u32(&bars->empty[stage]), phase ^ 1u, abort_flag, status)) { ok = false; break; }
            const uint32_t full = smem_u32(&bars->full[stage]);
            uint8_t* st = smem + stage * stage_bytes;
            mbar_expect_tx(full, (e[j].y < 0 ? 1 : 2) * kUpBytes);
            mbar_arrive(smem_u32(&bars->ready[stage]));
            tma_load_3d(smem_u32(st), &tm_up, 0, n0, up_block(e[j].x, la.rank_pad), full);
            if (e[j].y >= 0) tma_load_3d(smem_u32(st + kUpBytes), &tm_up, 0, n0, up_block(e[j].y, la.rank_pad), full);
            if (++stage == stages) { stage = 0; phase ^= 1u; }
          }
          c0 += kLookAhead * splits * kStep;
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t idesc = make_idesc_bf16(128, npad);
      int stage = 0; uint32_t phase = 0;
      bool ok = true;
      int chain = 0, acc = 0, chain_end = kb0 + (kb1 - kb0) / chains;      // the chain ends before K step chain_end
      uint32_t first = 1, emptied = 0;
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!mbar_wait(smem_u32(&bars->full[stage]), phase, abort_flag, status)) { ok = false; break; }
        tc_fence_after();
        if (kb == chain_end) {
          ++chain; chain_end = kb0 + (int)((long long)(kb1 - kb0) * (chain + 1) / chains); first = 1;
          if (++acc == n_acc && kEmpty) {                // all in use
            acc = 0;
            tc_commit(smem_u32(&bars->acc_full));
            if (!mbar_wait(smem_u32(&bars->acc_empty), emptied, abort_flag, status)) { ok = false; break; }
            emptied ^= 1u;
            tc_fence_after();
          }
        }
        const uint32_t d = tmem + (uint32_t)(acc * npad);
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
        const int total = __ldcg(la.n_chunks + blockIdx.z);
        const uint32_t last_acc = tmem + (uint32_t)(acc * npad);
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
            const uint64_t sdesc = make_smem_desc(up + kWStage) + (uint64_t)(i * 2 * kTerms);
#pragma unroll
            for (int t = 0; t < kTerms; ++t) tc_mma_f16(last_acc, udesc, sdesc + 2 * t, idesc, 1u);
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
    const int cols = min(tok, T - t0);                 // token columns that exist
    const uint32_t taddr = tmem + ((uint32_t)(lane_grp * 32) << 16);
    bool ok = true;
    // Columns c..c+15 of this lane: d = accumulator a, or d += it.
    auto take_accumulator = [&](int a, int c, float (&d)[16], bool add) {
      __syncwarp();                                    // the load is warp-collective
      uint32_t e[16];
      tc_ld16(taddr + a * npad + c, e);
      tc_wait_ld();
#pragma unroll
      for (int i = 0; i < 16; ++i) d[i] = add ? d[i] + __uint_as_float(e[i]) : __uint_as_float(e[i]);
    };
    constexpr int kSums = kEmpty ? kMostF32 / 16 : 1;
    float sum[kSums][16];                              // kEmpty: the sum of the chains before the last accumulators'
    uint32_t full = 0;
    int left = chains;                                 // not yet added
    if (!la.has && tid == 0) pdl_release();
    if constexpr (kEmpty) {
#pragma unroll
      for (int q = 0; q < kSums; ++q)
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[q][i] = 0.f;
      for (; left > n_acc; left -= n_acc) {
        ok = ok && mbar_wait_relaxed(smem_u32(&bars->acc_full), full, abort_flag, status);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        full ^= 1u;
        tc_fence_after();
#pragma unroll
        for (int q = 0; q < kSums; ++q)
          if (q * 16 < cols)
            for (int a = 0; a < n_acc; ++a) take_accumulator(a, q * 16, sum[q], true);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bars->acc_empty));
      }
    }
    if (la.has) {
      pdl_wait();
      if (tid == 0) pdl_release();
      const int32_t* list = la.chunks + (size_t)t0 * kLoraMaxChunks;
      const int cap = tok * kLoraMaxChunks;
      int2 e = list_step<kStep>(list, (split + lane * splits) * kStep, cap);      // lane i: the i-th of the next 32 steps
      const int total = __ldcg(la.n_chunks + blockIdx.z);
      SRow<kEmpty ? 1 : 4, kTerms> row;
      row.fetch(la, tid < npad && t0 + tid < T ? t0 + tid : -1);
      int stage = (kb1 - kb0) % stages;                // where the K steps end
      uint32_t phase = 0;                              // one parity bit per stage
      int step = 0;
      for (int c0 = split * kStep; ok && c0 < total;) {
        const int first = stage;
        int n = 0;
        for (; n < kBatch && c0 < total; ++n, c0 += splits * kStep, ++step) {
          if ((step & 31) == 0) e = up_to(step == 0 ? e : list_step<kStep>(list, c0 + lane * splits * kStep, cap), c0 + lane * splits * kStep, total);
          const int v0 = __shfl_sync(0xffffffffu, e.x, step & 31), v1 = __shfl_sync(0xffffffffu, e.y, step & 31);
          ok = mbar_wait(smem_u32(&bars->ready[stage]), (phase >> stage) & 1u, abort_flag, status);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          phase ^= 1u << stage;
          uint8_t* rows = smem + stage * stage_bytes + kWStage;
          if (tid < npad) {
            row.put(rows, tid, 0, v0);
            if (v1 >= 0) row.put(rows, tid, 1, v1);
          }
          if (++stage == stages) stage = 0;
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0)
          for (int i = 0, s = first; i < n; ++i) { mbar_arrive(smem_u32(&bars->sfull[s])); if (++s == stages) s = 0; }
      }
    }
    const bool got = ok && mbar_wait_relaxed(smem_u32(&bars->acc_full), full, abort_flag, status);
    const bool all = __all_sync(0xffffffffu, got);
    float* mine = reinterpret_cast<float*>(smem) + lane_grp * 32 + lane;       // [token][128] sums, in the ring: every load has been consumed
    if (all) {
      tc_fence_after();
      auto finish = [&](int c, float (&d)[16]) {
        take_accumulator(0, c, d, kEmpty);
        for (int a = 1; a < left; ++a) take_accumulator(a, c, d, true);
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (c + i < cols) mine[(c + i) * 128] = d[i];
      };
      if constexpr (kEmpty) {
#pragma unroll
        for (int q = 0; q < kSums; ++q)
          if (q * 16 < cols) finish(q * 16, sum[q]);
      } else {
        for (int c = 0; c < cols; c += 16) finish(c, sum[0]);
      }
    }
  }
  {
    // (a CTA that gave up still takes both barriers; its sums are then meaningless and the status word says so)
    if (splits > 1) cluster_sync_all(); else __syncthreads();
    const int cols = min(tok, T - t0);
    const int c0 = cols * split / splits, c1 = cols * (split + 1) / splits;
    const uint32_t base = smem_u32(smem);
    const bool several = c1 - c0 > kSmallThreads / 32;                // more than one token per warp
    if (splits <= 2 && several) add_splits<2, 4>(base, splits, c0 + warp, c1, t0, n0, N, y, y_stride, vec_ok);
    else add_splits<kMaxSplits, 1>(base, splits, c0 + warp, c1, t0, n0, N, y, y_stride, vec_ok);
    if (splits > 1) cluster_sync_reads();              // no CTA leaves while another reads its sums
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(tmem_cols) : "memory");
  }
}

// ------------------------------------------------------------------ host side
constexpr int kMaxDevices = 64;
int g_clusters[kMaxDevices][kMaxSplits + 1];           // co-resident clusters by size; [0]: set up

struct Plan { int npad, tok, n_tiles, t_tiles, num_kb, splits; long long cost; };

// The cluster size with the least work for the busiest SM, in K steps: a cluster needs that many free SMs in one GPC, so
// fewer SMs are usable for some sizes.
Plan plan(const int* clusters, int T, int N, int K, int out_f32) {
  constexpr long long kExchange = 6;                   // what the exchange of partial sums costs (2 us)
  constexpr long long kStart = 5;                      // a round's start and end
  Plan p{};
  p.npad = project_small_tokens(T, out_f32); p.tok = project_small_tile(out_f32);
  p.n_tiles = (N + 127) / 128; p.t_tiles = (T + p.tok - 1) / p.tok; p.num_kb = (K + 63) / 64;
  const long long tiles = (long long)p.n_tiles * p.t_tiles;
  p.splits = 1; p.cost = 1ll << 60;
  for (int c = 1; c <= kMaxSplits && c <= p.num_kb; ++c) {
    if (clusters[c] < 2) continue;
    // (of clusters of odd size a few fewer run at once than the occupancy query says: 48 of three took two rounds)
    const long long at_once = c > 1 && c % 2 ? clusters[c] * 15 / 16 : clusters[c];
    const long long cost = (tiles + at_once - 1) / at_once * ((p.num_kb + c - 1) / c + kStart) + (c > 1 ? kExchange : 0) - kStart;
    if (cost < p.cost) { p.cost = cost; p.splits = c; }
  }
  return p;
}

}  // namespace

int project_small_tile(int out_f32) { return out_f32 ? kMostF32 : kSmallTok; }       // (8 accumulators of 64 columns fill the tensor memory)
int project_small_tokens(int T, int out_f32) { return T >= project_small_tile(out_f32) ? project_small_tile(out_f32) : (T + 15) / 16 * 16; }

cudaError_t project_small_setup(int dev) {
  if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
  int* clusters = g_clusters[dev];
  if (clusters[0]) return cudaSuccess;
  cudaError_t e = cudaFuncSetAttribute(project_small_kernel<__nv_bfloat16, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmallRing + 2048);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(project_small_kernel<float, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmallRing + 2048);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(project_small_kernel<float, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmallRing + 2048);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 1; attr[0].val.clusterDim.z = 1;
  cfg.blockDim = dim3(kSmallThreads, 1, 1); cfg.dynamicSmemBytes = kSmallRing + 2048; cfg.attrs = attr; cfg.numAttrs = 1;
  for (int c = 1; c <= kMaxSplits; ++c) {
    attr[0].val.clusterDim.y = (unsigned)c;
    cfg.gridDim = dim3(kSms, c, 1);
    e = cudaOccupancyMaxActiveClusters(&clusters[c], project_small_kernel<__nv_bfloat16, false>, &cfg);
    if (e != cudaSuccess) return e;
  }
  clusters[0] = 1;
  return cudaSuccess;
}

long long project_small_cost(int dev, int T, int N, int K, int out_f32) { return plan(g_clusters[dev], T, N, K, out_f32).cost; }

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
                                 int dev, cudaStream_t s) {
  const Plan p = plan(g_clusters[dev], a.T, a.N, a.K, a.out_f32);
  const int steps = p.num_kb / p.splits;               // K steps a CTA has at least
  // Chains of kSlabSteps K steps, or of up to kLongestChain where the accumulators then suffice.
  int chains = a.out_f32 ? (steps + kSlabSteps - 1) / kSlabSteps : 1;
  int n_acc = kSmTmemColumns / p.npad;
  if (chains <= n_acc) n_acc = chains;
  else if ((p.num_kb + p.splits - 1) / p.splits <= n_acc * kLongestChain) chains = n_acc;
  int tmem_cols = 32;
  while (tmem_cols < n_acc * p.npad) tmem_cols *= 2;
  const int ring = a.bank && lora_beside(a.T) && tmem_cols <= kSharedColumns ? kSharedRing : kSmallRing;
  const int stages = stages_for(ring, p.npad);
  const size_t elt = a.out_f32 ? 4 : 2;
  const int vec_ok = reinterpret_cast<uintptr_t>(a.y) % (4 * elt) == 0 && a.y_stride % 4 == 0;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 1; attr[0].val.clusterDim.y = (unsigned)p.splits; attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = dim3(p.n_tiles, p.splits, p.t_tiles); cfg.blockDim = dim3(kSmallThreads, 1, 1);
  cfg.dynamicSmemBytes = smem_for(ring, p.npad); cfg.stream = s; cfg.attrs = attr;
  cfg.numAttrs = 2;
  const CUtensorMap& w = reinterpret_cast<const CUtensorMap&>(tm_w);
  const CUtensorMap& x = reinterpret_cast<const CUtensorMap&>(tm_x);
  const CUtensorMap& u = reinterpret_cast<const CUtensorMap&>(tm_up);
  const LoraArgs la = lora_args(a);
  if (a.out_f32)
    return cudaLaunchKernelEx(&cfg, chains > n_acc ? project_small_kernel<float, true> : project_small_kernel<float, false>, w, x, u, a.T, a.N, p.num_kb, p.tok, p.npad, stages, n_acc, chains, tmem_cols, la, (float*)a.y, a.y_stride,
                              vec_ok, a.status);
  return cudaLaunchKernelEx(&cfg, project_small_kernel<__nv_bfloat16, false>, w, x, u, a.T, a.N, p.num_kb, p.tok, p.npad, stages, n_acc, chains, tmem_cols, la,
                            (__nv_bfloat16*)a.y, a.y_stride, vec_ok, a.status);
}

}  // namespace cep
