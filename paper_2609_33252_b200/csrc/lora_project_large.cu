// The shared projection with the adapters' up projection inside its accumulator, for long batches (the formula and the
// adapters' steps: lora_project_small.cu).
//
// CTA pairs on 256 tokens x 256 columns (tcgen05 cta_group::2: each CTA loads its 128 tokens and half of the columns), fp32
// accumulators in tensor memory, two of them so that a tile's epilogue overlaps the next tile's K steps.  Tiles go out from a
// counter in an order that keeps a group of column blocks in the L2.  A batch whose tiles do not fill the last round of CTA
// pairs would leave most SMs idle for a whole tile; those tiles go to a second launch of the same kernel that splits K over
// the CTA pairs of a cluster (kSplit), which exchange partial sums through shared memory and add them in order.  The same
// kernel with one split takes a batch that is less than a round: one tile per pair needs no counter, and whole rows leave from
// shared memory (300 tokens of 7168x7168: 43 us against 48).
//
// fp32 outputs are summed from chains of kSlabSteps K steps (the tensor core's additions truncate): the epilogue keeps the
// running sum in registers, which takes the s-row warps as a second half of the epilogue.
#include <cuda.h>
#include <cuda_bf16.h>

#include "lora_device.cuh"

namespace cep {
namespace {

using namespace ptx;

constexpr int kStages = 6;
constexpr int kHalf = 128 * kKBytes;                   // one CTA's 128 rows of either operand: 16 KiB
constexpr int kRing = 4;                               // tile ids in flight
constexpr int kPoison = -2;
constexpr int kAsk = 10;                               // K steps before a tile's end at which the next id is fetched
constexpr int kThreads = 352;                          // warp 0 loads, 1 MMA, 2-5 epilogue, 6 tile ids, 7-10 rows of s
constexpr int kReaders = 19;                           // leader: loads, MMA, 4 epilogue, 4 s-row warps; peer: loads, 4, 4
constexpr int kBatch = 4;                              // (1000 tokens, 24 adapters in every tile: 157 us with four, 164 with two)
constexpr int kMaxSplits = 4;                          // CTA pairs of a portable cluster
constexpr int kPitch = 260;                            // floats per row of exchanged sums: rows four banks apart
struct __align__(8) Barriers {
  uint64_t full[kStages], empty[kStages], ready[kStages], sfull[kStages], acc_full[2], acc_empty[2];
  uint64_t ring_full[kRing], ring_empty[kRing], want;
  int32_t ring_tile[kRing];
  uint32_t tmem_base;
  int abort_flag;
};
static_assert(sizeof(Barriers) <= 512, "barrier block");
constexpr int kSmem = kStages * 2 * kHalf + 512 + 1024;
static_assert(alone_on_its_sm(kSmem), "takes all of the tensor memory");
static_assert(kSmem <= 227 * 1024 && 128 * kPitch * 4 <= kStages * 2 * kHalf, "shared memory");

// The tiles of a CTA pair, in the order every role of it walks them: from the ring of ids that the leader's warp 6 fills in
// both CTAs, or (kSplit) the one tile of the cluster.  -1 ends.
template <bool kSplit>
struct Tiles {
  int slot = 0; uint32_t phase = 0;
  int one;
  __device__ __forceinline__ explicit Tiles(int only) : one(only) {}
  __device__ __forceinline__ int next(Barriers* bars, bool is_peer, volatile int* abort_flag, int32_t* status) {
    if (kSplit) { const int t = one; one = -1; return t; }
    const uint32_t bar = smem_u32(&bars->ring_full[slot]);
    const bool ok = is_peer ? mbar_wait_acq_cluster(bar, phase, abort_flag, status) : mbar_wait_relaxed(bar, phase, abort_flag, status);
    if (!ok) return -1;
    const int t = *reinterpret_cast<volatile int32_t*>(&bars->ring_tile[slot]);
    if (t < -1) { atomicExch(&status[kStTimeout], 1); *abort_flag = 1; return -1; }
    return t;
  }
  __device__ __forceinline__ void done(Barriers* bars, bool signal) {
    if (kSplit) return;
    if (signal) mbar_arrive_cluster(mapa(smem_u32(&bars->ring_empty[slot]), 0));
    if (++slot == kRing) { slot = 0; phase ^= 1u; }
  }
};

struct Shape {
  int T, N, num_kb, slab_steps, m_tiles, n_blocks, n_group;
  int tile0, n_tiles;                                  // the tiles of this launch
};
// Linear tile -> (token tile, column block): column blocks in groups whose weight panel stays in the L2, each group swept
// over all token tiles with the column block as the fast index.
__device__ __forceinline__ void tile_at(const Shape& sh, int tile, int* m, int* nb) {
  const int g = tile / (sh.m_tiles * sh.n_group);
  const int rem = tile - g * sh.m_tiles * sh.n_group;
  const int gn = min(sh.n_group, sh.n_blocks - g * sh.n_group);
  *m = rem / gn;
  *nb = g * sh.n_group + rem % gn;
}

// 4 consecutive values of y, the first at column n of N
template <typename OT>
__device__ __forceinline__ void put4(OT* p, float4 v, int left, bool vec_ok) {
  if (left >= 4 && vec_ok) {
    if (sizeof(OT) == 2) *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
    else *reinterpret_cast<float4*>(p) = v;
    return;
  }
  if (left > 0) put_out(p, v.x);
  if (left > 1) put_out(p + 1, v.y);
  if (left > 2) put_out(p + 2, v.z);
  if (left > 3) put_out(p + 3, v.w);
}

// kLora: the call may have adapters.  (Without, an fp32 output's running sums fit the registers.)
template <typename OT, bool kSplit, bool kLora>
__global__ void __launch_bounds__(kThreads, 1)
project_large_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_x,
                     const __grid_constant__ CUtensorMap tm_up, const Shape sh, int splits, int after_peer, const LoraArgs la_, OT* __restrict__ y,
                     int64_t y_stride, int vec_ok, int32_t* __restrict__ tile_counter, int32_t* __restrict__ status) {
  constexpr bool kF32 = sizeof(OT) == 4;
  // (without adapters neither is of use, but with those of fp32 the compiler spills registers: 2048 tokens of 7168 -> 256 21.0 -> 22.8 us)
  constexpr int kStep = kLora ? UpStep<OT>::kChunks : 2, kTerms = kLora ? UpStep<OT>::kTerms : 2;
  constexpr bool kBothHalves = kF32 || kSplit;           // the s-row warps read half of the accumulator
  LoraArgs la = la_;
  if (!kLora) la.has = 0;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* smem_x = smem;
  uint8_t* smem_w = smem + kStages * kHalf;
  Barriers* bars = reinterpret_cast<Barriers*>(smem_w + kStages * kHalf);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t crank = cluster_ctarank(), lead = crank & ~1u;         // this pair's leader in the cluster
  const int half = (int)(crank & 1u), part = (int)(crank >> 1);
  const bool is_peer = half != 0;
  const uint16_t both = (uint16_t)(3u << lead);
  volatile int* abort_flag = &bars->abort_flag;
  const int only = kSplit ? sh.tile0 + (int)blockIdx.x / (2 * splits) : -1;
  // this pair's K steps, and its steps of the up projection: every splits-th
  const int kb0 = kSplit ? (int)((long long)sh.num_kb * part / splits) : 0;
  const int kb1 = kSplit ? (int)((long long)sh.num_kb * (part + 1) / splits) : sh.num_kb;
  const int c_first = part * kStep, c_stride = (kSplit ? splits : 1) * kStep;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(smem_u32(&bars->full[s]), 1); mbar_init(smem_u32(&bars->empty[s]), 1);
      mbar_init(smem_u32(&bars->ready[s]), 1); mbar_init(smem_u32(&bars->sfull[s]), 8);
    }
    for (int s = 0; s < 2; ++s) { mbar_init(smem_u32(&bars->acc_full[s]), 1); mbar_init(smem_u32(&bars->acc_empty[s]), kBothHalves ? 16 : 8); }
    for (int s = 0; s < kRing; ++s) {
      mbar_init(smem_u32(&bars->ring_full[s]), 1); mbar_init(smem_u32(&bars->ring_empty[s]), kReaders);
      bars->ring_tile[s] = kPoison;
    }
    mbar_init(smem_u32(&bars->want), 1);
    bars->abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (threadIdx.x == 64) { prefetch_map(&tm_x); prefetch_map(&tm_w); }
  if (!la.has && !after_peer) pdl_wait();                // (what wrote x)
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
  // What precedes this launch may be the down projection.  The K steps do not need it and start at once (it began after what
  // wrote x had ended); who reads its lists and s waits for it.  Or (after_peer) the launch with the full rounds of tiles, which
  // touches nothing of this one's and let it start only after the down projection's end.
  const bool wait = la.has && !after_peer;
  if (wait ? warp >= 7 : true) {
    if (wait) pdl_wait();
    if (threadIdx.x == 7 * 32) pdl_release();
  }

  if (warp == 0) {
    // ---------------------------------------------------------------- TMA loads (both CTAs)
    if (lane == 0) {
      int stage = 0; uint32_t phase = 0;
      bool ok = true;
      Tiles<kSplit> tiles(only);
      while (ok) {
        const int tile = tiles.next(bars, is_peer, abort_flag, status);
        tiles.done(bars, true);
        if (tile < 0) break;
        int m, nb;
        tile_at(sh, tile, &m, &nb);
        const int t0 = m * kLargeTok + half * 128, n0 = nb * 256 + half * 128;
        const int ask = max(kb0, kb1 - kAsk);
        for (int kb = kb0; kb < kb1; ++kb) {
          if (!mbar_wait(smem_u32(&bars->empty[stage]), phase ^ 1u, abort_flag, status)) { ok = false; break; }
          const uint32_t full = mapa(smem_u32(&bars->full[stage]), lead);
          if (!is_peer) mbar_expect_tx(smem_u32(&bars->full[stage]), 4 * kHalf);       // both CTAs' bytes
          tma_load_2d_pair(smem_u32(smem_x + stage * kHalf), &tm_x, kb * (kKBytes / 2), t0, full);
          tma_load_2d_pair(smem_u32(smem_w + stage * kHalf), &tm_w, kb * (kKBytes / 2), n0, full);
          if (++stage == kStages) { stage = 0; phase ^= 1u; }
          if (!kSplit && !is_peer && kb == ask) mbar_arrive(smem_u32(&bars->want));
        }
        if (wait) pdl_wait();
        const int total = la.has ? __ldcg(la.n_chunks + m) : 0;
        const int32_t* list = la.chunks + (size_t)m * kLargeTok * kLoraMaxChunks;
        for (int c0 = c_first; ok && c0 < total; c0 += kLookAhead * c_stride) {
          int2 e[kLookAhead];
#pragma unroll
          for (int j = 0; j < kLookAhead; ++j) e[j] = up_to(list_step<kStep>(list, c0 + j * c_stride, kLargeTok * kLoraMaxChunks), c0 + j * c_stride, total);
#pragma unroll
          for (int j = 0; j < kLookAhead; ++j) {
            if (e[j].x < 0) break;
            if (!mbar_wait(smem_u32(&bars->empty[stage]), phase ^ 1u, abort_flag, status)) { ok = false; break; }
            const uint32_t full = mapa(smem_u32(&bars->full[stage]), lead);
            if (!is_peer) mbar_expect_tx(smem_u32(&bars->full[stage]), (e[j].y < 0 ? 2 : 4) * kUpBytes);
            mbar_arrive(smem_u32(&bars->ready[stage]));
            uint8_t* st = smem_w + stage * kHalf;
            tma_load_3d_pair(smem_u32(st), &tm_up, 0, n0, up_block(e[j].x, la.rank_pad), full);
            if (e[j].y >= 0) tma_load_3d_pair(smem_u32(st + kUpBytes), &tm_up, 0, n0, up_block(e[j].y, la.rank_pad), full);
            if (++stage == kStages) { stage = 0; phase ^= 1u; }
          }
        }
      }
    }
  } else if (warp == 1) {
    // ---------------------------------------------------------------- MMA issuer (leaders only)
    if (lane == 0 && !is_peer) {
      constexpr uint32_t idesc = make_idesc_bf16(256, 256);
      int stage = 0; uint32_t phase = 0;
      int acc = 0; uint32_t acc_phase = 0;
      uint32_t sphase = 0;                               // one parity bit per stage
      bool ok = true;
      Tiles<kSplit> tiles(only);
      while (ok) {
        const int tile = tiles.next(bars, false, abort_flag, status);
        tiles.done(bars, true);
        if (tile < 0) break;
        if (!mbar_wait(smem_u32(&bars->acc_empty[acc]), acc_phase ^ 1u, abort_flag, status)) break;
        tc_fence_after();
        uint32_t d = tmem + (uint32_t)(acc * 256);
        uint32_t more = 0;                               // 0: the accumulator starts with this step
        for (int kb = kb0, left = sh.slab_steps; kb < kb1; ++kb, --left) {
          if (kF32 && left == 0) {                       // this chain is complete
            tc_commit_pair_both(smem_u32(&bars->acc_full[acc]), both);
            if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
            if (!mbar_wait(smem_u32(&bars->acc_empty[acc]), acc_phase ^ 1u, abort_flag, status)) { ok = false; break; }
            tc_fence_after();
            d = tmem + (uint32_t)(acc * 256);
            more = 0; left = sh.slab_steps;
          }
          if (!mbar_wait(smem_u32(&bars->full[stage]), phase, abort_flag, status)) { ok = false; break; }
          tc_fence_after();
          const uint64_t xdesc = make_smem_desc(smem_u32(smem_x + stage * kHalf));
          const uint64_t wdesc = make_smem_desc(smem_u32(smem_w + stage * kHalf));
#pragma unroll
          for (int k4 = 0; k4 < 4; ++k4)
            tc_mma_f16_pair(d, xdesc + (uint64_t)(k4 * 2), wdesc + (uint64_t)(k4 * 2), idesc, k4 != 0 ? 1u : more);
          more = 1;
          tc_commit_pair_both(smem_u32(&bars->empty[stage]), both);
          if (++stage == kStages) { stage = 0; phase ^= 1u; }
        }
        if (ok && la.has) {
          if (wait) pdl_wait();
          int m, nb;
          tile_at(sh, tile, &m, &nb);
          const int total = __ldcg(la.n_chunks + m);
          for (int c0 = c_first; c0 < total; c0 += c_stride) {
            if (!mbar_wait(smem_u32(&bars->full[stage]), phase, abort_flag, status) ||
                !mbar_wait_acq_cluster(smem_u32(&bars->sfull[stage]), (sphase >> stage) & 1u, abort_flag, status)) { ok = false; break; }
            sphase ^= 1u << stage;
            tc_fence_after();
            const uint64_t sdesc = make_smem_desc(smem_u32(smem_x + stage * kHalf));
            const int n = min(kStep, total - c0);
            for (int i = 0; i < n; ++i) {
              const uint64_t udesc = make_smem_desc_32b(smem_u32(smem_w + stage * kHalf) + i * kUpBytes);
              tc_mma_f16_pair(d, sdesc + (uint64_t)(i * 2 * kTerms), udesc, idesc, 1u);
              tc_mma_f16_pair(d, sdesc + (uint64_t)(i * 2 * kTerms + 2), udesc, idesc, 1u);
              if (kTerms == 3) tc_mma_f16_pair(d, sdesc + (uint64_t)(i * 2 * kTerms + 4), udesc, idesc, 1u);
            }
            tc_commit_pair_both(smem_u32(&bars->empty[stage]), both);
            if (++stage == kStages) { stage = 0; phase ^= 1u; }
          }
        }
        if (!ok) break;
        tc_commit_pair_both(smem_u32(&bars->acc_full[acc]), both);
        if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
      }
    }
  } else if (warp == 6) {
    // ---------------------------------------------------------------- tile ids (leader only)
    if (!kSplit && lane == 0 && !is_peer) {
      int slot = 0; uint32_t phase = 0;
      // The next id is fetched shortly before the loading thread needs it, not as soon as there is room for it: pairs start at
      // different times, and the first ones would take the tiles of those that start later.
      for (uint32_t n = 0;; ++n) {
        if (n > 0 && !mbar_wait_relaxed(smem_u32(&bars->want), (n - 1) & 1u, abort_flag, status)) break;
        if (!mbar_wait_relaxed(smem_u32(&bars->ring_empty[slot]), phase ^ 1u, abort_flag, status)) break;
        int t = atomicAdd(tile_counter, 1);
        t = t < sh.n_tiles ? sh.tile0 + t : -1;
        bars->ring_tile[slot] = t;
        st_shared_cluster_u32(mapa(smem_u32(&bars->ring_tile[slot]), 1), (uint32_t)t);
        mbar_arrive(smem_u32(&bars->ring_full[slot]));
        mbar_arrive_release_cluster(mapa(smem_u32(&bars->ring_full[slot]), 1));
        if (t < 0) break;
        if (++slot == kRing) { slot = 0; phase ^= 1u; }
      }
    }
  } else {
    // ---------------------------------------------------------------- rows of s (warps 7..10) and epilogue (warps 2..5; fp32
    // outputs and kSplit: 2..5 columns 0-127, 7..10 columns 128-255), both CTAs, one token per thread
    const bool s_warp = warp >= 7;
    const int lane_grp = warp & 3;                       // the tensor-memory lanes a warp may read
    const int r = threadIdx.x - 7 * 32;                  // an s-row warp's row
    int stage = 0; uint32_t phase = 0;                   // the ring, for rows of s (phase: one parity bit per stage)
    int acc = 0; uint32_t acc_phase = 0;
    bool ok = true;
    Tiles<kSplit> tiles(only);
    while (ok) {
      const int tile = tiles.next(bars, is_peer, abort_flag, status);
      __syncwarp();
      tiles.done(bars, lane == 0);
      if (!__all_sync(0xffffffffu, tile >= 0)) break;
      int m, nb;
      tile_at(sh, tile, &m, &nb);
      const int t = m * kLargeTok + half * 128 + lane_grp * 32 + lane;
      const int left = sh.N - nb * 256;                  // columns of this block that exist
      constexpr int kSum = kF32 ? 128 : 1;
      float sum[kSum];
#pragma unroll
      for (int c = 0; c < kSum; ++c) sum[c] = 0.f;
#pragma unroll 1
      for (int kb = kb0; ok && kb < kb1; kb += sh.slab_steps) {          // one accumulation chain after the other
        if (s_warp && la.has && kb + sh.slab_steps >= kb1) {
          // the adapters' steps end the last chain
          if (wait) pdl_wait();
          const int ts = m * kLargeTok + half * 128 + r;
          SRow<kF32 ? 0 : 4, kTerms> row;                // (fp32: the sums need the registers; 519 tokens with nine
                                                         // adapters 26.9 us, with one chunk ahead 29.0)
          row.fetch(la, ts < sh.T ? ts : -1);
          const int total = __ldcg(la.n_chunks + m);
          const int32_t* list = la.chunks + (size_t)m * kLargeTok * kLoraMaxChunks;
          stage = (stage + kb1 - kb0) % kStages;         // past the tile's K steps
          int2 e = make_int2(-1, -1);                    // lane i: the i-th of the next 32 steps
          int step = 0;
          for (int c0 = c_first; ok && c0 < total;) {
            const int first = stage;
            int n = 0;
            for (; n < kBatch && c0 < total; ++n, c0 += c_stride, ++step) {
              if ((step & 31) == 0) e = up_to(list_step<kStep>(list, c0 + lane * c_stride, kLargeTok * kLoraMaxChunks), c0 + lane * c_stride, total);
              const int v0 = __shfl_sync(0xffffffffu, e.x, step & 31), v1 = __shfl_sync(0xffffffffu, e.y, step & 31);
              ok = mbar_wait(smem_u32(&bars->ready[stage]), (phase >> stage) & 1u, abort_flag, status);
              ok = __all_sync(0xffffffffu, ok);
              if (!ok) break;
              phase ^= 1u << stage;
              row.put(smem_x + stage * kHalf, r, 0, v0);
              if (v1 >= 0) row.put(smem_x + stage * kHalf, r, 1, v1);
              if (++stage == kStages) stage = 0;
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0)
              for (int i = 0, s = first; i < n; ++i) {
                mbar_arrive_release_cluster(mapa(smem_u32(&bars->sfull[s]), lead));
                if (++s == kStages) s = 0;
              }
          }
        }
        if (s_warp && !kBothHalves) continue;
        ok = ok && mbar_wait_relaxed(smem_u32(&bars->acc_full[acc]), acc_phase, abort_flag, status);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tc_fence_after();
        const uint32_t taddr = tmem + ((uint32_t)(lane_grp * 32) << 16) + (uint32_t)(acc * 256);
        if constexpr (kF32) {
#pragma unroll
          for (int c = 0; c < 128; c += 16) {
            uint32_t d[16];
            tc_ld16(taddr + (s_warp ? 128 : 0) + c, d);
            tc_wait_ld();
#pragma unroll
            for (int i = 0; i < 16; ++i) sum[c + i] += __uint_as_float(d[i]);
          }
        } else {
          OT* row = y + (size_t)t * y_stride + nb * 256;
          float* sums = reinterpret_cast<float*>(smem) + (lane_grp * 32 + lane) * kPitch;   // (kSplit: the ring, all consumed)
          const int c_end = min(left, kBothHalves && !s_warp ? 128 : 256);
#pragma unroll 1
          for (int c = kBothHalves && s_warp ? 128 : 0; c < c_end; c += 32) {
            __syncwarp();                                // the load is warp-collective
            uint32_t d[32];
            tc_ld32(taddr + c, d);
            tc_wait_ld();
            if (kSplit) {
#pragma unroll
              for (int q = 0; q < 8; ++q) *reinterpret_cast<uint4*>(sums + c + 4 * q) = make_uint4(d[4 * q], d[4 * q + 1], d[4 * q + 2], d[4 * q + 3]);
            } else if (t >= sh.T) {
            } else if (vec_ok && c + 32 <= left) {
              uint4* dst = reinterpret_cast<uint4*>(row + c);
#pragma unroll
              for (int q = 0; q < 4; ++q)
                dst[q] = make_uint4(pack_bf16(__uint_as_float(d[8 * q]), __uint_as_float(d[8 * q + 1])),
                                    pack_bf16(__uint_as_float(d[8 * q + 2]), __uint_as_float(d[8 * q + 3])),
                                    pack_bf16(__uint_as_float(d[8 * q + 4]), __uint_as_float(d[8 * q + 5])),
                                    pack_bf16(__uint_as_float(d[8 * q + 6]), __uint_as_float(d[8 * q + 7])));
            } else {
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (c + i < left) put_out(row + c + i, __uint_as_float(d[i]));
            }
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(mapa(smem_u32(&bars->acc_empty[acc]), lead));
        if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
      }
      if constexpr (kF32) {
        const int c0 = s_warp ? 128 : 0;
        if (ok && kSplit) {
          float* sums = reinterpret_cast<float*>(smem) + (lane_grp * 32 + lane) * kPitch + c0;
#pragma unroll
          for (int q = 0; q < 32; ++q) *reinterpret_cast<float4*>(sums + 4 * q) = make_float4(sum[4 * q], sum[4 * q + 1], sum[4 * q + 2], sum[4 * q + 3]);
        } else if (ok && t < sh.T) {
          OT* row = y + (size_t)t * y_stride + nb * 256 + c0;
#pragma unroll
          for (int q = 0; q < 32; ++q) put4(row + 4 * q, make_float4(sum[4 * q], sum[4 * q + 1], sum[4 * q + 2], sum[4 * q + 3]), left - c0 - 4 * q, vec_ok);
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                 // no CTA leaves while another may still signal it; kSplit: the partial sums are there
  if (!kSplit && !is_peer && threadIdx.x == 0) {
    // the last pair puts the counters back (every pair has fetched its last id)
    if (atomicInc(reinterpret_cast<unsigned*>(tile_counter) + 1, gridDim.x / 2 - 1) == gridDim.x / 2 - 1) atomicExch(tile_counter, 0);
  }
  if (kSplit) {
    // this pair adds its share of the tile's rows over the cluster's pairs, in order (after a wait that ran out the sums mean
    // nothing and the status word says so)
    int m, nb;
    tile_at(sh, only, &m, &nb);
    const int t0 = m * kLargeTok + half * 128, rows = min(128, sh.T - t0);
    const int r1 = 128 * (part + 1) / splits;
    const uint32_t base = smem_u32(smem);
    const int end = min(r1, rows);
    constexpr int kWarps = kThreads / 32, kTogether = 2;  // rows read at once: a remote read takes 0.3 us whatever it brings
    const int left = sh.N - nb * 256;                     // columns that exist.  Only what is used is read: the barrier below
                                                          // does not wait for a read whose value nothing needs
    for (int r = 128 * part / splits + warp; r < end; r += kTogether * kWarps) {
      float4 v[kTogether][2][kMaxSplits];
#pragma unroll
      for (int u = 0; u < kTogether; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int p = 0; p < kMaxSplits; ++p)
            if (p < splits && r + u * kWarps < end && h * 128 + lane * 4 < left)
              v[u][h][p] = ld_cluster_f4(mapa(base + (uint32_t)(((r + u * kWarps) * kPitch + h * 128 + lane * 4) * 4), (uint32_t)(2 * p + half)));
#pragma unroll
      for (int u = 0; u < kTogether; ++u) {
        if (r + u * kWarps >= end) break;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int c = h * 128 + lane * 4;
          if (c >= left) break;
          float4 o = v[u][h][0];
#pragma unroll
          for (int p = 1; p < kMaxSplits; ++p)
            if (p < splits) { o.x += v[u][h][p].x; o.y += v[u][h][p].y; o.z += v[u][h][p].z; o.w += v[u][h][p].w; }
          put4(y + (size_t)(t0 + r + u * kWarps) * y_stride + nb * 256 + c, o, left - c, vec_ok);
        }
      }
    }
    cluster_sync_reads();             // no CTA leaves while another reads its sums
  }
  if (after_peer) pdl_wait();         // this launch ends after the one it ran beside
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(512) : "memory");
  }
}

// ------------------------------------------------------------------ host side
constexpr int kMaxDevices = 64;
int g_clusters[kMaxDevices][kMaxSplits + 1];           // co-resident clusters by CTA pairs; [0]: set up

struct Plan { int m_tiles, n_blocks, num_kb, full, rest, splits; long long cost; };

// Full rounds of tiles go to one launch, what is left over to a second one with the number of splits that has the least K
// steps for the busiest SM.  A second launch only if it saves more than it costs (kSecond).
Plan plan(const int* clusters, int T, int N, int K) {
  constexpr long long kTile = 4;                       // a tile's start and end, in K steps
  constexpr long long kExchange = 12;                  // exchanging partial sums (3.5 us)
  constexpr long long kAlone = 3;                      // one tile per pair, stored through shared memory: whole rows of 256 columns
  constexpr long long kSecond = 10;
  Plan p{};
  p.m_tiles = (T + kLargeTok - 1) / kLargeTok; p.n_blocks = (N + 255) / 256; p.num_kb = (K + 63) / 64;
  const long long total = (long long)p.m_tiles * p.n_blocks, round = clusters[1];
  const long long whole = (total + round - 1) / round * (p.num_kb + kTile);
  p.full = (int)total; p.rest = 0; p.splits = 1; p.cost = whole;
  const long long rounds = total / round, rest = total - rounds * round;
  for (int s = 1; s <= kMaxSplits && s <= p.num_kb && rest > 0; ++s) {
    if (clusters[s] < 1) continue;
    const long long cost = rounds * (p.num_kb + kTile) + (rounds > 0 ? kSecond : 0) +
                           (rest + clusters[s] - 1) / clusters[s] * ((p.num_kb + s - 1) / s + (s > 1 ? kExchange + kTile : kAlone));
    if (cost < p.cost) { p.cost = cost; p.full = (int)(rounds * round); p.rest = (int)rest; p.splits = s; }
  }
  return p;
}

template <typename OT>
cudaError_t launch(const ProjectArgs& a, const Plan& p, const CUtensorMap& w, const CUtensorMap& x, const CUtensorMap& u, int dev, cudaStream_t s) {
  const size_t elt = sizeof(OT);
  const int vec_ok = reinterpret_cast<uintptr_t>(a.y) % 16 == 0 && (size_t)a.y_stride * elt % 16 == 0;
  const LoraArgs la = lora_args(a);
  // (an fp32 output without adapters has kernels of its own, see there)
  const auto rounds = a.bank || elt == 2 ? project_large_kernel<OT, false, true> : project_large_kernel<OT, false, sizeof(OT) == 2>;
  const auto shared = a.bank || elt == 2 ? project_large_kernel<OT, true, true> : project_large_kernel<OT, true, sizeof(OT) == 2>;
  Shape sh{a.T, a.N, p.num_kb, sizeof(OT) == 4 ? kSlabSteps : p.num_kb, p.m_tiles, p.n_blocks, n_group_for(p.n_blocks, 256, a.K, 2), 0, p.full};
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.blockDim = dim3(kThreads, 1, 1); cfg.dynamicSmemBytes = kSmem; cfg.stream = s; cfg.attrs = attr;
  cfg.numAttrs = 2;
  if (p.full) {
    const int resident = g_clusters[dev][1];
    cfg.gridDim = dim3(2 * (unsigned)(p.full < resident ? p.full : resident), 1, 1);
    const cudaError_t e = cudaLaunchKernelEx(&cfg, rounds, w, x, u, sh, 1, 0, la, static_cast<OT*>(a.y), a.y_stride, vec_ok,
                                             a.tile_counter, a.status);
    if (e != cudaSuccess) return e;
  }
  if (p.rest) {                                        // after full rounds: starts on SMs as they run out of tiles
    sh.tile0 = p.full; sh.n_tiles = p.rest;
    attr[0].val.clusterDim.x = (unsigned)(2 * p.splits);
    cfg.gridDim = dim3((unsigned)(p.rest * 2 * p.splits), 1, 1);
    return cudaLaunchKernelEx(&cfg, shared, w, x, u, sh, p.splits, p.full > 0 ? 1 : 0, la, static_cast<OT*>(a.y), a.y_stride,
                              vec_ok, a.tile_counter, a.status);
  }
  return cudaSuccess;
}

}  // namespace

cudaError_t project_large_setup(int dev, int n_sms) {
  if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
  int* clusters = g_clusters[dev];
  if (clusters[0]) return cudaSuccess;
  const void* kernels[6] = {(const void*)project_large_kernel<__nv_bfloat16, false, true>, (const void*)project_large_kernel<__nv_bfloat16, true, true>,
                            (const void*)project_large_kernel<float, false, true>, (const void*)project_large_kernel<float, true, true>,
                            (const void*)project_large_kernel<float, false, false>, (const void*)project_large_kernel<float, true, false>};
  for (const void* k : kernels) {
    const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e != cudaSuccess) return e;
  }
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.blockDim = dim3(kThreads, 1, 1); cfg.dynamicSmemBytes = kSmem; cfg.attrs = attr; cfg.numAttrs = 1;
  for (int c = 1; c <= kMaxSplits; ++c) {
    attr[0].val.clusterDim.x = (unsigned)(2 * c);
    cfg.gridDim = dim3((unsigned)(n_sms / (2 * c) * 2 * c), 1, 1);
    const cudaError_t e = cudaOccupancyMaxActiveClusters(&clusters[c], project_large_kernel<__nv_bfloat16, true, true>, &cfg);
    if (e != cudaSuccess) return e;
  }
  if (clusters[1] < 1) return cudaErrorNotSupported;
  clusters[0] = 1;
  return cudaSuccess;
}

FreeSms project_large_free(int dev, int T, int N, int K) {
  const Plan p = plan(g_clusters[dev], T, N, K);
  const int blocks = 2 * p.splits * p.rest;
  if (p.full > 0 || blocks >= kSms) return FreeSms{0, 0};
  // clusters of four and more leave fewer whole groups of SMs than pairs do (measured: 16 blocks of 4 find room beside 28
  // clusters of four, not beside 30; 12 of four beside 48 pairs)
  const int lost = p.splits > 1 ? 16 : 2;
  return FreeSms{kSms - blocks, kSms - blocks > lost ? kSms - blocks - lost : 0};
}

long long project_large_cost(int dev, int T, int N, int K) { return plan(g_clusters[dev], T, N, K).cost; }

cudaError_t launch_project_large(const ProjectArgs& a, const GemmTensorMap& tm_w, const GemmTensorMap& tm_x, const GemmTensorMap& tm_up,
                                 int dev, cudaStream_t s) {
  const Plan p = plan(g_clusters[dev], a.T, a.N, a.K);
  if ((long long)p.m_tiles * p.n_blocks > (1ll << 30)) return cudaErrorInvalidValue;
  const CUtensorMap& w = reinterpret_cast<const CUtensorMap&>(tm_w);
  const CUtensorMap& x = reinterpret_cast<const CUtensorMap&>(tm_x);
  const CUtensorMap& u = reinterpret_cast<const CUtensorMap&>(tm_up);
  return a.out_f32 ? launch<float>(a, p, w, x, u, dev, s) : launch<__nv_bfloat16>(a, p, w, x, u, dev, s);
}

}  // namespace cep
