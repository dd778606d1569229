// Down projection of the low-rank adapters: s[t] = scale_a * A_a x[t] for every token t with adapter a, and the lists of
// adapters per token tile that the projection kernel walks.  Also packs an adapter into the bank.
//
// The work is 2 T r K operations against 2 T K bytes of x: at most r operations per byte, so memory (long batches) or
// latency (a few tokens) bounds it.  A block takes 128 consecutive tokens as the M side of a matrix product whose N side is
// the rows of every adapter among them, 16 ranks at a time: x is read once however many adapters the tokens have (up to
// 64 or 128 ranks a pass, for fp32 outputs and a long K fewer; more take further passes), and of the product each token keeps the columns of its own adapter.
// Operands come by TMA, accumulators are fp32 in tensor memory.  While there are few token tiles, K is split over the CTAs
// of a cluster, which add their partial sums in order through shared memory, so results do not depend on timing.
//
// A short batch's latency is 7 to 8 us (lists 2, loads and products 3 to 5, exchange 2): up to 128 tokens its blocks run beside
// the projection's on the same SMs and the weight streams meanwhile.  16384 tokens of 7168 with 30 adapters: 55 us, against 36
// for reading x once (tiles with many adapters take several passes); matrix instructions of one warp (16x8x16, fragments by
// copies through shared memory) took 120.  Fragments straight from global memory, no copy stages: 28 against 30 us with eight
// rank-16 adapters and 64 tokens, 51 against 37 with ranks up to 64; not kept.
#include <cuda.h>
#include <cuda_bf16.h>

#include "lora.h"
#include "lora_ptx.cuh"

namespace cep {
namespace {

using namespace ptx;

constexpr int kThreads = 192;                        // warp 0 loads, 1 MMA, 2-5 read the accumulator
constexpr int kRows = 128;                           // tokens per block
constexpr int kXStage = kRows * 128;                 // 64 bf16 of K
constexpr int kChunkStage = kLoraChunk * 128;
constexpr int kMaxStages = 8;
// K steps per accumulation chain (the tensor core's additions truncate): kChainSteps while the accumulators last, at most
// kLongestChain (1024 products) for an fp32 output.  A bf16 output does not see longer ones (7168 products end 8e-6 low).
constexpr int kChainSteps = 12, kLongestChain = 16;
constexpr int kMaxParts = 8;
struct __align__(8) ShrinkBarriers {
  uint64_t full[kMaxStages], empty[kMaxStages], acc_full;
  uint32_t tmem_base;
  int abort_flag;
};
struct ShrinkLists {                                 // scratch of the list building
  int id[kLargeTok], job[kLargeTok], n_chunks, warp_count[8];
  int first[kRows], count[kRows];                    // a token's own chunks among the pass's (they are consecutive)
  int chunk[kRows * kLoraMaxChunks];    // adapter * 16 + chunk of its ranks
};

// The slot a token's adapter id names, -1 for none; an id that names nothing loaded is reported and treated as none.
__device__ __forceinline__ int usable_id(const int32_t* __restrict__ ids, int t, const LoraBank& b, int32_t* status, bool report) {
  const int id = __ldg(ids + t);
  if (id >= 0 && id < b.slots && __ldg(b.rank + id) > 0) return id;
  if (id != -1 && report) atomicExch(&status[kStBadRouting], 1);
  return -1;
}

// Distinct non-negative values of v[0..n), n <= 256, in order of first appearance -> out; returns their number.  All threads.
// table: one int per slot.
__device__ int distinct_in_order(const int* v, int n, int* table, int* out, int* warp_count) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int i = threadIdx.x; i < n; i += kThreads) if (v[i] >= 0) table[v[i]] = n;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kThreads) if (v[i] >= 0) atomicMin(&table[v[i]], i);
  __syncthreads();
  int total = 0;
  for (int base = 0; base < n; base += kThreads) {
    const int i = base + threadIdx.x;
    const bool first = i < n && v[i] >= 0 && table[v[i]] == i;
    const unsigned m = __ballot_sync(0xffffffffu, first);
    if (lane == 0) warp_count[warp] = __popc(m);
    __syncthreads();
    int before = total;
    for (int w = 0; w < kThreads / 32; ++w) { if (w < warp) before += warp_count[w]; total += warp_count[w]; }
    if (first) out[before + __popc(m & ((1u << lane) - 1))] = v[i];
    __syncthreads();
  }
  return total;
}

// The adapters job[0..m) as chunks of 16 ranks, in order -> out; returns their number (warp 0 only, all lanes).
__device__ int expand_chunks(const int* job, int m, const LoraBank& bank, int* out) {
  const int lane = threadIdx.x & 31;
  int base = 0;
  for (int j0 = 0; j0 < m; j0 += 32) {
    const int a = j0 + lane < m ? job[j0 + lane] : -1;
    const int nc = a >= 0 ? (bank.rank[a] + kLoraChunk - 1) / kLoraChunk : 0;
    int incl = nc;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int v = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += v; }
    for (int c = 0; c < nc; ++c) out[base + incl - nc + c] = a * kLoraMaxChunks + c;
    base += __shfl_sync(0xffffffffu, incl, 31);
  }
  return base;
}

// Grid (token tiles, pass stripes, K parts); the parts are a cluster.  box: rows of x one TMA load brings.  With token_tile
// other than 128 the first stripe only builds the projection kernel's lists, beside the others' work.
__global__ void __launch_bounds__(kThreads, 3)              // (few registers: blocks of the projection kernel share the SM)
lora_shrink_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_down, int T, int K, int N,
                   const int32_t* __restrict__ ids, const LoraBank bank, int token_tile, int box, int x_stage, int ring, int chunks, int n_acc,
                   int tmem_cols, int32_t* __restrict__ out_ids, int32_t* __restrict__ n_chunks, int32_t* __restrict__ chunk_lists,
                   float* __restrict__ s_out, int32_t* __restrict__ status) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  __shared__ ShrinkBarriers bars;
  __shared__ ShrinkLists L;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  volatile int* abort_flag = &bars.abort_flag;
  const int t0 = blockIdx.x * kRows, rows = min(kRows, T - t0);
  const int part = blockIdx.z, parts = gridDim.z;
  const bool reporter = blockIdx.y == 0 && part == 0;
  const int list_stripes = token_tile != kRows;

  if (threadIdx.x == 32) { prefetch_map(&tm_x); prefetch_map(&tm_down); }
  if (threadIdx.x == 0) {
    for (int s = 0; s < kMaxStages; ++s) { mbar_init(smem_u32(&bars.full[s]), 1); mbar_init(smem_u32(&bars.empty[s]), 1); }
    mbar_init(smem_u32(&bars.acc_full), 1);
    bars.abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32(&bars.tmem_base)), "r"(tmem_cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }

  // What precedes this launch has ended.  The projection kernel may be scheduled from here on; its first loads rely on that end.
  // Not earlier for another reason too: its blocks allocate tensor memory and wait for this grid, so every block of this grid
  // has to hold its own first.
  __syncthreads();
  pdl_enter();

  // ---------------------------------------------------------------- lists (the ring is not in use yet and holds the table)
  int* table = reinterpret_cast<int*>(smem);
  if (reporter && token_tile != kRows) {
    // the projection kernel's tiles that start among these tokens: two of 64, every other time one of 256
    for (int a = t0; a < t0 + rows && a % token_tile == 0; a += token_tile) {
      const int n = min(token_tile, T - a);
      for (int i = threadIdx.x; i < n; i += kThreads) L.id[i] = usable_id(ids, a + i, bank, status, false);
      __syncthreads();
      const int m = distinct_in_order(L.id, n, table, L.job, L.warp_count);
      if (warp == 0) {
        const int nc = expand_chunks(L.job, m, bank, chunk_lists + (size_t)a * kLoraMaxChunks);
        if (lane == 0) n_chunks[a / token_tile] = nc;
      }
      __syncthreads();
    }
  }
  for (int i = threadIdx.x; i < kRows; i += kThreads) {
    const int id = i < rows ? usable_id(ids, t0 + i, bank, status, reporter) : -1;
    L.id[i] = id;
    if (reporter && i < rows) out_ids[t0 + i] = id;
  }
  __syncthreads();
  const int m = distinct_in_order(L.id, rows, table, L.job, L.warp_count);
  if (warp == 0) {
    const int nc = expand_chunks(L.job, m, bank, L.chunk);
    if (lane == 0) L.n_chunks = nc;
  }
  fence_proxy_async_smem();                          // the table's words become TMA destinations
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bars.tmem_base;
  const int total = L.n_chunks, steps = (K + 63) >> 6;
  if (reporter && token_tile == kRows) {
    for (int i = threadIdx.x; i < total; i += kThreads) chunk_lists[(size_t)t0 * kLoraMaxChunks + i] = L.chunk[i];
    if (threadIdx.x == 0) n_chunks[blockIdx.x] = total;
  }
  const int k0 = (int)((long long)steps * part / parts), k1 = (int)((long long)steps * (part + 1) / parts);
  const int cols = chunks * kLoraChunk;              // columns of an accumulator
  const int pitch = cols + 4;                        // floats per row of exchanged sums
  uint32_t phase = 0, acc_phase = 0;                 // phase: a parity bit per stage, of `empty` (loading warp) or `full` (issuing thread)

  for (int c0 = ((int)blockIdx.y - list_stripes) * chunks; c0 < total; c0 += ((int)gridDim.y - list_stripes) * chunks) {
    if (c0 < 0) break;                               // (the stripe that builds lists)
    const int n = min(chunks, total - c0);
    // as many stages as the pass's chunks leave room for.  With fewer than 128 tokens the M side's missing rows are whatever
    // follows in shared memory (their products are not read): a stage may be smaller than the operand, the ring as a whole not.
    const int stage_bytes = x_stage + n * kChunkStage;
    const int stages = min(kMaxStages, 1 + (ring - max(stage_bytes, kXStage)) / stage_bytes);
    int stage = 0;
    if (N > 0 && warp >= 2 && (int)threadIdx.x - 64 < n * kLoraChunk) {
      // a short batch meets its adapters' rows of A for the first time here, while the projection kernel beside this one keeps
      // the memory busy: ask for all of them now, not a stage at a time
      const int r = threadIdx.x - 64, v = L.chunk[c0 + r / kLoraChunk], a = v / kLoraMaxChunks, row = v % kLoraMaxChunks * kLoraChunk + r % kLoraChunk;
      if (row < bank.rank[a])
        prefetch_l2(bank.down + ((size_t)a * bank.rank_pad + row) * K + k0 * 64, (uint32_t)(min(K, k1 * 64) - k0 * 64) * 2);
    }
    if (N > 0 && warp == 5 && lane < n) {
      // a short batch meets each adapter's columns of B for the first time in the projection's last steps: have them in the
      // L2 by then (each part asks for its share)
      const size_t block = (size_t)N * kLoraChunk * 2;
      const size_t b0 = block * part / parts / 16 * 16, b1 = part + 1 == parts ? block : block * (part + 1) / parts / 16 * 16;
      const int v = L.chunk[c0 + lane];
      const uint8_t* up = reinterpret_cast<const uint8_t*>(bank.up) + (size_t)(v / kLoraMaxChunks * (bank.rank_pad / kLoraChunk) + v % kLoraMaxChunks) * block;
      if (b1 > b0) prefetch_l2(up + b0, (uint32_t)(b1 - b0));
    }
    if (warp == 0) {
      // lane i brings chunk i's rows of A; lane 0 the tokens' rows of x too
      const int boxes = (rows + box - 1) / box;
      const int v = lane < n ? L.chunk[c0 + lane] : 0, down_row = v / kLoraMaxChunks * bank.rank_pad + v % kLoraMaxChunks * kLoraChunk;
      for (int k = k0; k < k1; ++k) {
        const bool ok = mbar_wait(smem_u32(&bars.empty[stage]), ~(phase >> stage) & 1u, abort_flag, status);
        if (!__all_sync(0xffffffffu, ok)) break;
        const uint32_t full = smem_u32(&bars.full[stage]);
        uint8_t* st = smem + stage * stage_bytes;
        if (lane == 0) {
          mbar_expect_tx(full, boxes * box * 128 + n * kChunkStage);
          for (int b = 0; b < boxes; ++b) tma_load_2d(smem_u32(st + b * box * 128), &tm_x, k * 64, t0 + b * box, full);
        }
        __syncwarp();
        if (lane < n) tma_load_2d(smem_u32(st + x_stage + lane * kChunkStage), &tm_down, k * 64, down_row, full);
        phase ^= 1u << stage;
        if (++stage == stages) stage = 0;
      }
    } else if (warp == 1 && lane == 0) {
      const uint32_t idesc = make_idesc_bf16(kRows, n * kLoraChunk);
      int slab = 0, slab_end = k0 + (k1 - k0) / n_acc;
      uint32_t more = 0;
      bool ok = true;
      for (int k = k0; k < k1; ++k) {
        if (!mbar_wait(smem_u32(&bars.full[stage]), (phase >> stage) & 1u, abort_flag, status)) { ok = false; break; }
        tc_fence_after();
        if (k == slab_end) { ++slab; slab_end = k0 + (int)((long long)(k1 - k0) * (slab + 1) / n_acc); more = 0; }
        const uint64_t xdesc = make_smem_desc(smem_u32(smem + stage * stage_bytes));
        const uint64_t adesc = make_smem_desc(smem_u32(smem + stage * stage_bytes + x_stage));
#pragma unroll
        for (int k4 = 0; k4 < 4; ++k4)
          tc_mma_f16(tmem + (uint32_t)(slab * cols), xdesc + (uint64_t)(k4 * 2), adesc + (uint64_t)(k4 * 2), idesc, k4 != 0 ? 1u : more);
        more = 1;
        tc_commit(smem_u32(&bars.empty[stage]));
        phase ^= 1u << stage;
        if (++stage == stages) stage = 0;
      }
      if (ok) tc_commit(smem_u32(&bars.acc_full));
    } else if (warp >= 2) {
      bool got = mbar_wait_relaxed(smem_u32(&bars.acc_full), acc_phase, abort_flag, status);
      got = __all_sync(0xffffffffu, got);
      const int row = (warp & 3) * 32 + lane, my = L.id[row];
      const uint32_t taddr = tmem + ((uint32_t)((warp & 3) * 32) << 16);
      int first = 0, count = 0;
      if (got) {
        tc_fence_after();
        const float scale = my >= 0 ? bank.scale[my] : 0.f;
        const int rank = my >= 0 ? bank.rank[my] : 0;
        for (int i = 0; i < n; ++i) {
          const int v = L.chunk[c0 + i];
          const bool mine = my == v / kLoraMaxChunks;
          if (!__any_sync(0xffffffffu, mine)) continue;                    // (the loads are warp-collective)
          uint32_t d[16];
          tc_ld16(taddr + i * kLoraChunk, d);
          tc_wait_ld();
          for (int s = 1; s < n_acc; ++s) {
            uint32_t e[16];
            tc_ld16(taddr + s * cols + i * kLoraChunk, e);
            tc_wait_ld();
#pragma unroll
            for (int j = 0; j < 16; ++j) d[j] = __float_as_uint(__uint_as_float(d[j]) + __uint_as_float(e[j]));
          }
          if (mine) {
            if (count++ == 0) first = i;
            const int c = v % kLoraMaxChunks, left = rank - c * kLoraChunk;
            float4* dst = reinterpret_cast<float4*>(parts == 1 ? s_out + (size_t)(t0 + row) * bank.rank_pad + c * kLoraChunk
                                                               : reinterpret_cast<float*>(smem) + row * pitch + i * kLoraChunk);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              // ranks between the adapter's and the chunk's end are zero
              float4 f;
              f.x = 4 * q + 0 < left ? scale * __uint_as_float(d[4 * q + 0]) : 0.f;
              f.y = 4 * q + 1 < left ? scale * __uint_as_float(d[4 * q + 1]) : 0.f;
              f.z = 4 * q + 2 < left ? scale * __uint_as_float(d[4 * q + 2]) : 0.f;
              f.w = 4 * q + 3 < left ? scale * __uint_as_float(d[4 * q + 3]) : 0.f;
              dst[q] = f;
            }
          }
          __syncwarp();
        }
      }
      L.first[row] = first;
      L.count[row] = count;
    }
    acc_phase ^= 1u;
    if (parts > 1) {
      // the ring holds the partial sums: every load of this pass has been consumed
      cluster_sync_all();
      const int r0 = rows * part / parts, r1 = rows * (part + 1) / parts;
      const uint32_t base = smem_u32(smem);
      // a row per half warp and four ranks per lane: up to four of the row's chunks at a time
      for (int row = r0 + 2 * warp + (lane >> 4); row < r1; row += 2 * kThreads / 32) {
        const int end = L.first[row] + L.count[row];
        for (int i = L.first[row] + ((lane & 15) >> 2); i < end; i += 4) {
          float4 f[kMaxParts];
#pragma unroll
          for (int p = 0; p < kMaxParts; ++p)
            if (p < parts) f[p] = ld_cluster_f4(mapa(base + (uint32_t)((row * pitch + i * kLoraChunk + (lane & 3) * 4) * 4), (uint32_t)p));
          float4 o = f[0];
#pragma unroll
          for (int p = 1; p < kMaxParts; ++p)
            if (p < parts) { o.x += f[p].x; o.y += f[p].y; o.z += f[p].z; o.w += f[p].w; }
          *reinterpret_cast<float4*>(s_out + (size_t)(t0 + row) * bank.rank_pad + L.chunk[c0 + i] % kLoraMaxChunks * kLoraChunk + (lane & 3) * 4) = o;
        }
      }
      fence_proxy_async_smem();                      // the next pass's loads write where the partial sums were
      tc_fence_before();
      cluster_sync_reads();
      tc_fence_after();
    } else {
      tc_fence_before();
      __syncthreads();                               // the accumulator is read before the next pass writes it
      tc_fence_after();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(tmem_cols) : "memory");
  }
}

// up [N, rank] -> [rank_pad/16][N][16] (missing ranks zero), down [rank, K] -> dense rows.  An adapter's columns of B also meet
// the zero rows of other tokens in the accumulator, and 0 * inf is NaN there: values of B that are not finite are stored as
// zeros and marked (bad), and the adapter is then left out (lora_publish_kernel).
__global__ void __launch_bounds__(256)
lora_pack_kernel(const uint16_t* __restrict__ down, int64_t down_stride, const uint16_t* __restrict__ up, int64_t up_stride, int rank,
                 int slot, int K, int N, int rank_pad, uint16_t* __restrict__ bank_down, uint16_t* __restrict__ bank_up, int32_t* __restrict__ bad) {
  const size_t stride = (size_t)gridDim.x * blockDim.x, first = (size_t)blockIdx.x * blockDim.x + threadIdx.x;
  uint16_t* d = bank_down + (size_t)slot * rank_pad * K;
  for (size_t i = first; i < (size_t)rank * K; i += stride) d[i] = down[(i / K) * down_stride + i % K];
  uint16_t* u = bank_up + (size_t)slot * rank_pad * N;
  bool odd = false;
  for (size_t i = first; i < (size_t)rank_pad * N; i += stride) {
    const int r = (int)(i % kLoraChunk);
    const size_t cn = i / kLoraChunk, n = cn % N;
    const int rr = (int)(cn / N) * kLoraChunk + r;
    uint16_t v = rr < rank ? up[n * up_stride + rr] : (uint16_t)0;
    if ((v & 0x7f80) == 0x7f80) { odd = true; v = 0; }                // bf16 exponent all ones
    u[i] = v;
  }
  if (odd) atomicExch(bad, 1);
}
__global__ void lora_publish_kernel(int rank, float scale, int slot, int32_t* bank_rank, float* bank_scale, int32_t* bad, int32_t* status) {
  const bool usable = atomicExch(bad, 0) == 0;
  if (!usable) atomicExch(&status[kStBoundsViolation], 1);
  bank_rank[slot] = usable ? rank : 0;
  bank_scale[slot] = scale;
}

constexpr int kShortSmem = 76 * 1024, kLongSmem = 97 * 1024;     // beside the projection's blocks; two blocks per SM
constexpr int kShortAcc = 8, kLongAcc = 16;                      // chunks of 16 columns in all accumulators of a block
static_assert(kShortSmem >= kLeastTmemBlock && kLongSmem >= kLeastTmemBlock && kLongAcc * kLoraChunk <= kSmTmemColumns / 2 &&
              kShortAcc * kLoraChunk <= kSmTmemColumns / 2, "blocks that share an SM");

}  // namespace

cudaError_t launch_lora_pack(const uint16_t* down, int64_t down_stride, const uint16_t* up, int64_t up_stride, int rank, float scale, int slot,
                             int K, int N, const LoraBank& b, int32_t* bad, int32_t* status, cudaStream_t s) {
  if (rank > 0)
    lora_pack_kernel<<<296, 256, 0, s>>>(down, down_stride, up, up_stride, rank, slot, K, N, b.rank_pad, const_cast<uint16_t*>(b.down),
                                         const_cast<uint16_t*>(b.up), bad);
  lora_publish_kernel<<<1, 1, 0, s>>>(rank, scale, slot, const_cast<int32_t*>(b.rank), const_cast<float*>(b.scale), bad, status);
  return cudaGetLastError();
}

bool lora_beside(int T) { return T <= 128; }

cudaError_t lora_shrink_setup() {
  cudaError_t e = cudaFuncSetAttribute(lora_shrink_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kLongSmem);
  if (e != cudaSuccess) return e;
  // all of the SM's memory as shared memory: with a smaller split the projection kernel's blocks would have to wait for the
  // SM to run empty before the split can change
  return cudaFuncSetAttribute(lora_shrink_kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
}

cudaError_t launch_lora_shrink(const GemmTensorMap& tm_x, const GemmTensorMap& tm_down, int box, const FreeSms& free, int T, int K, int N, int out_f32,
                               const int32_t* ids, const LoraBank& bank, int token_tile, int32_t* out_ids, int32_t* n_chunks, int32_t* chunk_lists, float* s_out,
                               int32_t* status, cudaStream_t s) {
  // Up to 128 tokens the blocks leave shared memory for the projection kernel's on the same SM (lora_beside).
  const bool beside = lora_beside(T);
  int chunks = beside ? 4 : 8;
  const int smem = beside ? kShortSmem : kLongSmem;
  const int acc_chunks = beside ? kShortAcc : kLongAcc;
  const int x_stage = T < kRows ? (T + box - 1) / box * box * 128 : kXStage;
  const int tiles = (T + kRows - 1) / kRows, steps = (K + 63) / 64;
  // passes a tile can need
  const int n = T < kRows ? T : kRows, adapters = bank.slots < n ? bank.slots : n;
  const int most_chunks = adapters * (bank.rank_pad / kLoraChunk);
  int passes = (most_chunks + chunks - 1) / chunks;
  // Blocks that find SMs of their own beside the projection's run while it multiplies (free): then as many parts as still find
  // them, a cluster of `parts` SMs in one GPC per tile (700 tokens of 7168 -> 2048 with eight adapters: 31 us with six parts, 42
  // with eight; 1500: 49 with four, 62 with eight; 512 of 7168 -> 3584: 35 with four, 39 with six, 42 with eight).  Otherwise
  // the projection waits for most of them and their latency counts (1000 tokens: 44 with eight, 50 with four), unless the bank
  // holds so many adapters that the blocks may not run at once (30 of rank 64 in every tile: 82 with eight, 66 with four;
  // beside the projection, 700 tokens: 68 with six, 62 with four).
  int parts = 2 * kSms / tiles;
  if (parts > kMaxParts) parts = kMaxParts;
  if (tiles > 1 && 4 * tiles <= free.in_clusters) {
    if (parts > 6 && (2 * tiles * parts > free.sms || tiles * parts > free.in_clusters)) parts = 6;
    if (parts > 4 && (10 * tiles * parts > 7 * free.sms || tiles * parts > free.in_clusters || (long long)passes * tiles * parts > 3 * kSms)) parts = 4;
  } else if (tiles > 1 && parts > 4 && (long long)passes * tiles * parts > 4 * kSms) {
    parts = 4;
  }
  // Long batches: at least 8 steps a part, fewer blocks leave SMs to the projection's first tiles (6821 tokens of 896 -> 640:
  // 28 us with, 33 without; 4096 of 2048 -> 7168: 102 and 105).
  const int least = tiles >= 16 ? 8 : 1;
  if (parts > steps / least) parts = steps / least;
  if (parts < 1) parts = 1;
  if (out_f32) {
    // chains short enough for the output: fewer chunks a pass leave room for more accumulators (up to K = 65536 beside the
    // projection and 131072 in long batches, from where on chains grow)
    const int longest = kLongestChain * acc_chunks;
    if (parts < (steps + longest - 1) / longest) parts = (steps + longest - 1) / longest < kMaxParts ? (steps + longest - 1) / longest : kMaxParts;
    const int chains = ((steps + parts - 1) / parts + kLongestChain - 1) / kLongestChain;
    if (chunks > acc_chunks / chains) chunks = acc_chunks / chains > 1 ? acc_chunks / chains : 1;
    passes = (most_chunks + chunks - 1) / chunks;
  }
  // how many blocks share the passes
  int stripes = 4 * kSms / (tiles * parts);
  if (stripes > passes) stripes = passes;
  if (stripes < 1) stripes = 1;
  const int part_steps = steps / parts;
  int n_acc = (part_steps + kChainSteps - 1) / kChainSteps;
  const int most = acc_chunks / chunks;
  if (n_acc > most) n_acc = most;
  if (n_acc < 1) n_acc = 1;
  int tmem_cols = 32;
  while (tmem_cols < n_acc * chunks * kLoraChunk) tmem_cols *= 2;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 1; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = (unsigned)parts;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = dim3(tiles, stripes + (token_tile != kRows), parts); cfg.blockDim = dim3(kThreads, 1, 1); cfg.dynamicSmemBytes = smem; cfg.stream = s;
  cfg.attrs = attr; cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, lora_shrink_kernel, reinterpret_cast<const CUtensorMap&>(tm_x), reinterpret_cast<const CUtensorMap&>(tm_down), T, K,
                            token_tile == kLargeTok ? 0 : N, ids, bank, token_tile, box, x_stage, smem - 1024, chunks, n_acc, tmem_cols, out_ids, n_chunks, chunk_lists, s_out, status);
}

}  // namespace cep
