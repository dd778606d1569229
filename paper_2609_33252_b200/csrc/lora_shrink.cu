// Down projection of the low-rank adapters: s[t] = scale_a * A_a x[t] for every token t with adapter a, and the lists of
// adapters per token tile that the projection kernel walks.  Also packs an adapter into the bank.
//
// One block takes 64 tokens and one part of K, and one adapter present among them after the other: the tokens' rows of x
// (only those with this adapter) times the adapter's rows, 16x8x16 matrix instructions with fp32 accumulators, four
// asynchronous copy stages.  The work is 2 T r K operations against 2 T K bytes of x, at most r operations per byte: memory
// (long batches) or latency (a few tokens) bounds it, not the matrix pipe.  With few tokens K is split over several
// blocks: each part's partial sum is stored and the reader adds the parts in order, so the result does not depend on timing.
#include <cuda_bf16.h>

#include "lora.h"

namespace cep {
namespace {

constexpr int kStages = 3;
constexpr int kTileBytes = 64 * 128;                 // 64 rows x 64 bf16
constexpr int kShrinkSmem = kStages * 2 * kTileBytes;

__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool in) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// 16-byte chunk c of row r in a tile of 128-byte rows, chunks exchanged so that eight rows of a column hit all banks
__device__ __forceinline__ uint32_t tile_at(uint32_t base, int r, int c) { return base + r * 128 + ((c ^ (r & 7)) << 4); }

// The slot a token's adapter id names, -1 for none; an id that names nothing loaded is reported and treated as none.
__device__ __forceinline__ int usable_id(const int32_t* __restrict__ ids, int t, const LoraBank& b, int32_t* status, bool report) {
  const int id = __ldg(ids + t);
  if (id >= 0 && id < b.slots && __ldg(b.rank + id) > 0) return id;
  if (id != -1 && report) atomicExch(&status[kStBadRouting], 1);
  return -1;
}

// Distinct non-negative values of v[0..n), n <= 256, in order of first appearance; returns their number.  All 128 threads.
__device__ int distinct_in_order(const int* v, int n, int* out, int* warp_count) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int total = 0;
  for (int base = 0; base < n; base += 128) {
    const int i = base + threadIdx.x;
    bool first = i < n && v[i] >= 0;
    for (int j = 0; first && j < i; ++j) first = v[j] != v[i];
    const unsigned m = __ballot_sync(0xffffffffu, first);
    if (lane == 0) warp_count[warp] = __popc(m);
    __syncthreads();
    int before = total;
    for (int w = 0; w < 4; ++w) { if (w < warp) before += warp_count[w]; total += warp_count[w]; }
    if (first) out[before + __popc(m & ((1u << lane) - 1))] = v[i];
    __syncthreads();
  }
  return total;
}

// Blocks (token tile, K part, job stripe): job j of the tile belongs to stripe j mod gridDim.z.
__global__ void __launch_bounds__(128, 3)
lora_shrink_kernel(const uint16_t* __restrict__ x, int64_t x_stride, int T, int K, const int32_t* __restrict__ ids, const LoraBank bank,
                   int token_tile, int32_t* __restrict__ out_ids, int32_t* __restrict__ n_jobs, int32_t* __restrict__ jobs,
                   float* __restrict__ s_out, int32_t* __restrict__ tile_counter, int32_t* __restrict__ status) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int id_s[kLargeTok], job_s[kLargeTok], warp_count[4];
  const int t0 = blockIdx.x * kShrinkRows;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const bool reporter = blockIdx.y == 0 && blockIdx.z == 0;
  if (reporter && blockIdx.x == 0 && threadIdx.x == 0) *tile_counter = 0;
  if (reporter && t0 % token_tile == 0) {
    const int n = min(token_tile, T - t0), tile = t0 / token_tile;
    for (int i = threadIdx.x; i < n; i += 128) id_s[i] = usable_id(ids, t0 + i, bank, status, false);
    __syncthreads();
    const int m = distinct_in_order(id_s, n, job_s, warp_count);
    for (int i = threadIdx.x; i < m; i += 128) jobs[(size_t)tile * token_tile + i] = job_s[i];
    if (threadIdx.x == 0) n_jobs[tile] = m;
    __syncthreads();
  }
  const int rows = min(kShrinkRows, T - t0);
  for (int i = threadIdx.x; i < kShrinkRows; i += 128) {
    const int id = i < rows ? usable_id(ids, t0 + i, bank, status, reporter) : -1;
    id_s[i] = id;
    if (reporter && i < rows) out_ids[t0 + i] = id;
  }
  __syncthreads();
  const int m = distinct_in_order(id_s, rows, job_s, warp_count);

  const int steps = (K + 63) >> 6;
  const int k0 = (int)((long long)steps * blockIdx.y / gridDim.y), k1 = (int)((long long)steps * (blockIdx.y + 1) / gridDim.y);
  const uint32_t base = (uint32_t)__cvta_generic_to_shared(smem);
  float* s_part = s_out + (size_t)blockIdx.y * T * bank.rank_pad;
  for (int j = blockIdx.z; j < m; j += gridDim.z) {
    const int a = job_s[j], rank = bank.rank[a];
    const float scale = bank.scale[a];
    const uint16_t* down = bank.down + (size_t)a * bank.rank_pad * K;
    const bool live = __any_sync(0xffffffffu, id_s[warp * 16 + (lane & 15)] == a);    // this warp's 16 tokens
    for (int r0 = 0; r0 < rank; r0 += 64) {
      const int cols = min(64, (rank - r0 + kLoraChunk - 1) / kLoraChunk * kLoraChunk);
      auto load = [&](int step, int buf) {
        const uint32_t xs = base + buf * 2 * kTileBytes, as = xs + kTileBytes;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int i = q * 128 + threadIdx.x, r = i >> 3, c = i & 7, k = step * 64 + c * 8;
          // rows that are not read keep whatever is there: they meet only outputs that are not written
          if (id_s[r] == a) cp16(tile_at(xs, r, c), x + (size_t)(t0 + r) * x_stride + (k < K ? k : 0), k < K);
          if (r0 + r < rank) cp16(tile_at(as, r, c), down + (size_t)(r0 + r) * K + (k < K ? k : 0), k < K);
        }
      };
      float acc[8][4], sum[8][4];
#pragma unroll
      for (int n = 0; n < 8; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[n][i] = sum[n][i] = 0.f;
#pragma unroll
      for (int p = 0; p < kStages - 1; ++p) {
        if (k0 + p < k1) load(k0 + p, p);
        asm volatile("cp.async.commit_group;" ::: "memory");
      }
      for (int step = k0, buf = 0; step < k1; ++step) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
        __syncthreads();
        const int next = step + kStages - 1;
        if (next < k1) load(next, buf == 0 ? kStages - 1 : buf - 1);
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (live) {
          const uint32_t xs = base + buf * 2 * kTileBytes, as = xs + kTileBytes;
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) {
            uint32_t af[4];
            ldmatrix4(af, tile_at(xs, warp * 16 + (lane & 15), kk * 2 + (lane >> 4)));
#pragma unroll
            for (int n = 0; n < 8; n += 2) {
              if (n * 8 < cols) {                       // cols is a multiple of 16: both column groups are there
                uint32_t bf[4];
                ldmatrix4(bf, tile_at(as, n * 8 + (lane & 7) + ((lane >> 4) << 3), kk * 2 + ((lane >> 3) & 1)));
                mma16816(acc[n], af, bf[0], bf[1]);
                mma16816(acc[n + 1], af, bf[2], bf[3]);
              }
            }
          }
        }
        if (++buf == kStages) buf = 0;
        if (((step - k0) & 15) == 15 || step + 1 == k1) {         // the matrix unit's additions truncate: chains of 1024 products
#pragma unroll
          for (int n = 0; n < 8; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) { sum[n][i] += acc[n][i]; acc[n][i] = 0.f; }
        }
      }
      asm volatile("cp.async.wait_group 0;" ::: "memory");
      __syncthreads();                                  // the next round overwrites the stages
      if (live) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int r = warp * 16 + (lane >> 2) + h * 8;
          if (id_s[r] != a) continue;
          float* dst = s_part + (size_t)(t0 + r) * bank.rank_pad + r0;
#pragma unroll
          for (int n = 0; n < 8; ++n) {
            const int c = n * 8 + (lane & 3) * 2;
            if (c < cols) {
              // ranks between the adapter's and the next multiple of 16 are exact zeros
              float2 v = make_float2(r0 + c < rank ? scale * sum[n][2 * h] : 0.f, r0 + c + 1 < rank ? scale * sum[n][2 * h + 1] : 0.f);
              *reinterpret_cast<float2*>(dst + c) = v;
            }
          }
        }
      }
    }
  }
}

// up [N, rank] -> [rank_pad/16][N][16] (missing ranks zero), down [rank, K] -> dense rows; thread 0 publishes the adapter.
__global__ void __launch_bounds__(256)
lora_pack_kernel(const uint16_t* __restrict__ down, int64_t down_stride, const uint16_t* __restrict__ up, int64_t up_stride, int rank,
                 float scale, int slot, int K, int N, int rank_pad, uint16_t* __restrict__ bank_down, uint16_t* __restrict__ bank_up,
                 int32_t* __restrict__ bank_rank, float* __restrict__ bank_scale) {
  const size_t stride = (size_t)gridDim.x * blockDim.x, first = (size_t)blockIdx.x * blockDim.x + threadIdx.x;
  uint16_t* d = bank_down + (size_t)slot * rank_pad * K;
  for (size_t i = first; i < (size_t)rank * K; i += stride) d[i] = down[(i / K) * down_stride + i % K];
  uint16_t* u = bank_up + (size_t)slot * rank_pad * N;
  for (size_t i = first; i < (size_t)rank_pad * N; i += stride) {
    const int r = (int)(i % kLoraChunk);
    const size_t cn = i / kLoraChunk, n = cn % N;
    const int rr = (int)(cn / N) * kLoraChunk + r;
    u[i] = rr < rank ? up[n * up_stride + rr] : (uint16_t)0;
  }
  if (first == 0) { bank_rank[slot] = rank; bank_scale[slot] = scale; }
}

}  // namespace

cudaError_t launch_lora_pack(const uint16_t* down, int64_t down_stride, const uint16_t* up, int64_t up_stride, int rank, float scale, int slot,
                             int K, int N, const LoraBank& b, cudaStream_t s) {
  lora_pack_kernel<<<296, 256, 0, s>>>(down, down_stride, up, up_stride, rank, scale, slot, K, N, b.rank_pad, const_cast<uint16_t*>(b.down),
                                       const_cast<uint16_t*>(b.up), const_cast<int32_t*>(b.rank), const_cast<float*>(b.scale));
  return cudaGetLastError();
}

cudaError_t lora_shrink_setup() {
  return cudaFuncSetAttribute(lora_shrink_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kShrinkSmem);
}

cudaError_t launch_lora_shrink(const uint16_t* x, int64_t x_stride, int T, int K, const int32_t* ids, const LoraBank& bank, int parts,
                               int token_tile, int32_t* out_ids, int32_t* n_jobs, int32_t* jobs, float* s_out, int32_t* tile_counter,
                               int32_t* status, cudaStream_t s) {
  const int tiles = (T + kShrinkRows - 1) / kShrinkRows;
  int stripes = 592 / (tiles * parts);                   // enough blocks to fill the device when a tile has many adapters
  stripes = stripes < 1 ? 1 : stripes > 32 ? 32 : stripes;
  if (stripes > bank.slots) stripes = bank.slots;
  lora_shrink_kernel<<<dim3(tiles, parts, stripes), 128, kShrinkSmem, s>>>(x, x_stride, T, K, ids, bank, token_tile, out_ids, n_jobs, jobs,
                                                                           s_out, tile_counter, status);
  return cudaGetLastError();
}

}  // namespace cep
