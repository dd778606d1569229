// Attention of a batch of sequences that share long prefixes, keys and values in a paged cache (attn.h has the cutting of the
// work).  Per row: o = sum_j p_j v_j / sum_j p_j, p_j = exp(scale q.k_j - m), one pass over the keys with a running m.
//
// One CTA per SM.  Two warpgroups hold a row tile of 128 rows each (tokens x query heads of a kv head); a tile of 128 keys is
// fetched page by page by TMA into a ring that K and V tiles share, S = Q K^T and O += P V run on the tensor core with S, P and
// O in tensor memory (P takes S's place).  Each thread of a warpgroup owns one row of S: maximum and sum need no exchange.
//   two row tiles: both warpgroups use every key tile, the tensor core works for one while the other takes its exponentials
//   one row tile (decoding): the warpgroups take the key tiles in turn, with a maximum, sum and O of their own, joined at the
//     end through shared memory
#include <cuda.h>
#include <cuda_bf16.h>
#include <math_constants.h>

#include "attn.h"
#include "lora_ptx.cuh"

namespace cep {
namespace {

using namespace ptx;

constexpr int kMmaWarp = 8, kLoadWarp = 9, kItemWarp = 10, kCodeWarp = 12;     // (kCodeWarp and the next three: e4m3 only)
constexpr int kItemSlots = 4;
constexpr int kMaxShared = 227 * 1024;
constexpr int kHalfBytes = kAttnTile * 128;                 // 128 rows of 64 bf16: what a 128-byte swizzled box column is

// Shared memory: Q of two row tiles, the ring of K and V tiles, barriers and the like, the schedule; in an e4m3 cache's kernel the
// ring is shorter, and what the schedule leaves holds tiles of codes on their way in.
template <int DP, bool E4M3> struct Layout {
  static constexpr int threads = E4M3 ? 512 : 384;
  static constexpr int halves = DP / 64;
  static constexpr int tile_bytes = halves * kHalfBytes;    // a K, V or Q tile
  static constexpr int stages = (E4M3 ? 96 : 128) * 1024 / tile_bytes;
  static constexpr int code_bytes = kAttnTile * DP, max_codes = 8;
  static constexpr int q = 0, ring = 2 * tile_bytes, misc = ring + stages * tile_bytes, codes = misc + 3072, align = 1024;
  // tiles of codes beside a schedule of `words` words: at least two, for the largest
  __host__ __device__ static constexpr int code_slots(int words) {
    return E4M3 ? ((kMaxShared - align - codes - words * 4) / code_bytes < max_codes ? (kMaxShared - align - codes - words * 4) / code_bytes : max_codes) : 0;
  }
  __host__ __device__ static constexpr int smem(int words) { return codes + code_slots(words) * code_bytes + words * 4 + align; }
};
constexpr int kLeastWords = attn_sched_words(1, 0), kMostWords = attn_sched_words(kAttnMaxSeqs, kAttnMaxPrefixes);
template <int DP, bool E4M3> constexpr bool layout_ok() {
  typedef Layout<DP, E4M3> L;
  return alone_on_its_sm(L::smem(kLeastWords)) && L::smem(kMostWords) <= kMaxShared && (!E4M3 || L::code_slots(kMostWords) >= 2) && L::codes % 16 == 0;
}
static_assert(layout_ok<64, false>() && layout_ok<128, false>() && layout_ok<64, true>() && layout_ok<128, true>(),
              "all tensor memory: no other block may share the SM");

__device__ __forceinline__ float ex2(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ float max3(float a, float b, float c) { float r; asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c)); return r; }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_st32(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]),
        "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tc_st16(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
               ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
                 "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
               : "memory");
}
// Columns of S at or behind `see` count for nothing.
__device__ __forceinline__ void hide(uint32_t (&r)[32], int see) {
  if (see < 32) {
#pragma unroll
    for (int i = 0; i < 32; ++i) r[i] = i < see ? r[i] : 0xff800000u;
  }
}
// Four e4m3 codes as four bf16.  A code's exponent and mantissa, moved to bf16's places, read as the value times 2^-120 (the
// exponents' offsets are 7 and 127), subnormals too; NaN is the one code that needs a look.
__device__ __forceinline__ void decode4(uint32_t x, uint32_t& lo, uint32_t& hi) {
  auto two = [](uint32_t h) {                              // codes in the upper bytes of both halves
    const uint32_t bits = (h & 0x80008000u) | ((h >> 4) & 0x07f007f0u);
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(bits), "r"(0x7b807b80u));      // 2^120
    return r;
  };
  const uint32_t a = __byte_perm(x, 0, 0x1404), b = __byte_perm(x, 0, 0x3424);
  lo = two(a); hi = two(b);
  if (((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) {
    if ((a & 0x7f00u) == 0x7f00u) lo |= 0x7fc0u;
    if ((a & 0x7f000000u) == 0x7f000000u) lo |= 0x7fc00000u;
    if ((b & 0x7f00u) == 0x7f00u) hi |= 0x7fc0u;
    if ((b & 0x7f000000u) == 0x7f000000u) hi |= 0x7fc00000u;
  }
}
// A from tensor memory (lane = row, two bf16 per 32-bit column), B from shared memory
__device__ __forceinline__ void tc_mma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
               ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
               ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar) : "memory");
}
// V as the MMA's B operand: keys are the contraction, columns contiguous (64 per 128-byte row, the next 64 a half further)
__device__ __forceinline__ uint64_t make_v_desc(uint32_t saddr) {
  uint64_t d = 0;
  d |= (uint64_t)((saddr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(kHalfBytes >> 4) << 16;            // the next 64 columns
  d |= (uint64_t)(1024 >> 4) << 32;                  // the next 8 keys
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}
constexpr uint32_t kTransposeB = 1u << 16;           // instruction descriptor: B's rows are contiguous along N


// ---------------------------------------------------------------- the schedule
// Exclusive scan of n values over the block with `op`; put(i, before, through); returns the total.
template <typename V, typename Op, typename Get, typename Put>
__device__ __forceinline__ V block_scan(int n, V identity, Op op, Get get, Put put, V* warp_totals) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n_warps = blockDim.x >> 5;
  V carry = identity;
  for (int base = 0; base < n; base += blockDim.x) {
    const int i = base + tid;
    V v = i < n ? get(i) : identity;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const V o = __shfl_up_sync(0xffffffffu, v, d);
      if (lane >= d) v = op(o, v);
    }
    if (lane == 31) warp_totals[warp] = v;
    V before = __shfl_up_sync(0xffffffffu, v, 1);
    if (lane == 0) before = identity;
    __syncthreads();
    V ahead = carry;
    for (int w = 0; w < warp; ++w) ahead = op(ahead, warp_totals[w]);
    for (int w = 0; w < n_warps; ++w) carry = op(carry, warp_totals[w]);
    if (i < n) put(i, op(ahead, before), op(ahead, v));
    __syncthreads();
  }
  return carry;
}

// Every CTA computes the whole schedule from the lengths.  What does not fit the call is cut to what does and reported.
__device__ void build_schedule(const AttnArgs& a, AttnSched& s, long long* scratch) {
  const AttnShape& p = a.p;
  const int tid = threadIdx.x, nt = blockDim.x;
  int bad = 0;
  auto larger = [](int x, int y) { return x > y ? x : y; };
  auto clamp = [](int v, int hi) { return v < 0 ? 0 : v > hi ? hi : v; };
  int* totals = reinterpret_cast<int*>(scratch);
  // first tokens and first sequences never fall
  block_scan<int>(p.B + 1, 0, larger, [&](int i) { const int v = a.q_start[i], c = clamp(v, p.T); bad |= v != c; return c; },
                  [&](int i, int before, int v) { bad |= before > a.q_start[i]; s.q0[i] = v; }, totals);
  if (p.G)
    block_scan<int>(p.G + 1, 0, larger, [&](int i) { const int v = a.prefix_start ? a.prefix_start[i] : i ? p.B : 0, c = clamp(v, p.B); bad |= v != c; return c; },
                    [&](int i, int before, int v) { bad |= a.prefix_start && before > a.prefix_start[i]; s.gfirst[i] = v; }, totals);
  else if (tid == 0) s.gfirst[0] = 0;
  for (int g = tid; g < p.G; g += nt) { const int v = a.prefix_len[g]; s.glen[g] = clamp(v, p.prefix_cap); bad |= s.glen[g] != v; }
  for (int b = tid; b < p.B; b += nt) { const int v = a.kv_len[b]; s.kv[b] = clamp(v, p.own_cap); bad |= s.kv[b] != v; }
  __syncthreads();
  for (int b = tid; b < p.B; b += nt) {
    int g = -1;
    if (p.G && b >= s.gfirst[0] && b < s.gfirst[p.G]) {                // the last group that starts at or before b
      int lo = 0, hi = p.G;
      while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (s.gfirst[mid] <= b) lo = mid; else hi = mid; }
      g = lo;
    }
    s.group[b] = g;
  }
  __syncthreads();
  auto add = [](int x, int y) { return x + y; };
  const int n_short = block_scan<int>(p.B, 0, add, [&](int b) { return attn_is_short(p, s, b) ? s.q0[b + 1] - s.q0[b] : 0; },
                                      [&](int b, int before, int) { s.scum[b] = before; }, totals);
  if (tid == 0) s.scum[p.B] = n_short;
  __syncthreads();
  const int n_tiles = block_scan<int>(p.G, 0, add, [&](int g) { return attn_div_up(s.scum[s.gfirst[g + 1]] - s.scum[s.gfirst[g]], 2 * p.tps); },
                                      [&](int g, int before, int) { s.grt[g] = before; }, totals);
  if (tid == 0) s.grt[p.G] = n_tiles;
  __syncthreads();
  const long long total = block_scan<long long>(p.G + p.B, 0ll, [](long long x, long long y) { return x + y; },
      [&](int e) { const AttnEntity x = attn_entity(p, s, e); return p.Hkv * attn_items_cost(x, x.items); },
      [&](int e, long long before, long long) { s.cost[e] = before; }, scratch);
  if (tid == 0) s.cost[p.G + p.B] = total;
  s.share = attn_share(p, total);
  if (bad) atomicExch(&a.status[kStBoundsViolation], 1);
  __syncthreads();
}

// The sequence among whose short tokens number `i` of all short tokens is.
__device__ __forceinline__ int short_sequence(const AttnSched& s, int lo, int hi, int i) {
  while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (s.scum[mid] <= i) lo = mid; else hi = mid; }
  return lo;
}

// What a CTA has of an item, as the warp that walks the schedule hands it to the others.
struct alignas(16) Work {
  int32_t n, s0;                             // steps (0: no more items), the first of them
  int32_t head, tok, n_tok;                  // kv head; token of the batch (own, joint) or number among all short tokens (group); tokens
  int32_t ahead, own, n_ahead;               // as in AttnItem
  int32_t seen;                              // own keys that the first token sees
  int32_t b, g;
  int32_t lo, hi;                            // group: its sequences
  int32_t whole;                             // nothing to join: the rows are final
  long long prow;                            // first partial row
};
static_assert(sizeof(Work) == 64, "");

// Places in the ring, in the order in which the tensor core needs them: K0 K1 V0 K2 V1 ... K(n-1) V(n-2) V(n-1).
__device__ __forceinline__ uint32_t pos_k(uint32_t base, int j) { return base + (j ? 2 * j - 1 : 0); }
__device__ __forceinline__ uint32_t pos_v(uint32_t base, int j, int n) { return base + (j == n - 1 ? 2 * n - 1 : 2 * j + 2); }

// ---------------------------------------------------------------- the kernel
template <int DP, bool E4M3>
__global__ void __launch_bounds__(Layout<DP, E4M3>::threads, 1)
attn_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v) {
  using L = Layout<DP, E4M3>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t sbase = smem_u32(smem);
  const uint32_t bar0 = sbase + L::misc;
  const uint32_t full = bar0, empty = bar0 + 64, s_full = bar0 + 128, p_ready = bar0 + 144, o_done = bar0 + 160, q_ready = bar0 + 176, rows_meet = bar0 + 184,
                 w_full = bar0 + 192, w_empty = bar0 + 224, code_full = bar0 + 256, code_empty = bar0 + 320;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + L::misc + 384);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + L::misc + 388);
  long long* scratch = reinterpret_cast<long long*>(smem + L::misc + 512);             // a block's warps' totals
  const Work* work = reinterpret_cast<const Work*>(smem + L::misc + 640);
  float2* exchange = reinterpret_cast<float2*>(smem + L::misc + 1024);                 // [128] maximum and sum of the other warpgroup's rows
  const int words = attn_sched_words(a.p.B, a.p.G), n_codes = L::code_slots(words);
  uint8_t* sched_at = smem + L::codes + n_codes * L::code_bytes;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < L::stages; ++i) { mbar_init(full + 8 * i, E4M3 ? 4 : 1); mbar_init(empty + 8 * i, 1); }
    for (int i = 0; i < n_codes; ++i) { mbar_init(code_full + 8 * i, 1); mbar_init(code_empty + 8 * i, 4); }
    for (int i = 0; i < 2; ++i) { mbar_init(s_full + 8 * i, 1); mbar_init(p_ready + 8 * i, 4); mbar_init(o_done + 8 * i, 1); }
    mbar_init(q_ready, 8);
    mbar_init(rows_meet, 8);
    for (int i = 0; i < kItemSlots; ++i) { mbar_init(w_full + 8 * i, 1); mbar_init(w_empty + 8 * i, E4M3 ? 14 : 10); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (warp == kLoadWarp && lane == 0) { prefetch_map(&tm_k); prefetch_map(&tm_v); }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  pdl_enter();
  const AttnShape& p = a.p;
  AttnSched s = attn_carve(sched_at, p.B, p.G);
  build_schedule(a, s, scratch);
  if (blockIdx.x == 0) {                                    // for the kernel that joins partial results
    int32_t* dst = static_cast<int32_t*>(a.sched);
    const int32_t* src = reinterpret_cast<const int32_t*>(sched_at);
    for (int i = tid; i < words; i += L::threads) dst[i] = src[i];
  }

  const long long x0 = (long long)blockIdx.x * s.share, x1 = x0 + s.share;
  uint32_t ring = 0, turn = 0;                              // places of the ring and items used so far
  // the next item; every warp that took it gives it back after its last look
  auto take = [&]() -> const Work& {
    mbar_wait(w_full + 8 * (turn % kItemSlots), (turn / kItemSlots) & 1, abort_flag, a.status);
    return work[turn % kItemSlots];
  };
  auto give_back = [&]() {
    __syncwarp();
    if (lane == 0) mbar_arrive(w_empty + 8 * (turn % kItemSlots));
    ++turn;
  };

  if (warp == kLoadWarp) {
    // ------------------------------------------------------ keys and values, page by page
    const int page = 1 << a.page_shift, box = page < kAttnTile ? page : kAttnTile, box_shift = page < kAttnTile ? a.page_shift : 7;
    int bad = 0;
    bool alive = true;
    uint32_t issued = 0;
    while (alive) {
      const Work it = take();
      if (it.n == 0) break;
      give_back();
      const int s0 = it.s0, n = it.n;
      const int32_t* own_table = it.b >= 0 ? a.page_table + (long long)it.b * a.table_stride : nullptr;
      const int32_t* ahead_table = it.g >= 0 ? a.prefix_pages + (long long)it.g * a.prefix_stride : nullptr;
      // a lane's page of a step (up to 8), or -1 where the step has no keys any more
      auto page_of = [&](int j) -> int {
        const int step = s0 + j;
        const bool in_ahead = step < it.n_ahead;
        const int key = (in_ahead ? step : step - it.n_ahead) * kAttnTile + (lane << box_shift), keys = in_ahead ? it.ahead : it.own;
        if (j >= n || lane >= (kAttnTile >> box_shift) || key >= keys) return -1;
        int pg = (in_ahead ? ahead_table : own_table)[key >> a.page_shift];
        if (pg < 0 || pg >= a.n_pages) { bad = 1; pg = a.n_pages; }                    // (reads zeros)
        return pg;
      };
      auto load = [&](uint32_t pos, const CUtensorMap* tm, int j, int pg) {
        const int places = E4M3 ? n_codes : L::stages, st = pos % places;
        const uint32_t landed = (E4M3 ? code_full : full) + 8 * st, free = (E4M3 ? code_empty : empty) + 8 * st;
        alive = __all_sync(0xffffffffu, mbar_wait(free, ((pos / places) & 1) ^ 1, abort_flag, a.status));
        if (!alive) return;
        issued = pos + 1;
        const int step = s0 + j, in_page = ((step < it.n_ahead ? step : step - it.n_ahead) * kAttnTile) & (page - 1);
        const int pages = __popc(__ballot_sync(0xffffffffu, pg >= 0));
        if (lane == 0) mbar_expect_tx(landed, pages * box * (E4M3 ? DP : 128 * L::halves));
        __syncwarp();
        if (pg >= 0) {
          if (E4M3) {
            tma_load_4d(sbase + L::codes + st * L::code_bytes + (lane << box_shift) * DP, tm, 0, in_page, it.head, pg, landed);
          } else {
#pragma unroll
            for (int h = 0; h < L::halves; ++h)
              tma_load_4d(sbase + L::ring + st * L::tile_bytes + h * kHalfBytes + ((lane << box_shift) * 128), tm, h * 64, in_page, it.head, pg, landed);
          }
        }
        __syncwarp();
      };
      int cur = page_of(0), next = page_of(1);
      load(pos_k(ring, 0), &tm_k, 0, cur);
      for (int j = 0; j < n && alive; ++j) {
        const int after = page_of(j + 2);
        if (j + 1 < n) load(pos_k(ring, j + 1), &tm_k, j + 1, next);
        if (alive) load(pos_v(ring, j, n), &tm_v, j, cur);
        cur = next; next = after;
      }
      ring += 2 * n;
    }
    if (bad) atomicExch(&a.status[kStBadRouting], 1);
    if (!alive) {                                           // copies in flight land before the block's memory is given up
      const unsigned long long t0 = globaltimer();
      const uint32_t places = E4M3 ? n_codes : L::stages;
      for (uint32_t pos = issued > places ? issued - places : 0; pos < issued; ++pos)
        while (!mbar_try_wait((E4M3 ? code_full : full) + 8 * (pos % places), (pos / places) & 1) && globaltimer() - t0 < 100000000ull) {}
    }
  } else if (warp == kItemWarp) {
    // ------------------------------------------------------ the CTA's share of the schedule, item by item
    if (lane == 0) {
      AttnWalk k = attn_walk_at(p, s, x0);
      Work* out = const_cast<Work*>(work);
      for (;;) {
        Work w;
        w.n = 0; w.n_tok = 0;
        for (; !k.done && k.at < x1 && w.n == 0; attn_walk_next(p, s, &k)) {
          const AttnItem it = attn_item(p, s, k);
          const int s0 = attn_steps_before(k, it.n, x0), s1 = attn_steps_before(k, it.n, x1);
          w.n = s1 - s0; w.s0 = s0;
          if (w.n == 0) continue;
          w.head = it.head; w.n_tok = it.n_tok; w.ahead = it.ahead; w.own = it.own; w.n_ahead = it.n_ahead; w.b = it.b; w.g = it.g;
          w.whole = it.kind == kAttnJoint && w.n == it.n;
          w.prow = attn_part_row(it, blockIdx.x, s0);
          if (it.kind == kAttnGroup) {
            w.lo = s.gfirst[it.g]; w.hi = s.gfirst[it.g + 1];
            w.tok = s.scum[w.lo] + it.tok; w.seen = 0;
          } else {
            w.lo = w.hi = 0;
            w.tok = s.q0[it.b] + it.tok;
            w.seen = s.kv[it.b] - (s.q0[it.b + 1] - s.q0[it.b]) + it.tok + 1;
          }
        }
        if (!mbar_wait(w_empty + 8 * (turn % kItemSlots), ((turn / kItemSlots) & 1) ^ 1, abort_flag, a.status)) w.n = 0;
        out[turn % kItemSlots] = w;
        mbar_arrive(w_full + 8 * (turn % kItemSlots));
        ++turn;
        if (w.n == 0) break;
      }
    }
    __syncwarp();
  } else if (warp == kMmaWarp) {
    // ------------------------------------------------------ tensor core, one thread
    if (lane == 0) {
      constexpr uint32_t idesc_s = make_idesc_bf16(128, 128), idesc_o = make_idesc_bf16(128, DP) | kTransposeB;
      bool alive = true;
      uint32_t items = 0, p_phase[2] = {0, 0};
      auto wait_stage = [&](uint32_t pos) { alive = alive && mbar_wait(full + 8 * (pos % L::stages), (pos / L::stages) & 1, abort_flag, a.status); tc_fence_after(); };
      auto wait_p = [&](int w) { alive = alive && mbar_wait(p_ready + 8 * w, p_phase[w] & 1, abort_flag, a.status); ++p_phase[w]; tc_fence_after(); };
      auto free_stage = [&](uint32_t pos) { tc_commit(empty + 8 * (pos % L::stages)); };
      auto qk = [&](int w, int q_tile, uint32_t pos) {
        const uint64_t qd = make_smem_desc(sbase + L::q + q_tile * L::tile_bytes);
        const uint64_t kd = make_smem_desc(sbase + L::ring + (pos % L::stages) * L::tile_bytes);
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) {
          const uint64_t off = ((i >> 2) * kHalfBytes + (i & 3) * 32) >> 4;
          tc_mma_f16(tmem + w * 128, qd + off, kd + off, idesc_s, i > 0);
        }
        tc_commit(s_full + 8 * w);
      };
      auto pv = [&](int w, uint32_t pos, bool first) {
        const uint64_t vd = make_v_desc(sbase + L::ring + (pos % L::stages) * L::tile_bytes);
#pragma unroll
        for (int i = 0; i < kAttnTile / 16; ++i)
          tc_mma_f16_ts(tmem + 256 + w * 128, tmem + w * 128 + i * 8, vd + ((i * 16 * 128) >> 4), idesc_o, !first || i > 0);
      };
      while (alive) {
        const Work& it = take();
        const int n = it.n;
        const bool dual = it.n_tok > p.tps;
        if (n == 0) break;
        mbar_arrive(w_empty + 8 * (turn % kItemSlots));
        ++turn;
        alive = alive && mbar_wait(q_ready, items & 1, abort_flag, a.status);
        ++items;
        tc_fence_after();
        if (dual) {
          wait_stage(pos_k(ring, 0));
          if (!alive) break;
          qk(0, 0, pos_k(ring, 0));
          qk(1, 1, pos_k(ring, 0));
          free_stage(pos_k(ring, 0));
          for (int j = 0; j < n; ++j) {
            const bool more = j + 1 < n;
            const uint32_t pv_at = pos_v(ring, j, n), pk_at = pos_k(ring, j + 1);
            wait_p(0);
            if (more) wait_stage(pk_at);                    // (loaded before this step's V)
            wait_stage(pv_at);
            if (!alive) break;
            pv(0, pv_at, j == 0);
            if (more) qk(0, 0, pk_at); else tc_commit(o_done);
            wait_p(1);
            if (!alive) break;
            pv(1, pv_at, j == 0);
            free_stage(pv_at);
            if (more) { qk(1, 1, pk_at); free_stage(pk_at); } else tc_commit(o_done + 8);
          }
        } else {
          for (int j = 0; j < 2 && j < n; ++j) {
            wait_stage(pos_k(ring, j));
            if (!alive) break;
            qk(j, 0, pos_k(ring, j));
            free_stage(pos_k(ring, j));
          }
          for (int j = 0; j < n && alive; ++j) {
            const int w = j & 1;
            wait_p(w);
            wait_stage(pos_v(ring, j, n));
            if (!alive) break;
            pv(w, pos_v(ring, j, n), j < 2);
            free_stage(pos_v(ring, j, n));
            if (j + 2 >= n) { tc_commit(o_done + 8 * w); continue; }
            wait_stage(pos_k(ring, j + 2));
            if (!alive) break;
            qk(w, 0, pos_k(ring, j + 2));
            free_stage(pos_k(ring, j + 2));
          }
        }
        ring += 2 * n;
      }
    }
    __syncwarp();
  } else if (E4M3 && warp >= kCodeWarp) {
    // ------------------------------------------------------ codes to bf16, which holds every e4m3 value
    const int ct = tid & 127;
    bool alive = true;
    while (alive) {
      const Work it = take();
      if (__any_sync(0xffffffffu, it.n == 0)) break;
      give_back();
      for (int i = 0; i < 2 * it.n && alive; ++i) {
        const uint32_t pos = ring + i;
        const int j = i == 0 ? 0 : i == 2 * it.n - 1 ? it.n - 1 : (i & 1) ? (i + 1) >> 1 : (i >> 1) - 1;             // the order of pos_k and pos_v
        const int step = it.s0 + j, keys = (step < it.n_ahead ? it.ahead - step * kAttnTile : it.own - (step - it.n_ahead) * kAttnTile);
        const int st = pos % L::stages, slot = pos % n_codes;
        const bool ok = mbar_wait(code_full + 8 * slot, (pos / n_codes) & 1, abort_flag, a.status) &&
                        mbar_wait(empty + 8 * st, ((pos / L::stages) & 1) ^ 1, abort_flag, a.status);
        alive = __all_sync(0xffffffffu, ok);
        if (!alive) break;
        const uint8_t* src = smem + L::codes + slot * L::code_bytes;
        uint8_t* dst = smem + L::ring + st * L::tile_bytes;
        constexpr int per_row = DP / 16;                   // 16 codes at a time
#pragma unroll
        for (int u = 0; u < kAttnTile * per_row / 128; ++u) {
          const int id = u * 128 + ct, row = id / per_row, c = id % per_row;
          uint4 v = *reinterpret_cast<const uint4*>(src + id * 16);
          if (row >= keys) v = make_uint4(0, 0, 0, 0);     // what lies behind the last key may be anything: its weight 0 needs a finite value
          uint4 lo, hi;
          decode4(v.x, lo.x, lo.y); decode4(v.y, lo.z, lo.w);
          decode4(v.z, hi.x, hi.y); decode4(v.w, hi.z, hi.w);
          uint8_t* at = dst + (c >> 2) * kHalfBytes + row * 128;
          const int first = (((c & 3) * 2) ^ (row & 7)) << 4, second = first ^ 16;
          if (c & 4) {                                     // (the other order: both halves' stores share no bank)
            *reinterpret_cast<uint4*>(at + second) = hi;
            *reinterpret_cast<uint4*>(at + first) = lo;
          } else {
            *reinterpret_cast<uint4*>(at + first) = lo;
            *reinterpret_cast<uint4*>(at + second) = hi;
          }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) { mbar_arrive(code_empty + 8 * slot); mbar_arrive(full + 8 * st); }
      }
      ring += 2 * it.n;
    }
  } else if (warp < kMmaWarp) {
    // ------------------------------------------------------ rows: softmax, corrections, results
    // (After a wait that was given up an item's steps run on with what is there: what a warp does must not differ by lane.)
    const int wg = warp >> 2, row = tid & 127, row_tok = row / p.Gh, row_head = row - row_tok * p.Gh;
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;      // this warp's 32 lanes of tensor memory
    const uint32_t t_s = tmem + lanes + wg * 128, t_o = tmem + lanes + 256 + wg * 128;
    uint32_t s_phase = 0, o_phase = 0, m_phase = 0;
    auto meet = [&]() {                                     // both warpgroups
      __syncwarp();
      if (lane == 0) mbar_arrive(rows_meet);
      mbar_wait(rows_meet, m_phase & 1, abort_flag, a.status);
      ++m_phase;
    };
    for (;;) {
      const Work& it = take();
      const int n = it.n;
      if (__any_sync(0xffffffffu, n == 0 || *abort_flag)) break;
      const int s0 = it.s0, n_ahead = it.n_ahead, ahead = it.ahead, own = it.own, kvh = it.head;
      const bool dual = it.n_tok > p.tps, whole = it.whole;
      const int tt = (dual ? wg * p.tps : 0) + row_tok;     // token of the item
      const bool mine = row_tok < p.tps && tt < it.n_tok;
      const bool active = __any_sync(0xffffffffu, mine);
      int token = it.tok + tt, own_seen = own;
      if (mine) {
        if (it.hi > 0) {
          const int b = short_sequence(s, it.lo, it.hi, token);
          token = s.q0[b] + (token - s.scum[b]);
        } else if (p.causal) {
          own_seen = it.seen + tt;
        }
      }
      const int head = kvh * p.Gh + row_head;
      const long long prow = it.prow + (long long)tt * p.Gh + row_head;
      give_back();
      // Q into shared memory, columns beyond D as zeros (rows of nobody stay as they are: rows do not mix)
      if (mine && (dual || wg == 0)) {
        const uint16_t* src = a.q + (long long)token * a.q_tok + (long long)head * a.q_head;
        uint8_t* dst = smem + L::q + (dual ? wg : 0) * L::tile_bytes + row * 128;
#pragma unroll
        for (int c = 0; c < DP / 8; ++c) {
          const uint4 v = c * 8 < a.D ? __ldg(reinterpret_cast<const uint4*>(src + c * 8)) : make_uint4(0, 0, 0, 0);
          *reinterpret_cast<uint4*>(dst + (c >> 3) * kHalfBytes + (((c & 7) ^ (row & 7)) << 4)) = v;
        }
      }
      fence_proxy_async_smem();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(q_ready);

      const float sl2 = a.scale_log2 * (a.k_scale ? a.k_scale[kvh] : 1.f);
      float m = -CUDART_INF_F, l = 0.f;                     // maximum that the sums refer to (unscaled), sum
      bool any = false;                                     // O holds something
      for (int j = dual ? 0 : wg; j < n; j += dual ? 1 : 2) {
        const int step = s0 + j;
        const bool in_ahead = step < n_ahead;
        const int key0 = (in_ahead ? step : step - n_ahead) * kAttnTile, keys = (in_ahead ? ahead : own) - key0;
        mbar_wait(s_full + 8 * wg, s_phase & 1, abort_flag, a.status);
        ++s_phase;
        tc_fence_after();
        if (!E4M3 && keys < kAttnTile) {                    // what lies behind the last key may be anything: its weight 0 needs a finite value.
          // (Not before S: only then has this stage's use before last ended, and the parity tells the uses apart.)
          const uint32_t pos = pos_v(ring, j, n);
          mbar_wait(full + 8 * (pos % L::stages), (pos / L::stages) & 1, abort_flag, a.status);
          uint8_t* v = smem + L::ring + (pos % L::stages) * L::tile_bytes;
          const int from = keys < 0 ? 0 : keys;
#pragma unroll
          for (int h = 0; h < L::halves; ++h)
            for (int i = from * 8 + (tid & 127); i < kAttnTile * 8; i += 128) *reinterpret_cast<uint4*>(v + h * kHalfBytes + i * 16) = make_uint4(0, 0, 0, 0);
          fence_proxy_async_smem();
        }
        if (active) {
          const int see = in_ahead ? keys : (own_seen - key0 < keys ? own_seen - key0 : keys);
          float m_new = m;
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            uint32_t r[32];
            tc_ld32(t_s + c * 32, r);
            tc_wait_ld();
            hide(r, see - c * 32);
            float top = __uint_as_float(r[0]);
#pragma unroll
            for (int i = 1; i < 31; i += 2) top = max3(top, __uint_as_float(r[i]), __uint_as_float(r[i + 1]));
            m_new = max3(m_new, top, __uint_as_float(r[31]));
          }
          // The sums keep referring to an older maximum until weights could pass 2^8: fp32 and bf16 carry that exactly as well.
          const bool raise = m_new > m && (m_new - m) * sl2 > 8.f;
          if (!any) {
            m = m_new;
          } else if (__any_sync(0xffffffffu, raise)) {
            const float f = raise ? ex2((m - m_new) * sl2) : 1.f;
            if (raise) { m = m_new; l *= f; }
#pragma unroll
            for (int c = 0; c < DP / 32; ++c) {
              uint32_t o[32];
              tc_ld32(t_o + c * 32, o);
              tc_wait_ld();
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
              tc_st32(t_o + c * 32, o);
            }
            tc_wait_st();
          }
          any = true;
          const float shift = m == -CUDART_INF_F ? 0.f : m * sl2;
          float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            uint32_t r[32], w[16];
            tc_ld32(t_s + c * 32, r);
            tc_wait_ld();
            hide(r, see - c * 32);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float p0 = ex2(fmaf(__uint_as_float(r[2 * i]), sl2, -shift)), p1 = ex2(fmaf(__uint_as_float(r[2 * i + 1]), sl2, -shift));
              sum[i & 1] += p0; sum[2 + (i & 1)] += p1;
              w[i] = pack_bf16(p0, p1);
            }
            tc_st16(t_s + c * 16, w);
          }
          l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
          tc_wait_st();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_ready + 8 * wg);
      }

      // ---- the item's result
      const bool worked = dual || wg < n;                   // (of one step, the second warpgroup has none)
      if (worked) { mbar_wait(o_done + 8 * wg, o_phase & 1, abort_flag, a.status); ++o_phase; tc_fence_after(); }
      const float m2 = m == -CUDART_INF_F ? m : m * sl2;
      // 32 columns of O at a time
      auto finish = [&](float m2, float l, auto get) {
        if (whole) {
          const float inv = l > 0.f ? (a.v_scale ? a.v_scale[kvh] : 1.f) / l : l;        // (a NaN stays)
          uint16_t* dst = a.out + (long long)token * a.out_tok + (long long)head * a.out_head;
#pragma unroll
          for (int c = 0; c < DP / 32; ++c) {
            float o[32];
            get(c, o);
            if (mine) {
#pragma unroll
              for (int i = 0; i < 32; i += 8)
                if (c * 32 + i < a.D) {
                  uint4 v;
                  v.x = l == 0.f ? 0u : pack_bf16(o[i] * inv, o[i + 1] * inv); v.y = l == 0.f ? 0u : pack_bf16(o[i + 2] * inv, o[i + 3] * inv);
                  v.z = l == 0.f ? 0u : pack_bf16(o[i + 4] * inv, o[i + 5] * inv); v.w = l == 0.f ? 0u : pack_bf16(o[i + 6] * inv, o[i + 7] * inv);
                  *reinterpret_cast<uint4*>(dst + c * 32 + i) = v;
                }
            }
          }
          if (mine && a.lse) a.lse[(long long)token * a.lse_tok + head] = (m2 + __log2f(l)) * 0.6931471805599453f;
        } else {
          float* dst = a.part_o + prow * DP;
#pragma unroll
          for (int c = 0; c < DP / 32; ++c) {
            float o[32];
            get(c, o);
            if (mine) {
#pragma unroll
              for (int i = 0; i < 32; i += 4) *reinterpret_cast<float4*>(dst + c * 32 + i) = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
            }
          }
          if (mine) a.part_ml[prow] = make_float2(m2, l);
        }
      };
      if (dual) {
        if (active) finish(m2, l, [&](int c, float (&o)[32]) {
          uint32_t r[32];
          tc_ld32(t_o + c * 32, r);
          tc_wait_ld();
#pragma unroll
          for (int i = 0; i < 32; ++i) o[i] = __uint_as_float(r[i]);
        });
        // (the other warpgroup may still read its Q: each overwrites its own only)
      } else {
        // the second warpgroup's O goes through the memory of Q, which nothing reads any more
        constexpr int chunks = DP / 4;
        float4* pool = reinterpret_cast<float4*>(smem + L::q) + row * chunks;
        meet();
        if (wg == 1) {
          if (active && worked) {
#pragma unroll
            for (int c = 0; c < DP / 32; ++c) {
              uint32_t r[32];
              tc_ld32(t_o + c * 32, r);
              tc_wait_ld();
#pragma unroll
              for (int i = 0; i < 8; ++i)
                pool[(c * 8 + i) ^ (row & (chunks - 1))] = make_float4(__uint_as_float(r[4 * i]), __uint_as_float(r[4 * i + 1]), __uint_as_float(r[4 * i + 2]),
                                                                       __uint_as_float(r[4 * i + 3]));
            }
          }
          exchange[row] = make_float2(m2, l);
        }
        meet();
        if (wg == 0 && active) {
          const float2 other = exchange[row];
          const bool two = n > 1;
          const float mm = two ? fmaxf(m2, other.x) : m2, base = mm == -CUDART_INF_F ? 0.f : mm;
          const float f0 = two ? ex2(m2 - base) : 1.f, f1 = two ? ex2(other.x - base) : 0.f;
          finish(mm, two ? l * f0 + other.y * f1 : l, [&](int c, float (&o)[32]) {
            uint32_t r[32];
            tc_ld32(t_o + c * 32, r);
            tc_wait_ld();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float4 x = two ? pool[(c * 8 + i) ^ (row & (chunks - 1))] : make_float4(0.f, 0.f, 0.f, 0.f);
              o[4 * i] = __uint_as_float(r[4 * i]) * f0 + x.x * f1; o[4 * i + 1] = __uint_as_float(r[4 * i + 1]) * f0 + x.y * f1;
              o[4 * i + 2] = __uint_as_float(r[4 * i + 2]) * f0 + x.z * f1; o[4 * i + 3] = __uint_as_float(r[4 * i + 3]) * f0 + x.w * f1;
            }
          });
        }
        meet();
      }
      tc_fence_before();
      ring += 2 * n;
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kMmaWarp) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

// ---------------------------------------------------------------- rows whose keys were in several places
constexpr int kJoinThreads = 256, kJoinBlocks = 4 * 148;

// The partial results of one item for one of its rows, joined into (m, l, o) of a warp; o: this lane's columns 4 lane .. + 3.
template <int DP>
__device__ __forceinline__ void join_item(const AttnArgs& a, const AttnSched& s, const AttnWalk& k, const AttnItem& it, int row, float& m, float& l, float4& o) {
  const int lane = threadIdx.x & 31;
  const int c_lo = (int)(k.at / s.share), c_hi = (int)((k.at + k.w - 1) / s.share);
  for (int c0 = c_lo; c0 <= c_hi; c0 += 32) {
    const int c = c0 + lane;
    long long at = -1;
    float2 ml = make_float2(-CUDART_INF_F, 0.f);
    if (c <= c_hi) {
      const int s0 = attn_steps_before(k, it.n, c * s.share), s1 = attn_steps_before(k, it.n, (c + 1) * s.share);
      if (s0 < s1) { at = attn_part_row(it, c, s0) + row; ml = a.part_ml[at]; }
    }
    float top = ml.x;
#pragma unroll
    for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    top = fmaxf(top, m);
    const float base = top == -CUDART_INF_F ? 0.f : top;
    const float keep = ex2(m - base);
    o.x *= keep; o.y *= keep; o.z *= keep; o.w *= keep; l *= keep;
    m = top;
    const float f = ex2(ml.x - base);
    float add = ml.y * f;
#pragma unroll
    for (int d = 16; d; d >>= 1) add += __shfl_xor_sync(0xffffffffu, add, d);
    l += add;
    unsigned have = __ballot_sync(0xffffffffu, at >= 0);
    while (have) {
      const int src = __ffs(have) - 1;
      have &= have - 1;
      const long long r = __shfl_sync(0xffffffffu, at, src);
      const float g = __shfl_sync(0xffffffffu, f, src);
      if (lane < DP / 4) {
        const float4 v = *reinterpret_cast<const float4*>(a.part_o + r * DP + lane * 4);
        o.x += v.x * g; o.y += v.y * g; o.z += v.z * g; o.w += v.w * g;
      }
    }
  }
}

template <int DP>
__device__ __forceinline__ void write_row(const AttnArgs& a, int token, int head, float m, float l, float4 o) {
  const int lane = threadIdx.x & 31;
  const float inv = l > 0.f ? (a.v_scale ? a.v_scale[head / a.p.Gh] : 1.f) / l : l;
  if (lane * 4 < a.D) {
    const uint2 v = l == 0.f ? make_uint2(0, 0) : make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
    *reinterpret_cast<uint2*>(a.out + (long long)token * a.out_tok + (long long)head * a.out_head + lane * 4) = v;
  }
  if (lane == 0 && a.lse) a.lse[(long long)token * a.lse_tok + head] = (m + __log2f(l)) * 0.6931471805599453f;
}

template <int DP>
__global__ void __launch_bounds__(kJoinThreads)
attn_join_kernel(const __grid_constant__ AttnArgs a) {
  extern __shared__ uint8_t join_smem[];
  pdl_enter();
  const AttnShape& p = a.p;
  const int tid = threadIdx.x, warp = tid >> 5, warps = kJoinThreads / 32;
  {
    int32_t* dst = reinterpret_cast<int32_t*>(join_smem);
    const int32_t* src = static_cast<const int32_t*>(a.sched);
    for (int i = tid; i < attn_sched_words(p.B, p.G); i += kJoinThreads) dst[i] = src[i];
    __syncthreads();
  }
  AttnSched s = attn_carve(join_smem, p.B, p.G);
  s.share = attn_share(p, s.cost[p.G + p.B]);
  // tokens of short sequences: their group's prefix, then their own keys
  const int n_rows = s.scum[p.B] * p.Hq;                    // (at most 2^31: checked by the plan)
  for (int u = blockIdx.x * warps + warp; u < n_rows; u += gridDim.x * warps) {
    const int i = u / p.Hq, head = u - i * p.Hq, b = short_sequence(s, 0, p.B, i), g = s.group[b];
    const int kvh = head / p.Gh, rh = head - kvh * p.Gh;
    float m = -CUDART_INF_F, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    AttnWalk k;
    k.done = false;
    k.e = g; k.head = kvh;
    k.x = attn_entity(p, s, g);
    const int in_group = i - s.scum[s.gfirst[g]];
    k.r = in_group / (2 * p.tps);
    k.w = k.x.a;
    k.at = s.cost[g] + (long long)(kvh * k.x.items + k.r) * k.x.a;
    join_item<DP>(a, s, k, attn_item(p, s, k), (in_group - k.r * 2 * p.tps) * p.Gh + rh, m, l, o);
    if (s.kv[b] > 0) {
      k.e = p.G + b; k.r = 0;
      k.x = attn_entity(p, s, k.e);
      k.w = k.x.a;
      k.at = s.cost[k.e] + kvh * k.x.a;
      join_item<DP>(a, s, k, attn_item(p, s, k), (i - s.scum[b]) * p.Gh + rh, m, l, o);
    }
    write_row<DP>(a, s.q0[b] + (i - s.scum[b]), head, m, l, o);
  }
  // joint items that a cut between two CTAs' shares went through: found at their first cut
  for (int c = 1 + blockIdx.x; c < p.n_ctas; c += gridDim.x) {
    const long long x = c * s.share;
    const AttnWalk k = attn_walk_at(p, s, x);
    if (k.done) break;
    const AttnItem it = attn_item(p, s, k);
    if (it.kind != kAttnJoint) continue;
    const int before = attn_steps_before(k, it.n, x);
    if (before == 0 || before == it.n || attn_steps_before(k, it.n, x - s.share) > 0) continue;
    for (int r = warp; r < it.n_tok * p.Gh; r += warps) {
      float m = -CUDART_INF_F, l = 0.f;
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
      join_item<DP>(a, s, k, it, r, m, l, o);
      const int tt = r / p.Gh;
      write_row<DP>(a, s.q0[it.b] + it.tok + tt, it.head * p.Gh + (r - tt * p.Gh), m, l, o);
    }
  }
}

template <int DP, bool E4M3>
cudaError_t launch_dim(const AttnArgs& a, const CUtensorMap& tk, const CUtensorMap& tv, cudaStream_t s) {
  const int words = attn_sched_words(a.p.B, a.p.G);
  cudaError_t e = launch_pdl(attn_kernel<DP, E4M3>, dim3(a.p.n_ctas), dim3(Layout<DP, E4M3>::threads), Layout<DP, E4M3>::smem(words), s, 1, a, tk, tv);
  if (e != cudaSuccess) return e;
  return launch_pdl(attn_join_kernel<DP>, dim3(kJoinBlocks), dim3(kJoinThreads), words * 4, s, 1, a);
}

}  // namespace

int attn_padded_dim(int D) { return D <= 64 ? 64 : 128; }

cudaError_t attn_setup() {
  cudaError_t e = cudaFuncSetAttribute(attn_kernel<64, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxShared);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(attn_kernel<128, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxShared);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(attn_kernel<64, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxShared);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(attn_kernel<128, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxShared);
  return e;
}

int make_cache_map(GemmTensorMap* out, const void* base, const cep_attn_config& c, const int64_t* stride) {
  typedef CUresult (*Encode)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                             const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static Encode enc = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    const bool ok = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess;
    return ok ? reinterpret_cast<Encode>(p) : nullptr;
  }();
  if (!enc) return -1;
  const bool e4m3 = c.cache_elem == CEP_ELEM_E4M3;
  const int elt = e4m3 ? 1 : 2, box_rows = c.page_size < kAttnTile ? c.page_size : kAttnTile;
  const long long room = (c.head_dim * elt + 15) / 16 * 16;           // (the stride of a single element means nothing)
  auto bytes = [&](int64_t n, int64_t st) { return (cuuint64_t)(n > 1 ? st * elt : room); };
  cuuint64_t dims[4] = {(cuuint64_t)c.head_dim, (cuuint64_t)c.page_size, (cuuint64_t)c.n_kv_heads, (cuuint64_t)c.n_pages};
  cuuint64_t strides[3] = {bytes(c.page_size, stride[1]), bytes(c.n_kv_heads, stride[2]), bytes(c.n_pages, stride[0])};
  cuuint32_t box[4] = {(cuuint32_t)(e4m3 ? attn_padded_dim(c.head_dim) : 64), (cuuint32_t)box_rows, 1, 1}, es[4] = {1, 1, 1, 1};
  const CUresult r = enc(reinterpret_cast<CUtensorMap*>(out), e4m3 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4,
                         const_cast<void*>(base), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                         e4m3 ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? 0 : -2;
}

cudaError_t launch_attn(const AttnArgs& a, int e4m3, const GemmTensorMap& tm_k, const GemmTensorMap& tm_v, cudaStream_t s) {
  const CUtensorMap& tk = reinterpret_cast<const CUtensorMap&>(tm_k);
  const CUtensorMap& tv = reinterpret_cast<const CUtensorMap&>(tm_v);
  const bool narrow = attn_padded_dim(a.D) == 64;
  if (e4m3) return narrow ? launch_dim<64, true>(a, tk, tv, s) : launch_dim<128, true>(a, tk, tv, s);
  return narrow ? launch_dim<64, false>(a, tk, tv, s) : launch_dim<128, false>(a, tk, tv, s);
}

}  // namespace cep
