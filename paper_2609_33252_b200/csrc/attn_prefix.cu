// Attention of a batch of sequences that share long prefixes, keys and values in a paged cache (attn.h has the cutting of the
// work).  Per row: o = sum_j p_j v_j / sum_j p_j, p_j = exp(scale q.k_j - m), one pass over the keys with a running m.
//
// One CTA per SM.  Two warpgroups hold a row tile of 128 rows each (tokens x query heads of a kv head); a tile of 128 keys is
// fetched page by page by TMA into a ring that K and V tiles share, S = Q K^T and O += P V run on the tensor core with S, P and
// O in tensor memory (P takes S's place).  Each thread of a warpgroup owns one row of S: maximum and sum need no exchange.
//   two row tiles: both warpgroups use every key tile, the tensor core works for one while the other takes its exponentials
//   one row tile (decoding): the warpgroups take the key tiles in turn, with a Q, maximum, sum and O of their own
// The CTA's items form one stream of key tiles, so that loads, products and row work of neighbouring items overlap; the thread
// that issues the products serves whichever warpgroup is ready.
#include <cuda.h>
#include <cuda_bf16.h>
#include <math_constants.h>

#include <algorithm>

#include "attn.h"
#include "lora_ptx.cuh"

namespace cep {
namespace {

using namespace ptx;

constexpr int kMmaWarp = 8, kLoadWarp = 9, kItemWarp = 10, kMmaWarp2 = 11, kCodeWarp = 12;     // (kCodeWarp and the next three: e4m3 only)
constexpr int kItemSlots = 8;                               // items between the warp that walks the schedule and the slowest reader
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
  static constexpr int q = 0, ring = 2 * tile_bytes, misc = ring + stages * tile_bytes, codes = misc + 2048, align = 1024;
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
__device__ __forceinline__ float ex2_here(float x) { float r; asm volatile("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_st16(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
               ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
                 "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
               : "memory");
}
// Four e4m3 codes as four fp16, exactly.
__device__ __forceinline__ void decode4(uint32_t x, uint32_t& lo, uint32_t& hi) {
  asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.rn.f16x2.e4m3x2 %0, a;\n cvt.rn.f16x2.e4m3x2 %1, b;\n}" : "=r"(lo), "=r"(hi) : "r"(x));
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


// The bounded wait of tcgen05_ptx.cuh in few instructions: the kernel's roles share an instruction cache.
__device__ __forceinline__ bool wait_bar(uint32_t bar, uint32_t parity, volatile int* abort_flag, int32_t* status) {
  uint32_t spin = 0;
  unsigned long long t0 = 0;
#pragma unroll 1
  while (!mbar_try_wait(bar, parity)) {
    if ((++spin & 255u) != 0u) continue;
    const unsigned long long now = globaltimer();
    if (t0 == 0) t0 = now;
    if (now - t0 > kWaitLimitNs) { *abort_flag = 1; atomicExch(&status[kStTimeout], 1); }
    if (*abort_flag) return false;
  }
  return true;
}

__device__ __forceinline__ bool elect_one() {
  uint32_t yes;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(yes));
  return yes != 0;
}

// ---------------------------------------------------------------- the schedule
// Exclusive scan of n pairs over the block: put(i, before); returns the totals.
struct Pair { int a, b; };
template <typename Get, typename Put>
__device__ __forceinline__ Pair block_scan(int n, Get get, Put put, Pair* warp_totals) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n_warps = blockDim.x >> 5;
  Pair carry{0, 0};
#pragma unroll 1
  for (int base = 0; base < n; base += blockDim.x) {
    const int i = base + tid;
    Pair v{0, 0};
    if (i < n) v = get(i);
    const Pair own = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int a = __shfl_up_sync(0xffffffffu, v.a, d);
      const int b = __shfl_up_sync(0xffffffffu, v.b, d);
      if (lane >= d) { v.a += a; v.b += b; }
    }
    if (lane == 31) warp_totals[warp] = v;
    __syncthreads();
    Pair w{0, 0};
    if (lane < n_warps) w = warp_totals[lane];
    const bool ahead = lane < warp;
    Pair mine;
    mine.a = carry.a + __reduce_add_sync(0xffffffffu, ahead ? w.a : 0) + v.a - own.a;
    mine.b = carry.b + __reduce_add_sync(0xffffffffu, ahead ? w.b : 0) + v.b - own.b;
    carry.a += __reduce_add_sync(0xffffffffu, w.a);
    carry.b += __reduce_add_sync(0xffffffffu, w.b);
    if (i < n) put(i, mine);
    __syncthreads();
  }
  return carry;
}

// Starts that fall are held at the largest before them (this is not what a correct call needs: one thread).
__device__ __forceinline__ void never_fall(int32_t* v, int n) {
#pragma unroll 1
  for (int i = 1; i < n; ++i) if (v[i] < v[i - 1]) v[i] = v[i - 1];
}

// Every CTA computes the whole schedule from the lengths.  What does not fit the call is cut to what does and reported.
// first_entity: where this CTA's share begins (-1: behind the end).
__device__ __forceinline__ void build_schedule(const AttnArgs& a, AttnSched& s, Pair* scratch, volatile int* first_entity) {
  const AttnShape& p = a.p;
  const int tid = threadIdx.x, nt = blockDim.x;
  int bad = 0, falls = 0;
  auto take = [&](int v, int hi) { const int c = v < 0 ? 0 : v > hi ? hi : v; bad |= c != v; return c; };
#pragma unroll 1
  for (int i = tid; i <= p.B; i += nt) {
    const int v = a.q_start[i];
    if (i < p.B) { falls |= a.q_start[i + 1] < v; s.kv[i] = take(a.kv_len[i], p.own_cap); }
    s.q0[i] = take(v, p.T);
  }
#pragma unroll 1
  for (int i = tid; i <= p.G; i += nt) {
    if (i < p.G) s.glen[i] = take(a.prefix_len[i], p.prefix_cap);
    if (!a.prefix_start) { s.gfirst[i] = i && p.G ? p.B : 0; continue; }
    const int v = a.prefix_start[i];
    if (i < p.G) falls |= a.prefix_start[i + 1] < v;
    s.gfirst[i] = take(v, p.B);
  }
  if (__syncthreads_or(falls)) {
    bad = 1;
    if (tid == 0) { never_fall(s.q0, p.B + 1); never_fall(s.gfirst, p.G + 1); }
    __syncthreads();
  }
  const Pair places = block_scan(p.B,
      [&](int b) {
        int g = -1;
        if (b >= s.gfirst[0] && b < s.gfirst[p.G]) {       // the last group that starts at or before b
          int lo = 0, hi = p.G;
#pragma unroll 1
          while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (s.gfirst[mid] <= b) lo = mid; else hi = mid; }
          g = lo;
        }
        s.group[b] = (int16_t)g;
        const int n = s.q0[b + 1] - s.q0[b];
        return Pair{attn_has_rows(p, s, b) ? n : 0, attn_is_short(p, s, b) ? n : 0};
      },
      [&](int b, const Pair& before) { s.pcum[b] = before.a; s.scum[b] = before.b; }, scratch);
  if (tid == 0) { s.pcum[p.B] = places.a; s.scum[p.B] = places.b; }
  __syncthreads();
  const Pair total = block_scan(p.G + p.B,
      [&](int e) { const AttnEntity x = attn_entity(p, s, e); return Pair{p.Hkv * attn_items_cost(x, x.items), e < p.G ? x.items : 0}; },
      [&](int e, const Pair& before) { s.cost[e] = before.a; if (e < p.G) s.grt[e] = before.b; }, scratch);
  if (tid == 0) { s.cost[p.G + p.B] = total.a; s.grt[p.G] = total.b; *first_entity = -1; }
  s.share = attn_share(p, total.a);
  __syncthreads();
  const int x0 = blockIdx.x * s.share;
#pragma unroll 1
  for (int e = tid; e < p.G + p.B; e += nt)
    if (s.cost[e] <= x0 && x0 < s.cost[e + 1]) *first_entity = e;
  if (bad) atomicExch(&a.status[kStBoundsViolation], 1);
  __syncthreads();
}

// The sequence (lo <= b < hi) with before[b] <= i < before[b + 1].
__device__ __forceinline__ int sequence_of(const int32_t* before, int lo, int hi, int i) {
#pragma unroll 1
  while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (before[mid] <= i) lo = mid; else hi = mid; }
  return lo;
}

// ---------------------------------------------------------------- records for the kernel that joins partial results
// Where the partial results of an item are.
struct JoinPart {
  long long rows;                            // first partial row
  int32_t at, w, n, n_tok, dual, joint;      // its place and length on the cost axis, steps, tokens; two row tiles; prefix and own keys in one
};
struct alignas(16) JoinSeq {                 // a sequence with partial rows of its own: its (only) item of kv head 0
  JoinPart part;                             // n = 0: no own keys
  int32_t q0, first, g, in_group;            // first token; first among those of such sequences; group (-1: shares nothing); first among the group's short ones
};
struct alignas(16) JoinGroup { JoinPart part; int32_t items, n_short, pad[2]; };       // item 0 of kv head 0; items per kv head; tokens
struct alignas(16) JoinCut { JoinPart part; int32_t token, head, pad[2]; };            // part.n = 0: no item to join at the start of this CTA's share
struct JoinRecords { int32_t* head; JoinSeq* seq; JoinGroup* group; JoinCut* cut; int32_t* seq_of; };    // head: share, tokens
static_assert(sizeof(JoinPart) == 32 && sizeof(JoinSeq) == 48 && sizeof(JoinGroup) == 48 && sizeof(JoinCut) == 48, "");
__device__ __forceinline__ JoinRecords records_of(const AttnArgs& a) {
  JoinRecords r;
  uint8_t* p = static_cast<uint8_t*>(a.records);
  r.head = reinterpret_cast<int32_t*>(p); p += 16;
  r.cut = reinterpret_cast<JoinCut*>(p); p += kAttnMaxCtas * sizeof(JoinCut);
  r.group = reinterpret_cast<JoinGroup*>(p); p += a.p.G * sizeof(JoinGroup);
  r.seq = reinterpret_cast<JoinSeq*>(p); p += a.p.B * sizeof(JoinSeq);
  r.seq_of = reinterpret_cast<int32_t*>(p);
  return r;
}
// By a warp of every CTA that has nothing else to do by then; each writes its part.
__device__ __forceinline__ void write_records(const AttnArgs& a, const AttnSched& s, const JoinPart& cut, int cut_token, int cut_head) {
  const AttnShape& p = a.p;
  const JoinRecords r = records_of(a);
  const int lane = threadIdx.x & 31, worker = blockIdx.x * 32 + lane, workers = gridDim.x * 32;
  if (lane == 0) r.cut[blockIdx.x] = JoinCut{cut, cut_token, cut_head, {0, 0}};
  if (worker == 0) { r.head[0] = s.share; r.head[1] = s.pcum[p.B]; }
#pragma unroll 1
  for (int e = worker; e < p.G + p.B; e += workers) {
    AttnWalk k;
    k.done = false; k.e = e; k.head = 0; k.r = 0; k.at = s.cost[e];
    k.x = attn_entity(p, s, e);
    k.w = attn_item_cost(k.x, 0);
    JoinPart part{};
    if (k.x.items > 0) {
      const AttnItem it = attn_item(p, s, k);
      part = JoinPart{it.rows, k.at, k.w, it.n, it.n_tok, it.dual, it.kind == kAttnJoint};
    }
    if (e < p.G) {
      r.group[e] = JoinGroup{part, k.x.items, s.scum[s.gfirst[e + 1]] - s.scum[s.gfirst[e]], {0, 0}};
    } else {
      const int b = e - p.G, g = attn_is_short(p, s, b) ? s.group[b] : -1;
      r.seq[b] = JoinSeq{part, s.q0[b], s.pcum[b], g, g >= 0 ? s.scum[b] - s.scum[s.gfirst[g]] : 0};
    }
  }
  // tokens of sequences with partial rows of their own -> their sequence
#pragma unroll 1
  for (int i = worker; i < s.pcum[p.B]; i += workers) r.seq_of[i] = sequence_of(s.pcum, 0, p.B, i);
}

// What a CTA has of an item, as the warp that walks the schedule hands it to the others.
struct alignas(16) Work {
  int32_t n, s0;                             // steps (0: no more items), the first of them
  int32_t head, tok, n_tok;                  // kv head; token of the batch (own, joint) or number among all short tokens (group); tokens
  int32_t ahead, own, n_ahead;               // as in AttnItem
  int32_t seen;                              // own keys that the first token sees
  int32_t b, g;
  int32_t lo, hi;                            // group: its sequences
  int32_t flags;                             // 1: two row tiles; 2: the rows are final
  long long prow;                            // first partial row
};
static_assert(sizeof(Work) == 64, "");
enum { kDual = 1, kWhole = 2 };

// Weights are fp32 in the sums and enter the product with V in the 16 bits that its operands have: bf16 with V's own bf16 (2^-8 of a weight at most;
// its exponents are fp32's), fp16 with decoded codes (2^-11).  fp16 ends at 2^-24, which a row with one strong key reaches, so its weights
// are all multiplied by 2^kLift: with maxima that lag by 2^8 at most they stay below 2^15, and those from 2^-21 of the
// largest on keep all of their bits, from 2^-32 on some.  (Without: 2^-14 and 2^-25.)
constexpr float kLift = 7.f;

// The CTA's key tiles are numbered through, t = 0, 1, ...  Places in the ring, in the order in which the tensor core needs them:
// K0 K1 V0 K2 V1 K3 V2 ...
__device__ __forceinline__ uint32_t pos_k(uint32_t t) { return t ? 2 * t - 1 : 0; }
__device__ __forceinline__ uint32_t pos_v(uint32_t t) { return 2 * t + 2; }
// Of an item whose first tile is t0, a warpgroup has all tiles (two row tiles) or those with its parity.
__device__ __forceinline__ int first_step(uint32_t t0, bool dual, int wg) { return dual ? 0 : (int)((t0 + wg) & 1); }

// The tensor-memory lane of a warpgroup's first row.  Two row tiles: 0.  One with few rows: the second warpgroup's lie half a tile further, as
// they would otherwise be the work of one scheduler's warps.
__device__ __forceinline__ int first_row(bool dual, int wg, int rows) { return !dual && wg && rows <= 64 ? 64 : 0; }

// Two fp32 values in one 64-bit register pair: one instruction multiplies and adds both.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair2(float lo, float hi) { f32x2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi)); return r; }
__device__ __forceinline__ void unpair2(f32x2 v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) { f32x2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }

// (volatile: the order in the source is the order that is wanted)
__device__ __forceinline__ f32x2 fma2_here(f32x2 a, f32x2 b, f32x2 c) { f32x2 r; asm volatile("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ f32x2 add2_here(f32x2 a, f32x2 b) { f32x2 r; asm volatile("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ uint32_t pack_bf16_here(float lo, float hi) { uint32_t r; asm volatile("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo)); return r; }
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) { uint32_t r; asm volatile("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo)); return r; }
__device__ __forceinline__ uint32_t pack_f16_finite(float lo, float hi) { uint32_t r; asm volatile("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo)); return r; }

__device__ __forceinline__ float max3_nan(float a, float b, float c) { float r; asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c)); return r; }
__device__ __forceinline__ float max_nan(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }

// What tcgen05.ld brought may be used from here on (the wait before this has seen it arrive).
__device__ __forceinline__ void arrived(uint32_t (&r)[32]) {
#pragma unroll
  for (int i = 0; i < 32; ++i) asm volatile("" : "+r"(r[i]));
}

// ---------------------------------------------------------------- the kernel
template <int DP, bool E4M3>
__global__ void __launch_bounds__(Layout<DP, E4M3>::threads, 1)
attn_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
            const __grid_constant__ CUtensorMap tm_q1, const __grid_constant__ CUtensorMap tm_qn) {
  using L = Layout<DP, E4M3>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t sbase = smem_u32(smem);
  const uint32_t bar0 = sbase + L::misc;
  const uint32_t full = bar0, empty = bar0 + 64, s_full = bar0 + 128, o_done = bar0 + 160, q_ready = bar0 + 176,
                 w_full = bar0 + 192, w_empty = bar0 + 256, code_full = bar0 + 320, code_empty = bar0 + 384, p_ready = bar0 + 464, o_mid = bar0 + 496;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + L::misc + 448);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + L::misc + 452);
  volatile int* first_entity = reinterpret_cast<volatile int*>(smem + L::misc + 456);
  const uint32_t loaded = bar0 + 460;                                                  // ring places whose copies have been asked for
  Pair* scratch = reinterpret_cast<Pair*>(smem + L::misc + 512);                       // a block's warps' totals
  const uint32_t ex_turn = bar0 + 768;                                                 // [2][4] a warp of each warpgroup may take its exponentials
  const uint32_t q_free = bar0 + 832, q_raw = bar0 + 848;
  const Work* work = reinterpret_cast<const Work*>(smem + L::misc + 1024);
  const int words = attn_sched_words(a.p.B, a.p.G), n_codes = L::code_slots(words);
  uint8_t* sched_at = smem + L::codes + n_codes * L::code_bytes;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < L::stages; ++i) { mbar_init(full + 8 * i, E4M3 ? 4 : 1); mbar_init(empty + 8 * i, 2); }
    for (int i = 0; i < n_codes; ++i) { mbar_init(code_full + 8 * i, 1); mbar_init(code_empty + 8 * i, 4); }
    for (int i = 0; i < 4; ++i) { mbar_init(s_full + 8 * i, 1); mbar_init(p_ready + 8 * i, 4); }
    for (int i = 0; i < 8; ++i) mbar_init(ex_turn + 8 * i, 1);
    for (int i = 0; i < 2; ++i) { mbar_init(o_mid + 8 * i, 1); mbar_init(o_done + 8 * i, 1); mbar_init(q_free + 8 * i, 1); mbar_init(q_raw + 8 * i, 1); mbar_init(q_ready + 8 * i, E4M3 ? 4 : 1); }
    // readers of an item: the loading warp, the products of each warpgroup, eight row warps, four decoding warps
    for (int i = 0; i < kItemSlots; ++i) { mbar_init(w_full + 8 * i, 1); mbar_init(w_empty + 8 * i, E4M3 ? 15 : 11); }
    *abort_flag = 0;
    *reinterpret_cast<volatile uint32_t*>(smem + L::misc + 460) = 0;
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
  build_schedule(a, s, scratch, first_entity);

  // A stage of the ring has landed.  The barrier's parity tells two uses apart, not three: where the use before this one was the other
  // warpgroup's, it may not even have landed yet.  Once the copies of `pos` are asked for it has, and has been freed.  (Decoded codes
  // land in the order of their places: who has seen a later one has seen it.)  seen: places known to be asked for.
  auto wait_ring = [&](uint32_t pos, uint32_t& seen) -> bool {
    if (!E4M3 && seen <= pos) {
      uint32_t spin = 0;
      unsigned long long since = 0;
#pragma unroll 1
      for (;;) {
        asm volatile("ld.acquire.cta.shared::cta.u32 %0, [%1];" : "=r"(seen) : "r"(loaded) : "memory");
        if (seen > pos) break;
        if ((++spin & 255u) != 0u) continue;
        const unsigned long long now = globaltimer();
        if (since == 0) since = now;
        if (now - since > kWaitLimitNs) { *abort_flag = 1; atomicExch(&a.status[kStTimeout], 1); }
        if (*abort_flag) return false;
      }
    }
    return wait_bar(full + 8 * (pos % L::stages), (pos / L::stages) & 1, abort_flag, a.status);
  };
  // the next item; every reader gives it back after its last look
  uint32_t turn = 0;
  auto take = [&]() -> const Work& {
    wait_bar(w_full + 8 * (turn % kItemSlots), (turn / kItemSlots) & 1, abort_flag, a.status);
    return work[turn % kItemSlots];
  };
  auto give_back = [&]() {
    __syncwarp();
    if (lane == 0) mbar_arrive(w_empty + 8 * (turn % kItemSlots));
    ++turn;
  };
  // a key tile of an item: where its keys begin, and how many there are from there on
  auto keys_of = [](const Work& it, int j, int& key0) {
    const int step = it.s0 + j;
    const bool in_ahead = step < it.n_ahead;
    key0 = (in_ahead ? step : step - it.n_ahead) * kAttnTile;
    return (in_ahead ? it.ahead : it.own) - key0;
  };

  if (warp == kLoadWarp) {
    // ------------------------------------------------------ keys and values, page by page
    const int page = 1 << a.page_shift, box = page < kAttnTile ? page : kAttnTile, box_shift = page < kAttnTile ? a.page_shift : 7;
    const int places = E4M3 ? n_codes : L::stages;
    int bad = 0;
    bool alive = true;
    uint32_t issued = 0;
    Work it;
    int j = 0;
    // What a lane has to fetch of the tile (item `it`, step j).
    struct Fetch { int page, in_page, head; bool want; };
    auto look = [&]() -> Fetch {
      int key0;
      const int keys = keys_of(it, j, key0), key = lane << box_shift;
      Fetch f{0, key0 & (page - 1), it.head, lane < (kAttnTile >> box_shift) && key < keys};
      if (f.want) {
        const int32_t* table = it.s0 + j < it.n_ahead ? a.prefix_pages + (long long)it.g * a.prefix_stride : a.page_table + (long long)it.b * a.table_stride;
        f.page = table[(key0 + key) >> a.page_shift];
      }
      return f;
    };
    auto load = [&](uint32_t pos, const CUtensorMap* tm, const Fetch& f) {
      const int st = pos % places;
      const uint32_t landed = (E4M3 ? code_full : full) + 8 * st, free = (E4M3 ? code_empty : empty) + 8 * st;
      alive = __all_sync(0xffffffffu, wait_bar(free, ((pos / places) & 1) ^ 1, abort_flag, a.status));
      if (!alive) return;
      issued = pos + 1;
      const int pages = __popc(__ballot_sync(0xffffffffu, f.want));
      const bool known = f.page >= 0 && f.page < a.n_pages;
      const int from = known ? f.page : a.n_pages;          // (behind the last page: reads zeros)
      bad |= f.want && !known;
      if (lane == 0) mbar_expect_tx(landed, pages * box * (E4M3 ? DP : 128 * L::halves));
      __syncwarp();
      if (f.want) {
        if (E4M3) {
          tma_load_4d(sbase + L::codes + st * L::code_bytes + (lane << box_shift) * DP, tm, 0, f.in_page, f.head, from, landed);
        } else {
#pragma unroll
          for (int h = 0; h < L::halves; ++h)
            tma_load_4d(sbase + L::ring + st * L::tile_bytes + h * kHalfBytes + ((lane << box_shift) * 128), tm, h * 64, f.in_page, f.head, from, landed);
        }
      }
      __syncwarp();
      if (!E4M3 && lane == 0) asm volatile("st.release.cta.shared::cta.u32 [%0], %1;" ::"r"(loaded), "r"(pos + 1) : "memory");
    };
    auto next_tile = [&]() -> bool {                        // moves on to the next tile, if there is one
      if (++j < it.n) return true;
      it = take();
      if (__any_sync(0xffffffffu, it.n == 0 || *abort_flag)) return false;
      give_back();
      j = 0;
      return true;
    };
    it.n = 0;
    bool more = true;
    Fetch next, now, last;
    next.want = false;
    // tile t's K, then tile t - 1's V; the page ids of tile t + 1 arrive while tile t waits for its place
    for (uint32_t t = 0; alive; ++t) {
      last = now; now = next;
      const bool have = more;                               // (in the first round: a tile that is none)
      more = more && next_tile();
      if (more) next = look();
      if (t == 0) { if (!more) break; continue; }
#pragma unroll 1
      for (int v = 0; v < 2; ++v) {                         // tiles are numbered from 0, rounds from 1
        if (v == 0 ? have : t > 1) { if (alive) load(v == 0 ? pos_k(t - 1) : pos_v(t - 2), v == 0 ? &tm_k : &tm_v, v == 0 ? now : last); }
      }
      if (!have) break;
    }
    if (bad) atomicExch(&a.status[kStBadRouting], 1);
    if (!alive) {                                           // copies in flight land before the block's memory is given up
      const unsigned long long t0 = globaltimer();
      for (uint32_t pos = issued > (uint32_t)places ? issued - places : 0; pos < issued; ++pos)
        while (!mbar_try_wait((E4M3 ? code_full : full) + 8 * (pos % places), (pos / places) & 1) && globaltimer() - t0 < 100000000ull) {}
    }
  } else if (__builtin_expect(warp == kItemWarp, 0)) {
    // ------------------------------------------------------ the CTA's share of the schedule, item by item, and the items' Q
    // (Not expected: so its code is laid out behind the others' loops.  Between them its length moves these about in the instruction cache that
    // all share, which made up to 8 % of an e4m3 batch's decoding: 159 us for 128 requests over 5000 shared and 1500 own keys against 172.)
    const int x0 = blockIdx.x * s.share, x1 = x0 + s.share;
    AttnWalk k;
    k.done = *first_entity < 0;
    if (!k.done) k = attn_walk_in(p, s, *first_entity, x0);
    Work* out = const_cast<Work*>(work);
    uint32_t t0 = 0, q_turn[2] = {0, 0};
    bool alive = true;
#pragma unroll 1
    while (alive) {
      Work w;
      w.n = 0; w.n_tok = 0; w.flags = 0; w.hi = 0; w.lo = 0; w.tok = 0; w.head = 0;
#pragma unroll 1
      for (; !k.done && k.at < x1 && w.n == 0; attn_walk_next(p, s, &k)) {
        const AttnItem it = attn_item(p, s, k);
        const int s0 = attn_steps_before(k, it.n, x0), s1 = attn_steps_before(k, it.n, x1);
        w.n = s1 - s0; w.s0 = s0;
        if (w.n == 0) continue;
        w.head = it.head; w.n_tok = it.n_tok; w.ahead = it.ahead; w.own = it.own; w.n_ahead = it.n_ahead; w.b = it.b; w.g = it.g;
        w.flags = (it.dual ? kDual : 0) | (attn_is_whole(it, s0, s1) ? kWhole : 0);
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
      alive = __all_sync(0xffffffffu, wait_bar(w_empty + 8 * (turn % kItemSlots), ((turn / kItemSlots) & 1) ^ 1, abort_flag, a.status));
      if (!alive) break;
      if (lane == 0) { out[turn % kItemSlots] = w; mbar_arrive(w_full + 8 * (turn % kItemSlots)); }
      ++turn;
      if (w.n == 0) break;
      // Q of each warpgroup with a part in the item, as soon as the products with its last Q are through.  Rows are tokens x heads, as the
      // tensor maps' boxes lay them: one box for tokens side by side that fill at least half a row tile, else one for each token.
#pragma unroll 1
      for (int wg = 0; wg < 2; ++wg) {
        const bool dual = w.flags & kDual;
        if (first_step(t0, dual, wg) >= w.n) continue;
        const int from = dual ? wg * p.tps : 0, count = max(0, min(dual ? p.tps : w.n_tok, w.n_tok - from));
        const uint32_t landed = (E4M3 ? q_raw : q_ready) + 8 * wg, dst = sbase + L::q + wg * L::tile_bytes + first_row(dual, wg, w.n_tok * p.Gh) * 128;
        alive = __all_sync(0xffffffffu, wait_bar(q_free + 8 * wg, (q_turn[wg]++ & 1) ^ 1, abort_flag, a.status));
        if (!alive) break;
        const bool box = w.hi == 0 && 2 * count > p.tps;
        if (lane == 0) mbar_expect_tx(landed, (box ? p.tps : count) * p.Gh * 128 * L::halves);
        __syncwarp();
        if (box) {
          if (lane < L::halves) tma_load_3d(dst + lane * kHalfBytes, &tm_qn, lane * 64, w.head * p.Gh, w.tok + from, landed);
          continue;
        }
#pragma unroll 1
        for (int i = lane; i < count * L::halves; i += 32) {
          const int tt = i / L::halves, h = i % L::halves;
          int token = w.tok + from + tt;
          if (w.hi > 0) { const int b = sequence_of(s.scum, w.lo, w.hi, token); token = s.q0[b] + (token - s.scum[b]); }
          tma_load_3d(dst + h * kHalfBytes + tt * p.Gh * 128, &tm_q1, h * 64, w.head * p.Gh, token, landed);
        }
      }
      t0 += w.n;
    }
    __syncwarp();
    if (!alive) {                                           // copies in flight land before the block's memory is given up
      const unsigned long long since = globaltimer();
      for (int wg = 0; wg < 2; ++wg)
        while (q_turn[wg] && !mbar_try_wait((E4M3 ? q_raw : q_ready) + 8 * wg, (q_turn[wg] - 1) & 1) && globaltimer() - since < 100000000ull) {}
    }
    // For the kernel that joins partial results: does this CTA's first item begin in the share before, and use the rows at the cuts?
    JoinPart cut{};
    k.done = *first_entity < 0;
    if (!k.done) k = attn_walk_in(p, s, *first_entity, x0);
    int cut_token = 0, cut_head = 0;
    if (!k.done && k.e >= p.G && x0 > 0 && !attn_has_rows(p, s, k.e - p.G)) {
      const AttnItem it = attn_item(p, s, k);
      const int before = attn_steps_before(k, it.n, x0);
      if (before > 0 && before < it.n && attn_steps_before(k, it.n, x0 - s.share) == 0) {
        cut = JoinPart{it.rows, k.at, k.w, it.n, it.n_tok, it.dual, 1};
        cut_token = s.q0[it.b] + it.tok; cut_head = it.head;
      }
    }
    write_records(a, s, cut, cut_token, cut_head);
  } else if (warp == kMmaWarp || warp == kMmaWarp2) {
    // ------------------------------------------------------ tensor core: one thread for each warpgroup's products
    // (Elected, not picked by its number: the compiler then knows that one thread issues, and a product of 128 x 128 x 16 takes its 64
    // cycles of the tensor core; from a thread picked by number every tcgen05 instruction takes 66 of its own, whatever its size.)
    if (elect_one()) {
      constexpr uint32_t type = E4M3 ? (1u << 7) | (1u << 10) : 0u;         // codes are decoded to fp16, whose type bits are 0 (bf16: 1)
      constexpr uint32_t idesc_s = make_idesc_bf16(128, 64) ^ type, idesc_o = (make_idesc_bf16(128, DP) | kTransposeB) ^ type;
      const int w = warp == kMmaWarp2;
      const uint32_t t_s = tmem + w * 128, t_o = tmem + 256 + w * 128;
      const uint64_t qd = make_smem_desc(sbase + L::q + w * L::tile_bytes);
      uint32_t t0 = 0, q_phase = 0, p_phase = 0, seen = 0;
      bool alive = true;
      auto wait = [&](uint32_t bar, uint32_t parity) { alive = alive && wait_bar(bar, parity & 1, abort_flag, a.status); };
      // A stage is free when both threads say so; a tile of one warpgroup is none of the other's business.
      auto free_stage = [&](bool dual, int st) {
        tc_commit(empty + 8 * st);
        if (!dual) mbar_arrive(empty + 8 * st);
      };
#pragma unroll 1
      while (alive) {
        const Work& it = take();
        const int n = it.n;
        const bool dual = it.flags & kDual;
        if (n == 0 || *abort_flag) break;
        mbar_arrive(w_empty + 8 * (turn % kItemSlots));
        ++turn;
        const int j0 = first_step(t0, dual, w), step = dual ? 1 : 2;
        // scores of half a tile's keys
        auto scores = [&](int j, int h) {
          const int sk = pos_k(t0 + j) % L::stages;
          const uint64_t kd = make_smem_desc(sbase + L::ring + sk * L::tile_bytes + h * (kHalfBytes / 2));
#pragma unroll
          for (int i = 0; i < DP / 16; ++i) {
            const uint64_t off = ((i >> 2) * kHalfBytes + (i & 3) * 32) >> 4;
            tc_mma_f16(t_s + h * 64, qd + off, kd + off, idesc_s, i > 0);
          }
          tc_commit(s_full + 16 * w + 8 * h);
          if (h) {
            free_stage(dual, sk);
            if (j + step >= n) tc_commit(q_free + 8 * w);
          }
        };
        auto wait_stage = [&](uint32_t pos) { alive = alive && wait_ring(pos, seen); tc_fence_after(); };
        if (j0 < n) {
          wait(q_ready + 8 * w, q_phase++);
          wait_stage(pos_k(t0 + j0));
          if (!alive) break;
          scores(j0, 0);
          scores(j0, 1);
        }
#pragma unroll 1
        for (int j = j0; j < n && alive; j += step) {
          const uint32_t pv = pos_v(t0 + j);
          const int sv = pv % L::stages;
          const bool more = j + step < n;
          wait_stage(pv);
          const uint64_t vd = make_v_desc(sbase + L::ring + sv * L::tile_bytes);
#pragma unroll 1
          for (int h = 0; h < 2; ++h) {                     // the other half's weights are on their way meanwhile
            wait(p_ready + 16 * w + 8 * h, p_phase);
            if (!alive) break;
            tc_fence_after();
#pragma unroll
            for (int i = 0; i < 4; ++i)
              tc_mma_f16_ts(t_o, t_s + h * 64 + i * 8, vd + ((h * 64 + i * 16) * 128 >> 4), idesc_o, i + h ? 1u : (uint32_t)(j != j0));
            if (h == 0) tc_commit(o_mid + 8 * w); else free_stage(dual, sv);
            if (more) {
              if (h == 0) wait_stage(pos_k(t0 + j + step));
              if (!alive) break;
              scores(j + step, h);
            }
          }
          ++p_phase;
          if (!more && alive) tc_commit(o_done + 8 * w);
        }
        t0 += n;
      }
    }
    __syncwarp();
  } else if (E4M3 && warp >= kCodeWarp) {
    // ------------------------------------------------------ codes to fp16, which holds every e4m3 value
    const int ct = tid & 127;
    bool alive = true;
    auto decode = [&](uint32_t pos, int keys) {
      const int st = pos % L::stages, slot = pos % n_codes;
      const bool ok = wait_bar(code_full + 8 * slot, (pos / n_codes) & 1, abort_flag, a.status) &&
                      wait_bar(empty + 8 * st, ((pos / L::stages) & 1) ^ 1, abort_flag, a.status);
      alive = __all_sync(0xffffffffu, ok);
      if (!alive) return;
      const uint8_t* src = smem + L::codes + slot * L::code_bytes;
      uint8_t* dst = smem + L::ring + st * L::tile_bytes;
      // 16 codes at a time.  Eight neighbouring threads take the left half of one row and the right half of the next (then the other way
      // round), so that neither their loads nor their stores meet in a bank.
      constexpr int rounds = kAttnTile * DP / 16 / 128;
      const int sub = ct >> 2 & 1, row0 = (ct >> 3) * 2 + sub;
      uint4 v[rounds];
#pragma unroll
      for (int u = 0; u < rounds; ++u) {
        const int row = DP == 64 ? u * 32 + (ct >> 2) : (u >> 1) * 32 + row0, c = DP == 64 ? ct & 3 : (ct & 3) + 4 * ((sub + u) & 1);
        v[u] = *reinterpret_cast<const uint4*>(src + row * DP + c * 16);
        if (row >= keys) v[u] = make_uint4(0, 0, 0, 0);    // what lies behind the last key may be anything: its weight 0 needs a finite value
      }
#pragma unroll
      for (int u = 0; u < rounds; ++u) {
        const int row = DP == 64 ? u * 32 + (ct >> 2) : (u >> 1) * 32 + row0, c = DP == 64 ? ct & 3 : (ct & 3) + 4 * ((sub + u) & 1);
        uint4 lo, hi;
        decode4(v[u].x, lo.x, lo.y); decode4(v[u].y, lo.z, lo.w);
        decode4(v[u].z, hi.x, hi.y); decode4(v[u].w, hi.z, hi.w);
        uint8_t* at = dst + (c >> 2) * kHalfBytes + row * 128;
        const int first = (((c & 3) * 2) ^ (row & 7)) << 4;
        *reinterpret_cast<uint4*>(at + first) = lo;
        *reinterpret_cast<uint4*>(at + (first ^ 16)) = hi;
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) { mbar_arrive(code_empty + 8 * slot); mbar_arrive(full + 8 * st); }
    };
    uint32_t t = 0;
    int before = 0, j = 0;
    bool more = true;
    Work it;
    it.n = 0;
#pragma unroll 1
    while (more && alive) {
      if (j == it.n) {
        it = take();
        more = !__any_sync(0xffffffffu, it.n == 0 || *abort_flag);
        if (more) give_back();
        j = 0;
      }
      int key0, keys = 0;
      if (more) keys = keys_of(it, j, key0);
#pragma unroll 1
      for (int v = 0; v < 2; ++v)                           // a tile's K, then the tile before's V
        if ((v == 0 ? more : t > 0) && alive) decode(v == 0 ? pos_k(t) : pos_v(t - 1), v == 0 ? keys : before);
      before = keys;
      ++t; ++j;
    }
  } else if (warp < kMmaWarp) {
    // ------------------------------------------------------ rows: softmax, corrections, results
    // (After a wait that was given up an item's steps run on with what is there: what a warp does must not differ by lane.)
    const int wg = warp >> 2, row = tid & 127;
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;      // this warp's 32 lanes of tensor memory
    const uint32_t t_s = tmem + lanes + wg * 128, t_o = tmem + lanes + 256 + wg * 128;
    const uint32_t my_turn = ex_turn + 32 * wg + 8 * (warp & 3), other_turn = ex_turn + 32 * (wg ^ 1) + 8 * (warp & 3);
    const uint32_t gh_magic = 65536u / p.Gh + 1;            // x / Gh for x < 128: (x * gh_magic) >> 16
    uint32_t s_phase = 0, o_phase = 0, t0 = 0, e_phase = 0, q_phase = 0;
    // This thread's row of an item.
    struct Row { int n, j, s0, n_ahead, ahead, own, seen, kvh, head, token; bool dual, whole, mine, active; uint32_t t0; long long prow; float sl2; };
    // The next item that this warpgroup has a part in.
    auto next_item = [&](Row& r) -> bool {
      for (;;) {
        const Work& it = take();
        const int n = it.n;
        if (__any_sync(0xffffffffu, n == 0 || *abort_flag)) return false;
        const bool dual = it.flags & kDual;
        const int j = first_step(t0, dual, wg);
        if (j >= n) { give_back(); t0 += n; continue; }
        r.n = n; r.j = j; r.t0 = t0; r.dual = dual; r.whole = it.flags & kWhole;
        r.s0 = it.s0; r.n_ahead = it.n_ahead; r.ahead = it.ahead; r.own = it.own;
        const int at = row - first_row(dual, wg, it.n_tok * p.Gh);
        const int row_tok = (int)(((uint32_t)at * gh_magic) >> 16), row_head = at - row_tok * p.Gh;
        const int tt = (dual ? wg * p.tps : 0) + row_tok, kvh = it.head;      // token of the item
        r.mine = at >= 0 && row_tok < p.tps && tt < it.n_tok;
        r.token = it.tok + tt;
        r.seen = it.own;
        if (r.mine) {
          if (it.hi > 0) {
            const int b = sequence_of(s.scum, it.lo, it.hi, r.token);
            r.token = s.q0[b] + (r.token - s.scum[b]);
          } else if (p.causal) {
            r.seen = it.seen + tt;
          }
        }
        r.kvh = kvh; r.head = kvh * p.Gh + row_head;        // (the head of nobody's row is not one)
        // partial rows: those of the item's tokens; where the warpgroups take turns, once for the one with the first tile and once for the other
        r.prow = it.prow + (long long)(tt + (dual ? 0 : j * it.n_tok)) * p.Gh + row_head;
        t0 += n;
        give_back();
        r.active = __any_sync(0xffffffffu, r.mine);
        r.sl2 = a.scale_log2 * (a.k_scale ? a.k_scale[kvh] : 1.f);
        return true;
      }
    };
    // e4m3 caches: a row of Q as fp16, times the power of two that brings its largest value to 2^14 (exact; what falls below fp16's range
    // then is 2^-38 of the largest).  The scores are taken back by sl2.
    auto convert_q = [&](Row& r) {
      wait_bar(q_raw + 8 * wg, q_phase++ & 1, abort_flag, a.status);
      if (r.active) {
        uint8_t* mine = smem + L::q + wg * L::tile_bytes + row * 128;
        auto part = [&](int c) { return reinterpret_cast<uint4*>(mine + (c >> 3) * kHalfBytes + (((c & 7) ^ (row & 7)) << 4)); };
        uint32_t top = 0;
#pragma unroll 4
        for (int c = 0; c < DP / 8; ++c) {
          const uint4 v = *part(c);
          const uint32_t w4[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int k = 0; k < 4; ++k) top = max(top, max(w4[k] & 0x7fffu, w4[k] >> 16 & 0x7fffu));
        }
        const int e = (int)(top >> 7);                      // biased exponent of the largest
        const int shift = e == 0 || e == 255 ? 0 : min(100, 127 + 14 - e);
        const float up = __int_as_float((127 + shift) << 23);
        r.sl2 *= __int_as_float((127 - shift) << 23);
        auto half2 = [&](uint32_t w2) { return pack_f16(__uint_as_float(w2 << 16) * up, __uint_as_float(w2 & 0xffff0000u) * up); };
#pragma unroll 4
        for (int c = 0; c < DP / 8; ++c) {
          const uint4 v = *part(c);
          *part(c) = make_uint4(half2(v.x), half2(v.y), half2(v.z), half2(v.w));
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(q_ready + 8 * wg);
    };
    Row r{}, next{};
    float m = 0.f, l = 0.f;                                 // maximum that the sums refer to (unscaled), sum
    bool first_round = true;
    // the item's result: its rows, or partial ones
    auto result = [&]() {
      wait_bar(o_done + 8 * wg, o_phase & 1, abort_flag, a.status);
      ++o_phase;
      tc_fence_after();
      if (r.active) {
        const float m2 = m == -CUDART_INF_F ? m : E4M3 ? m * r.sl2 - kLift : m * r.sl2;
        const float inv = l > 0.f ? (a.v_scale ? a.v_scale[r.kvh] : 1.f) / l : l;        // (a NaN stays)
        // (A row per lane: 32 lines with every access, 4 us for two full row tiles; the other warpgroup works meanwhile.)
        if (r.whole) {
          uint16_t* dst = a.out + (long long)r.token * a.out_tok + (long long)r.head * a.out_head;
#pragma unroll 1
          for (int c = 0; c < DP; c += 32) {
            uint32_t o[32];
            tc_ld32(t_o + c, o);
            tc_wait_ld();
#pragma unroll
            for (int i = 0; i < 32; i += 8) {
              uint32_t w[4];
#pragma unroll
              for (int q = 0; q < 4; ++q) w[q] = l == 0.f ? 0u : pack_bf16(__uint_as_float(o[i + 2 * q]) * inv, __uint_as_float(o[i + 2 * q + 1]) * inv);
              if (r.mine && c + i < a.D) *reinterpret_cast<uint4*>(dst + c + i) = make_uint4(w[0], w[1], w[2], w[3]);
            }
          }
        } else {
          float* dst = a.part_o + r.prow * DP;
#pragma unroll 1
          for (int c = 0; c < DP; c += 32) {
            uint32_t o[32];
            tc_ld32(t_o + c, o);
            tc_wait_ld();
#pragma unroll
            for (int i = 0; i < 32; i += 4)
              if (r.mine) *reinterpret_cast<uint4*>(dst + c + i) = make_uint4(o[i], o[i + 1], o[i + 2], o[i + 3]);
          }
        }
        if (r.mine && !r.whole) a.part_ml[r.prow] = make_float2(m2, l);
        if (r.mine && r.whole && a.lse) a.lse[(long long)r.token * a.lse_tok + r.head] = (m2 + __log2f(l)) * 0.6931471805599453f;
      }
      tc_fence_before();
    };
#pragma unroll 1
    for (;;) {
      const bool more = next_item(next);
      if (E4M3 && more) convert_q(next);                    // (while the last item's last product runs)
      if (!first_round) result();
      if (!more) break;
      first_round = false;
      r = next;
      m = -CUDART_INF_F; l = 0.f;
      bool any = false;                                     // O holds something
#pragma unroll 1
      for (int j = r.j; j < r.n; j += r.dual ? 1 : 2) {
        const int step = r.s0 + j;
        const bool in_ahead = step < r.n_ahead;
        const int key0 = (in_ahead ? step : step - r.n_ahead) * kAttnTile, keys = (in_ahead ? r.ahead : r.own) - key0;
        // Two warps, one of each warpgroup, share a scheduler and its unit for exponentials, and fall into step: with heads above 64 they
        // take turns at it (4096 tokens behind 8192 keys: 983 against 1022 us; heads of 64 lose, 941 against 891, and so do e4m3 caches,
        // 1127 against 1095, where other warps' work fills the gaps).
        constexpr bool turns = DP == 128 && !E4M3;
        auto take_turn = [&]() {
          if (turns && r.dual) wait_bar(my_turn, (e_phase & 1) ^ (wg ^ 1), abort_flag, a.status);
        };
        auto pass_turn = [&]() {
          if (!turns || !r.dual) return;
          ++e_phase;
          if (lane == 0) mbar_arrive(other_turn);
        };
        const int see = in_ahead ? keys : (r.seen - key0 < keys ? r.seen - key0 : keys);
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {                       // half the keys; the tensor core works on the other half
          wait_bar(s_full + 16 * wg + 8 * h, s_phase & 1, abort_flag, a.status);
          tc_fence_after();
          if (!E4M3 && h == 0 && keys < kAttnTile) {                    // what lies behind the last key may be anything: its weight 0 needs a finite value.
            const uint32_t pos = pos_v(r.t0 + j);
            uint32_t seen = 0;
            wait_ring(pos, seen);
            uint8_t* v = smem + L::ring + (pos % L::stages) * L::tile_bytes;
            const int from = keys < 0 ? 0 : keys;
#pragma unroll 1
            for (int h = 0; h < L::halves; ++h)
#pragma unroll 1
              for (int i = from * 8 + (tid & 127); i < kAttnTile * 8; i += 128) *reinterpret_cast<uint4*>(v + h * kHalfBytes + i * 16) = make_uint4(0, 0, 0, 0);
            fence_proxy_async_smem();
          }
          if (r.active) {
            uint32_t x[2][32];
            tc_ld32(t_s + h * 64, x[0]);
            tc_ld32(t_s + h * 64 + 32, x[1]);
            tc_wait_ld();
            arrived(x[0]); arrived(x[1]);
            if (__any_sync(0xffffffffu, see < h * 64 + 64)) {
#pragma unroll
              for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int i = 0; i < 32; ++i) x[c][i] = h * 64 + c * 32 + i < see ? x[c][i] : 0xff800000u;
            }
            float top[4] = {m, __uint_as_float(x[0][31]), __uint_as_float(x[1][31]), m};
#pragma unroll
            for (int i = 0; i < 31; ++i) {
              if ((i & 1) == 0 && i + 1 < 31) {
                top[i & 2 ? 0 : 1] = max3_nan(top[i & 2 ? 0 : 1], __uint_as_float(x[0][i]), __uint_as_float(x[0][i + 1]));
                top[i & 2 ? 3 : 2] = max3_nan(top[i & 2 ? 3 : 2], __uint_as_float(x[1][i]), __uint_as_float(x[1][i + 1]));
              }
            }
            top[0] = max3_nan(top[0], top[1], __uint_as_float(x[0][30]));
            top[3] = max3_nan(top[3], top[2], __uint_as_float(x[1][30]));
            const float m_new = max_nan(top[0], top[3]);
            // The sums keep referring to an older maximum until weights could pass 2^8: fp32 and the weights' type carry that exactly as well.
            // (A NaN raises too: it then is in the sums.)
            const bool raise = r.mine && m_new != m && !((m_new - m) * r.sl2 <= 8.f);
            if (!any) {
              m = m_new;
            } else if (__any_sync(0xffffffffu, raise)) {
              // O stands still once the product before is through, which comes before the other half's next scores (o_mid: this tile's first half)
              if (h == 0) wait_bar(s_full + 16 * wg + 8, s_phase & 1, abort_flag, a.status);
              else wait_bar(o_mid + 8 * wg, s_phase & 1, abort_flag, a.status);
              tc_fence_after();
              const float f = raise ? ex2((m - m_new) * r.sl2) : 1.f;
              if (raise) { m = m_new; l *= f; }
#pragma unroll 1
              for (int c = 0; c < DP / 16; ++c) {
                uint32_t o[16];
                tc_ld16(t_o + c * 16, o);
                tc_wait_ld();
#pragma unroll
                for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                tc_st16(t_o + c * 16, o);
              }
              tc_wait_st();
            }
            any = true;
            // no key seen yet: all weights 0; an infinite score: NaN
            const float shift = m == -CUDART_INF_F ? 0.f : m == CUDART_INF_F ? CUDART_NAN_F : E4M3 ? kLift - m * r.sl2 : -m * r.sl2;
            const f32x2 scale2 = pair2(r.sl2, r.sl2), shift2 = pair2(shift, shift);
            f32x2 sum[4] = {0, 0, 0, 0};
            // The unit for exponentials takes 8 cycles a warp for each: what comes before and after them is put between them (a
            // pair's scaling kAhead pairs ahead, its sum and rounding kBehind pairs behind), in this order, in place.
            auto scaled = [&](int i) {
              float z0, z1;
              unpair2(fma2_here(pair2(__uint_as_float(x[i >> 4][2 * i & 31]), __uint_as_float(x[i >> 4][(2 * i & 31) + 1])), scale2, shift2), z0, z1);
              x[i >> 4][2 * i & 31] = __float_as_uint(z0); x[i >> 4][(2 * i & 31) + 1] = __float_as_uint(z1);
            };
            constexpr int kAhead = 4, kBehind = 4;
            uint32_t w[2][16];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) scaled(i);
            take_turn();
#pragma unroll
            for (int i = 0; i < 32 + kBehind; ++i) {
              if (i + kAhead < 32) scaled(i + kAhead);
              if (i < 32) {
                uint32_t &u = x[i >> 4][2 * i & 31], &v = x[i >> 4][(2 * i & 31) + 1];
                u = __float_as_uint(ex2_here(__uint_as_float(u)));
                v = __float_as_uint(ex2_here(__uint_as_float(v)));
              }
              if (i == 31) pass_turn();
              if (i >= kBehind) {
                const int k = i - kBehind;
                const float p0 = __uint_as_float(x[k >> 4][2 * k & 31]), p1 = __uint_as_float(x[k >> 4][(2 * k & 31) + 1]);
                w[k >> 4][k & 15] = E4M3 ? pack_f16_finite(p0, p1) : pack_bf16_here(p0, p1);
                sum[k & 3] = add2_here(sum[k & 3], pair2(p0, p1));
                if (k == 15) tc_st16(t_s + h * 64, w[0]);
              }
            }
            tc_st16(t_s + h * 64 + 16, w[1]);
            float s0, s1;
            unpair2(add2(add2(sum[0], sum[1]), add2(sum[2], sum[3])), s0, s1);
            l += s0 + s1;
            tc_wait_st();
          } else {
            take_turn();
            pass_turn();
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(p_ready + 16 * wg + 8 * h);
        }
        ++s_phase;
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kMmaWarp) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

// ---------------------------------------------------------------- rows whose keys were in several places

// A row's running (maximum, sum, output), in log2 and unscaled; o: a lane's columns 4 lane .. + 3.
struct Joined { float m, l; float4 o; };

// Lane i has the first row of the i-th partial result of a round of 32 (-1: none), two for each CTA from c0 on.
__device__ __forceinline__ long long part_place(const AttnArgs& a, int share, const JoinPart& j, int c0, int c_hi) {
  const int lane = threadIdx.x & 31, c = c0 + (lane >> 1);
  if (c > c_hi) return -1;
  AttnWalk k;
  k.at = j.at; k.w = j.w;
  AttnItem it;
  it.rows = j.rows; it.dual = j.dual;
  const int s0 = attn_steps_before(k, j.n, c * share), s1 = attn_steps_before(k, j.n, (c + 1) * share);
  return s0 < s1 && (lane & 1) < attn_part_count(it, s0, s1) ? attn_part_row(it, c, s0) + (lane & 1) * j.n_tok * a.p.Gh : -1;
}

// Joins a round of partial results into `n` (up to N) rows, row0 and those behind it; every lane's loads for all rows go out together.
template <int DP, int N>
__device__ __forceinline__ void join_rows(const AttnArgs& a, long long place, int row0, int n, Joined (&j)[N]) {
  const int lane = threadIdx.x & 31;
  float2 ml[N];
  float f[N];
#pragma unroll
  for (int i = 0; i < N; ++i) ml[i] = place >= 0 && i < n ? a.part_ml[place + row0 + i] : make_float2(-CUDART_INF_F, 0.f);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float top = ml[i].x;
#pragma unroll
    for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    top = fmaxf(top, j[i].m);
    const float base = top == -CUDART_INF_F ? 0.f : top, keep = ex2(j[i].m - base);
    j[i].o.x *= keep; j[i].o.y *= keep; j[i].o.z *= keep; j[i].o.w *= keep;
    j[i].m = top;
    f[i] = ex2(ml[i].x - base);
    float add = ml[i].y * f[i];
#pragma unroll
    for (int d = 16; d; d >>= 1) add += __shfl_xor_sync(0xffffffffu, add, d);
    j[i].l = j[i].l * keep + add;
  }
  unsigned have = __ballot_sync(0xffffffffu, place >= 0);
#pragma unroll 4
  while (have) {
    const int src = __ffs(have) - 1;
    have &= have - 1;
    const long long r = __shfl_sync(0xffffffffu, place, src) + row0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float g = __shfl_sync(0xffffffffu, f[i], src);
      if (i < n && lane < DP / 4) {
        const float4 v = *reinterpret_cast<const float4*>(a.part_o + (r + i) * DP + lane * 4);
        j[i].o.x += v.x * g; j[i].o.y += v.y * g; j[i].o.z += v.z * g; j[i].o.w += v.w * g;
      }
    }
  }
}

template <int DP>
__device__ __forceinline__ void write_row(const AttnArgs& a, int token, int head, int kvh, const Joined& j) {
  const int lane = threadIdx.x & 31;
  const float inv = j.l > 0.f ? (a.v_scale ? a.v_scale[kvh] : 1.f) / j.l : j.l;
  if (lane * 4 < a.D) {
    const uint2 v = j.l == 0.f ? make_uint2(0, 0) : make_uint2(pack_bf16(j.o.x * inv, j.o.y * inv), pack_bf16(j.o.z * inv, j.o.w * inv));
    *reinterpret_cast<uint2*>(a.out + (long long)token * a.out_tok + (long long)head * a.out_head + lane * 4) = v;
  }
  if (lane == 0 && a.lse) a.lse[(long long)token * a.lse_tok + head] = (j.m + __log2f(j.l)) * 0.6931471805599453f;
}

// Rows of two kinds.  A token of a sequence with partial rows of its own: its group's prefix and its own keys, or both in one item; a
// unit of work is up to kJoinRows of its heads that share a kv head.  A longer sequence's item that a cut between two CTAs' shares went
// through, found at its first cut: a unit is kJoinRows of its rows.
constexpr int kJoinThreads = 256, kJoinRows = 4;

template <int DP>
__global__ void __launch_bounds__(kJoinThreads, 2)
attn_join_kernel(const __grid_constant__ AttnArgs a) {
  pdl_enter();
  const AttnShape& p = a.p;
  const int tid = threadIdx.x, warp = tid >> 5, warps = kJoinThreads / 32;
  const JoinRecords rec = records_of(a);
  const int share = rec.head[0], tokens = rec.head[1];
  const int per_head = (p.Gh + kJoinRows - 1) / kJoinRows, per_token = p.Hkv * per_head;
  const int n_own = tokens * per_token;                     // (below 2^31: checked by the plan)
  const int tile = 2 * p.tps, per_cut = (tile * p.Gh + kJoinRows - 1) / kJoinRows;
  const int n_units = n_own + (p.T > tile ? (p.n_ctas - 1) * per_cut : 0);
#pragma unroll 1
  for (int u = blockIdx.x * warps + warp; u < n_units; u += gridDim.x * warps) {
    Joined j[kJoinRows];
#pragma unroll
    for (int i = 0; i < kJoinRows; ++i) j[i] = Joined{-CUDART_INF_F, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
    const bool own = u < n_own;
    int row0, n, token, kvh, head = 0;                      // row of the token (of the cut item); rows; token of row 0; its head
    JoinPart part, ahead;
    int rows_ahead = 0;                                     // rows of the group's item before row 0's
    ahead.n = 0;
    if (own) {
      const int i = u / per_token, in_token = u - i * per_token;
      const JoinSeq q = rec.seq[rec.seq_of[i]];
      kvh = in_token / per_head;
      row0 = (in_token - kvh * per_head) * kJoinRows;
      n = min(kJoinRows, p.Gh - row0);
      head = kvh * p.Gh + row0;
      const int t = i - q.first;
      token = q.q0 + t;
      part = q.part;
      part.at += kvh * part.w;
      part.rows += 2ll * kvh * part.n_tok * p.Gh;
      row0 += t * p.Gh;
      if (q.g >= 0) {
        const JoinGroup g = rec.group[q.g];
        const int in_group = q.in_group + t, r = attn_div(in_group, tile);
        ahead = g.part;
        ahead.at += (kvh * g.items + r) * ahead.w;
        ahead.rows += (long long)(kvh * g.items + r) * tile * p.Gh;
        ahead.n_tok = min(tile, g.n_short - r * tile);
        rows_ahead = (in_group - r * tile - t) * p.Gh;
      }
    } else {
      const int cut = (u - n_own) / per_cut;
      row0 = (u - n_own - cut * per_cut) * kJoinRows;
      const JoinCut c = rec.cut[cut + 1];
      part = c.part;
      n = min(kJoinRows, part.n_tok * p.Gh - row0);
      token = c.token; kvh = c.head;
      if (part.n == 0 || n <= 0) continue;
    }
    bool final = false;
#pragma unroll 1
    for (int side = 0; side < 2; ++side) {
      const JoinPart x = side ? part : ahead;
      if (x.n == 0) continue;
      const int c_lo = x.at / share, c_hi = (x.at + x.w - 1) / share;
      if (own && x.joint) {                                 // all in one part, which wrote the rows themselves?
        AttnWalk k;
        k.at = x.at; k.w = x.w;
        final = attn_steps_before(k, x.n, (c_lo + 1) * share) == x.n && (x.dual || x.n == 1);
        if (final) break;
      }
      const int row = row0 + (side ? 0 : rows_ahead);
#pragma unroll 1
      for (int c0 = c_lo; c0 <= c_hi; c0 += 16) join_rows<DP>(a, part_place(a, share, x, c0, c_hi), row, n, j);
    }
    if (final) continue;
#pragma unroll
    for (int i = 0; i < kJoinRows; ++i) {
      if (i >= n) break;
      const int r = row0 + i, tt = own ? 0 : attn_div(r, p.Gh);
      write_row<DP>(a, token + tt, own ? head + i : kvh * p.Gh + (r - tt * p.Gh), kvh, j[i]);
    }
  }
}

// A warp per unit up to four blocks per SM, which the host bounds by what the tokens may need: it does not know the lengths.
int join_blocks(const AttnArgs& a) {
  const long long per_token = (long long)a.p.Hkv * ((a.p.Gh + kJoinRows - 1) / kJoinRows);
  const long long units = std::min<long long>(a.p.T, 2ll * a.p.tps * a.p.B) * per_token + (a.p.n_ctas - 1) * (long long)((2 * a.p.tps * a.p.Gh + kJoinRows - 1) / kJoinRows);
  return (int)std::min<long long>(4 * a.p.n_ctas, (units + kJoinThreads / 32 - 1) / (kJoinThreads / 32));
}

template <int DP, bool E4M3>
cudaError_t launch_dim(const AttnArgs& a, const CUtensorMap& tk, const CUtensorMap& tv, const CUtensorMap& q1, const CUtensorMap& qn, cudaStream_t s) {
  const int words = attn_sched_words(a.p.B, a.p.G);
  cudaError_t e = launch_pdl(attn_kernel<DP, E4M3>, dim3(a.p.n_ctas), dim3(Layout<DP, E4M3>::threads), Layout<DP, E4M3>::smem(words), s, 1, a, tk, tv, q1, qn);
  if (e != cudaSuccess) return e;
  return launch_pdl(attn_join_kernel<DP>, dim3(join_blocks(a)), dim3(kJoinThreads), 0, s, 1, a);
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

namespace {
// A tensor map of 16-byte aligned elements in 128-byte swizzled (bf16) or plain (e4m3) boxes; a stride counts where there is a second
// element along it.
int encode(GemmTensorMap* out, const void* base, bool e4m3, int rank, const long long* n, const int64_t* stride, const int* box_of) {
  typedef CUresult (*Encode)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                             const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static Encode enc = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    const bool ok = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess;
    return ok ? reinterpret_cast<Encode>(p) : nullptr;
  }();
  if (!enc) return -1;
  const int elt = e4m3 ? 1 : 2;
  cuuint64_t dims[4], strides[3];
  cuuint32_t box[4], es[4] = {1, 1, 1, 1};
  for (int i = 0; i < rank; ++i) { dims[i] = (cuuint64_t)n[i]; box[i] = (cuuint32_t)box_of[i]; }
  for (int i = 1; i < rank; ++i) strides[i - 1] = (cuuint64_t)(n[i] > 1 ? stride[i] * elt : (n[0] * elt + 15) / 16 * 16);
  const CUresult r = enc(reinterpret_cast<CUtensorMap*>(out), e4m3 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank,
                         const_cast<void*>(base), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                         e4m3 ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? 0 : -2;
}
}  // namespace

int make_cache_map(GemmTensorMap* out, const void* base, const cep_attn_config& c, const int64_t* stride) {
  const bool e4m3 = c.cache_elem == CEP_ELEM_E4M3;
  const long long n[4] = {c.head_dim, c.page_size, c.n_kv_heads, c.n_pages};
  const int64_t st[4] = {1, stride[1], stride[2], stride[0]};
  const int box[4] = {e4m3 ? attn_padded_dim(c.head_dim) : 64, c.page_size < kAttnTile ? c.page_size : kAttnTile, 1, 1};
  return encode(out, base, e4m3, 4, n, st, box);
}

int make_q_map(GemmTensorMap* out, const AttnArgs& a, int tokens) {
  const long long n[3] = {a.D, a.p.Hq, a.p.T};
  const int64_t st[3] = {1, a.q_head, a.q_tok};
  const int box[3] = {64, a.p.Gh, tokens};
  return encode(out, a.q, false, 3, n, st, box);
}

cudaError_t launch_attn(const AttnArgs& a, int e4m3, const GemmTensorMap (&maps)[4], cudaStream_t s) {
  auto map = [&](int i) -> const CUtensorMap& { return reinterpret_cast<const CUtensorMap&>(maps[i]); };
  const bool narrow = attn_padded_dim(a.D) == 64;
  if (e4m3) return narrow ? launch_dim<64, true>(a, map(0), map(1), map(2), map(3), s) : launch_dim<128, true>(a, map(0), map(1), map(2), map(3), s);
  return narrow ? launch_dim<64, false>(a, map(0), map(1), map(2), map(3), s) : launch_dim<128, false>(a, map(0), map(1), map(2), map(3), s);
}

}  // namespace cep
