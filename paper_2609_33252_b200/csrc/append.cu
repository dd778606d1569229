// New tokens on their way into attention: rotation of q and k by position, k and v to their slots in a paged cache.
//
// Per token: sines and cosines of R/2 angles, shared by all heads, then (n_heads + 2 n_kv_heads) heads that are read once and
// written once; memory is the bound.  A thread has the same parts of a token's heads for every token that its block comes to, so
// that all divisions are done once; it asks for them before the angles are computed, which then cost no time of their own.
// 16384 tokens of 56 + 2 x 8 heads of 128 (604 MB): 135 us, 4.5 TB/s (151 us with the parts found anew for each token, which is better
// for 1531 tokens of 36 heads of 80: 6.1 against 7.6 us).  Few warps bound it: 107 to 111 registers let an SM hold two blocks, 12 to 16 warps,
// which spend a third of their time at the barrier behind the angles.
// Heads that cannot be taken 16 bytes at a time go element by element: the same 16384 tokens 550 us.
//
// Angles: position * inv_freq reaches 10^6 and more, where fp32 has lost the turn's fraction.  The product with 1/(2 pi) is
// taken in fp64 (4 instructions a pair, B200 has them at half rate), the whole turns are dropped, and the rest, below half a
// turn, goes to sincospif.
#include <cuda_bf16.h>

#include <algorithm>

#include "cep_common.h"

namespace cep {
namespace {

// Threads per SM that the blocks which come to tokens again are counted for (768: 11.1 us where 1536 take 12.4, but 39.5 against 35.5 with small
// heads).  Registers let about 576 run at a time: the rest of the blocks start when the first have ended.
constexpr int kAppendPerSm = 1024;
constexpr int kAppendMaxThreads = 512, kAppendMaxDim = 1024;

struct AppendArgs {
  const uint16_t *q, *k, *v; uint16_t* q_out;
  uint8_t *k_cache, *v_cache;
  const int32_t* positions; const int64_t* slots; const float* inv_freq;
  const float *k_scale, *v_scale;
  int32_t* status;
  long long q_tok, q_head, qo_tok, qo_head, k_tok, k_head, v_tok, v_head;
  long long kc[3], vc[3];                    // page, position, head
  long long n_slots;
  int T, Hq, Hk, D, R, page_shift;
  int units;                                 // of a head: pairs of vectors
  int tokens;                                // that a block takes at a time
  int parts;                                 // blocks that share a token's heads (when there are few tokens)
  int groups;                                // of blocks, each with every groups-th round of tokens
};

template <int V> struct Vec;
template <> struct Vec<8> { typedef uint4 T; };
template <> struct Vec<1> { typedef uint16_t T; };

__device__ __forceinline__ float bf16_bits(uint32_t b) { return __uint_as_float(b << 16); }
__device__ __forceinline__ void unpack(uint16_t v, float (&f)[1]) { f[0] = bf16_bits(v); }
__device__ __forceinline__ void unpack(const uint4& v, float (&f)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { f[2 * i] = bf16_bits(w[i] & 0xffffu); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ uint32_t two_bf16(float lo, float hi) {
  __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t two_e4m3(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ void put_bf16(uint16_t* p, const float (&f)[1]) { *p = (uint16_t)two_bf16(f[0], 0.f); }
__device__ __forceinline__ void put_bf16(uint16_t* p, const float (&f)[8]) {
  *reinterpret_cast<uint4*>(p) = make_uint4(two_bf16(f[0], f[1]), two_bf16(f[2], f[3]), two_bf16(f[4], f[5]), two_bf16(f[6], f[7]));
}
__device__ __forceinline__ void put_e4m3(uint8_t* p, const float (&f)[1], float s) { *p = (uint8_t)two_e4m3(__fdiv_rn(f[0], s), 0.f); }
__device__ __forceinline__ void put_e4m3(uint8_t* p, const float (&f)[8], float s) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = two_e4m3(__fdiv_rn(f[2 * i], s), __fdiv_rn(f[2 * i + 1], s));
  *reinterpret_cast<uint2*>(p) = make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
}

// Cosines and sines of a token in shared memory: eight threads read eight neighbouring angles each, two 16-byte chunks at a time, which
// the swizzle keeps apart (angles as pairs of cosine and sine met four to a bank: the kernel waited for them).
__device__ __forceinline__ int angle_room(int half) { return (half + 7) / 8 * 8; }
__device__ __forceinline__ int angle_at(int i) { return (((i >> 2) ^ (i >> 5 & 1)) << 2) + (i & 3); }
__device__ __forceinline__ void put_turn(float* cosines, int room, int i, int position, float inv_freq) {
  const double turn = (double)position * ((double)inv_freq * 0.15915494309189533577);
  float s, c;
  sincospif((float)(2.0 * (turn - rint(turn))), &s, &c);
  cosines[angle_at(i)] = c;
  cosines[room + angle_at(i)] = s;
}
template <int V> __device__ __forceinline__ void get_turns(const float* p, int i, float (&f)[V]) {
  if (V == 8) {
    const float4 a = *reinterpret_cast<const float4*>(p + angle_at(i)), b = *reinterpret_cast<const float4*>(p + angle_at(i + 4));
    const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int j = 0; j < V; ++j) f[j] = v[j];
  } else {
    f[0] = p[angle_at(i)];
  }
}

// A unit of a head: two vectors of V columns.  Rotated columns: the vectors that turn with one another (halves), or 2V
// neighbouring columns (interleaved); behind them, and in v, 2V neighbouring columns that are copied.
struct Place { int head, first, second, angle; };          // column of each vector (second < 0: none), first angle (-1: copied)
template <int V, bool INTERLEAVED>
__device__ __forceinline__ Place place(const AppendArgs& a, int unit, int rotated) {
  Place p;
  p.head = unit / a.units;
  const int u = unit - p.head * a.units, turning = rotated / (2 * V);
  if (u < turning) {
    p.first = INTERLEAVED ? 2 * V * u : V * u;
    p.second = INTERLEAVED ? p.first + V : p.first + rotated / 2;
    p.angle = V * u;
  } else {
    p.first = rotated + 2 * V * (u - turning);
    p.second = p.first + V < a.D ? p.first + V : -1;
    p.angle = -1;
    if (p.first >= a.D) p.first = -1;
  }
  return p;
}

template <int V, bool INTERLEAVED, bool E4M3, int UNROLL>
__global__ void __launch_bounds__(kAppendMaxThreads) append_kernel(const __grid_constant__ AppendArgs a) {
  extern __shared__ __align__(16) float turns[];                        // [2][tokens][2][R/2 rounded up] cosines, sines
  typedef typename Vec<V>::T T;
  pdl_enter();
  const int group = blockIdx.x / a.parts, part = blockIdx.x - group * a.parts, half = a.R / 2, room = angle_room(half);
  const int per_token = (a.Hq + 2 * a.Hk) * a.units, n_units = a.tokens * per_token;
  const int tid = threadIdx.x, threads = blockDim.x, step = a.parts * threads;
  int buffer = 0;
#pragma unroll 1
  for (int base = part * threads; base < n_units; base += UNROLL * step) {
    // this thread's parts: columns, head, which of the tokens at a time; its tensors' base and strides
    Place pl[UNROLL];
    int tok[UNROLL];
    const uint16_t* src[UNROLL];
    long long src_tok[UNROLL];
#pragma unroll
    for (int i = 0; i < UNROLL; ++i) {
      const int u = base + i * step + tid;
      pl[i].first = -1; tok[i] = 0; src[i] = nullptr; src_tok[i] = 0;
      if (u >= n_units) continue;
      tok[i] = u / per_token;
      const int in_token = u - tok[i] * per_token;
      pl[i] = place<V, INTERLEAVED>(a, in_token, in_token < (a.Hq + a.Hk) * a.units ? a.R : 0);
      if (pl[i].first < 0) continue;
      const int h = pl[i].head;
      src[i] = h < a.Hq ? a.q + h * a.q_head : h < a.Hq + a.Hk ? a.k + (h - a.Hq) * a.k_head : a.v + (h - a.Hq - a.Hk) * a.v_head;
      src_tok[i] = h < a.Hq ? a.q_tok : h < a.Hq + a.Hk ? a.k_tok : a.v_tok;
    }
#pragma unroll 1
    for (long long t0 = (long long)group * a.tokens; t0 < a.T; t0 += (long long)a.groups * a.tokens) {
      const int n_tok = (int)min((long long)a.tokens, a.T - t0);
      T x[UNROLL], y[UNROLL];
      long long slot[UNROLL];
#pragma unroll
      for (int i = 0; i < UNROLL; ++i) {
        if (pl[i].first < 0 || tok[i] >= n_tok) continue;
        const uint16_t* from = src[i] + (t0 + tok[i]) * src_tok[i];
        x[i] = *reinterpret_cast<const T*>(from + pl[i].first);
        if (pl[i].second >= 0) y[i] = *reinterpret_cast<const T*>(from + pl[i].second);
        slot[i] = pl[i].head < a.Hq ? 0 : a.slots[t0 + tok[i]];
      }
      float* cs_of = turns + buffer * a.tokens * 2 * room;
      buffer ^= 1;                                         // (the other one may still be read)
      for (int i = tid; i < n_tok * half; i += threads) {
        const int t = i / half, f = i - t * half;
        put_turn(cs_of + t * 2 * room, room, f, a.positions[t0 + t], a.inv_freq[f]);
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < UNROLL; ++i) {
        if (pl[i].first < 0 || tok[i] >= n_tok) continue;
        float f[V], g[V];
        unpack(x[i], f);
        if (pl[i].second >= 0) unpack(y[i], g);
        if (pl[i].angle >= 0) {
          float co[V], si[V];
          get_turns<V>(cs_of + tok[i] * 2 * room, pl[i].angle, co);
          get_turns<V>(cs_of + tok[i] * 2 * room + room, pl[i].angle, si);
          if (INTERLEAVED && V > 1) {
#pragma unroll
            for (int j = 0; j < V; j += 2) {
              const float c0 = co[j / 2], s0 = si[j / 2], c1 = co[V / 2 + j / 2], s1 = si[V / 2 + j / 2];
              const float p0 = f[j], p1 = f[(j + 1) % V], r0 = g[j], r1 = g[(j + 1) % V];
              f[j] = p0 * c0 - p1 * s0; f[(j + 1) % V] = p0 * s0 + p1 * c0;
              g[j] = r0 * c1 - r1 * s1; g[(j + 1) % V] = r0 * s1 + r1 * c1;
            }
          } else {
#pragma unroll
            for (int j = 0; j < V; ++j) {
              const float p0 = f[j], p1 = g[j];
              f[j] = p0 * co[j] - p1 * si[j]; g[j] = p0 * si[j] + p1 * co[j];
            }
          }
        }
        int h = pl[i].head;
        if (h < a.Hq) {
          uint16_t* dst = a.q_out + (t0 + tok[i]) * a.qo_tok + h * a.qo_head;
          put_bf16(dst + pl[i].first, f);
          if (pl[i].second >= 0) put_bf16(dst + pl[i].second, g);
          continue;
        }
        if (slot[i] < 0 || slot[i] >= a.n_slots) {
          if (slot[i] != -1 && a.status) *a.status = 1;
          continue;
        }
        h -= a.Hq;
        const bool is_k = h < a.Hk;
        if (!is_k) h -= a.Hk;
        const long long page = slot[i] >> a.page_shift, pos = slot[i] & ((1 << a.page_shift) - 1);
        const long long at = is_k ? page * a.kc[0] + pos * a.kc[1] + h * a.kc[2] : page * a.vc[0] + pos * a.vc[1] + h * a.vc[2];
        uint8_t* cache = is_k ? a.k_cache : a.v_cache;
        if (E4M3) {
          const float* scale = is_k ? a.k_scale : a.v_scale;
          const float s = scale ? scale[h] : 1.f;
          put_e4m3(cache + at + pl[i].first, f, s);
          if (pl[i].second >= 0) put_e4m3(cache + at + pl[i].second, g, s);
        } else {
          uint16_t* dst = reinterpret_cast<uint16_t*>(cache) + at;
          put_bf16(dst + pl[i].first, f);
          if (pl[i].second >= 0) put_bf16(dst + pl[i].second, g);
        }
      }
    }
  }
}

constexpr int unroll_of(int v) { return v == 8 ? 3 : 4; }

template <int V, bool INTERLEAVED>
cudaError_t launch(const AppendArgs& a, bool e4m3, int threads, size_t smem, cudaStream_t s) {
  constexpr int U = unroll_of(V);
  const dim3 grid(a.groups * a.parts), block(threads);
  if (e4m3) return launch_pdl(append_kernel<V, INTERLEAVED, true, U>, grid, block, smem, s, 1, a);
  return launch_pdl(append_kernel<V, INTERLEAVED, false, U>, grid, block, smem, s, 1, a);
}

bool on(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

}  // namespace
}  // namespace cep

using namespace cep;

extern "C" int attn_append(const cep_append_desc* d, const void* q, const void* k, const void* v, const int32_t* positions, const int64_t* slots,
                           const float* inv_freq, void* q_out, void* k_cache, void* v_cache, const float* k_scale, const float* v_scale,
                           int32_t* status, void* stream) {
  if (!d) return record_error(CEP_ERR_ARG, "append: the description is NULL");
  if (d->n_tokens < 0 || d->n_heads < 0 || d->n_kv_heads <= 0) return record_error(CEP_ERR_ARG, "append: need n_tokens >= 0, n_heads >= 0 and n_kv_heads > 0");
  if (d->head_dim <= 0 || d->head_dim % 2 || d->rotary_dim < 0 || d->rotary_dim % 2 || d->rotary_dim > d->head_dim)
    return record_error(CEP_ERR_ARG, "append: head_dim and rotary_dim must be even, 0 <= rotary_dim <= head_dim, head_dim > 0");
  if (d->head_dim > kAppendMaxDim || (long long)(d->n_heads + 2ll * d->n_kv_heads) * d->head_dim > (1 << 24))
    return record_error(CEP_ERR_UNSUPPORTED, "append: head_dim above %d or heads of 2^24 columns and more in all", kAppendMaxDim);
  if (d->cache_elem != CEP_ELEM_BF16 && d->cache_elem != CEP_ELEM_E4M3) return record_error(CEP_ERR_ARG, "append: unknown cache_elem %d", d->cache_elem);
  if (d->page_size <= 0 || (d->page_size & (d->page_size - 1)) || d->n_pages <= 0 || d->n_pages > (1ll << 40) / d->page_size)
    return record_error(CEP_ERR_ARG, "append: page_size must be a power of two, n_pages positive");
  const bool e4m3 = d->cache_elem == CEP_ELEM_E4M3;
  if (!e4m3 && (k_scale || v_scale)) return record_error(CEP_ERR_ARG, "append: a bf16 cache has no scales");
  if (d->n_tokens == 0) return CEP_OK;                       // nothing to do: empty tensors may have no address
  if (!k || !v || !positions || !slots || !k_cache || !v_cache || (d->rotary_dim && !inv_freq)) return record_error(CEP_ERR_ARG, "append: a pointer is NULL");
  if ((d->n_heads > 0) != (q != nullptr) || (d->n_heads > 0) != (q_out != nullptr)) return record_error(CEP_ERR_ARG, "append: q, q_out and n_heads go together");
  const int64_t D = d->head_dim, T = d->n_tokens;
  // 16-byte accesses need every head of every tensor to start on 16 bytes (8 for codes) and whole vectors
  bool wide = d->rotary_dim % 16 == 0 && (D - d->rotary_dim) % 8 == 0, strides = true, aligned = true;
  struct Side { const void* p; int64_t bytes, vec, n[3], st[3]; };
  const int64_t cb = e4m3 ? 1 : 2;
  const Side sides[6] = {{q, 2, 16, {T, d->n_heads, 0}, {d->q_token_stride, d->q_head_stride, 0}},
                         {q_out, 2, 16, {T, d->n_heads, 0}, {d->q_out_token_stride, d->q_out_head_stride, 0}},
                         {k, 2, 16, {T, d->n_kv_heads, 0}, {d->k_token_stride, d->k_head_stride, 0}},
                         {v, 2, 16, {T, d->n_kv_heads, 0}, {d->v_token_stride, d->v_head_stride, 0}},
                         {k_cache, cb, 8 * cb, {d->n_pages, d->page_size, d->n_kv_heads}, {d->k_cache_stride[0], d->k_cache_stride[1], d->k_cache_stride[2]}},
                         {v_cache, cb, 8 * cb, {d->n_pages, d->page_size, d->n_kv_heads}, {d->v_cache_stride[0], d->v_cache_stride[1], d->v_cache_stride[2]}}};
  for (const Side& s : sides) {
    if (!s.p) continue;
    aligned = aligned && on(s.p, s.bytes);
    wide = wide && on(s.p, s.vec);
    for (int i = 0; i < 3; ++i)
      if (s.n[i] > 1) { strides = strides && s.st[i] >= D; wide = wide && s.st[i] * s.bytes % s.vec == 0; }    // (of a single element it means nothing)
  }
  if (!strides) return record_error(CEP_ERR_ARG, "append: a stride is smaller than head_dim");
  // a rotated head is written by the thread that has read it, others may be read later
  const HeadRows q_new = head_rows(q_out, T, d->n_heads, d->q_out_token_stride, d->q_out_head_stride, D);
  const bool in_place = q == q_out && (T == 1 || d->q_token_stride == d->q_out_token_stride) && (d->n_heads == 1 || d->q_head_stride == d->q_out_head_stride);
  if ((!in_place && rows_meet(head_rows(q, T, d->n_heads, d->q_token_stride, d->q_head_stride, D), q_new)) ||
      rows_meet(head_rows(k, T, d->n_kv_heads, d->k_token_stride, d->k_head_stride, D), q_new) ||
      rows_meet(head_rows(v, T, d->n_kv_heads, d->v_token_stride, d->v_head_stride, D), q_new))
    return record_error(CEP_ERR_ARG, "append: q_out overlaps k, v or a part of q");
  if (!aligned || !on(positions, 4) || !on(slots, 8) || !on(inv_freq, 4) || !on(k_scale, 4) || !on(v_scale, 4) || !on(status, 4))
    return record_error(CEP_ERR_ARG, "append: a pointer is not aligned to its element type");
  AppendArgs a{};
  a.q = static_cast<const uint16_t*>(q); a.k = static_cast<const uint16_t*>(k); a.v = static_cast<const uint16_t*>(v); a.q_out = static_cast<uint16_t*>(q_out);
  a.k_cache = static_cast<uint8_t*>(k_cache); a.v_cache = static_cast<uint8_t*>(v_cache);
  a.positions = positions; a.slots = slots; a.inv_freq = inv_freq; a.k_scale = k_scale; a.v_scale = v_scale; a.status = status;
  a.q_tok = d->q_token_stride; a.q_head = d->q_head_stride; a.qo_tok = d->q_out_token_stride; a.qo_head = d->q_out_head_stride;
  a.k_tok = d->k_token_stride; a.k_head = d->k_head_stride; a.v_tok = d->v_token_stride; a.v_head = d->v_head_stride;
  for (int i = 0; i < 3; ++i) { a.kc[i] = d->k_cache_stride[i]; a.vc[i] = d->v_cache_stride[i]; }
  a.n_slots = d->n_pages * d->page_size;
  a.T = d->n_tokens; a.Hq = d->n_heads; a.Hk = d->n_kv_heads; a.D = d->head_dim; a.R = d->rotary_dim;
  while ((1 << a.page_shift) < d->page_size) ++a.page_shift;
  const int V = wide ? 8 : 1;
  a.units = (a.R / (2 * V)) + (a.D - a.R + 2 * V - 1) / (2 * V);
  const int v_units = (a.D + 2 * V - 1) / (2 * V);
  if (v_units > a.units) a.units = v_units;
  const int per_token = (a.Hq + 2 * a.Hk) * a.units, unroll = unroll_of(V);
  auto warps = [](int n) { return (n + 31) / 32 * 32; };
  // Few tokens: a token's heads are shared by blocks whose threads have a part each.  Many: as many tokens at a time as give 256 threads
  // their parts, and blocks that come to tokens again and again, up to kAppendPerSm threads an SM.
  int threads;
  a.tokens = 1; a.parts = 1;
  if (a.T < 2 * 148) {
    threads = std::min(256, warps(per_token));
    a.parts = (per_token + threads - 1) / threads;
  } else {
    while (a.tokens < 16 && a.tokens * 2 * per_token <= 256 * unroll) a.tokens *= 2;
    threads = std::min(kAppendMaxThreads, warps((a.tokens * per_token + unroll - 1) / unroll));
  }
  a.groups = (int)std::min<long long>(((long long)a.T + a.tokens - 1) / a.tokens, 148 * std::max(1, kAppendPerSm / threads));
  if (a.parts > 1) a.groups = a.T;
  const size_t smem = 2 * (size_t)a.tokens * 2 * ((a.R / 2 + 7) / 8 * 8) * sizeof(float);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = wide ? (d->interleaved ? launch<8, true>(a, e4m3, threads, smem, s) : launch<8, false>(a, e4m3, threads, smem, s))
                             : (d->interleaved ? launch<1, true>(a, e4m3, threads, smem, s) : launch<1, false>(a, e4m3, threads, smem, s));
  if (e != cudaSuccess) return record_error(CEP_ERR_CUDA, "append launch failed: %s", cudaGetErrorString(e));
  return CEP_OK;
}
