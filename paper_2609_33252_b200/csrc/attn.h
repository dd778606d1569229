// Attention behind a shared prefix: what its translation units share (attn.cu: plan and C ABI; attn_prefix.cu: the kernels).
//
// Work is cut into items.  An item is up to two row tiles (tokens x query heads of one kv head) against a run of keys, in steps
// of 128 keys:
//   group items   the prefix of one group against the tokens of ALL its short sequences, packed: the prefix is read once per
//                 row tile instead of once per sequence
//   own items     a short sequence against its own keys
//   joint items   a sequence that fills row tiles by itself (or has no one to share with): prefix, then own keys
// Two row tiles' items occupy both warpgroups of a CTA; items of one row tile are taken by the warpgroups in turn, step by step, so
// that a CTA's part of such an item leaves up to two partial results.
//
// The items lie on one axis of estimated cost, which is cut into equal shares, one per CTA; a cut inside an item falls on a
// step.  A row whose keys ended up in several places is put together from partial results (sums, maxima) by a second kernel,
// in the order of the cuts: nothing depends on timing.
#pragma once
#include "cep_common.h"
#include <math.h>

#include "gemm_tcgen05.h"

namespace cep {

constexpr int kAttnTile = 128;               // keys of a step, rows of a row tile
constexpr int kAttnMaxSeqs = 1024, kAttnMaxPrefixes = 256;
constexpr int kAttnMaxCtas = 148;
constexpr int kAttnSplitRows = 2 * 2 * kAttnTile;                      // partial rows that a CTA's two cut items may need
// Estimated cost of four keys for one row tile (taken by the warpgroups in turn) and for two, and of an item beside its keys; a unit is 5 ns.
// So 128 keys count 1.44 us for one and 2.56 for two, an item 2.8 and 6 us beside them.  8 and 600 for one, 16 and 1600 for two fit each kind alone;
// what counts is the ratio of both kinds where they run side by side.  These, those, and these with 14 in the place of 16, us:
//   256 tokens over 32768 shared, up to 4096 own keys   707   760   749      4096 tokens, prompts and decoding over 8192 shared  1284  1340  1320
//    64 over 8192, up to 2000                            80    81    85      the same over 2048, 16 heads, 4 kv heads             142   141   138
//    96 over 16384, up to 1000                          129   124   124      256 over 4096, up to 512                             141   142   143
//   128 over 5000, up to 1500, e4m3                     160   154   164      48 x 1..8 over 8192, up to 2000                       64    64    65
constexpr int kAttnCostSingle = 9, kAttnCostDual = 16, kAttnItemSingle = 560, kAttnItemDual = 1200;

struct AttnShape {
  int T, B, G;                               // tokens, sequences, groups
  int Hq, Hkv, Gh;                           // query heads, kv heads, query heads per kv head
  int tps;                                   // tokens of a row tile: 128 / Gh
  int causal;
  int own_cap, prefix_cap;                   // keys that the page tables have room for
  int n_ctas;
  float per_cta;                             // 1 / n_ctas
  int cost_shift;                            // keeps the sum of all costs below 2^31
  uint32_t tile_magic;                       // division by 2 tps: (x * tile_magic) >> 32
};

// The schedule of one call.
struct AttnSched {
  int32_t* q0;                               // [B+1] first token of each sequence
  int32_t* kv;                               // [B] own keys
  int32_t* scum;                             // [B+1] tokens of short sequences before this one
  int32_t* pcum;                             // [B+1] tokens of sequences with partial rows of their own before this one
  int32_t* gfirst;                           // [G+1] first sequence of each group
  int32_t* glen;                             // [G] prefix keys
  int32_t* grt;                              // [G+1] group items of a kv head before this group
  int16_t* group;                            // [B] -1: no prefix
  int32_t* cost;                             // [G+B+1] cost before each entity (a group or a sequence)
  int32_t share;                             // of one CTA
};
// The arrays of a schedule carved from `base`.
__host__ __device__ inline AttnSched attn_carve(void* base, int B, int G) {
  AttnSched s;
  int32_t* p = static_cast<int32_t*>(base);
  s.cost = p; p += G + B + 1;
  s.q0 = p; p += B + 1;
  s.kv = p; p += B;
  s.scum = p; p += B + 1;
  s.pcum = p; p += B + 1;
  s.gfirst = p; p += G + 1;
  s.glen = p; p += G;
  s.grt = p; p += G + 1;
  s.group = reinterpret_cast<int16_t*>(p);
  s.share = 0;
  return s;
}
__host__ __device__ constexpr int attn_sched_words(int B, int G) { return G + B + 1 + 4 * B + 3 + 3 * G + 2 + (B + 1) / 2; }      // 4-byte words
constexpr int kAttnSchedBytes = attn_sched_words(kAttnMaxSeqs, kAttnMaxPrefixes) * 4;
// Records of the joining kernel: a head, 48 bytes per CTA, group and sequence, 4 per token of a sequence of up to two row tiles.
inline size_t attn_record_bytes(int max_seqs, int max_prefixes, long long tokens) { return 16 + 48ull * (kAttnMaxCtas + max_prefixes + max_seqs) + 4ull * tokens; }

__host__ __device__ inline int attn_key_tiles(int keys) { return (keys + kAttnTile - 1) / kAttnTile; }

__host__ __device__ inline int attn_tiles(const AttnShape& p, int tokens) {     // of 2 tps tokens
#ifdef __CUDA_ARCH__
  return __umulhi((uint32_t)(tokens + 2 * p.tps - 1), p.tile_magic);
#else
  return (int)((uint64_t)(uint32_t)(tokens + 2 * p.tps - 1) * p.tile_magic >> 32);
#endif
}
// a / b without the long division: an estimate, put right by products.
__host__ __device__ inline int attn_div(int a, int b) {
  int q = (int)((float)a / (float)b);
  while ((long long)q * b > a) --q;
  while ((long long)(q + 1) * b <= a) ++q;
  return q;
}

// Tokens that a group's prefix is shared by: sequences short enough to leave a row tile's rows empty, in a group of two or more.
__host__ __device__ inline bool attn_is_short(const AttnShape& p, const AttnSched& s, int b) {
  const int n = s.q0[b + 1] - s.q0[b], g = s.group[b];
  return g >= 0 && n > 0 && n <= 2 * p.tps && s.glen[g] > 0 && s.gfirst[g + 1] - s.gfirst[g] >= 2;
}

// Sequences of up to two row tiles have partial rows of their own; longer ones use those of the CTAs whose cut goes through them.
__host__ __device__ inline bool attn_has_rows(const AttnShape& p, const AttnSched& s, int b) { return s.q0[b + 1] - s.q0[b] <= 2 * p.tps; }

// An entity's items per kv head, and what the first r of them cost: r a + (slope r (r + 1) / 2 >> shift), as item r sees slope more than the one before.
// (The slope is not shifted by itself: with few tokens per row tile, and a shift for wide page tables, nothing would be left of it, and the last
// items of a long prompt would count as much as the first.)
struct AttnEntity { int items, a, slope, shift; };
__host__ __device__ inline AttnEntity attn_entity(const AttnShape& p, const AttnSched& s, int e) {
  int n, keys, slope = 0;
  bool some = true;
  if (e < p.G) {
    n = s.scum[s.gfirst[e + 1]] - s.scum[s.gfirst[e]];
    keys = s.glen[e];
  } else {
    const int b = e - p.G, g = s.group[b], kv = s.kv[b];
    n = s.q0[b + 1] - s.q0[b];
    keys = kv;
    if (attn_is_short(p, s, b)) {
      some = kv > 0;
    } else {
      if (p.causal) { keys = kv > n ? kv - n : 0; slope = 1; }
      if (g >= 0) keys += s.glen[g];
    }
  }
  const int unit = n > p.tps ? kAttnCostDual : kAttnCostSingle, fixed = n > p.tps ? kAttnItemDual : kAttnItemSingle;
  AttnEntity x;
  x.items = some ? attn_tiles(p, n) : 0;
  x.a = (int)((fixed + (long long)unit * (keys >> 2)) >> p.cost_shift) + 1;
  x.slope = slope ? unit * 2 * p.tps >> 2 : 0;
  x.shift = p.cost_shift;
  return x;
}
__host__ __device__ inline int attn_items_cost(const AttnEntity& x, int r) { return r * x.a + (x.slope ? (int)(x.slope * ((long long)r * (r + 1) >> 1) >> x.shift) : 0); }
__host__ __device__ inline int attn_item_cost(const AttnEntity& x, int r) { return x.slope ? attn_items_cost(x, r + 1) - attn_items_cost(x, r) : x.a; }

// Where a CTA's walk over its items stands.
struct AttnWalk {
  int e, head, r;                            // entity, kv head, item of these
  int at, w;                                 // cost before the item, of the item
  AttnEntity x;
  bool done;
};
// The item that the point `x` of the cost axis lies in, which is in entity `e`.
__host__ __device__ inline AttnWalk attn_walk_in(const AttnShape& p, const AttnSched& s, int e, int x) {
  AttnWalk k;
  k.e = e; k.done = false;
  k.x = attn_entity(p, s, e);
  const int per_head = attn_items_cost(k.x, k.x.items);
  int rest = x - s.cost[e];
  k.head = attn_div(rest, per_head);
  rest -= k.head * per_head;
  int r;                                     // items_cost(r) <= rest < items_cost(r + 1)
  if (k.x.slope == 0) {
    r = attn_div(rest, k.x.a);
  } else {                                   // the root of slope r^2 / 2 + (a + slope / 2) r = rest, put right by the sums themselves
    const float slope = (float)k.x.slope / (float)(1u << k.x.shift), h = (float)k.x.a / slope + 0.5f, x2 = 2.f * (float)rest / slope;
    r = (int)(x2 / (sqrtf(h * h + x2) + h));
    if (r > k.x.items - 1) r = k.x.items - 1;
    while (r > 0 && attn_items_cost(k.x, r) > rest) --r;
    while (attn_items_cost(k.x, r + 1) <= rest) ++r;
  }
  k.r = r;
  k.at = x - (rest - attn_items_cost(k.x, r));
  k.w = attn_item_cost(k.x, r);
  return k;
}
__host__ __device__ inline AttnWalk attn_walk_at(const AttnShape& p, const AttnSched& s, int x) {
  const int E = p.G + p.B;
  if (x >= s.cost[E]) { AttnWalk k; k.done = true; return k; }
  int lo = 0, hi = E;                        // cost[lo] <= x < cost[hi]
#pragma unroll 1
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (s.cost[mid] <= x) lo = mid; else hi = mid;
  }
  return attn_walk_in(p, s, lo, x);
}
__host__ __device__ inline void attn_walk_next(const AttnShape& p, const AttnSched& s, AttnWalk* k) {
  k->at += k->w;
  if (++k->r == k->x.items) {
    k->r = 0;
    if (++k->head == p.Hkv) {
      k->head = 0;
      do ++k->e; while (k->e < p.G + p.B && s.cost[k->e + 1] == s.cost[k->e]);       // entities without items
      k->done = k->e >= p.G + p.B;
      if (k->done) return;
      k->x = attn_entity(p, s, k->e);
    }
  }
  k->w = attn_item_cost(k->x, k->r);
}

enum AttnKind { kAttnGroup = 0, kAttnOwn = 1, kAttnJoint = 2 };
struct AttnItem {
  int kind, b, g, head;                      // sequence (-1 for a group item), group (-1: none)
  int tok;                                   // first token: among the group's short tokens, or in the sequence
  int n_tok;                                 // tokens
  bool dual;                                 // two row tiles (the second may be empty in an entity's last item)
  int ahead, own;                            // prefix keys, own keys that the item's last token sees
  int n_ahead, n;                            // steps over the prefix, all steps
  long long rows;                            // first partial row
};
__host__ __device__ inline AttnItem attn_item(const AttnShape& p, const AttnSched& s, const AttnWalk& k) {
  AttnItem it;
  it.head = k.head;
  const int tile_tokens = 2 * p.tps, tile_rows = tile_tokens * p.Gh;
  const long long group_rows = (long long)p.Hkv * s.grt[p.G] * tile_rows;
  if (k.e < p.G) {
    it.kind = kAttnGroup; it.b = -1; it.g = k.e;
    it.tok = k.r * tile_tokens;
    const int n = s.scum[s.gfirst[k.e + 1]] - s.scum[s.gfirst[k.e]];
    it.n_tok = n - it.tok < tile_tokens ? n - it.tok : tile_tokens;
    it.dual = n > p.tps;
    it.ahead = s.glen[k.e]; it.own = 0;
    it.rows = ((long long)p.Hkv * s.grt[k.e] + (long long)k.head * k.x.items + k.r) * tile_rows;
  } else {
    it.b = k.e - p.G;
    const int n = s.q0[it.b + 1] - s.q0[it.b], kv = s.kv[it.b];
    it.g = s.group[it.b];
    it.dual = n > p.tps;
    it.rows = group_rows + 2ll * s.pcum[it.b] * p.Hq + (attn_has_rows(p, s, it.b) ? 2ll * k.head * n * p.Gh : 0);
    if (attn_is_short(p, s, it.b)) {
      it.kind = kAttnOwn;
      it.tok = 0; it.n_tok = n;
      it.ahead = 0; it.own = kv;
    } else {
      it.kind = kAttnJoint;
      it.tok = k.r * tile_tokens;
      it.n_tok = n - it.tok < tile_tokens ? n - it.tok : tile_tokens;
      it.ahead = it.g >= 0 ? s.glen[it.g] : 0;
      const int seen = p.causal ? kv - n + it.tok + it.n_tok : kv;
      it.own = seen < 0 ? 0 : seen < kv ? seen : kv;
    }
  }
  it.n_ahead = attn_key_tiles(it.ahead);
  it.n = it.n_ahead + attn_key_tiles(it.own);
  if (it.n == 0) it.n = 1;                   // rows that see nothing are written all the same
  return it;
}
// Steps of the item that lie before the point x.
__host__ __device__ inline int attn_steps_before(const AttnWalk& k, int n, int x) {
  if (x <= k.at) return 0;
  if (x >= k.at + k.w) return n;
  // (in fp32: what counts is that it never falls with x, and that all who ask get the same)
  const int steps = (int)ceilf((float)(x - k.at) * ((float)n / (float)k.w));
  return steps < n ? steps : n;
}
// First partial row of what CTA c has of an item, steps from s0 on; and how many partial results that is, tok rows apart.
__host__ __device__ inline long long attn_part_row(const AttnItem& it, int c, int s0) {
  return it.rows + (long long)c * kAttnSplitRows + (s0 == 0 ? kAttnSplitRows / 2 : 0);
}
__host__ __device__ inline int attn_part_count(const AttnItem& it, int s0, int s1) { return it.dual || s1 - s0 == 1 ? 1 : 2; }
__host__ __device__ inline bool attn_is_whole(const AttnItem& it, int s0, int s1) {
  return it.kind == kAttnJoint && s1 - s0 == it.n && attn_part_count(it, s0, s1) == 1;
}
// Tokens of sequences with partial rows of their own, at most.
__host__ __device__ inline long long attn_most_own(int max_tokens, int max_seqs, int Hq, int Hkv) {
  const long long most = (long long)max_seqs * 2 * (kAttnTile / (Hq / Hkv));
  return most < max_tokens ? most : max_tokens;
}
__host__ __device__ inline long long attn_max_part_rows(int max_tokens, int max_seqs, int max_prefixes, int Hq, int Hkv, int n_ctas) {
  const int Gh = Hq / Hkv, tps = kAttnTile / Gh;
  const long long most = attn_most_own(max_tokens, max_seqs, Hq, Hkv);
  return 2 * most * Hq + (long long)Hkv * (most / (2 * tps) + max_prefixes) * 2 * tps * Gh + (long long)(n_ctas + 1) * kAttnSplitRows;
}

// The cost that each CTA gets: equal shares, and about a step at least (one token over 777 shared and 33 own keys:
// 17.0 us; with three steps at least 19.5).
__host__ __device__ inline int attn_share(const AttnShape& p, int total) {
  // (fp32 is off by 2^-23 of the sum at most, which is less than one part in 10^4 of a share)
  int share = (int)((float)total * p.per_cta) + 1 + (total >> 21);
  const int least = (kAttnTile / 4 * kAttnCostSingle + kAttnItemSingle / 16) >> p.cost_shift;
  return share > least ? share : least;
}

inline AttnShape attn_shape(int T, int B, int G, int Hq, int Hkv, int causal, long long own_cap, long long prefix_cap, int n_ctas) {
  AttnShape p{};
  p.T = T; p.B = B; p.G = G; p.Hq = Hq; p.Hkv = Hkv; p.Gh = Hq / Hkv; p.tps = kAttnTile / p.Gh; p.causal = causal;
  p.own_cap = (int)own_cap; p.prefix_cap = (int)prefix_cap;
  p.n_ctas = n_ctas; p.per_cta = 1.f / n_ctas;
  p.tile_magic = (uint32_t)(0x100000000ull / (2 * p.tps) + 1);
  // more than all items can cost: every item with as many keys as the tables hold, and the slope's rounding
  const double items = (double)Hkv * ((double)T / (2 * p.tps) + B + G);
  const double most = items * (kAttnItemDual + 2 + kAttnCostDual * 0.25 * ((double)own_cap + (double)prefix_cap + T + 4 * p.tps));
  while (ldexp(most, -p.cost_shift) + items > 2.0e9) ++p.cost_shift;
  return p;
}

struct AttnArgs {
  AttnShape p;
  int D, page_shift, n_pages;                // page_size = 1 << page_shift
  const uint16_t* q; long long q_tok, q_head;
  const int32_t *q_start, *kv_len, *page_table, *prefix_start, *prefix_len, *prefix_pages;
  long long table_stride, prefix_stride;
  uint16_t* out; long long out_tok, out_head;
  float* lse; long long lse_tok;
  const float *k_scale, *v_scale;            // [Hkv] or NULL
  float scale_log2;                          // softmax scale * log2(e)
  float* part_o;                             // [rows][padded D]
  float2* part_ml;                           // [rows] maximum (in log2), sum
  void* records;                             // attn_record_bytes: what the joining kernel needs of the schedule
  int32_t* status;
};

int attn_padded_dim(int D);                  // 64 or 128
cudaError_t attn_setup();                  // once per plan, with its device current
cudaError_t launch_attn(const AttnArgs& a, int e4m3, const GemmTensorMap (&maps)[4], cudaStream_t s);       // k, v, q by single tokens, q by row tiles
int make_q_map(GemmTensorMap* out, const AttnArgs& a, int tokens);         // boxes of `tokens` tokens' query heads of a kv head
int make_cache_map(GemmTensorMap* out, const void* base, const cep_attn_config& c, const int64_t* stride);    // stride: page, position, head

}  // namespace cep
