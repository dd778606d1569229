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
#include "gemm_tcgen05.h"

namespace cep {

constexpr int kAttnTile = 128;               // keys of a step, rows of a row tile
constexpr int kAttnMaxSeqs = 1024, kAttnMaxPrefixes = 256;
constexpr int kAttnMaxCtas = 148;
constexpr int kAttnSplitRows = 2 * 2 * kAttnTile;                      // partial rows that a CTA's two cut items may need
// Estimated cost of a key for one row tile's pair of warpgroups and for two row tiles, and of an item beside its keys.
constexpr int kAttnCostSingle = 10, kAttnCostDual = 16, kAttnCostItem = 2400;

struct AttnShape {
  int T, B, G;                               // tokens, sequences, groups
  int Hq, Hkv, Gh;                           // query heads, kv heads, query heads per kv head
  int tps;                                   // tokens of a row tile: 128 / Gh
  int causal;
  int own_cap, prefix_cap;                   // keys that the page tables have room for
  int n_ctas;
};

// The schedule of one call, in shared or in global memory.  
struct AttnSched {
  int32_t* q0;                               // [B+1] first token of each sequence
  int32_t* kv;                               // [B] own keys
  int32_t* scum;                             // [B+1] tokens of short sequences before this one
  int32_t* pcum;                             // [B+1] tokens of sequences with partial rows of their own before this one
  int32_t* gfirst;                           // [G+1] first sequence of each group
  int32_t* glen;                             // [G] prefix keys
  int32_t* grt;                              // [G+1] group items of a kv head before this group
  int16_t* group;                            // [B] -1: no prefix
  long long* cost;                           // [G+B+1] cost before each entity (a group or a sequence)
  long long share;                           // of one CTA
};
// The arrays of a schedule carved from `base` (8-byte aligned).
__host__ __device__ inline AttnSched attn_carve(void* base, int B, int G) {
  AttnSched s;
  s.cost = static_cast<long long*>(base);
  int32_t* p = reinterpret_cast<int32_t*>(s.cost + G + B + 1);
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
__host__ __device__ constexpr int attn_sched_words(int B, int G) { return 2 * (G + B + 1) + (4 * B + 3 + 3 * G + 2 + (B + 1) / 2 + 1) / 2 * 2; }   // 4-byte words, an even number
constexpr int kAttnSchedBytes = attn_sched_words(kAttnMaxSeqs, kAttnMaxPrefixes) * 4;

__host__ __device__ inline int attn_div_up(int a, int b) { return (a + b - 1) / b; }

// Tokens that a group's prefix is shared by: sequences short enough to leave a row tile's rows empty, in a group of two or more.
__host__ __device__ inline bool attn_is_short(const AttnShape& p, const AttnSched& s, int b) {
  const int n = s.q0[b + 1] - s.q0[b], g = s.group[b];
  return g >= 0 && n > 0 && n <= 2 * p.tps && s.glen[g] > 0 && s.gfirst[g + 1] - s.gfirst[g] >= 2;
}

// Sequences of up to two row tiles have partial rows of their own; longer ones use those of the CTAs whose cut goes through them.
__host__ __device__ inline bool attn_has_rows(const AttnShape& p, const AttnSched& s, int b) { return s.q0[b + 1] - s.q0[b] <= 2 * p.tps; }

// An entity's items per kv head, and what item r (0-based) of them costs: a + slope * (r + 1).
struct AttnEntity { int items; long long a, slope; };
__host__ __device__ inline AttnEntity attn_entity(const AttnShape& p, const AttnSched& s, int e) {
  AttnEntity x;
  x.slope = 0;
  if (e < p.G) {
    const int n = s.scum[s.gfirst[e + 1]] - s.scum[s.gfirst[e]];
    x.items = attn_div_up(n, 2 * p.tps);
    x.a = kAttnCostItem + (long long)(n > p.tps ? kAttnCostDual : kAttnCostSingle) * s.glen[e];
    return x;
  }
  const int b = e - p.G, n = s.q0[b + 1] - s.q0[b], kv = s.kv[b];
  const long long unit = n > p.tps ? kAttnCostDual : kAttnCostSingle;
  if (attn_is_short(p, s, b)) {
    x.items = kv > 0;
    x.a = kAttnCostItem + unit * kv;
    return x;
  }
  x.items = attn_div_up(n, 2 * p.tps);
  const int g = s.group[b], ahead = g >= 0 ? s.glen[g] : 0;
  x.a = kAttnCostItem + unit * ((long long)ahead + (p.causal ? (kv > n ? kv - n : 0) : kv));
  if (p.causal) x.slope = unit * 2 * p.tps;
  return x;
}
__host__ __device__ inline long long attn_items_cost(const AttnEntity& x, long long r) { return r * x.a + x.slope * (r * (r + 1) / 2); }

// Where a CTA's walk over its items stands.
struct AttnWalk {
  int e, head, r;                            // entity, kv head, item of these
  long long at, w;                           // cost before the item, of the item
  AttnEntity x;
  bool done;
};
__host__ __device__ inline void attn_walk_entity(const AttnShape& p, const AttnSched& s, AttnWalk* k) {
  while (k->e < p.G + p.B && s.cost[k->e + 1] == s.cost[k->e]) ++k->e;       // entities without items
  k->done = k->e >= p.G + p.B;
  if (!k->done) k->x = attn_entity(p, s, k->e);
}
// The item that the point `x` of the cost axis lies in.
__host__ __device__ inline AttnWalk attn_walk_at(const AttnShape& p, const AttnSched& s, long long x) {
  AttnWalk k;
  k.e = 0; k.head = 0; k.r = 0; k.at = 0; k.w = 0;
  const int E = p.G + p.B;
  k.done = x >= s.cost[E];
  if (k.done) return k;
  int lo = 0, hi = E;                        // cost[lo] <= x < cost[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (s.cost[mid] <= x) lo = mid; else hi = mid;
  }
  k.e = lo;
  k.x = attn_entity(p, s, lo);
  const long long per_head = attn_items_cost(k.x, k.x.items);
  long long rest = x - s.cost[lo];
  k.head = (int)(rest / per_head);
  rest -= k.head * per_head;
  int a = 0, b = k.x.items;                  // items_cost(a) <= rest < items_cost(b)
  while (b - a > 1) {
    const int mid = (a + b) >> 1;
    if (attn_items_cost(k.x, mid) <= rest) a = mid; else b = mid;
  }
  k.r = a;
  k.at = x - (rest - attn_items_cost(k.x, a));
  k.w = k.x.a + k.x.slope * (a + 1);
  return k;
}
__host__ __device__ inline void attn_walk_next(const AttnShape& p, const AttnSched& s, AttnWalk* k) {
  k->at += k->w;
  if (++k->r == k->x.items) {
    k->r = 0;
    if (++k->head == p.Hkv) {
      k->head = 0;
      ++k->e;
      attn_walk_entity(p, s, k);
      if (k->done) return;
    }
  }
  k->w = k->x.a + k->x.slope * (k->r + 1);
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
  it.n_ahead = attn_div_up(it.ahead, kAttnTile);
  it.n = it.n_ahead + attn_div_up(it.own, kAttnTile);
  if (it.n == 0) it.n = 1;                   // rows that see nothing are written all the same
  return it;
}
// Steps of the item that lie before the point x.
__host__ __device__ inline int attn_steps_before(const AttnWalk& k, int n, long long x) {
  if (x <= k.at) return 0;
  if (x >= k.at + k.w) return n;
  return (int)(((x - k.at) * n + k.w - 1) / k.w);
}
// First partial row of what CTA c has of an item, steps from s0 on; and how many partial results that is, tok rows apart.
__host__ __device__ inline long long attn_part_row(const AttnItem& it, int c, int s0) {
  return it.rows + (long long)c * kAttnSplitRows + (s0 == 0 ? kAttnSplitRows / 2 : 0);
}
__host__ __device__ inline int attn_part_count(const AttnItem& it, int s0, int s1) { return it.dual || s1 - s0 == 1 ? 1 : 2; }
__host__ __device__ inline bool attn_is_whole(const AttnItem& it, int s0, int s1) {
  return it.kind == kAttnJoint && s1 - s0 == it.n && attn_part_count(it, s0, s1) == 1;
}
__host__ __device__ inline long long attn_max_part_rows(int max_tokens, int max_seqs, int max_prefixes, int Hq, int Hkv, int n_ctas) {
  const int Gh = Hq / Hkv, tps = kAttnTile / Gh;
  long long most = (long long)max_seqs * 2 * tps;                      // tokens of sequences with rows of their own
  if (most > max_tokens) most = max_tokens;
  return 2 * most * Hq + (long long)Hkv * (most / (2 * tps) + max_prefixes) * 2 * tps * Gh + (long long)(n_ctas + 1) * kAttnSplitRows;
}

// The cost that each CTA gets: equal shares, and no less than two steps, which two warpgroups take at the same time.
__host__ __device__ inline long long attn_share(const AttnShape& p, long long total) {
  const long long share = (total + p.n_ctas - 1) / p.n_ctas, least = 2ll * kAttnTile * kAttnCostSingle;
  return share > least ? share : least;
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
  void* sched;                               // kAttnSchedBytes: the schedule as the merge kernel reads it
  int32_t* status;
};

int attn_padded_dim(int D);                  // 64 or 128
cudaError_t attn_setup();                  // once per plan, with its device current
cudaError_t launch_attn(const AttnArgs& a, int e4m3, const GemmTensorMap& tm_k, const GemmTensorMap& tm_v, cudaStream_t s);
int make_cache_map(GemmTensorMap* out, const void* base, const cep_attn_config& c, const int64_t* stride);    // stride: page, position, head

}  // namespace cep
