// Plan object and C ABI of the attention behind shared prefixes (include/cascade_ffn.h, attn_*).  Host code only checks,
// carves and enqueues; it waits for the device in attn_status and attn_plan_destroy alone.
#include <math.h>

#include <algorithm>
#include <new>
#include <vector>

#include "attn.h"

using namespace cep;

struct cep_attn_plan {
  cep_attn_config cfg;
  int device, n_ctas;
  GemmTensorMap tm_k, tm_v;
  const float *k_scale, *v_scale;
  int32_t* status; void* records; float* part_o; float2* part_ml;
  // The plan's last enqueued work.  Work on another stream waits for it: the workspace is shared.
  cudaEvent_t last; unsigned long long last_stream; bool have_last;    // (by id: a handle can come back as another stream's)
};

namespace {

size_t up_to(size_t v, size_t a) { return (v + a - 1) / a * a; }
bool on(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

int check_config(const cep_attn_config* c) {
  if (!c) return record_error(CEP_ERR_ARG, "attn: the configuration is NULL");
  if (c->n_heads <= 0 || c->n_kv_heads <= 0 || c->n_heads % c->n_kv_heads) return record_error(CEP_ERR_ARG, "attn: n_heads must be a positive multiple of n_kv_heads");
  if (c->n_heads / c->n_kv_heads > kAttnTile) return record_error(CEP_ERR_UNSUPPORTED, "attn: more than %d query heads per kv head", kAttnTile);
  if (c->cache_elem != CEP_ELEM_BF16 && c->cache_elem != CEP_ELEM_E4M3) return record_error(CEP_ERR_ARG, "attn: unknown cache_elem %d", c->cache_elem);
  const int per16 = c->cache_elem == CEP_ELEM_E4M3 ? 16 : 8;           // elements in 16 bytes
  if (c->head_dim <= 0 || c->head_dim > 128 || c->head_dim % per16) return record_error(CEP_ERR_UNSUPPORTED, "attn: head_dim must be a multiple of %d up to 128", per16);
  if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128 && c->page_size != 256)
    return record_error(CEP_ERR_UNSUPPORTED, "attn: page_size must be 16, 32, 64, 128 or 256");
  if (c->n_pages <= 0) return record_error(CEP_ERR_ARG, "attn: n_pages must be positive");
  if (c->max_tokens <= 0 || c->max_tokens > (1 << 22) || (long long)c->max_tokens * c->n_heads > 0x7fffffffll)
    return record_error(CEP_ERR_ARG, "attn: max_tokens must be in 1..2^22, max_tokens * n_heads below 2^31");
  if (c->max_seqs <= 0 || c->max_seqs > kAttnMaxSeqs) return record_error(CEP_ERR_ARG, "attn: max_seqs must be in 1..%d", kAttnMaxSeqs);
  if (c->max_prefixes < 0 || c->max_prefixes > kAttnMaxPrefixes) return record_error(CEP_ERR_ARG, "attn: max_prefixes must be in 0..%d", kAttnMaxPrefixes);
  if (!(c->scale > 0.f) || c->scale > 3.402823466e38f) return record_error(CEP_ERR_ARG, "attn: the scale must be finite and positive");
  // a stride counts where there is a second element along it
  for (const int64_t* st : {c->k_stride, c->v_stride}) {
    const int64_t count[3] = {c->n_pages, c->page_size, c->n_kv_heads};
    for (int i = 0; i < 3; ++i)
      if (count[i] > 1 && (st[i] < c->head_dim || st[i] % per16 || st[i] >= (1ll << 38)))
        return record_error(CEP_ERR_ARG, "attn: the cache's strides must be multiples of 16 bytes, and at least head_dim");
  }
  return CEP_OK;
}

struct Carve { size_t status, records, ml, o, total; };
Carve carve(const cep_attn_config& c) {
  Carve w{};
  size_t o = 0;
  auto take = [&](size_t& f, size_t bytes) { f = o; o = up_to(o + bytes, 256); };
  const size_t rows = (size_t)attn_max_part_rows(c.max_tokens, c.max_seqs, c.max_prefixes, c.n_heads, c.n_kv_heads, kAttnMaxCtas);
  take(w.status, kStWords * 4);
  take(w.records, attn_record_bytes(c.max_seqs, c.max_prefixes, attn_most_own(c.max_tokens, c.max_seqs, c.n_heads, c.n_kv_heads)));
  take(w.ml, rows * sizeof(float2));
  take(w.o, rows * attn_padded_dim(c.head_dim) * sizeof(float));
  w.total = o;
  return w;
}

int enter(cep_attn_plan* p, cudaStream_t s, bool* capturing) {
  int dev = -1;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return record_error(CEP_ERR_CUDA, "attn: cudaGetDevice failed: %s", cudaGetErrorString(e));
  if (dev != p->device) return record_error(CEP_ERR_ARG, "attn: the plan was made on device %d, device %d is current", p->device, dev);
  cudaStreamCaptureStatus st = cudaStreamCaptureStatusNone;
  e = cudaStreamIsCapturing(s, &st);
  if (e != cudaSuccess) return record_error(CEP_ERR_CUDA, "attn: cudaStreamIsCapturing failed: %s", cudaGetErrorString(e));
  *capturing = st != cudaStreamCaptureStatusNone;
  unsigned long long id = 0;
  if (!*capturing && (e = cudaStreamGetId(s, &id)) != cudaSuccess) return record_error(CEP_ERR_CUDA, "attn: cudaStreamGetId failed: %s", cudaGetErrorString(e));
  if (!*capturing && p->have_last && p->last_stream != id) {
    e = cudaStreamWaitEvent(s, p->last, 0);
    if (e != cudaSuccess) return record_error(CEP_ERR_CUDA, "attn: cudaStreamWaitEvent failed: %s", cudaGetErrorString(e));
  }
  return CEP_OK;
}
int leave(cep_attn_plan* p, cudaStream_t s, bool capturing) {
  if (capturing) return CEP_OK;
  cudaError_t e = cudaEventRecord(p->last, s);
  if (e == cudaSuccess) e = cudaStreamGetId(s, &p->last_stream);
  if (e != cudaSuccess) return record_error(CEP_ERR_CUDA, "attn: cudaEventRecord failed: %s", cudaGetErrorString(e));
  p->have_last = true;
  return CEP_OK;
}

}  // namespace

extern "C" {

int attn_plan_workspace_bytes(const cep_attn_config* cfg, size_t* bytes) {
  const int rc = check_config(cfg);
  if (rc) return rc;
  if (!bytes) return record_error(CEP_ERR_ARG, "attn: bytes is NULL");
  *bytes = carve(*cfg).total;
  return CEP_OK;
}

int attn_plan(const cep_attn_config* cfg, const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale, void* workspace,
              size_t workspace_bytes, void* stream, cep_attn_plan** out) {
  const int rc0 = check_config(cfg);
  if (rc0) return rc0;
  if (!out) return record_error(CEP_ERR_ARG, "attn: out is NULL");
  *out = nullptr;
  if (!k_cache || !v_cache || !workspace) return record_error(CEP_ERR_ARG, "attn: a cache or the workspace is NULL");
  if (!on(k_cache, 16) || !on(v_cache, 16)) return record_error(CEP_ERR_ARG, "attn: the caches must start on 16 bytes");
  if (!on(k_scale, 4) || !on(v_scale, 4)) return record_error(CEP_ERR_ARG, "attn: a scale pointer is misaligned");
  const Carve w = carve(*cfg);
  if (workspace_bytes < w.total || !on(workspace, 256)) return record_error(CEP_ERR_WORKSPACE, "attn: the workspace needs %zu bytes on a 256-byte boundary", w.total);
  cep_attn_plan* p = new (std::nothrow) cep_attn_plan();
  if (!p) return record_error(CEP_ERR_ARG, "attn: out of host memory");
  p->cfg = *cfg; p->k_scale = k_scale; p->v_scale = v_scale;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  p->status = reinterpret_cast<int32_t*>(ws + w.status);
  p->records = ws + w.records;
  p->part_ml = reinterpret_cast<float2*>(ws + w.ml);
  p->part_o = reinterpret_cast<float*>(ws + w.o);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  auto give_up = [&](int code, const char* what, cudaError_t e) {
    attn_plan_destroy(p);
    return record_error(code, "attn: %s failed: %s", what, cudaGetErrorString(e));
  };
  cudaError_t e = cudaGetDevice(&p->device);
  if (e != cudaSuccess) return give_up(CEP_ERR_CUDA, "cudaGetDevice", e);
  // A capture would only record the clearing of the status word: the plan's first calls would find it as it is.
  cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
  e = cudaStreamIsCapturing(st, &capture);
  if (e != cudaSuccess) return give_up(CEP_ERR_CUDA, "cudaStreamIsCapturing", e);
  if (capture != cudaStreamCaptureStatusNone) {
    attn_plan_destroy(p);
    return record_error(CEP_ERR_STATE, "attn: a plan cannot be made on a stream that is being captured");
  }
  const void* given[5] = {k_cache, v_cache, workspace, k_scale ? k_scale : workspace, v_scale ? v_scale : workspace};
  for (const void* m : given) {                            // kernels of one device never get another one's memory
    cudaPointerAttributes at{};
    e = cudaPointerGetAttributes(&at, m);
    if (e != cudaSuccess) return give_up(CEP_ERR_CUDA, "cudaPointerGetAttributes", e);
    if (at.type == cudaMemoryTypeDevice && at.device != p->device) {
      const int current = p->device;
      attn_plan_destroy(p);
      return record_error(CEP_ERR_ARG, "attn: a cache, a scale or the workspace is on device %d, device %d is current", at.device, current);
    }
  }
  int sms = 0;
  e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, p->device);
  if (e != cudaSuccess) return give_up(CEP_ERR_CUDA, "cudaDeviceGetAttribute", e);
  p->n_ctas = std::min(sms, kAttnMaxCtas);
  e = cudaEventCreateWithFlags(&p->last, cudaEventDisableTiming);
  if (e != cudaSuccess) { p->last = nullptr; return give_up(CEP_ERR_CUDA, "cudaEventCreateWithFlags", e); }
  e = attn_setup();
  if (e != cudaSuccess) return give_up(CEP_ERR_CUDA, "setting up the kernels", e);
  int m = make_cache_map(&p->tm_k, k_cache, *cfg, cfg->k_stride);
  if (!m) m = make_cache_map(&p->tm_v, v_cache, *cfg, cfg->v_stride);
  if (m) { attn_plan_destroy(p); return record_error(CEP_ERR_CUDA, "attn: cuTensorMapEncodeTiled failed (%d)", m); }
  e = cudaMemsetAsync(p->status, 0, kStWords * 4, st);
  if (e != cudaSuccess) return give_up(CEP_ERR_CUDA, "cudaMemsetAsync", e);
  const int rc = leave(p, st, false);
  if (rc) { attn_plan_destroy(p); return rc; }
  *out = p;
  return CEP_OK;
}

int attn_prefix(cep_attn_plan* p, const cep_attn_batch* b, const void* q, const int32_t* q_start, const int32_t* kv_len, const int32_t* page_table,
                const int32_t* prefix_start, const int32_t* prefix_len, const int32_t* prefix_pages, void* out, float* lse, void* stream) {
  if (!p) return record_error(CEP_ERR_ARG, "attn: the plan is NULL");
  if (!b) return record_error(CEP_ERR_ARG, "attn: the batch is NULL");
  const cep_attn_config& c = p->cfg;
  if (b->n_tokens < 0 || b->n_seqs < 0 || b->n_prefixes < 0) return record_error(CEP_ERR_ARG, "attn: n_tokens, n_seqs and n_prefixes may not be negative");
  if (b->n_tokens > c.max_tokens || b->n_seqs > c.max_seqs || b->n_prefixes > c.max_prefixes)
    return record_error(CEP_ERR_CAPACITY, "attn: %d tokens, %d sequences, %d prefixes; the plan was made for %d, %d, %d", b->n_tokens, b->n_seqs, b->n_prefixes,
                        c.max_tokens, c.max_seqs, c.max_prefixes);
  if (b->n_tokens == 0 || b->n_seqs == 0) return CEP_OK;
  if (!q || !q_start || !kv_len || !out) return record_error(CEP_ERR_ARG, "attn: q, q_start, kv_len or out is NULL");
  if (b->table_width < 0 || b->prefix_width < 0 || (b->table_width > 0 && !page_table) || (b->n_prefixes > 0 && (!prefix_len || (b->prefix_width > 0 && !prefix_pages))))
    return record_error(CEP_ERR_ARG, "attn: a page table or the prefix lengths are missing");
  if ((b->n_seqs > 1 && b->table_stride < b->table_width) || (b->n_prefixes > 1 && b->prefix_stride < b->prefix_width))
    return record_error(CEP_ERR_ARG, "attn: the rows of a page table lie less than its width apart");
  if ((long long)b->table_width * c.page_size > 0x3fffffffll || (long long)b->prefix_width * c.page_size > 0x3fffffffll)
    return record_error(CEP_ERR_UNSUPPORTED, "attn: a page table holds 2^30 keys or more");
  const int64_t strides[4] = {b->q_token_stride, b->q_head_stride, b->out_token_stride, b->out_head_stride};
  const int count[4] = {b->n_tokens, c.n_heads, b->n_tokens, c.n_heads};
  for (int i = 0; i < 4; ++i)
    if (count[i] > 1 && (strides[i] < c.head_dim || strides[i] % 8)) return record_error(CEP_ERR_ARG, "attn: heads of q and out must lie multiples of 16 bytes and at least head_dim apart");
  if (!on(q, 16) || !on(out, 16)) return record_error(CEP_ERR_ARG, "attn: q and out must start on 16 bytes");
  // a block writes rows of out while another still reads q
  if (rows_meet(head_rows(q, b->n_tokens, c.n_heads, b->q_token_stride, b->q_head_stride, c.head_dim),
                head_rows(out, b->n_tokens, c.n_heads, b->out_token_stride, b->out_head_stride, c.head_dim)))
    return record_error(CEP_ERR_ARG, "attn: out overlaps q");
  if (lse && b->n_tokens > 1 && b->lse_token_stride < c.n_heads) return record_error(CEP_ERR_ARG, "attn: rows of lse lie less than n_heads apart");
  for (const void* i : {(const void*)q_start, (const void*)kv_len, (const void*)page_table, (const void*)prefix_start, (const void*)prefix_len, (const void*)prefix_pages, (const void*)lse})
    if (!on(i, 4)) return record_error(CEP_ERR_ARG, "attn: a pointer is not aligned to its element type");
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  bool capturing = false;
  const int rc = enter(p, st, &capturing);
  if (rc) return rc;
  AttnArgs a{};
  a.p = attn_shape(b->n_tokens, b->n_seqs, b->n_prefixes, c.n_heads, c.n_kv_heads, b->causal != 0, (long long)b->table_width * c.page_size,
                   (long long)b->prefix_width * c.page_size, p->n_ctas);
  a.D = c.head_dim;
  while ((1 << a.page_shift) < c.page_size) ++a.page_shift;
  a.n_pages = c.n_pages;
  a.q = static_cast<const uint16_t*>(q); a.q_tok = b->q_token_stride; a.q_head = b->q_head_stride;
  a.q_start = q_start; a.kv_len = kv_len; a.page_table = page_table;
  a.prefix_start = prefix_start; a.prefix_len = prefix_len; a.prefix_pages = prefix_pages;
  a.table_stride = b->table_stride; a.prefix_stride = b->prefix_stride;
  a.out = static_cast<uint16_t*>(out); a.out_tok = b->out_token_stride; a.out_head = b->out_head_stride;
  a.lse = lse; a.lse_tok = b->lse_token_stride;
  a.k_scale = p->k_scale; a.v_scale = p->v_scale;
  a.scale_log2 = (float)((double)c.scale * 1.4426950408889634);
  a.part_o = p->part_o; a.part_ml = p->part_ml; a.records = p->records; a.status = p->status;
  GemmTensorMap maps[4] = {p->tm_k, p->tm_v, {}, {}};
  int m = make_q_map(&maps[2], a, 1);
  if (!m) m = make_q_map(&maps[3], a, a.p.tps);
  if (m) return record_error(CEP_ERR_CUDA, "attn: cuTensorMapEncodeTiled failed (%d)", m);
  const cudaError_t e = launch_attn(a, c.cache_elem == CEP_ELEM_E4M3, maps, st);
  if (e != cudaSuccess) return record_error(CEP_ERR_CUDA, "attn: a launch failed: %s", cudaGetErrorString(e));
  return leave(p, st, capturing);
}

int attn_status(cep_attn_plan* p) {
  if (!p) return record_error(CEP_ERR_ARG, "attn: the plan is NULL");
  int32_t st[kStWords] = {};
  cudaError_t e = p->have_last ? cudaEventSynchronize(p->last) : cudaSuccess;
  if (e == cudaSuccess) e = cudaMemcpy(st, p->status, sizeof st, cudaMemcpyDeviceToHost);
  if (e == cudaSuccess && (st[kStTimeout] || st[kStBadRouting] || st[kStBoundsViolation])) {
    e = cudaMemset(p->status, 0, sizeof st);
    // the next call's stream may not wait for the default one: what its kernels report must not be cleared with this
    if (e == cudaSuccess) e = cudaStreamSynchronize(nullptr);
  }
  if (e != cudaSuccess) return record_error(CEP_ERR_CUDA, "attn: reading the status failed: %s", cudaGetErrorString(e));
  if (st[kStTimeout]) return record_error(CEP_ERR_DEVICE_TIMEOUT, "attn: a bounded wait inside a kernel expired");
  if (st[kStBoundsViolation]) return record_error(CEP_ERR_CAPACITY, "attn: a length or start did not fit the call");
  if (st[kStBadRouting]) return record_error(CEP_ERR_BAD_ROUTING, "attn: a page table named a page outside the cache");
  return CEP_OK;
}

int attn_plan_destroy(cep_attn_plan* p) {
  if (!p) return CEP_OK;
  if (p->last) {
    if (p->have_last) cudaEventSynchronize(p->last);
    cudaEventDestroy(p->last);
  }
  delete p;
  return CEP_OK;
}

int cep_debug_attn_schedule(const cep_attn_config* c, int32_t n_tokens, int32_t n_seqs, int32_t n_prefixes, int32_t causal, int32_t n_ctas, const int32_t* q_start,
                            const int32_t* kv_len, const int32_t* prefix_start, const int32_t* prefix_len, int64_t* parts, int32_t max_parts, int64_t* part_rows) {
  if (check_config(c)) return CEP_ERR_ARG;
  if (!q_start || !kv_len || (n_prefixes > 0 && !prefix_len) || !parts || !part_rows || n_tokens < 1 || n_seqs < 1 || n_prefixes < 0 || n_ctas < 1 || max_parts < 0)
    return record_error(CEP_ERR_ARG, "attn: a schedule needs lengths, room and a positive grid");
  if (n_tokens > c->max_tokens || n_seqs > c->max_seqs || n_prefixes > c->max_prefixes || n_ctas > kAttnMaxCtas)
    return record_error(CEP_ERR_CAPACITY, "attn: more than the plan was made for");
  long long own_cap = 0, prefix_cap = 0;
  for (int i = 0; i < n_seqs; ++i) own_cap = std::max<long long>(own_cap, kv_len[i]);
  for (int i = 0; i < n_prefixes; ++i) prefix_cap = std::max<long long>(prefix_cap, prefix_len[i]);
  const AttnShape p = attn_shape(n_tokens, n_seqs, n_prefixes, c->n_heads, c->n_kv_heads, causal != 0, own_cap, prefix_cap, n_ctas);
  int32_t* store = new (std::nothrow) int32_t[kAttnSchedBytes / 4];
  if (!store) return record_error(CEP_ERR_ARG, "attn: out of host memory");
  AttnSched s = attn_carve(store, p.B, p.G);
  for (int i = 0; i <= p.B; ++i) s.q0[i] = std::max(i ? s.q0[i - 1] : 0, std::min(std::max(q_start[i], 0), p.T));
  for (int i = 0; i <= p.G; ++i) s.gfirst[i] = std::max(i ? s.gfirst[i - 1] : 0, std::min(std::max(prefix_start ? prefix_start[i] : i ? p.B : 0, 0), p.B));
  if (!p.G) s.gfirst[0] = 0;
  for (int g = 0; g < p.G; ++g) s.glen[g] = std::max(0, prefix_len[g]);
  for (int b = 0; b < p.B; ++b) {
    s.kv[b] = std::max(0, kv_len[b]);
    s.group[b] = -1;
    for (int g = 0; g < p.G; ++g) if (s.gfirst[g] <= b && b < s.gfirst[g + 1]) s.group[b] = g;
  }
  s.scum[0] = s.pcum[0] = 0;
  for (int b = 0; b < p.B; ++b) {
    s.scum[b + 1] = s.scum[b] + (attn_is_short(p, s, b) ? s.q0[b + 1] - s.q0[b] : 0);
    s.pcum[b + 1] = s.pcum[b] + (attn_has_rows(p, s, b) ? s.q0[b + 1] - s.q0[b] : 0);
  }
  s.grt[0] = 0;
  for (int g = 0; g < p.G; ++g) s.grt[g + 1] = s.grt[g] + attn_tiles(p, s.scum[s.gfirst[g + 1]] - s.scum[s.gfirst[g]]);
  s.cost[0] = 0;
  for (int e = 0; e < p.G + p.B; ++e) { const AttnEntity x = attn_entity(p, s, e); s.cost[e + 1] = s.cost[e] + p.Hkv * attn_items_cost(x, x.items); }
  s.share = attn_share(p, s.cost[p.G + p.B]);
  *part_rows = attn_max_part_rows(c->max_tokens, c->max_seqs, c->max_prefixes, c->n_heads, c->n_kv_heads, kAttnMaxCtas);
  int n = 0;
  for (int cta = 0; cta < n_ctas; ++cta) {
    const int x0 = cta * s.share, x1 = x0 + s.share;
    for (AttnWalk k = attn_walk_at(p, s, x0); !k.done && k.at < x1; attn_walk_next(p, s, &k)) {
      const AttnItem it = attn_item(p, s, k);
      const int s0 = attn_steps_before(k, it.n, x0), s1 = attn_steps_before(k, it.n, x1);
      if (s0 >= s1) continue;
      if (n < max_parts) {
        int64_t* r = parts + 13ll * n;
        r[0] = cta; r[1] = it.kind; r[2] = it.b; r[3] = it.g; r[4] = it.head; r[5] = it.tok; r[6] = it.n_tok; r[7] = s0; r[8] = s1; r[9] = it.n;
        r[10] = attn_is_whole(it, s0, s1) ? -1 : attn_part_row(it, cta, s0);
        r[11] = k.w;
        r[12] = attn_part_count(it, s0, s1);
      }
      ++n;
    }
  }
  delete[] store;
  return n;
}

}  // extern "C"
