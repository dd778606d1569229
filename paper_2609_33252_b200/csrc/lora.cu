// Plan object and C ABI of the projection with per-request low-rank adapters (include/cascade_ffn.h, lora_*).
// Host code only checks, carves and enqueues; it waits for the device in lora_status and lora_plan_destroy alone.
#include <algorithm>
#include <new>

#include "lora.h"

using namespace cep;

struct cep_lora_plan {
  cep_lora_config cfg;
  int device, n_sms;
  const void* weight; int64_t weight_stride;
  GemmTensorMap tm_w, tm_up, tm_down;
  LoraBank bank;
  uint8_t* ws;
  int32_t* status; int32_t* tile_counter;
  int32_t* ids; int32_t* n_chunks; int32_t* chunks;
  float* s;
  // The plan's last enqueued work.  Work on another stream waits for it: the workspace and the bank are shared.
  cudaEvent_t last; unsigned long long last_stream; bool have_last;    // (by id: a handle can come back as another stream's)
};

namespace {

size_t up_to(size_t v, size_t a) { return (v + a - 1) / a * a; }
bool on(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
int rank_pad_of(const cep_lora_config& c) { return (c.max_rank + kLoraChunk - 1) / kLoraChunk * kLoraChunk; }

int check_config(const cep_lora_config* c) {
  if (!c) return record_error(CEP_ERR_ARG, "lora: the configuration is NULL");
  if (c->in_features <= 0 || c->in_features % 8) return record_error(CEP_ERR_ARG, "lora: in_features must be a positive multiple of 8");
  if (c->out_features <= 0 || c->max_tokens <= 0) return record_error(CEP_ERR_ARG, "lora: out_features and max_tokens must be positive");
  if (c->max_adapters < 0 || c->max_adapters > kLoraMaxAdapters) return record_error(CEP_ERR_ARG, "lora: max_adapters must be in 0..%d", kLoraMaxAdapters);
  if (c->max_rank < 0 || c->max_rank > kLoraMaxRank || (c->max_adapters > 0) != (c->max_rank > 0))
    return record_error(CEP_ERR_ARG, "lora: max_rank must be in 1..%d with adapters, 0 without", kLoraMaxRank);
  if (c->out_elem != CEP_ELEM_BF16 && c->out_elem != CEP_ELEM_FP32) return record_error(CEP_ERR_ARG, "lora: unknown out_elem %d", c->out_elem);
  if ((long long)c->max_adapters * (rank_pad_of(*c) / kLoraChunk) > (1ll << 30)) return record_error(CEP_ERR_ARG, "lora: too many adapters");
  return CEP_OK;
}

struct Carve { size_t status, tile_counter, ids, n_chunks, chunks, s, total; };
Carve carve(const cep_lora_config& c) {
  Carve w{};
  size_t o = 0;
  auto take = [&](size_t& f, size_t bytes) { f = o; o = up_to(o + bytes, 256); };
  const size_t T = c.max_tokens;
  take(w.status, kStWords * 4);
  take(w.tile_counter, 12);                               // and the mark of a load under way
  if (c.max_adapters) {
    take(w.ids, T * 4);
    take(w.n_chunks, (T / 64 + 1) * 4);
    take(w.chunks, up_to(T, kLargeTok) * kLoraMaxChunks * 4);
    take(w.s, T * rank_pad_of(c) * 4);
  }
  w.total = o;
  return w;
}

struct BankLayout { size_t rank, scale, down, up, total; };
BankLayout bank_layout(const cep_lora_config& c) {
  BankLayout b{};
  size_t o = 0;
  auto take = [&](size_t& f, size_t bytes) { f = o; o = up_to(o + bytes, 256); };
  const size_t S = c.max_adapters, R = rank_pad_of(c);
  take(b.rank, S * 4);
  take(b.scale, S * 4);
  take(b.down, S * R * c.in_features * 2);
  take(b.up, S * R * c.out_features * 2);
  b.total = S ? o : 0;
  return b;
}

// Orders `s` after the plan's last work if that went to another stream.  Inside a stream capture the caller orders.
int enter(cep_lora_plan* p, cudaStream_t s, bool* capturing) {
  int dev = -1;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return record_error(CEP_ERR_CUDA, "lora: cudaGetDevice failed: %s", cudaGetErrorString(e));
  if (dev != p->device) return record_error(CEP_ERR_ARG, "lora: the plan was made on device %d, device %d is current", p->device, dev);
  cudaStreamCaptureStatus st = cudaStreamCaptureStatusNone;
  e = cudaStreamIsCapturing(s, &st);
  if (e != cudaSuccess) return record_error(CEP_ERR_CUDA, "lora: cudaStreamIsCapturing failed: %s", cudaGetErrorString(e));
  *capturing = st != cudaStreamCaptureStatusNone;
  unsigned long long id = 0;
  if (!*capturing && (e = cudaStreamGetId(s, &id)) != cudaSuccess) return record_error(CEP_ERR_CUDA, "lora: cudaStreamGetId failed: %s", cudaGetErrorString(e));
  if (!*capturing && p->have_last && p->last_stream != id) {
    e = cudaStreamWaitEvent(s, p->last, 0);
    if (e != cudaSuccess) return record_error(CEP_ERR_CUDA, "lora: cudaStreamWaitEvent failed: %s", cudaGetErrorString(e));
  }
  return CEP_OK;
}
int leave(cep_lora_plan* p, cudaStream_t s, bool capturing) {
  if (capturing) return CEP_OK;
  cudaError_t e = cudaEventRecord(p->last, s);
  if (e == cudaSuccess) e = cudaStreamGetId(s, &p->last_stream);
  if (e != cudaSuccess) return record_error(CEP_ERR_CUDA, "lora: cudaEventRecord failed: %s", cudaGetErrorString(e));
  p->have_last = true;
  return CEP_OK;
}

}  // namespace

extern "C" {

int lora_plan_workspace_bytes(const cep_lora_config* cfg, size_t* bytes) {
  const int rc = check_config(cfg);
  if (rc) return rc;
  if (!bytes) return record_error(CEP_ERR_ARG, "lora: bytes is NULL");
  *bytes = carve(*cfg).total;
  return CEP_OK;
}

int lora_bank_bytes(const cep_lora_config* cfg, size_t* bytes) {
  const int rc = check_config(cfg);
  if (rc) return rc;
  if (!bytes) return record_error(CEP_ERR_ARG, "lora: bytes is NULL");
  *bytes = bank_layout(*cfg).total;
  return CEP_OK;
}

int lora_plan(const cep_lora_config* cfg, const void* weight, int64_t weight_stride, void* bank, size_t bank_bytes, void* workspace,
              size_t workspace_bytes, void* stream, cep_lora_plan** out) {
  int rc = check_config(cfg);
  if (rc) return rc;
  if (!out) return record_error(CEP_ERR_ARG, "lora: out is NULL");
  *out = nullptr;
  if (!weight || !workspace) return record_error(CEP_ERR_ARG, "lora: weight or workspace is NULL");
  if (!on(weight, 16) || weight_stride < cfg->in_features || weight_stride % 8)
    return record_error(CEP_ERR_ARG, "lora: the weight's rows must start on 16 bytes and lie at least in_features apart");
  const Carve w = carve(*cfg);
  const BankLayout b = bank_layout(*cfg);
  if (workspace_bytes < w.total || !on(workspace, 256)) return record_error(CEP_ERR_WORKSPACE, "lora: the workspace needs %zu bytes on a 256-byte boundary", w.total);
  if (b.total && (!bank || bank_bytes < b.total || !on(bank, 256)))
    return record_error(CEP_ERR_WORKSPACE, "lora: the bank needs %zu bytes on a 256-byte boundary", b.total);
  cep_lora_plan* p = new (std::nothrow) cep_lora_plan();
  if (!p) return record_error(CEP_ERR_ARG, "lora: out of host memory");
  p->cfg = *cfg; p->weight = weight; p->weight_stride = weight_stride;
  p->ws = static_cast<uint8_t*>(workspace);
  auto ints = [&](size_t off) { return reinterpret_cast<int32_t*>(p->ws + off); };
  p->status = ints(w.status); p->tile_counter = ints(w.tile_counter);
  p->ids = ints(w.ids); p->n_chunks = ints(w.n_chunks); p->chunks = ints(w.chunks);
  p->s = reinterpret_cast<float*>(p->ws + w.s);
  uint8_t* bk = static_cast<uint8_t*>(bank);
  p->bank = LoraBank{reinterpret_cast<int32_t*>(bk + b.rank), reinterpret_cast<float*>(bk + b.scale), reinterpret_cast<uint16_t*>(bk + b.down),
                     reinterpret_cast<uint16_t*>(bk + b.up), cfg->max_adapters, rank_pad_of(*cfg)};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  auto give_up = [&](int code, const char* what, cudaError_t e) {
    lora_plan_destroy(p);
    return record_error(code, "lora: %s failed: %s", what, cudaGetErrorString(e));
  };
  cudaError_t e = cudaGetDevice(&p->device);
  if (e != cudaSuccess) return give_up(CEP_ERR_CUDA, "cudaGetDevice", e);
  // A capture would only record the clearing of the counters and slots: the plan's first calls would read them as they are.
  cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
  e = cudaStreamIsCapturing(st, &capture);
  if (e != cudaSuccess) return give_up(CEP_ERR_CUDA, "cudaStreamIsCapturing", e);
  if (capture != cudaStreamCaptureStatusNone) {
    lora_plan_destroy(p);
    return record_error(CEP_ERR_STATE, "lora: a plan cannot be made on a stream that is being captured");
  }
  // kernels of one device never get another one's memory
  const void* given[3] = {weight, workspace, b.total ? bank : workspace};
  for (const void* m : given) {
    cudaPointerAttributes at{};
    e = cudaPointerGetAttributes(&at, m);
    if (e != cudaSuccess) return give_up(CEP_ERR_CUDA, "cudaPointerGetAttributes", e);
    if (at.type == cudaMemoryTypeDevice && at.device != p->device) {
      const int current = p->device;
      lora_plan_destroy(p);
      return record_error(CEP_ERR_ARG, "lora: the weight, the bank or the workspace is on device %d, device %d is current", at.device, current);
    }
  }
  e = cudaDeviceGetAttribute(&p->n_sms, cudaDevAttrMultiProcessorCount, p->device);
  if (e != cudaSuccess) return give_up(CEP_ERR_CUDA, "cudaDeviceGetAttribute", e);
  e = cudaEventCreateWithFlags(&p->last, cudaEventDisableTiming);
  if (e != cudaSuccess) { p->last = nullptr; return give_up(CEP_ERR_CUDA, "cudaEventCreateWithFlags", e); }
  e = lora_shrink_setup();
  if (e == cudaSuccess) e = project_small_setup(p->device);
  if (e == cudaSuccess) e = project_large_setup(p->device, p->n_sms);
  if (e != cudaSuccess) return give_up(CEP_ERR_CUDA, "setting up the kernels", e);
  int m = make_tile_map(&p->tm_w, weight, cfg->in_features, cfg->out_features, weight_stride * 2, 0, 0, 64, 128, 128);
  p->tm_up = p->tm_down = p->tm_w;                        // (not read without adapters)
  if (!m && cfg->max_adapters)
    m = make_tile_map(&p->tm_down, p->bank.down, cfg->in_features, (long long)cfg->max_adapters * p->bank.rank_pad, cfg->in_features * 2ll, 0, 0, 64,
                      kLoraChunk, 128);
  if (!m && cfg->max_adapters)
    m = make_tile_map(&p->tm_up, p->bank.up, kLoraChunk, cfg->out_features, kLoraChunk * 2, (long long)cfg->max_adapters * (p->bank.rank_pad / kLoraChunk),
                      (long long)cfg->out_features * kLoraChunk * 2, kLoraChunk, 128, 32);
  if (m) { lora_plan_destroy(p); return record_error(CEP_ERR_CUDA, "lora: cuTensorMapEncodeTiled failed (%d)", m); }
  // the status word and the counters start at zero, every slot of the bank empty
  e = cudaMemsetAsync(p->ws, 0, w.tile_counter + 12, st);
  if (e == cudaSuccess && b.total) e = cudaMemsetAsync(bk, 0, b.down, st);
  if (e != cudaSuccess) return give_up(CEP_ERR_CUDA, "cudaMemsetAsync", e);
  rc = leave(p, st, false);
  if (rc) { lora_plan_destroy(p); return rc; }
  *out = p;
  return CEP_OK;
}

int lora_load_adapter(cep_lora_plan* p, int32_t slot, int32_t rank, float scale, const void* down, int64_t down_stride, const void* up,
                      int64_t up_stride, void* stream) {
  if (!p) return record_error(CEP_ERR_ARG, "lora: the plan is NULL");
  if (slot < 0 || slot >= p->cfg.max_adapters) return record_error(CEP_ERR_CAPACITY, "lora: slot %d is outside 0..%d", slot, p->cfg.max_adapters - 1);
  if (rank < 0 || rank > p->cfg.max_rank) return record_error(CEP_ERR_CAPACITY, "lora: rank %d is outside 0..%d", rank, p->cfg.max_rank);
  if (rank > 0) {
    if (!down || !up || !on(down, 2) || !on(up, 2)) return record_error(CEP_ERR_ARG, "lora: an adapter pointer is NULL or misaligned");
    if (down_stride < p->cfg.in_features || up_stride < rank) return record_error(CEP_ERR_ARG, "lora: an adapter's row stride is smaller than its rows");
    if (!(scale - scale == 0.f)) return record_error(CEP_ERR_ARG, "lora: the scale must be finite");
  }
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  bool capturing = false;
  int rc = enter(p, st, &capturing);
  if (rc) return rc;
  const cudaError_t e = launch_lora_pack(static_cast<const uint16_t*>(down), down_stride, static_cast<const uint16_t*>(up), up_stride, rank, scale, slot,
                                         p->cfg.in_features, p->cfg.out_features, p->bank, p->tile_counter + 2, p->status, st);
  if (e != cudaSuccess) return record_error(CEP_ERR_CUDA, "lora: the pack launch failed: %s", cudaGetErrorString(e));
  return leave(p, st, capturing);
}

int lora_project(cep_lora_plan* p, const void* x, int64_t x_stride, int32_t n_tokens, const int32_t* adapter_ids, void* y, int64_t y_stride,
                 void* stream) {
  if (!p) return record_error(CEP_ERR_ARG, "lora: the plan is NULL");
  const cep_lora_config& c = p->cfg;
  if (n_tokens < 0) return record_error(CEP_ERR_ARG, "lora: n_tokens is negative");
  if (n_tokens > c.max_tokens) return record_error(CEP_ERR_CAPACITY, "lora: %d tokens, the plan was made for %d", n_tokens, c.max_tokens);
  if (n_tokens == 0) return CEP_OK;
  if (!x || !y) return record_error(CEP_ERR_ARG, "lora: x or y is NULL");
  if (!on(x, 16) || x_stride % 8 || x_stride < c.in_features)
    return record_error(CEP_ERR_ARG, "lora: the rows of x must start on 16 bytes and lie at least in_features apart");
  if (!on(y, c.out_elem == CEP_ELEM_FP32 ? 4 : 2) || y_stride < c.out_features)
    return record_error(CEP_ERR_ARG, "lora: y is misaligned or its rows lie less than out_features apart");
  if (adapter_ids && !c.max_adapters) return record_error(CEP_ERR_ARG, "lora: adapter ids given to a plan without adapters");
  if (!on(adapter_ids, 4)) return record_error(CEP_ERR_ARG, "lora: adapter_ids is misaligned");
  // Up to 128 tokens the small kernel's tile is no wider than the batch; beyond, the kernel whose busiest SM has less to do.
  const bool small = n_tokens <= kSmallTok || (n_tokens <= 4 * kSmallTok &&
                     project_small_cost(p->device, n_tokens, c.out_features, c.in_features, c.out_elem == CEP_ELEM_FP32) + 3 <=
                     project_large_cost(p->device, n_tokens, c.out_features, c.in_features));
  const int f32 = c.out_elem == CEP_ELEM_FP32;
  const int token_tile = small ? project_small_tile(f32) : kLargeTok, box = small ? project_small_tokens(n_tokens, f32) : 128;
  GemmTensorMap tm_x;
  if (const int m = make_tile_map(&tm_x, x, c.in_features, n_tokens, x_stride * 2, 0, 0, 64, box, 128))
    return record_error(CEP_ERR_CUDA, "lora: cuTensorMapEncodeTiled failed (%d)", m);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  bool capturing = false;
  int rc = enter(p, st, &capturing);
  if (rc) return rc;
  ProjectArgs a{};
  a.T = n_tokens; a.K = c.in_features; a.N = c.out_features; a.out_f32 = f32;
  a.y = y; a.y_stride = y_stride; a.tile_counter = p->tile_counter; a.status = p->status;
  cudaError_t e = cudaSuccess;
  if (adapter_ids) {
    const FreeSms free = small ? FreeSms{0, 0} : project_large_free(p->device, n_tokens, c.out_features, c.in_features);
    e = launch_lora_shrink(tm_x, p->tm_down, box, free, n_tokens, c.in_features, c.out_features, f32, adapter_ids, p->bank, token_tile, p->ids, p->n_chunks, p->chunks, p->s,
                           p->status, st);
    a.bank = &p->bank;
    a.step = LoraStep{p->ids, p->n_chunks, p->chunks, p->s};
  }
  if (e == cudaSuccess) e = small ? launch_project_small(a, p->tm_w, tm_x, p->tm_up, p->device, st)
                                  : launch_project_large(a, p->tm_w, tm_x, p->tm_up, p->device, st);
  if (e != cudaSuccess) return record_error(CEP_ERR_CUDA, "lora: a launch failed: %s", cudaGetErrorString(e));
  return leave(p, st, capturing);
}

int lora_status(cep_lora_plan* p) {
  if (!p) return record_error(CEP_ERR_ARG, "lora: the plan is NULL");
  int32_t st[kStWords] = {};
  cudaError_t e = p->have_last ? cudaEventSynchronize(p->last) : cudaSuccess;
  if (e == cudaSuccess) e = cudaMemcpy(st, p->status, sizeof st, cudaMemcpyDeviceToHost);
  if (e == cudaSuccess && (st[kStTimeout] || st[kStBadRouting] || st[kStBoundsViolation])) {
    e = cudaMemset(p->status, 0, sizeof st);
    // the next call's stream may not wait for the default one: what its kernels report must not be cleared with this
    if (e == cudaSuccess) e = cudaStreamSynchronize(nullptr);
  }
  if (e != cudaSuccess) return record_error(CEP_ERR_CUDA, "lora: reading the status failed: %s", cudaGetErrorString(e));
  if (st[kStTimeout]) return record_error(CEP_ERR_DEVICE_TIMEOUT, "lora: a bounded wait inside a kernel expired");
  if (st[kStBoundsViolation]) return record_error(CEP_ERR_ARG, "lora: an adapter's B held a value that is not finite; its slot was left empty");
  if (st[kStBadRouting]) return record_error(CEP_ERR_BAD_ROUTING, "lora: an adapter id named no loaded adapter");
  return CEP_OK;
}

int lora_plan_destroy(cep_lora_plan* p) {
  if (!p) return CEP_OK;
  if (p->last) {
    if (p->have_last) cudaEventSynchronize(p->last);
    cudaEventDestroy(p->last);
  }
  delete p;
  return CEP_OK;
}

}  // extern "C"
