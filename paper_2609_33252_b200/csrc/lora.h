// Internal interface of the projection with per-request low-rank adapters (lora.cu: plan and C ABI; lora_shrink.cu: the
// down projection A x; lora_project_small.cu, lora_project_large.cu: the shared projection with the up projection inside its
// accumulator).
#pragma once
#include "cep_common.h"
#include "gemm_tcgen05.h"

namespace cep {

constexpr int kLoraChunk = 16;               // ranks per K step of the up projection (one bf16 MMA)
constexpr int kLoraMaxRank = 256;
constexpr int kLoraMaxChunks = kLoraMaxRank / kLoraChunk;
constexpr int kLoraMaxAdapters = 4096;
constexpr int kSms = 148;                    // K is split while the tiles are fewer than this
constexpr int kSmallTok = 128;               // tokens per tile of the small kernel (fp32 outputs: 64)
constexpr int kLargeTok = 256;               // tokens per tile of the large kernel

// One adapter's place in the bank, read by the kernels.
struct LoraBank {
  const int32_t* rank;                       // [slots], 0: nothing loaded
  const float* scale;                        // [slots]
  const uint16_t* down;                      // bf16 [slots][rank_pad][K]; rows at or beyond the rank count for nothing
  const uint16_t* up;                        // bf16 [slots][rank_pad/16][N][16]; ranks beyond the adapter's are zero
  int slots, rank_pad;
};

// What the down projection leaves for the projection kernel.
struct LoraStep {
  const int32_t* ids;                        // [T] usable adapter slot of each token, -1: none
  const int32_t* n_chunks;                   // [token tiles] chunks of 16 ranks of all distinct adapters of a tile
  const int32_t* chunks;                     // [token tiles][tile tokens * 16] slot * 16 + chunk, adapters in order of appearance
  const float* s;                            // [T][rank_pad] scale * A_a x
};

// SMs without a block of the projection kernel, and how many of them clusters of four or more can still use.
struct FreeSms { int sms, in_clusters; };
cudaError_t launch_lora_pack(const uint16_t* down, int64_t down_stride, const uint16_t* up, int64_t up_stride, int rank, float scale, int slot,
                             int K, int N, const LoraBank& bank, int32_t* bad, int32_t* status, cudaStream_t s);
bool lora_beside(int T);                     // the down projection runs beside the projection kernel on the same SMs
cudaError_t lora_shrink_setup();             // once per plan, with its device current
// tm_x: 64 columns x `box` rows; tm_down: the bank's down rows, 64 columns x 16 rows.  token_tile: tokens per tile of the
// projection kernel that follows (its lists are made here); free: what that kernel leaves.
cudaError_t launch_lora_shrink(const GemmTensorMap& tm_x, const GemmTensorMap& tm_down, int box, const FreeSms& free, int T, int K, int N, int out_f32,
                               const int32_t* ids, const LoraBank& bank, int token_tile, int32_t* out_ids, int32_t* n_chunks, int32_t* chunk_lists, float* s_out,
                               int32_t* status, cudaStream_t s);

struct ProjectArgs {
  int T, K, N;
  int out_f32;
  void* y; int64_t y_stride;
  const LoraBank* bank;                      // nullptr: no adapters in this call
  LoraStep step;
  int32_t* tile_counter;                     // [2], zero between calls: tiles handed out, CTA pairs done
  int32_t* status;
};
// Tensor maps are encoded per call for x and once for the weight and the up bank.
int make_tile_map(GemmTensorMap* out, const void* base, long long cols, long long rows, long long row_stride, long long depth,
                  long long depth_stride, int box_cols, int box_rows, int swizzle_bytes);
// Once per plan, with the device current: launch attributes and how many clusters fit.
cudaError_t project_small_setup(int dev);
cudaError_t project_large_setup(int dev, int n_sms);
// Work of the busiest SM, in K steps of a tile (both kernels' steps take about the same time).
long long project_small_cost(int dev, int T, int N, int K, int out_f32);
long long project_large_cost(int dev, int T, int N, int K);
FreeSms project_large_free(int dev, int T, int N, int K);
cudaError_t launch_project_small(const ProjectArgs& a, const GemmTensorMap& tm_w, const GemmTensorMap& tm_x, const GemmTensorMap& tm_up,
                                 int dev, cudaStream_t s);
cudaError_t launch_project_large(const ProjectArgs& a, const GemmTensorMap& tm_w, const GemmTensorMap& tm_x, const GemmTensorMap& tm_up,
                                 int dev, cudaStream_t s);
int project_small_tile(int out_f32);                // tokens per tile of the small kernel
int project_small_tokens(int T, int out_f32);       // token columns of its MMA: T rounded up to 16, at most the tile's

}  // namespace cep
