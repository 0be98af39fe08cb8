// Internal launcher declarations of the norm, 8-bit cache and cache attention operators.
// Every launcher enqueues on `stream` and returns the cudaError_t of the launch.
#pragma once

#include <cuda_runtime.h>
#include <cstdint>

namespace lrqat {

// Bit of the device status word that marks a batch or block table out of its bounds
// (lrqat_get_device_status reports it as LRQAT_ERR_RANGE; bit 0 marks a wait that gave up).
constexpr int kStatusRange = 2;

// ---- norm.cu -----------------------------------------------------------------
struct NormFwdArgs {
  int64_t T, k;
  float eps;
  const uint16_t* X;
  const uint16_t* R;        // residual or nullptr
  const uint16_t* gamma;
  uint16_t* H;              // X + R or nullptr
  uint16_t* Y;              // bf16 result or nullptr
  int8_t* Y_q;              // int8 codes or nullptr
  float* s_y;               // [T] scales, or nullptr with quant == 0
  int quant;                // 1: per-token 8-bit quantizer
};
cudaError_t launch_add_rmsnorm_fwd(const NormFwdArgs& a, int sms, cudaStream_t stream);

struct NormBwdArgs {
  int64_t T, k;
  float eps;
  const uint16_t* dY;
  const uint16_t* dH;       // gradient of the residual output or nullptr
  const uint16_t* H;
  const uint16_t* gamma;
  uint16_t* dX;
  float* dgamma;            // [k] or nullptr
  float* part;              // [norm_bwd_parts][k] partial sums of dgamma
  int accumulate;
};
// Rows of the partial sums of dgamma that a call which writes dgamma needs.
int64_t norm_bwd_parts(int64_t T, int64_t k, int sms);
cudaError_t launch_add_rmsnorm_bwd(const NormBwdArgs& a, int sms, cudaStream_t stream);
cudaError_t launch_act_dequant(const int8_t* codes, const float* scale, int64_t T, int64_t k, uint16_t* x_hat,
                               cudaStream_t stream);

// ---- kv_cache.cu, kv_attn.cu ---------------------------------------------------
// A paged cache and a ragged batch of its sequences (lrqat_kv_cache, lrqat_kv_batch).
struct KvArgs {
  int8_t* codes[2];         // keys, values: [n_blocks][heads][block][d]
  float* scale[2];          // [n_blocks][heads]
  int64_t n_blocks;
  int heads;                // key/value heads
  int d;
  int block_log2;
  int n_seqs;
  const int32_t* len;
  const int32_t* row_start;
  const int32_t* table;
  int max_blocks;           // columns of the table
  int64_t rows;
  int max_rows, max_len;
  int* status;
};
// Blocks that the last `max_rows` of `max_len` tokens can touch; at least one, whose thread block then reports
// sequences beyond a bound of zero.
inline int kv_touched_blocks(const KvArgs& a) {
  const int64_t all = (static_cast<int64_t>(a.max_len) + (1 << a.block_log2) - 1) >> a.block_log2;
  const int64_t some = ((static_cast<int64_t>(a.max_rows) + (1 << a.block_log2) - 2) >> a.block_log2) + 1;
  return static_cast<int>(all < 1 ? 1 : all < some ? all : some);
}
cudaError_t launch_kv_write(const KvArgs& a, const uint16_t* K, int64_t ldk, const uint16_t* V, int64_t ldv,
                            cudaStream_t stream);
cudaError_t launch_kv_read(const KvArgs& a, uint16_t* K, int64_t ldk, uint16_t* V, int64_t ldv, cudaStream_t stream);

struct AttnArgs {
  KvArgs kv;
  int group;                // query heads per key/value head
  const uint16_t* Q;
  int64_t ldq;
  uint16_t* O;
  int64_t ldo;
  float scale_log2;         // softmax scale times log2(e)
  int window;               // 0: none
  int chunk;                // keys of one split
  int splits;               // most splits of a row tile
  int tile_rows;            // (token, head) rows of a tile
  int row_tiles;            // tiles of one sequence and key/value head
  float* part;              // [seq][head][tile][split][tile_rows][d] unnormalised outputs (splits > 1)
  uint64_t timeout_ns;      // limit of one wait inside a kernel
  float* part_stat;         // [seq][head][tile][split][tile_rows][4] maxima m and n, denominator
};
// Sets chunk, splits, tile_rows and row_tiles for the batch's bounds.
void plan_attn(AttnArgs& a, int sms);
inline int64_t attn_part_rows(const AttnArgs& a) {
  return a.splits > 1 ? static_cast<int64_t>(a.kv.n_seqs) * a.kv.heads * a.row_tiles * a.splits * a.tile_rows
                      : 0;
}
constexpr int kPromptRows = 256;   // tile_rows of the prompt kernel (kv_prompt.cu)
cudaError_t launch_kv_prompt(const AttnArgs& a, cudaStream_t stream);
cudaError_t launch_kv_attn(const AttnArgs& a, cudaStream_t stream);

}  // namespace lrqat
