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

// ---- rope.cu -----------------------------------------------------------------
// [0]: queries, [1]: keys.
struct RopeArgs {
  int64_t T;
  int heads[2];             // 0: none
  int d, rot;
  float eps;
  const uint64_t* turns;    // [rot / 2] freq / (2 pi) as 64-bit fractions
  const int32_t* pos;       // [T] or nullptr: row t at position t
  const uint16_t* X[2];
  int64_t ldx[2];
  const uint16_t* gamma[2]; // or nullptr: no norm
  uint16_t* Y[2];           // backward: the gradient of X
  int64_t ldy[2];
};
struct RopeBwdArgs {
  RopeArgs f;
  const uint16_t* dY[2];
  int64_t lddy[2];
  float* dgamma[2];         // [d] or nullptr
  float* part;              // [rope_bwd_parts][2][d], nullptr without dgamma
  int accumulate;
};
// Rows of the partial sums of dgamma.
int64_t rope_bwd_parts(const RopeArgs& a, int sms);
// neighbours: pairs (2 i, 2 i + 1), else (i, i + rot / 2).
cudaError_t launch_rope_fwd(const RopeArgs& a, bool neighbours, int sms, cudaStream_t stream);
cudaError_t launch_rope_bwd(const RopeBwdArgs& a, bool neighbours, int sms, cudaStream_t stream);

// ---- kv_blocks.cu ------------------------------------------------------------
struct BlocksArgs {
  int n_seqs, max_blocks, block_log2, pinned;
  int64_t capacity;         // entries of free_ids
  int32_t* table;           // [n_seqs][max_blocks]
  int32_t* free_ids;
  const int32_t* len;       // [n_seqs]
  const int32_t* free_count;
  int32_t* len_out;         // may be len
  int32_t* free_out;        // may be free_count
  int4* info;               // [n_seqs + 1]
  int* status;
};
struct ExtendArgs {
  BlocksArgs b;
  const int32_t* add;
  int64_t rows;
  int32_t* batch_len;       // [n_seqs]
  int32_t* row_start;       // [n_seqs + 1]
  int32_t* pos;             // [rows]
  int64_t* slot;            // [rows] or nullptr
};
struct TruncateArgs {
  BlocksArgs b;
  const int32_t* keep;
};
int kv_extend_launches(const ExtendArgs& a);
int kv_truncate_launches(const TruncateArgs& a);
cudaError_t launch_kv_extend(const ExtendArgs& a, cudaStream_t stream);
cudaError_t launch_kv_truncate(const TruncateArgs& a, cudaStream_t stream);

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
  // What the kernels' general variants add; all 0 for kv_attn itself.
  int sinks;                // the first keys that a window leaves visible
  int sink_pad;             // and the rest of their last 16
  const int32_t* prefix_table;
  int prefix;               // keys before it lie in the prefix table's blocks, whatever the sequence
  int first;                // the first key of every tile: 0 or prefix
  int across;               // 1: the rows of all sequences are one sequence's, over the prefix alone
  int keep_parts;           // 1: outputs stay parts, even of tiles that are not cut
  int behind;               // 1: the launch may start beside the one before it, of which it needs nothing
};
// Launches `kernel`; lined_up: its blocks may start while the launch before it runs (which says when), and wait for it
// where they need it.
template <typename... Args>
cudaError_t launch_lined_up(void (*kernel)(Args...), dim3 grid, int threads, int smem, int lined_up, cudaStream_t stream,
                            const Args&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = lined_up ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}
inline bool attn_general(const AttnArgs& a) { return a.sinks || a.prefix; }
inline int attn_grid_seqs(const AttnArgs& a) { return a.across ? 1 : a.kv.n_seqs; }
// Sets chunk, splits, tile_rows, row_tiles and sink_pad for the batch's bounds.
void plan_attn(AttnArgs& a, int sms);
// A call in which each sequence goes over a shared prefix and its own keys, and one in which the rows of all go over the
// prefix together (planned here) and then each sequence over its own keys (`own`, planned): about how long they take.
// shared_together: whether they are compared at all, where no sequence may have many rows.
bool shared_together(const AttnArgs& a);
double apart_ns(const AttnArgs& a, int sms);
double plan_prefix(AttnArgs& a, const AttnArgs& own, int sms);
inline int64_t attn_part_rows(const AttnArgs& a) {
  return a.splits > 1 || a.keep_parts
             ? static_cast<int64_t>(attn_grid_seqs(a)) * a.kv.heads * a.row_tiles * a.splits * a.tile_rows
             : 0;
}
constexpr int kPromptRows = 256;   // tile_rows of the prompt kernel (kv_prompt.cu)
cudaError_t launch_kv_prompt(const AttnArgs& a, cudaStream_t stream);
cudaError_t launch_kv_attn(const AttnArgs& a, cudaStream_t stream);
// Attention whose rows go over the prefix together (`prefix`) and over their own keys (`own`), and the join of both.
cudaError_t launch_kv_attn_shared(const AttnArgs& prefix, const AttnArgs& own, cudaStream_t stream);

}  // namespace lrqat
