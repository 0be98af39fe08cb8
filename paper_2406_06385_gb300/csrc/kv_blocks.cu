// Cache blocks handed to growing sequences and taken back from shortened ones, on the device.
//
// With P tokens a block and the first `pinned` columns of a table the caller's own, a sequence of n tokens holds the
// columns pinned .. ceil(n / P) - 1.  Extending sequence b from len to len + add (add > 0):
//   need_b = columns that only the longer sequence holds,  base_b = sum of need over the sequences before b,
//   column (first new one) + i takes free_ids[free - 1 - (base_b + i)];
// a sequence is served where base_b + need_b <= free.  Its rows are row_start[b] + i at position len + i.
// Shortening: the j-th of all `total` blocks given back goes to free_ids[free + total - 1 - j], so that taking back
// what was just handed out leaves the list as it was.
//
// Both are a scan over the sequences and an expansion (rows; columns).  The scan is one thread block; where the
// expansion is small the same block does it, behind a barrier instead of a launch.
#include <cuda_runtime.h>
#include <cstdint>

#include "serve.cuh"

namespace lrqat {
namespace {

constexpr int kScanThreads = 1024, kScanWarps = kScanThreads / 32;

__device__ __forceinline__ int64_t warp_scan(int64_t v, int lane) {          // inclusive
#pragma unroll
  for (int o = 1; o < 32; o *= 2) {
    const int64_t u = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += u;
  }
  return v;
}
// Exclusive sums over the block's threads, which stand behind `carry`; carry becomes the sum of all so far.  Every
// thread calls it; `sm` is free again for the next call.
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t& carry, int64_t (*sm)[kScanWarps]) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t in = warp_scan(v, lane);
  if (lane == 31) sm[0][warp] = in;
  __syncthreads();
  if (warp == 0) {
    const int64_t w = sm[0][lane], up = warp_scan(w, lane);
    sm[0][lane] = up - w;
    if (lane == 31) sm[1][0] = up;
  }
  __syncthreads();
  const int64_t out = carry + sm[0][warp] + in - v;
  carry += sm[1][0];
  __syncthreads();
  return out;
}
__device__ __forceinline__ int64_t columns(int64_t tokens, int block_log2) {
  return (tokens + (1 << block_log2) - 1) >> block_log2;
}
// The number of free blocks, 0 (and the range bit) where it is none.
__device__ __forceinline__ int64_t free_blocks(const BlocksArgs& a) {
  const int n = *a.free_count;
  if (n >= 0 && n <= a.capacity) return n;
  if (threadIdx.x == 0) atomicOr(a.status, kStatusRange);
  return 0;
}

// What the expansion has to know of a sequence: x, extending: its first new position, or -1 for rows of padding;
// shortening: the first column it gives back.  y: its first row; the column behind the last one.  z: its first new
// column.  w: its base.
__device__ __forceinline__ int32_t clamp32(int64_t v) { return v > INT32_MAX ? INT32_MAX : static_cast<int32_t>(v); }

// One row: the sequence it belongs to by bisection of the first rows, its position and slot, and the table's entry where
// the row is the first of a new column.
__device__ __forceinline__ void extend_row(const ExtendArgs& a, int64_t row, int64_t rows_used, int64_t free) {
  int pos = -1;
  int64_t slot = -1;
  if (row < rows_used) {
    int lo = 0, hi = a.b.n_seqs;             // the last sequence whose first row is not behind `row`
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (__ldcg(&a.b.info[mid].y) <= row) lo = mid;
      else hi = mid;
    }
    const int4 s = __ldcg(a.b.info + lo);
    if (s.x >= 0) {
      pos = s.x + static_cast<int>(row - s.y);
      const int column = pos >> a.b.block_log2, in_block = pos & ((1 << a.b.block_log2) - 1);
      int32_t* entry = a.b.table + static_cast<int64_t>(lo) * a.b.max_blocks + column;
      int id;
      if (column >= s.z) {
        id = a.b.free_ids[free - 1 - (static_cast<int64_t>(s.w) + column - s.z)];
        if (in_block == 0) *entry = id;
      } else {
        id = *entry;
      }
      slot = (static_cast<int64_t>(id) << a.b.block_log2) + in_block;
    }
  }
  a.pos[row] = pos;
  if (a.slot) a.slot[row] = slot;
}

// info[n_seqs] holds {rows_used, free} for the expansion.
template <bool kAlone>
__global__ void __launch_bounds__(kScanThreads) kv_extend_scan_kernel(ExtendArgs a) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  __shared__ int64_t sm[2][kScanWarps];
  const int64_t free = free_blocks(a.b), most = static_cast<int64_t>(a.b.max_blocks) << a.b.block_log2;
  const int free_raw = *a.b.free_count;
  int64_t row = 0, base = 0, used = 0;       // carries; what served sequences take, by thread
  for (int b0 = 0; b0 < a.b.n_seqs; b0 += kScanThreads) {
    const int b = b0 + threadIdx.x;
    const bool in = b < a.b.n_seqs;
    const int64_t len = in ? a.b.len[b] : 0, add = in ? a.add[b] : 0;
    const int64_t r0 = block_scan(add < 0 ? -add : add, row, sm), r1 = r0 + (add < 0 ? -add : add);
    bool ok = len >= 0 && len <= most && (add <= 0 || len + add <= most) && r1 <= a.rows;
    const int64_t column = max(columns(len, a.b.block_log2), static_cast<int64_t>(a.b.pinned));
    const int64_t need = ok && add > 0 ? max(columns(len + add, a.b.block_log2) - column, int64_t{0}) : 0;
    const int64_t at = block_scan(need, base, sm);
    if (at + need > free && need > 0) ok = false;
    if (!in) continue;
    if (!ok) atomicOr(a.b.status, kStatusRange);
    if (ok && need > 0) used = at + need;
    a.b.info[b] = make_int4(ok && add > 0 ? static_cast<int>(len) : -1, clamp32(r0), static_cast<int>(column), clamp32(at));
    a.b.len_out[b] = static_cast<int>(ok && add > 0 ? len + add : len);
    a.batch_len[b] = static_cast<int>(ok && add >= 0 ? len + add : 0);
    a.row_start[b] = clamp32(r0);
    if (b == a.b.n_seqs - 1) a.row_start[a.b.n_seqs] = clamp32(r1);
  }
  // sequences are served in order, so the most that one of them reaches is the sum
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) used = max(used, __shfl_xor_sync(0xffffffffu, used, o));
  if ((threadIdx.x & 31) == 0) sm[0][threadIdx.x >> 5] = used;
  __syncthreads();
  const int64_t rows_used = min(row, a.rows);
  if (threadIdx.x == 0) {
    for (int w = 1; w < kScanWarps; ++w) used = max(used, sm[0][w]);
    *a.b.free_out = static_cast<int>(free_raw - used);
    if (!kAlone) a.b.info[a.b.n_seqs] = make_int4(static_cast<int>(rows_used), static_cast<int>(free), 0, 0);
  }
  if constexpr (kAlone) {
    for (int64_t r = threadIdx.x; r < a.rows; r += kScanThreads) extend_row(a, r, rows_used, free);
  }
}

constexpr int kExpandThreads = 256;
__global__ void __launch_bounds__(kExpandThreads) kv_extend_rows_kernel(ExtendArgs a) {
  asm volatile("griddepcontrol.wait;" ::: "memory");         // the scan is there
  const int64_t row = static_cast<int64_t>(blockIdx.x) * kExpandThreads + threadIdx.x;
  if (row >= a.rows) return;
  const int4 s = __ldcg(a.b.info + a.b.n_seqs);
  extend_row(a, row, s.x, s.y);
}

// The blocks of one sequence, by a warp.
__device__ __forceinline__ void truncate_columns(const BlocksArgs& a, int b, int64_t top, int lane) {
  const int4 s = __ldcg(a.info + b);
  const int32_t* row = a.table + static_cast<int64_t>(b) * a.max_blocks;
  for (int c = s.x + lane; c < s.y; c += 32) a.free_ids[top - 1 - (static_cast<int64_t>(s.w) + c - s.x)] = row[c];
}

template <bool kAlone>
__global__ void __launch_bounds__(kScanThreads) kv_truncate_scan_kernel(TruncateArgs a) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  __shared__ int64_t sm[2][kScanWarps];
  const int64_t free = free_blocks(a.b), most = static_cast<int64_t>(a.b.max_blocks) << a.b.block_log2;
  const int free_raw = *a.b.free_count;
  const bool known = free == free_raw;
  int64_t base = 0, total = 0;
  for (int b0 = 0; b0 < a.b.n_seqs; b0 += kScanThreads) {
    const int b = b0 + threadIdx.x;
    const bool in = b < a.b.n_seqs;
    const int64_t len = in ? a.b.len[b] : 0;
    int64_t keep = in ? max(a.keep[b], 0) : 0;
    if (keep > len) keep = len;
    bool ok = len >= 0 && len <= most;
    const int64_t lo = max(columns(keep, a.b.block_log2), static_cast<int64_t>(a.b.pinned));
    const int64_t back = ok ? max(columns(len, a.b.block_log2) - lo, int64_t{0}) : 0;
    const int64_t at = block_scan(back, base, sm);
    if (back > 0 && (!known || free + at + back > a.b.capacity)) ok = false;
    if (!in) continue;
    if (!ok) atomicOr(a.b.status, kStatusRange);
    if (ok && back > 0) total = at + back;
    a.b.info[b] = make_int4(static_cast<int>(lo), static_cast<int>(ok ? lo + back : lo), 0, clamp32(at));
    a.b.len_out[b] = static_cast<int>(ok ? keep : len);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) total = max(total, __shfl_xor_sync(0xffffffffu, total, o));
  if ((threadIdx.x & 31) == 0) sm[0][threadIdx.x >> 5] = total;
  __syncthreads();
  if (kAlone || threadIdx.x == 0)
    for (int w = 0; w < kScanWarps; ++w) total = max(total, sm[0][w]);
  if (threadIdx.x == 0) {
    *a.b.free_out = static_cast<int>(free_raw + total);
    if (!kAlone) a.b.info[a.b.n_seqs] = make_int4(static_cast<int>(free + total), 0, 0, 0);
  }
  if constexpr (kAlone) {
    for (int b = threadIdx.x >> 5; b < a.b.n_seqs; b += kScanWarps) truncate_columns(a.b, b, free + total, threadIdx.x & 31);
  }
}

__global__ void __launch_bounds__(kExpandThreads) kv_truncate_columns_kernel(TruncateArgs a) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int b = static_cast<int>((static_cast<int64_t>(blockIdx.x) * kExpandThreads + threadIdx.x) >> 5);
  if (b < a.b.n_seqs) truncate_columns(a.b, b, __ldcg(a.b.info + a.b.n_seqs).x, threadIdx.x & 31);
}

template <typename Args>
cudaError_t launch_behind(void (*kernel)(Args), const Args& a, int64_t threads, cudaStream_t stream) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>((threads + kExpandThreads - 1) / kExpandThreads));
  cfg.blockDim = dim3(kExpandThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

// The scan's block expands by itself up to this many rows (sequences, where blocks are given back).
constexpr int64_t kAloneRows = 4096, kAloneSeqs = 128;

}  // namespace

int kv_extend_launches(int64_t rows) { return rows <= kAloneRows ? 1 : 2; }
int kv_truncate_launches(int64_t n_seqs) { return n_seqs <= kAloneSeqs ? 1 : 2; }

cudaError_t launch_kv_extend(const ExtendArgs& a, cudaStream_t stream) {
  if (a.rows <= kAloneRows) {
    kv_extend_scan_kernel<true><<<1, kScanThreads, 0, stream>>>(a);
    return cudaGetLastError();
  }
  kv_extend_scan_kernel<false><<<1, kScanThreads, 0, stream>>>(a);
  const cudaError_t e = cudaGetLastError();
  return e != cudaSuccess ? e : launch_behind(kv_extend_rows_kernel, a, a.rows, stream);
}

cudaError_t launch_kv_truncate(const TruncateArgs& a, cudaStream_t stream) {
  if (a.b.n_seqs <= kAloneSeqs) {
    kv_truncate_scan_kernel<true><<<1, kScanThreads, 0, stream>>>(a);
    return cudaGetLastError();
  }
  kv_truncate_scan_kernel<false><<<1, kScanThreads, 0, stream>>>(a);
  const cudaError_t e = cudaGetLastError();
  return e != cudaSuccess ? e : launch_behind(kv_truncate_columns_kernel, a, 32 * static_cast<int64_t>(a.b.n_seqs), stream);
}

}  // namespace lrqat
