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

// Rows and blocks are counted up to 2^31 - 1, which is more than any array holds: sums of numbers that are not
// negative stay there, in whatever order they are formed.
struct Count {
  uint32_t rows, blocks;
};
__device__ __forceinline__ uint32_t upto(int64_t v) { return v > INT32_MAX ? INT32_MAX : static_cast<uint32_t>(v); }
__device__ __forceinline__ Count operator+(Count a, Count b) {
  return {min(a.rows + b.rows, static_cast<uint32_t>(INT32_MAX)), min(a.blocks + b.blocks, static_cast<uint32_t>(INT32_MAX))};
}
__device__ __forceinline__ Count shfl_up(Count v, int o) {
  return {__shfl_up_sync(0xffffffffu, v.rows, o), __shfl_up_sync(0xffffffffu, v.blocks, o)};
}
__device__ __forceinline__ Count warp_scan(Count v, int lane) {              // inclusive
#pragma unroll
  for (int o = 1; o < 32; o *= 2) {
    const Count u = shfl_up(v, o);
    if (lane >= o) v = v + u;
  }
  return v;
}
// What the threads before hold, behind `carry`; carry becomes the sum of all so far.  Every thread calls it.
__device__ __forceinline__ Count block_scan(Count v, Count& carry, Count (*sm)[kScanWarps]) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Count in = warp_scan(v, lane), up = shfl_up(in, 1);
  if (lane == 31) sm[0][warp] = in;
  __syncthreads();
  if (warp == 0) sm[1][lane] = warp_scan(sm[0][lane], lane);
  __syncthreads();
  Count out = carry;
  if (warp > 0) out = out + sm[1][warp - 1];
  if (lane > 0) out = out + up;
  carry = carry + sm[1][kScanWarps - 1];
  return out;
}
__device__ __forceinline__ int64_t columns(int64_t tokens, int block_log2) {
  return (tokens + (1 << block_log2) - 1) >> block_log2;
}
// The number of free blocks, 0 (and the range bit) where it is none.
__device__ __forceinline__ int64_t free_blocks(const BlocksArgs& a, int n) {
  if (n >= 0 && n <= a.capacity) return n;
  if (threadIdx.x == 0) atomicOr(a.status, kStatusRange);
  return 0;
}
// The largest v over the block, valid in every thread.
__device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t* sm) {
  v = __reduce_max_sync(0xffffffffu, v);
  if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = v;
  __syncthreads();
  return __reduce_max_sync(0xffffffffu, sm[threadIdx.x & 31]);
}

// What the expansion has to know of a sequence.  Extending, x: its first new position, or -1 for rows of padding;
// y: its first row; z: its first new column; w: its base.  Shortening, x and y: the columns it gives back; w: its base.

// One row of sequence b: its position and slot, and the table's entry where the row is the first of a new column.
__device__ __forceinline__ void extend_row(const ExtendArgs& a, int64_t row, int b, const int4& s, int64_t free) {
  int pos = -1;
  int64_t slot = -1;
  if (b >= 0 && s.x >= 0) {
    pos = s.x + static_cast<int>(row - s.y);
    const int column = pos >> a.b.block_log2, in_block = pos & ((1 << a.b.block_log2) - 1);
    int32_t* entry = a.b.table + static_cast<int64_t>(b) * a.b.max_blocks + column;
    int id;
    if (column >= s.z) {
      id = a.b.free_ids[free - 1 - (static_cast<int64_t>(s.w) + column - s.z)];
      if (in_block == 0) *entry = id;
    } else {
      id = *entry;
    }
    slot = (static_cast<int64_t>(id) << a.b.block_log2) + in_block;
  }
  a.pos[row] = pos;
  if (a.slot) a.slot[row] = slot;
}

// A thread takes kItems neighbouring sequences.  kAlone: at most kScanThreads sequences and few rows, which the block
// expands itself.  Otherwise info[n_seqs] holds {rows used, free blocks} for the expansion.
template <bool kAlone, int kItems>
__global__ void __launch_bounds__(kScanThreads) kv_extend_scan_kernel(ExtendArgs a) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  __shared__ Count sm[2][kScanWarps];
  __shared__ uint32_t top[kScanWarps];
  __shared__ int4 info[kAlone ? kScanThreads : 1];
  const int free_raw = *a.b.free_count;
  const int64_t most = static_cast<int64_t>(a.b.max_blocks) << a.b.block_log2;
  int64_t free = -1;
  Count carry{0, 0};
  uint32_t used = 0;                         // what sequences that are served reach, of this thread
  for (int b0 = 0; b0 < a.b.n_seqs; b0 += kItems * kScanThreads) {
    int len[kItems], add[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int b = b0 + kItems * threadIdx.x + i;
      len[i] = b < a.b.n_seqs ? a.b.len[b] : 0;
      add[i] = b < a.b.n_seqs ? a.add[b] : 0;
    }
    if (free < 0) free = free_blocks(a.b, free_raw);
    Count mine[kItems], sum{0, 0};
    bool ok[kItems];
    int column[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int64_t n = len[i], m = add[i];
      ok[i] = n >= 0 && n <= most && (m <= 0 || n + m <= most);
      column[i] = static_cast<int>(max(columns(ok[i] ? n : 0, a.b.block_log2), static_cast<int64_t>(a.b.pinned)));
      mine[i].rows = upto(m < 0 ? -m : m);
      mine[i].blocks = ok[i] && m > 0 ? upto(max(columns(n + m, a.b.block_log2) - column[i], int64_t{0})) : 0;
      sum = sum + mine[i];
    }
    Count at = block_scan(sum, carry, sm);
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int b = b0 + kItems * threadIdx.x + i;
      const Count end = at + mine[i];
      if (b < a.b.n_seqs) {
        // behind the first that does not fit the rows, or whose blocks run out, no other with rows or blocks fits
        if (end.rows > a.rows || (mine[i].blocks > 0 && end.blocks > free)) ok[i] = false;
        if (!ok[i]) atomicOr(a.b.status, kStatusRange);
        if (ok[i] && mine[i].blocks > 0) used = end.blocks;
        const bool grows = ok[i] && add[i] > 0;
        const int4 s = make_int4(grows ? len[i] : -1, static_cast<int>(at.rows), column[i], static_cast<int>(at.blocks));
        if (kAlone) info[b] = s;
        else a.b.info[b] = s;
        a.b.len_out[b] = grows ? len[i] + add[i] : len[i];
        a.batch_len[b] = ok[i] && add[i] >= 0 ? len[i] + add[i] : 0;
        a.row_start[b] = static_cast<int>(at.rows);
        if (b == a.b.n_seqs - 1) a.row_start[a.b.n_seqs] = static_cast<int>(end.rows);
      }
      at = end;
    }
    __syncthreads();                         // sm has been read
  }
  used = block_max(used, top);               // and info is there
  const int64_t rows_used = min(static_cast<int64_t>(carry.rows), a.rows);
  if (threadIdx.x == 0) {
    *a.b.free_out = static_cast<int>(free_raw - static_cast<int64_t>(used));
    if (!kAlone) a.b.info[a.b.n_seqs] = make_int4(static_cast<int>(rows_used), static_cast<int>(free), 0, 0);
  }
  if constexpr (kAlone) {
    for (int64_t row = threadIdx.x; row < a.rows; row += kScanThreads) {
      int lo = 0, hi = a.b.n_seqs;           // the last sequence whose first row is not behind `row`
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (info[mid].y <= row) lo = mid;
        else hi = mid;
      }
      extend_row(a, row, row < rows_used ? lo : -1, info[lo], free);
    }
  }
}

// A warp takes kWarpRows rows, 32 at a time.  The first one's sequence is found by probing 32 starts a time, the others'
// among the 32 starts behind it (all of them, where more than 32 sequences share 32 rows).
constexpr int kExpandThreads = 256;
constexpr int kWarpRows = 128;
__global__ void __launch_bounds__(kExpandThreads) kv_extend_rows_kernel(ExtendArgs a) {
  asm volatile("griddepcontrol.wait;" ::: "memory");         // the scan is there
  const int lane = threadIdx.x & 31, n = a.b.n_seqs;
  const int64_t row0 = (static_cast<int64_t>(blockIdx.x) * (kExpandThreads / 32) + (threadIdx.x >> 5)) * kWarpRows;
  if (row0 >= a.rows) return;
  const int4 total = __ldcg(a.b.info + n);
  int b = 0, end = n;
  while (end - b > 1) {
    const int step = (end - b + 31) >> 5, probe = b + step * lane;
    const uint32_t hit = __ballot_sync(0xffffffffu, probe < end && __ldcg(a.row_start + probe) <= row0);
    b += step * (31 - __clz(hit));           // the start of b itself is not behind row0
    end = min(b + step, end);
  }
#pragma unroll
  for (int i = 0; i < kWarpRows / 32; ++i) {
    const int64_t row = row0 + 32 * i + lane;
    const int start = __ldcg(a.row_start + min(b + 1 + lane, n));
    int behind = 0;                          // of those 32 starts, the number that are not behind the row
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
      if (__shfl_sync(0xffffffffu, start, behind + o - 1) <= row) behind += o;
    if (__shfl_sync(0xffffffffu, start, 31) <= row && behind == 31) behind = 32;
    int lo = min(b + behind, n - 1), hi = behind == 32 ? n : lo + 1;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (__ldcg(a.row_start + mid) <= row) lo = mid;
      else hi = mid;
    }
    if (row < a.rows) {
      const bool in = row < total.x;
      extend_row(a, row, in ? lo : -1, in ? __ldcg(a.b.info + lo) : total, total.y);
    }
    b = __shfl_sync(0xffffffffu, lo, 31);
  }
}

// The blocks of one sequence, by a warp.
__device__ __forceinline__ void truncate_columns(const BlocksArgs& a, int b, int64_t top, int lane) {
  const int4 s = __ldcg(a.info + b);
  const int32_t* row = a.table + static_cast<int64_t>(b) * a.max_blocks;
  for (int c = s.x + lane; c < s.y; c += 32) a.free_ids[top - 1 - (static_cast<int64_t>(s.w) + c - s.x)] = row[c];
}

template <bool kAlone, int kItems>
__global__ void __launch_bounds__(kScanThreads) kv_truncate_scan_kernel(TruncateArgs a) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  __shared__ Count sm[2][kScanWarps];
  __shared__ uint32_t top[kScanWarps];
  const int free_raw = *a.b.free_count;
  const int64_t most = static_cast<int64_t>(a.b.max_blocks) << a.b.block_log2;
  int64_t free = -1;
  Count carry{0, 0};
  uint32_t total = 0;                        // what sequences that are shortened reach, of this thread
  for (int b0 = 0; b0 < a.b.n_seqs; b0 += kItems * kScanThreads) {
    int len[kItems], keep[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int b = b0 + kItems * threadIdx.x + i;
      len[i] = b < a.b.n_seqs ? a.b.len[b] : 0;
      keep[i] = b < a.b.n_seqs ? a.keep[b] : 0;
    }
    if (free < 0) free = free_blocks(a.b, free_raw);
    Count mine[kItems], sum{0, 0};
    bool ok[kItems];
    int lo[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      ok[i] = len[i] >= 0 && len[i] <= most;
      keep[i] = min(max(keep[i], 0), max(len[i], 0));
      lo[i] = static_cast<int>(max(columns(keep[i], a.b.block_log2), static_cast<int64_t>(a.b.pinned)));
      mine[i].rows = 0;
      mine[i].blocks = ok[i] ? upto(max(columns(len[i], a.b.block_log2) - lo[i], int64_t{0})) : 0;
      sum = sum + mine[i];
    }
    Count at = block_scan(sum, carry, sm);
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int b = b0 + kItems * threadIdx.x + i;
      const Count end = at + mine[i];
      if (b < a.b.n_seqs) {
        if (mine[i].blocks > 0 && (free != free_raw || free + end.blocks > a.b.capacity)) ok[i] = false;
        if (!ok[i]) atomicOr(a.b.status, kStatusRange);
        if (ok[i] && mine[i].blocks > 0) total = end.blocks;
        a.b.info[b] = make_int4(lo[i], ok[i] ? lo[i] + static_cast<int>(mine[i].blocks) : lo[i], 0, static_cast<int>(at.blocks));
        a.b.len_out[b] = ok[i] ? keep[i] : len[i];
      }
      at = end;
    }
    __syncthreads();                         // sm has been read
  }
  total = block_max(total, top);             // and info is there
  if (threadIdx.x == 0) {
    *a.b.free_out = static_cast<int>(free_raw + static_cast<int64_t>(total));
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

// The scan's block expands by itself up to this many rows (of at most kScanThreads sequences; sequences, where blocks are
// given back).
constexpr int64_t kAloneRows = 4096, kAloneSeqs = 128;
bool extend_alone(const ExtendArgs& a) { return a.rows <= kAloneRows && a.b.n_seqs <= kScanThreads; }

}  // namespace

int kv_extend_launches(const ExtendArgs& a) { return extend_alone(a) || a.rows == 0 ? 1 : 2; }
int kv_truncate_launches(const TruncateArgs& a) { return a.b.n_seqs <= kAloneSeqs ? 1 : 2; }

cudaError_t launch_kv_extend(const ExtendArgs& a, cudaStream_t stream) {
  if (extend_alone(a)) {
    kv_extend_scan_kernel<true, 1><<<1, kScanThreads, 0, stream>>>(a);
    return cudaGetLastError();
  }
  if (a.b.n_seqs <= kScanThreads) kv_extend_scan_kernel<false, 1><<<1, kScanThreads, 0, stream>>>(a);
  else kv_extend_scan_kernel<false, 4><<<1, kScanThreads, 0, stream>>>(a);
  const cudaError_t e = cudaGetLastError();
  if (a.rows == 0) return e;                 // nothing to expand, and no grid is empty
  return e != cudaSuccess ? e : launch_behind(kv_extend_rows_kernel, a, (a.rows + kWarpRows - 1) / kWarpRows * 32, stream);
}

cudaError_t launch_kv_truncate(const TruncateArgs& a, cudaStream_t stream) {
  if (a.b.n_seqs <= kAloneSeqs) {
    kv_truncate_scan_kernel<true, 1><<<1, kScanThreads, 0, stream>>>(a);
    return cudaGetLastError();
  }
  if (a.b.n_seqs <= kScanThreads) kv_truncate_scan_kernel<false, 1><<<1, kScanThreads, 0, stream>>>(a);
  else kv_truncate_scan_kernel<false, 4><<<1, kScanThreads, 0, stream>>>(a);
  const cudaError_t e = cudaGetLastError();
  return e != cudaSuccess ? e : launch_behind(kv_truncate_columns_kernel, a, 32 * static_cast<int64_t>(a.b.n_seqs), stream);
}

}  // namespace lrqat
