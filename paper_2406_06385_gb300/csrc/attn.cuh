// What the cache attention kernels share: the codes as half precision numbers, the row tiles and
// their splits.
#pragma once

#include <cuda_runtime.h>
#include <cstdint>

#include "serve.cuh"

namespace lrqat {

constexpr int kKeyAlign = 32;      // a row tile's first key is a multiple of this

__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// Bytes `sel` of a word of codes biased by 128 as two halves: the half 0x6400 | u is 1024 + u.
template <uint32_t kSel>
__device__ __forceinline__ uint32_t half_codes(uint32_t biased) {
  const uint32_t h = __byte_perm(biased, 0x64646464u, kSel);
  uint32_t r;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(h), "r"(0x64806480u));   // 1024 + 128
  return r;
}
__device__ __forceinline__ float lg2(float x) {
  float y;
  asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.0f : m; }
// 2^up / l, 0 for a row that saw no key (l = 0); up = m - n is at most log2 of the largest scale, and -infinity
// where every value scale that the row saw is 0.
__device__ __forceinline__ float out_factor(float l, float up) {
  const float half = ex2(0.5f * up);                   // 2^up itself may be subnormal
  return l == 0.0f ? 0.0f : half / l * half;
}

// The tile of `tile_rows` rows `rt` of (sequence, key/value head): row i is token
// (tile_rows rt + i) / group of the sequence's rows and query head (tile_rows rt + i) % group of the
// head's group.  Its keys are numbered without the gap between the sinks and the window: number x is key x before
// sink_pad and key x + gap from there on.  Where there is a gap, x + gap may stand for the key in what hides keys
// behind a row's position or before its window, whatever x: every row lies behind the gap, and a number that is
// not below `sinks` but below sink_pad then counts as before the window, as it has to.
struct Tile {
  SeqRows seq;
  int rows;            // rows of the sequence and head, all tiles
  int r0;              // first row of this tile
  int pos_lo, pos_hi;  // positions of the tile's first and last row
  int lo, hi;          // keys [lo, hi) that some row may see; lo a multiple of 16
  int gap;             // general variants only
};
template <bool kGeneral>
__device__ __forceinline__ bool attn_tile(const AttnArgs& a, int b, int rt, Tile& t) {
  t.gap = 0;
  if (kGeneral && a.across) {
    t.seq.row0 = 0;
    t.seq.n = static_cast<int>(a.kv.rows);
    t.seq.len = t.seq.first = 0;
    t.rows = t.seq.n * a.group;
    t.r0 = rt * a.tile_rows;
    t.pos_lo = t.pos_hi = 0;
    t.lo = 0;
    t.hi = a.prefix;
    return t.r0 < t.rows;
  }
  if (!seq_rows(a.kv, b, t.seq)) return false;
  t.rows = t.seq.n * a.group;
  t.r0 = rt * a.tile_rows;
  if (t.r0 >= t.rows) return false;
  const int last = min(t.r0 + a.tile_rows, t.rows) - 1;
  t.pos_lo = t.seq.first + t.r0 / a.group;
  t.pos_hi = t.seq.first + last / a.group;
  t.hi = max(t.pos_hi + 1, 0);
  const int64_t seen = static_cast<int64_t>(t.pos_lo) - a.window + 1;   // pos_lo is negative for padding rows
  t.lo = a.window > 0 && seen > 0 ? static_cast<int>(seen) & ~(kKeyAlign - 1) : 0;
  if (kGeneral) {
    if (a.sinks > 0) {
      t.lo = a.window > 0 && seen > 0 ? static_cast<int>(seen) & ~15 : 0;
      if (t.lo > a.sink_pad) t.gap = t.lo - a.sink_pad;
      t.hi -= t.gap;
      t.lo = 0;
    }
    if (a.first > 0) t.lo = a.first;
  }
  return true;
}
// The key that number x stands for.
template <bool kGeneral>
__device__ __forceinline__ int key_at(const AttnArgs& a, const Tile& t, int x) {
  return kGeneral && x >= a.sink_pad ? x + t.gap : x;
}
// The entry of a block table that holds `key` of the sequence whose row of the table is given.
template <bool kGeneral>
__device__ __forceinline__ int table_entry(const AttnArgs& a, const int32_t* table, int key) {
  return __ldg((kGeneral && key < a.prefix ? a.prefix_table : table) + (key >> a.kv.block_log2));
}
// The block of the 16 keys from number x on.  The blocks between the sinks and the window, which may be anybody's, have no
// numbers: a tile's numbers go on from the sinks' last 16 keys to the 16 that hold the first key of its first row's window.
template <bool kGeneral>
__device__ __forceinline__ int group_block(const AttnArgs& a, const Tile& t, const int32_t* table, int x) {
  int key = key_at<kGeneral>(a, t, x);
  if (kGeneral) asm volatile("" : "+r"(key));   // kept apart from the other uses of x: merged, 8-row tiles spill 24 bytes
  return table_entry<kGeneral>(a, table, key);
}

// The sequence of a row of the batch and the row's position.  seq -1: a row behind the last sequence, or of a sequence that
// contradicts the bounds; pos below 0: padding.
struct RowPlace {
  int seq, pos;
};
__device__ __forceinline__ bool row_in(const KvArgs& a, int b, int64_t row) {
  return __ldg(a.row_start + b) <= row && row < __ldg(a.row_start + b + 1);
}
// The last sequence in [lo, hi) whose first row is not behind `row`, where row starts do not fall.
__device__ __forceinline__ int last_start(const KvArgs& a, int lo, int hi, int64_t row) {
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (__ldg(a.row_start + mid) <= row) lo = mid;
    else hi = mid;
  }
  return lo;
}
// The place of a row that sequence `b` should hold.  Where it does not, the arrays contradict themselves, and the row may
// still belong to a sequence that does not.
__device__ __forceinline__ RowPlace row_place(const KvArgs& a, int b, int64_t row) {
  if (!row_in(a, b, row)) {
    const int end = __ldg(a.row_start + b + 1);
    if (b == a.n_seqs - 1 && __ldg(a.row_start + b) <= end && end <= row) return {-1, -1};
    for (b = 0; b < a.n_seqs && !row_in(a, b, row); ++b) {
    }
    if (b == a.n_seqs) return {-1, -1};
  }
  const int64_t r0 = __ldg(a.row_start + b), r1 = __ldg(a.row_start + b + 1);
  const int len = __ldg(a.len + b);
  if (r0 < 0 || r1 > a.rows || r1 - r0 > a.max_rows || len < 0 || len > a.max_len) return {-1, -1};
  return {b, static_cast<int>(len - (r1 - row))};
}
__device__ __forceinline__ RowPlace find_row(const KvArgs& a, int64_t row) {
  return row_place(a, last_start(a, 0, a.n_seqs, row), row);
}
// The same for the rows of a warp's lanes, which do not fall from lane to lane: the first lane's sequence by probing 32
// starts at a time, the others' among the 32 starts behind it.
__device__ __forceinline__ RowPlace find_rows(const KvArgs& a, int64_t row) {
  const int lane = threadIdx.x & 31;
  const int64_t row0 = __shfl_sync(0xffffffffu, row, 0);
  int b = 0, end = a.n_seqs;
  while (end - b > 1) {
    const int step = (end - b + 31) >> 5, probe = b + step * lane;
    const uint32_t hit = __ballot_sync(0xffffffffu, probe < end && __ldg(a.row_start + probe) <= row0) | 1u;
    b += step * (31 - __clz(hit));
    end = min(b + step, end);
  }
  const int start = __ldg(a.row_start + min(b + 1 + lane, a.n_seqs));
  int behind = 0;                            // of those, how many are not behind the row
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    if (__shfl_sync(0xffffffffu, start, behind + o - 1) <= row) behind += o;
  const bool more = __shfl_sync(0xffffffffu, start, 31) <= row;
  b = min(b + behind, a.n_seqs - 1);
  if (more) b = last_start(a, b, a.n_seqs, row);
  return row_place(a, b, row);
}

// At the end of one block of a launch that runs beside the one before it: the launch ends behind that one, so that what
// comes next finds the results of both.
__device__ __forceinline__ void finish_behind() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// The end of the piece of a tile's keys that starts at k0.
__device__ __forceinline__ int piece_end(const AttnArgs& a, const Tile& t, int k0) {
  return t.hi - k0 > a.chunk ? k0 + a.chunk : t.hi;
}
__device__ __forceinline__ int tile_splits(const AttnArgs& a, const Tile& t) {
  return t.hi > t.lo ? (t.hi - t.lo - 1) / a.chunk + 1 : 0;   // lengths and a.chunk may be close to 2^31
}

}  // namespace lrqat
