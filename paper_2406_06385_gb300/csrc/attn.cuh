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
// head's group.
struct Tile {
  SeqRows seq;
  int rows;            // rows of the sequence and head, all tiles
  int r0;              // first row of this tile
  int pos_lo, pos_hi;  // positions of the tile's first and last row
  int lo, hi;          // keys [lo, hi) that some row may see; lo a multiple of kKeyAlign
};
__device__ __forceinline__ bool attn_tile(const AttnArgs& a, int b, int rt, Tile& t) {
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
  return true;
}

// The end of the piece of a tile's keys that starts at k0.
__device__ __forceinline__ int piece_end(const AttnArgs& a, const Tile& t, int k0) {
  return t.hi - k0 > a.chunk ? k0 + a.chunk : t.hi;
}
__device__ __forceinline__ int tile_splits(const AttnArgs& a, const Tile& t) {
  return t.hi > t.lo ? (t.hi - t.lo - 1) / a.chunk + 1 : 0;   // lengths and a.chunk may be close to 2^31
}

}  // namespace lrqat
