// Device helpers shared by the norm, 8-bit cache and cache attention kernels.
#pragma once

#include <cuda_runtime.h>
#include <cstdint>

#include "serve.h"

namespace lrqat {

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ void unpack8(const uint4& v, float (&x)[8]) {
  x[0] = bf16_lo(v.x), x[1] = bf16_hi(v.x), x[2] = bf16_lo(v.y), x[3] = bf16_hi(v.y);
  x[4] = bf16_lo(v.z), x[5] = bf16_hi(v.z), x[6] = bf16_lo(v.w), x[7] = bf16_hi(v.w);
}
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}

// 1.5 * 2^23: adding it to |y| < 2^22 rounds y to the nearest integer (ties to even) and
// leaves that integer, in two's complement, in the low bits of the sum.
constexpr float kRoundMagic = 12582912.0f;

// max(a, b) and max(|a|, |b|, |c|), NaN if one of them is.
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float max3_abs_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// t = round(fl32(x / s)) + kRoundMagic for 8 values with |x / s| < 2^10.  y = x r with r = fl32(1 / s) and
// fl32(x / s) both lie within 2^-22 |y| of x / s, below 2^-12: where y is more than 2^-11 away from a
// half-integer both round to the same integer; otherwise, and where r is infinite or a value is not a
// number, the division decides.  A scale below 2^-142 has too few bits for max|x| / s <= 127 (up to 190), which
// fp32 x can meet, bf16 x not (kFp32): r is infinite there, and the division's integers end at -128 and 127.
template <bool kFp32>
__device__ __forceinline__ void round_div8(const float (&x)[8], float s, float r, float (&t)[8]) {
  const float2 rr = make_float2(r, r), mm = make_float2(kRoundMagic, kRoundMagic);
  float off = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const float2 v = make_float2(x[e], x[e + 1]);
    const float2 u = __ffma2_rn(v, rr, mm);
    const float2 q = __fadd2_rn(mm, make_float2(-u.x, -u.y));              // minus the integer
    const float2 d = __ffma2_rn(v, rr, q);
    off = max3_abs_nan(off, d.x, d.y);
    t[e] = u.x, t[e + 1] = u.y;
  }
  if (!(off < 0.49951171875f)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float u = rintf(__fdiv_rn(x[e], s));
      t[e] = (kFp32 ? fminf(fmaxf(u, -128.0f), 127.0f) : u) + kRoundMagic;
    }
  }
}
// The codes of round_div8: the low bytes of whole numbers in [-128, 127] plus kRoundMagic.
__device__ __forceinline__ uint2 pack_codes8(const float (&t)[8]) {
  uint32_t b[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) b[e] = __float_as_uint(t[e]);
  return make_uint2(__byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410),
                    __byte_perm(__byte_perm(b[4], b[5], 0x0040), __byte_perm(b[6], b[7], 0x0040), 0x5410));
}
// Four int8 codes as floats: 2^23 + (c + 128) has the byte c + 128 as its low mantissa bits.
__device__ __forceinline__ void codes4(uint32_t w, float (&c)[4]) {
  const uint32_t u = w ^ 0x80808080u;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    c[e] = __uint_as_float(__byte_perm(u, 0x4B000000u, 0x7540 + e)) - 8388736.0f;
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Asynchronous copies into shared memory, in groups that a thread waits for.
__device__ __forceinline__ uint32_t smem_addr(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ void copy_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_async16(void* dst, const void* src) { copy_async16(smem_addr(dst), src); }
__device__ __forceinline__ void copy_async4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kPending>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(kPending) : "memory");
}

// The rows of sequence b: `n` rows from row `row0` of the batch, at positions first .. len - 1.
// Negative positions belong to padding rows.  False (and the range bit of the status word) where
// the arrays contradict the batch's bounds.
struct SeqRows {
  int64_t row0;
  int n, len, first;
};
__device__ __forceinline__ bool seq_rows(const KvArgs& a, int b, SeqRows& s) {
  const int64_t r0 = a.row_start[b], r1 = a.row_start[b + 1];
  const int len = a.len[b];
  s.row0 = r0;
  s.n = static_cast<int>(r1 - r0);
  s.len = len;
  s.first = len - s.n;
  if (r0 < 0 || r1 < r0 || r1 > a.rows || r1 - r0 > a.max_rows || len < 0 || len > a.max_len) {
    if (threadIdx.x == 0) atomicOr(a.status, kStatusRange);
    return false;
  }
  return true;
}
// The cache block that holds position `pos` of sequence b, or -1 (and the range bit).
__device__ __forceinline__ int seq_block(const KvArgs& a, int b, int pos) {
  const int blk = __ldg(a.table + static_cast<int64_t>(b) * a.max_blocks + (pos >> a.block_log2));
  if (static_cast<uint32_t>(blk) >= static_cast<uint64_t>(a.n_blocks)) {
    atomicOr(a.status, kStatusRange);
    return -1;
  }
  return blk;
}

}  // namespace lrqat
