// Attention of the newest tokens of each sequence over the paged 8-bit cache.
//
// With s_k, s_v the scales of a cache block and c_k, c_v its codes, query row q at position p:
//   z_j = scale s_k (q . c_k,j)   for the keys j <= p (and j > p - window),
//   o = sum_j e^{z_j} s_v c_v,j / sum_j e^{z_j},   0 for a row that sees no key.
// The kernels fold s_v into the exponent: with z'_j = z_j log2(e) + log2(s_v) and m their running maximum,
// P_j = 2^{z'_j - m} lies in [0, 1] and is what a key contributes to o, whatever the scales of the blocks
// are (the many-row kernel lets m stay below the maximum as long as half precision holds P, and scales
// within 2^32 of the first one share m with the denominator).  The denominator, the sum of P_j / s_v, is
// kept relative to a running maximum n of its own, that of z_j log2(e): scales of one sequence may lie as
// far apart as fp32 reaches. So P fits half precision (11 bits, fewer below 2^-14, zero below 2^-25: a long
// row loses at most its number of keys times 2^-25 of its largest contribution) and the codes (|c| <= 128)
// are exact in it; a row of q is first divided by the power of two of its largest magnitude, which half
// precision also holds (exact but for elements below 2^-14 of the largest).
// Scores, maxima, sums and outputs are 32-bit.
#include <cuda_runtime.h>
#include <cstdint>
#include <type_traits>

#include "attn.cuh"
#include "kernels.h"

namespace lrqat {
namespace {

constexpr int kWarps = 4;
constexpr int kStep = kKeyAlign;   // keys of one step of a warp, in two halves of 16
constexpr int kStages = 2, kValueStages = 1;   // steps of keys and of values in a warp's ring
constexpr int kPerSm = 16 / kWarps;        // thread blocks an SM holds (with 16 rows: half of them)

__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                          const uint32_t (&b)[2]) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b[0]), "r"(b[1]));
}
// Transposes an 8 x 8 matrix of halves whose row l / 4 lane l holds at columns 2 (l % 4), + 1.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t addr) {
  uint2 v;
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr) : "memory");
  return v;
}

// Where 16-byte piece q of token r (of 16) lies in a warp's shared memory, so that copying whole
// tokens and the lanes' reads below are free of bank conflicts.
template <int D>
__device__ __forceinline__ uint32_t key_place(uint32_t r, uint32_t q) {
  return D == 128 ? r * 128 + (q ^ (r & 1) << 2) * 16 : r * 64 + q * 16;
}
template <int D>
__device__ __forceinline__ uint32_t value_place(uint32_t r, uint32_t q) {
  return D == 128 ? r * 128 + (q ^ (r & 6)) * 16 : (r ^ (r >> 2 & 1)) * 64 + (q ^ (r & 2)) * 16;
}

template <int D, int NT>
struct SplitSmem {
  static constexpr int kHalf = 16 * D;                                      // bytes of 16 keys
  static constexpr int kWarpStage = 2 * kHalf;                              // 32 keys, or their values
  static constexpr int kRing = (kStages + kValueStages) * kWarps * kWarpStage;
  static constexpr int kOut = kWarps * 8 * NT * (D + 4) * 4;                // the join's outputs reuse the ring
  static constexpr int kScales = kRing > kOut ? kRing : kOut;
  static constexpr int kBytes = kScales + kStages * kWarps * 16;
};

// One thread block per (split, head and row tile, sequence); a tile has 8 NT (token, head) rows. A warp
// takes every fourth step of 32 keys and keeps its own maxima, sum and outputs; the warps join at the
// end.  Keys are the M of the first product (scores = K q^T) and the head's dimensions that of the
// second (o^T = V^T P^T), so a tile of 8 rows wastes no tensor work and few registers, and one 8 x 8
// transpose per 8 keys turns scores into the second product's operand.  The order of the dimensions
// inside a product is free: each lane takes 16 consecutive bytes of a token.  A step's codes come
// through a ring in shared memory filled by the warp that reads it: warps never wait for one another.
// Bound by the copies in flight (48 KB a block, four blocks an SM) and, close behind, by issue slots (58%
// in use, half of them for turning codes into halves): 64 ragged sequences at 72% of the memory's rate.
template <int D, int NT, bool kGeneral>
__device__ __forceinline__ void split_block(const AttnArgs& a) {
  using Sm = SplitSmem<D, NT>;
  constexpr int kC = D / 64;         // 64-dimension pieces of a token
  constexpr int kRows = 8 * NT;
  extern __shared__ __align__(16) uint8_t smem[];
  const int h = blockIdx.x % a.kv.heads, rt = blockIdx.x / a.kv.heads, b = blockIdx.y;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  Tile t;
  if (!attn_tile<kGeneral>(a, b, rt, t)) return;
  // Whole pieces first, every tile's shorter one (or its piece number a.splits - 1) in the end, where it fills
  // gaps: 20 ragged sequences of up to 5000 tokens with 40 heads 103 -> 97 us, 90 of up to 3000 with 8 heads
  // 65 -> 60, 64 of up to 8100 no faster (82 -> 83).
  const int ns = tile_splits(a, t);
  if (kGeneral && a.keep_parts && ns == 0) return;
  const bool last = blockIdx.z + 1 == gridDim.z;
  const int split = last ? max(ns - 1, 0) : static_cast<int>(blockIdx.z);
  if (last ? ns > 0 && ns < a.splits && (t.hi - t.lo) % a.chunk == 0
           : (split + 1) * static_cast<int64_t>(a.chunk) > t.hi - t.lo)
    return;
  const int k0 = t.lo + split * a.chunk, k1 = piece_end(a, t, k0);

  const uint32_t ring = smem_addr(smem) + warp * Sm::kWarpStage;
  const uint32_t scales = smem_addr(smem) + Sm::kScales + warp * 16;
  constexpr uint32_t kStageBytes = kWarps * Sm::kWarpStage, kStageScales = kWarps * 16;
  const int first_key = k0 + kStep * warp;
  const int steps = first_key < k1 ? (k1 - first_key + kStep * kWarps - 1) / (kStep * kWarps) : 0;
  const int32_t* table = a.kv.table + static_cast<int64_t>(b) * a.kv.max_blocks;
  const uint32_t in_block = (1u << a.kv.block_log2) - 1;
  // 16 keys from `key` on; the second half of a step may lie past the tile's keys, and then past the table
  auto block_of = [&](int key) { return key < k1 ? group_block<kGeneral>(a, t, table, key) : -2; };
  int next_blk[2] = {block_of(first_key), block_of(first_key + 16)};
  uint32_t skipped = 0;              // bit 2 s + u: half u of the step in stage s has no valid block
  const uint32_t piece = lane % (D / 16), tok = lane / (D / 16);            // a copy instruction covers 512 / D tokens
  int64_t off[2] = {-1, -1};         // where the keys copied last lie: the values that are copied next
  static_assert(kStages == 2 && kValueStages == 1, "order of the copies: keys 0, values 0, keys 1, values 1, keys 2, ...");
  // the keys and scales of step i, then its values
  auto issue_keys = [&](int i) {
    if (i < steps) {
      const int key = first_key + i * kStep * kWarps, stage = i % kStages;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int blk = next_blk[u];
        next_blk[u] = block_of(key + kStep * kWarps + 16 * u);
        const uint32_t bit = 1u << (2 * stage + u);
        off[u] = -1;
        if (static_cast<uint32_t>(blk) < static_cast<uint64_t>(a.kv.n_blocks)) {
          skipped &= ~bit;
          const int64_t at = static_cast<int64_t>(blk) * a.kv.heads + h;
          off[u] = ((at << a.kv.block_log2) + (key_at<kGeneral>(a, t, key + 16 * u) & in_block)) * D + lane * 16;
          const int8_t* p = a.kv.codes[0] + off[u];
          const uint32_t dst = ring + stage * kStageBytes + u * Sm::kHalf;
#pragma unroll
          for (int j = 0; j < D / 32; ++j) copy_async16(dst + key_place<D>(512 / D * j + tok, piece), p + 512 * j);
          if (lane < 2)
            copy_async4(scales + stage * kStageScales + u * 8 + lane * 4, (lane ? a.kv.scale[1] : a.kv.scale[0]) + at);
        } else {
          skipped |= bit;
          if (lane == 0 && blk != -2) atomicOr(a.kv.status, kStatusRange);
        }
      }
    }
    copy_commit();
  };
  auto issue_values = [&](int i) {
    if (i < steps) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if (off[u] < 0) continue;
        const int8_t* p = a.kv.codes[1] + off[u];
        const uint32_t dst = ring + (kStages + i % kValueStages) * kStageBytes + u * Sm::kHalf;
#pragma unroll
        for (int j = 0; j < D / 32; ++j) copy_async16(dst + value_place<D>(512 / D * j + tok, piece), p + 512 * j);
      }
    }
    copy_commit();
  };
  // q is asked for ahead of the ring's bytes, which would keep it waiting
  uint4 qw[NT][kC][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = t.r0 + 8 * nt + g;
    const uint16_t* q = a.Q + (t.seq.row0 + r / a.group) * a.ldq + static_cast<int64_t>(h * a.group + r % a.group) * D;
#pragma unroll
    for (int c = 0; c < kC; ++c)
#pragma unroll
      for (int u = 0; u < 2; ++u)
        qw[nt][c][u] = r < t.rows ? __ldg(reinterpret_cast<const uint4*>(q + 64 * c + 16 * t4) + u) : make_uint4(0u, 0u, 0u, 0u);
  }
  issue_keys(0);
  issue_values(0);
  issue_keys(1);

  // row g of each 8: its operand fragments; rows 2 t4, + 1: power of two and position
  uint32_t qf[NT][4 * kC][2];
  float qs[NT][2];
  int pos[NT][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    float x[kC][16], top = 0.0f;
#pragma unroll
    for (int c = 0; c < kC; ++c)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        float v[8];
        unpack8(qw[nt][c][u], v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[c][8 * u + e] = v[e];
          top = fmaxf(top, fabsf(v[e]));
        }
      }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const uint32_t e = min(max(__float_as_uint(top) >> 23, 1u), 253u);   // exponent of a normal power of two
    const float inv = __uint_as_float((254u - e) << 23);
#pragma unroll
    for (int c = 0; c < kC; ++c)
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int k = 0; k < 2; ++k)
          qf[nt][4 * c + u][k] = pack_half(x[c][4 * u + 2 * k] * inv, x[c][4 * u + 2 * k + 1] * inv);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      qs[nt][j] = __shfl_sync(0xffffffffu, __uint_as_float(e << 23), 4 * (2 * t4 + j));
      const int rr = t.r0 + 8 * nt + 2 * t4 + j;
      pos[nt][j] = rr < t.rows ? t.seq.first + rr / a.group : -1;
      if (kGeneral && a.across && rr < t.rows) pos[nt][j] = max(find_row(a.kv, rr / a.group).pos, -1);
    }
  }
  if (kGeneral && a.across) {                // padding does not count: nobody reads its parts
    int least = INT32_MAX;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (pos[nt][j] >= 0) least = min(least, pos[nt][j]);
    t.pos_lo = __reduce_min_sync(0xffffffffu, least);
  }

  float acc[NT][D / 16][4];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int j = 0; j < D / 16; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[nt][j][e] = 0.0f;
  // per row: the running maximum m; per row and lane (its own keys): the maximum n and the sum
  float m[NT][2], n[NT][2], l[NT][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int j = 0; j < 2; ++j) m[nt][j] = n[nt][j] = -INFINITY, l[nt][j] = 0.0f;

  for (int i = 0; i < steps; ++i) {
    copy_wait<2>();                  // in flight: this step's values and the next one's keys
    __syncwarp();                    // every lane's copies of this step's keys are here
    const int number = first_key + i * kStep * kWarps, key = kGeneral ? number + t.gap : number, stage = i % kStages;
    const uint32_t src = ring + stage * kStageBytes;
    const uint32_t skip = skipped >> (2 * stage) & 3u;   // before the stage takes another step's keys

    float s[2][NT][4] = {};          // keys g, g + 8 of a half by rows 2 t4, + 1
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int c = 0; c < kC; ++c) {
        const uint4 w0 = lds128(src + u * Sm::kHalf + key_place<D>(g, 4 * c + t4));
        const uint4 w1 = lds128(src + u * Sm::kHalf + key_place<D>(g + 8, 4 * c + t4));
        const uint32_t x0[4] = {w0.x, w0.y, w0.z, w0.w}, x1[4] = {w1.x, w1.y, w1.z, w1.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t y0 = x0[k] ^ 0x80808080u, y1 = x1[k] ^ 0x80808080u;
          const uint32_t a0 = half_codes<0x4140>(y0), a2 = half_codes<0x4342>(y0);
          const uint32_t a1 = half_codes<0x4140>(y1), a3 = half_codes<0x4342>(y1);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) mma_16816(s[u][nt], a0, a1, a2, a3, qf[nt][4 * c + k]);
        }
      }

    const uint4 sc = lds128(scales + stage * kStageScales);
    const float coef[2] = {a.scale_log2 * __uint_as_float(sc.x), a.scale_log2 * __uint_as_float(sc.z)};
    const float lsv[2] = {lg2(__uint_as_float(sc.y)), lg2(__uint_as_float(sc.w))};
    const bool all = skip == 0 && key + kStep - 1 <= t.pos_lo &&
                     (a.window == 0 || key > t.pos_hi - a.window || (kGeneral && number + kStep <= a.sinks));
    uint32_t p[2][NT][2];
    float alpha[NT][2];
    bool moved = false;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float P[2][4];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float z[2][2], x[2][2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const float cu = coef[u] * qs[nt][j];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            z[u][e] = s[u][nt][2 * e + j] * cu;
            x[u][e] = z[u][e] + lsv[u];
          }
        }
        if (!all) {
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int k = key + 16 * u + 8 * e + g;
              if (k > pos[nt][j] || (a.window > 0 && k <= pos[nt][j] - a.window && !(kGeneral && k - t.gap < a.sinks)) || (skip >> u & 1))
                z[u][e] = x[u][e] = -INFINITY;
            }
        }
        float mx = fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[1][0], x[1][1]));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
        const float m1 = fmaxf(m[nt][j], mx), base = finite_max(m1);
        const float n1 = fmaxf(fmaxf(n[nt][j], fmaxf(z[0][0], z[0][1])), fmaxf(z[1][0], z[1][1]));
        const float nbase = finite_max(n1);
        alpha[nt][j] = ex2(m[nt][j] - base);
        moved = moved || m1 != m[nt][j];
        float sum = 0.0f;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            P[u][2 * e + j] = ex2(x[u][e] - base);
            sum += ex2(z[u][e] - nbase);
          }
        l[nt][j] = fmaf(l[nt][j], ex2(n[nt][j] - nbase), sum);
        m[nt][j] = m1;
        n[nt][j] = n1;
      }
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 2; ++e) p[u][nt][e] = transpose8(pack_half(P[u][2 * e], P[u][2 * e + 1]));
    }
    if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < D / 16; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[nt][j][e] *= alpha[nt][e & 1];
    }
    copy_wait<1>();                  // in flight: the next step's keys
    __syncwarp();                    // and this step's values
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      uint32_t vw[4][D / 32];        // tokens 2 t4, 2 t4 + 1, 2 t4 + 8, 2 t4 + 9, dimensions g D/8 ..
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t r = 2 * t4 + (k & 1) + 8 * (k >> 1), at = ring + (kStages + i % kValueStages) * kStageBytes + u * Sm::kHalf;
        if constexpr (D == 128) {
          const uint4 w = lds128(at + value_place<D>(r, g));
          vw[k][0] = w.x ^ 0x80808080u, vw[k][1] = w.y ^ 0x80808080u;
          vw[k][2] = w.z ^ 0x80808080u, vw[k][3] = w.w ^ 0x80808080u;
        } else {
          const uint2 w = lds64(at + value_place<D>(r, g >> 1) + (g & 1) * 8);
          vw[k][0] = w.x ^ 0x80808080u, vw[k][1] = w.y ^ 0x80808080u;
        }
      }
#pragma unroll
      for (int w = 0; w < D / 32; ++w) {
        const uint32_t lo0 = __byte_perm(vw[0][w], vw[1][w], 0x5140), hi0 = __byte_perm(vw[0][w], vw[1][w], 0x7362);
        const uint32_t lo1 = __byte_perm(vw[2][w], vw[3][w], 0x5140), hi1 = __byte_perm(vw[2][w], vw[3][w], 0x7362);
        const uint32_t a0 = half_codes<0x4140>(lo0), a1 = half_codes<0x4342>(lo0);
        const uint32_t a2 = half_codes<0x4140>(lo1), a3 = half_codes<0x4342>(lo1);
        const uint32_t b0 = half_codes<0x4140>(hi0), b1 = half_codes<0x4342>(hi0);
        const uint32_t b2 = half_codes<0x4140>(hi1), b3 = half_codes<0x4342>(hi1);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          mma_16816(acc[nt][2 * w], a0, a1, a2, a3, p[u][nt]);
          mma_16816(acc[nt][2 * w + 1], b0, b1, b2, b3, p[u][nt]);
        }
      }
    }
    __syncwarp();                    // the step has been read
    issue_values(i + 1);
    issue_keys(i + 2);
  }

  // join the lanes' sums and then the warps
  __shared__ float stat_sm[kWarps][kRows][3];
  copy_wait<0>();
  __syncthreads();                   // the ring becomes the warps' outputs
  float (*o_sm)[kRows][D + 4] = reinterpret_cast<float (*)[kRows][D + 4]>(smem);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float nn = n[nt][j];
#pragma unroll
      for (int o = 4; o < 32; o *= 2) nn = fmaxf(nn, __shfl_xor_sync(0xffffffffu, nn, o));
      float ll = l[nt][j] * ex2(n[nt][j] - finite_max(nn));
#pragma unroll
      for (int o = 4; o < 32; o *= 2) ll += __shfl_xor_sync(0xffffffffu, ll, o);
      const int row = 8 * nt + 2 * t4 + j;
      if (g == 0) stat_sm[warp][row][0] = m[nt][j], stat_sm[warp][row][1] = nn, stat_sm[warp][row][2] = ll;
      // dimensions g D/8 + 2 i, + 1 lie in accumulator i
#pragma unroll
      for (int i = 0; i < D / 16; i += 2)
        *reinterpret_cast<float4*>(&o_sm[warp][row][g * (D / 8) + 2 * i]) =
            make_float4(acc[nt][i][j], acc[nt][i][2 + j], acc[nt][i + 1][j], acc[nt][i + 1][2 + j]);
    }
  __syncthreads();
  constexpr int kPer = kRows * D / (32 * kWarps);            // dimensions of one row a thread
  const int row = threadIdx.x / (D / kPer), d0 = threadIdx.x % (D / kPer) * kPer;
  const int r = t.r0 + row;
  if (r >= t.rows) return;
  float mm = -INFINITY, nn = -INFINITY;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    mm = fmaxf(mm, stat_sm[w][row][0]);
    nn = fmaxf(nn, stat_sm[w][row][1]);
  }
  const float base = finite_max(mm), nbase = finite_max(nn);
  float o[kPer] = {}, ll = 0.0f;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    const float f = ex2(stat_sm[w][row][0] - base);
    ll = fmaf(stat_sm[w][row][2], ex2(stat_sm[w][row][1] - nbase), ll);
#pragma unroll
    for (int e = 0; e < kPer; e += 4) {
      const float4 v = *reinterpret_cast<const float4*>(&o_sm[w][row][d0 + e]);
      o[e] = fmaf(v.x, f, o[e]), o[e + 1] = fmaf(v.y, f, o[e + 1]);
      o[e + 2] = fmaf(v.z, f, o[e + 2]), o[e + 3] = fmaf(v.w, f, o[e + 3]);
    }
  }
  if (ns <= 1 && !(kGeneral && a.keep_parts)) {
    const float inv = out_factor(ll, mm - nbase);
    uint16_t* out = a.O + (t.seq.row0 + r / a.group) * a.ldo + static_cast<int64_t>(h * a.group + r % a.group) * D + d0;
#pragma unroll
    for (int e = 0; e < kPer; e += 4)
      *reinterpret_cast<uint2*>(out + e) =
          make_uint2(pack_bf16(o[e] * inv, o[e + 1] * inv), pack_bf16(o[e + 2] * inv, o[e + 3] * inv));
    return;
  }
  const int64_t slot = ((((static_cast<int64_t>(b) * a.kv.heads + h) * a.row_tiles + rt) * a.splits + split) * kRows) + row;
#pragma unroll
  for (int e = 0; e < kPer; e += 4)
    *reinterpret_cast<float4*>(a.part + slot * D + d0 + e) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
  if (d0 == 0) *reinterpret_cast<float4*>(a.part_stat + slot * 4) = make_float4(mm, nn, ll, 0.0f);
}

template <int D, int NT, bool kGeneral>
__global__ void __launch_bounds__(32 * kWarps, NT == 1 ? kPerSm : kPerSm / 2) kv_attn_split_kernel(AttnArgs a) {
  split_block<D, NT, kGeneral>(a);
  if (kGeneral && a.keep_parts && blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0) finish_behind();
}

// Joins the splits of one row per thread block: the warps take interleaved splits, each relative to its own
// maxima, and are then added in order.
constexpr int kJoinWarps = 8;
template <int D, bool kGeneral>
__global__ void __launch_bounds__(32 * kJoinWarps) kv_attn_join_kernel(AttnArgs a) {
  constexpr int kPer = D / 32;
  const int h = blockIdx.y % a.kv.heads, rt = blockIdx.y / a.kv.heads, b = blockIdx.z, row = blockIdx.x;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  Tile t;
  const bool in = attn_tile<kGeneral>(a, b, rt, t);
  asm volatile("griddepcontrol.wait;" ::: "memory");         // the parts are there
  const int ns = in ? tile_splits(a, t) : 0, r = t.r0 + row;
  if (ns <= 1 || r >= t.rows) return;
  const int64_t slot0 = (((static_cast<int64_t>(b) * a.kv.heads + h) * a.row_tiles + rt) * a.splits) * a.tile_rows + row;
  float m = -INFINITY, n = -INFINITY, acc[kPer] = {}, l = 0.0f;
#pragma unroll 4
  for (int s = warp; s < ns; s += warps) {
    const int64_t slot = slot0 + static_cast<int64_t>(s) * a.tile_rows;
    const float4 v = *reinterpret_cast<const float4*>(a.part_stat + 4 * slot);
    const float* p = a.part + slot * D + lane * kPer;
    const float m1 = fmaxf(m, v.x), n1 = fmaxf(n, v.y);
    const float keep = ex2(m - finite_max(m1)), f = ex2(v.x - finite_max(m1));
    l = fmaf(l, ex2(n - finite_max(n1)), v.z * ex2(v.y - finite_max(n1)));
#pragma unroll
    for (int e = 0; e < kPer; e += 2) {
      const float2 x = *reinterpret_cast<const float2*>(p + e);
      acc[e] = fmaf(acc[e], keep, x.x * f), acc[e + 1] = fmaf(acc[e + 1], keep, x.y * f);
    }
    m = m1;
    n = n1;
  }
  __shared__ float part[kJoinWarps][D + 3];
#pragma unroll
  for (int e = 0; e < kPer; ++e) part[warp][lane * kPer + e] = acc[e];
  if (lane == 0) part[warp][D] = m, part[warp][D + 1] = n, part[warp][D + 2] = l;
  __syncthreads();
  if (threadIdx.x >= D / 2) return;
  m = n = -INFINITY;
  for (int w = 0; w < warps; ++w) m = fmaxf(m, part[w][D]), n = fmaxf(n, part[w][D + 1]);
  const float base = finite_max(m), nbase = finite_max(n);
  float o0 = 0.0f, o1 = 0.0f;
  l = 0.0f;
  for (int w = 0; w < warps; ++w) {
    const float f = ex2(part[w][D] - base);
    o0 = fmaf(part[w][2 * threadIdx.x], f, o0);
    o1 = fmaf(part[w][2 * threadIdx.x + 1], f, o1);
    l = fmaf(part[w][D + 2], ex2(part[w][D + 1] - nbase), l);
  }
  const float inv = out_factor(l, m - nbase);
  uint16_t* out = a.O + (t.seq.row0 + r / a.group) * a.ldo + static_cast<int64_t>(h * a.group + r % a.group) * D;
  reinterpret_cast<uint32_t*>(out)[threadIdx.x] = pack_bf16(o0 * inv, o1 * inv);
}

// Joins the parts of the rows' own keys (`a`) with those of the prefix (`p`), in that order: kShares warps have one row of the
// batch and head, each a share of its parts, a warp's lanes the statistics of 32 parts at a time and the row's dimensions.
// Many parts, which few rows have, in four shares: 2 sequences behind 16000 tokens (64 parts and their own) 23.8 -> 20.4
// us, behind 32000 28.9 -> 25.2, 4 x 2 tokens of 16 heads and one for keys behind 30000 28.2 -> 21.6.
constexpr int kJoinAhead = 8;
template <int D, int kShares>
__global__ void __launch_bounds__(32 * kJoinWarps) kv_attn_join_shared_kernel(AttnArgs a, AttnArgs p) {
  constexpr int kPer = D / 32;
  const int lane = threadIdx.x & 31, h = blockIdx.y;
  constexpr int kRows = kJoinWarps / kShares;
  const int warp = threadIdx.x >> 5, share = warp % kShares;
  const int64_t rr0 = static_cast<int64_t>(blockIdx.x) * kRows + warp / kShares, rows = a.kv.rows * a.group;
  const bool none = rr0 >= rows;
  const int64_t rr = none ? rows - 1 : rr0;
  const int64_t token = rr / a.group;
  const int head = static_cast<int>(rr - token * a.group);
  const RowPlace at = find_rows(a.kv, token);
  // the row's own keys: its tile of the sequence's rows, and the parts that tile was cut into
  int own = 0, tile = 0, row = 0;
  if (at.seq >= 0 && at.pos >= 0) {
    const int r = static_cast<int>(token - __ldg(a.kv.row_start + at.seq)) * a.group + head;
    tile = r / a.tile_rows, row = r - tile * a.tile_rows;
    Tile t;
    if (attn_tile<true>(a, at.seq, tile, t)) own = tile_splits(a, t);
  }
  const int all = at.seq >= 0 && at.pos >= 0 ? own + (p.prefix - 1) / p.chunk + 1 : 0;      // rows of padding see nothing
  const int64_t slot0 = ((static_cast<int64_t>(max(at.seq, 0)) * a.kv.heads + h) * a.row_tiles + tile) * a.splits * a.tile_rows + row;
  const int64_t slot1 = (static_cast<int64_t>(h) * p.row_tiles + rr / p.tile_rows) * p.splits * p.tile_rows + rr % p.tile_rows;
  auto slot_of = [&](int s) {
    return s < own ? slot0 + static_cast<int64_t>(s) * a.tile_rows : slot1 + static_cast<int64_t>(s - own) * p.tile_rows;
  };
  using Vec = typename std::conditional<kPer == 4, float4, float2>::type;
  union Dims {
    Vec v;
    float f[kPer];
  };
  asm volatile("griddepcontrol.wait;" ::: "memory");         // the parts are there
  const bool skip = none || at.seq < 0;
  if (kShares == 1 && skip) return;
  const int per = (all + kShares - 1) / kShares, end = skip ? 0 : min(all, (share + 1) * per);
  float m = -INFINITY, n = -INFINITY, l = 0.0f, acc[kPer] = {};
  for (int s0 = share * per; s0 < end; s0 += 32) {
    const int count = min(end - s0, 32);
    float4 v = make_float4(-INFINITY, -INFINITY, 0.0f, 0.0f);
    if (lane < count) v = __ldcg(reinterpret_cast<const float4*>((s0 + lane < own ? a : p).part_stat + slot_of(s0 + lane) * 4));
    float f = 0.0f;
    for (int u0 = 0; u0 < count; u0 += kJoinAhead) {
      Dims x[kJoinAhead];
#pragma unroll
      for (int u = 0; u < kJoinAhead; ++u) {
        const int s = s0 + min(u0 + u, count - 1);
        x[u].v = __ldcg(reinterpret_cast<const Vec*>((s < own ? a : p).part + slot_of(s) * D) + lane);
      }
      if (u0 == 0) {
        float m1 = v.x, n1 = v.y;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
          m1 = fmaxf(m1, __shfl_xor_sync(0xffffffffu, m1, o));
          n1 = fmaxf(n1, __shfl_xor_sync(0xffffffffu, n1, o));
        }
        m1 = fmaxf(m, m1), n1 = fmaxf(n, n1);
        const float base = finite_max(m1), nbase = finite_max(n1), keep = ex2(m - base);
        f = ex2(v.x - base);
        l *= ex2(n - nbase);
        float sum = v.z * ex2(v.y - nbase);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        l += sum;
#pragma unroll
        for (int e = 0; e < kPer; ++e) acc[e] *= keep;
        m = m1, n = n1;
      }
#pragma unroll
      for (int u = 0; u < kJoinAhead; ++u) {
        const float fu = __shfl_sync(0xffffffffu, f, (u0 + u) & 31);
        if (u0 + u < count)
#pragma unroll
          for (int e = 0; e < kPer; ++e) acc[e] = fmaf(x[u].f[e], fu, acc[e]);
      }
    }
  }
  if constexpr (kShares > 1) {
    __shared__ float4 stat[kJoinWarps];
    __shared__ float part[kJoinWarps][D];
    if (lane == 0) stat[warp] = make_float4(m, n, l, 0.0f);
#pragma unroll
    for (int e = 0; e < kPer; ++e) part[warp][lane * kPer + e] = acc[e];
    __syncthreads();
    if (share != 0 || skip) return;
#pragma unroll
    for (int w = 1; w < kShares; ++w) m = fmaxf(m, stat[warp + w].x), n = fmaxf(n, stat[warp + w].y);
    const float base = finite_max(m), nbase = finite_max(n);
    l = 0.0f;
#pragma unroll
    for (int e = 0; e < kPer; ++e) acc[e] = 0.0f;
#pragma unroll
    for (int w = 0; w < kShares; ++w) {
      const float4 v = stat[warp + w];
      const float f = ex2(v.x - base);
      l = fmaf(v.z, ex2(v.y - nbase), l);
#pragma unroll
      for (int e = 0; e < kPer; ++e) acc[e] = fmaf(part[warp + w][lane * kPer + e], f, acc[e]);
    }
  }
  const float inv = out_factor(l, m - finite_max(n));
  uint32_t* out = reinterpret_cast<uint32_t*>(a.O + token * a.ldo + static_cast<int64_t>(h * a.group + head) * D) + lane * (kPer / 2);
  if constexpr (kPer == 4) {
    *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16(acc[0] * inv, acc[1] * inv), pack_bf16(acc[2] * inv, acc[3] * inv));
  } else {
    *out = pack_bf16(acc[0] * inv, acc[1] * inv);
  }
}

template <int D, int NT, bool kGeneral>
cudaError_t launch_split(const AttnArgs& a, cudaStream_t stream) {
  using Sm = SplitSmem<D, NT>;
  const dim3 grid(a.kv.heads * a.row_tiles, attn_grid_seqs(a), a.splits);
  static bool smem_set[kMaxDevices];
  const cudaError_t e = ensure_smem_attr(reinterpret_cast<const void*>(kv_attn_split_kernel<D, NT, kGeneral>), Sm::kBytes, smem_set);
  if (e != cudaSuccess) return e;
  return launch_lined_up(kv_attn_split_kernel<D, NT, kGeneral>, grid, 32 * kWarps, Sm::kBytes, a.behind, stream, a);
}

template <int D, bool kGeneral>
cudaError_t launch_parts(const AttnArgs& a, cudaStream_t stream) {
  return a.tile_rows == kPromptRows ? launch_kv_prompt(a, stream)
         : a.tile_rows == 8         ? launch_split<D, 1, kGeneral>(a, stream)
                                    : launch_split<D, 2, kGeneral>(a, stream);
}

template <int D, bool kGeneral>
cudaError_t launch(const AttnArgs& a, cudaStream_t stream) {
  const cudaError_t e = launch_parts<D, kGeneral>(a, stream);
  if (e != cudaSuccess || a.splits <= 1) return e;
  const int threads = 32 * (a.splits > 32 ? kJoinWarps : a.splits > 8 ? kJoinWarps / 2 : 2);   // at least D / 2
  return launch_lined_up(kv_attn_join_kernel<D, kGeneral>, dim3(a.tile_rows, a.kv.heads * a.row_tiles, a.kv.n_seqs), threads,
                         0, 1, stream, a);
}

template <int D>
cudaError_t launch_shared(const AttnArgs& p, const AttnArgs& a, cudaStream_t stream) {
  cudaError_t e = launch_parts<D, true>(p, stream);
  if (e == cudaSuccess) e = launch_parts<D, true>(a, stream);
  if (e != cudaSuccess) return e;
  const int shares = a.splits + p.splits > 24 ? 4 : 1, per = kJoinWarps / shares;
  const dim3 grid(static_cast<unsigned>((a.kv.rows * a.group + per - 1) / per), a.kv.heads);
  return launch_lined_up(shares == 4 ? kv_attn_join_shared_kernel<D, 4> : kv_attn_join_shared_kernel<D, 1>, grid, 32 * kJoinWarps, 0,
                         1, stream, a, p);
}

}  // namespace

// Keys of a piece of 16- or 256-row tiles whose blocks come in waves of `slots`, and the call's time for it.  A block takes
// about 6.5 us and 13.1 ns a key (16 rows, two blocks an SM) or 7 us and 14.1 ns (256 rows), a launch 3 us and the join one
// more and its bytes; all are fitted to windows of 100 to 4000 keys and 4 sinks, 20 to 128 rows of 1, 16 and 64 sequences
// with 8 heads.
struct Pieces {
  int64_t chunk;
  double ns;
};
Pieces plan_pieces(const AttnArgs& a, int64_t keys, int tile_rows, int sms) {
  const bool prompt = tile_rows == kPromptRows;
  const int64_t rows = static_cast<int64_t>(a.kv.max_rows) * a.group, unit = 128, slots = prompt ? sms : sms * (kPerSm / 2);
  const int64_t tiles = static_cast<int64_t>(a.kv.n_seqs) * a.kv.heads * ((rows + tile_rows - 1) / tile_rows);
  Pieces best{(keys + unit) / unit * unit, 0.0};
  for (int64_t pieces = 1; pieces <= 64; ++pieces) {
    const int64_t chunk = ((keys + pieces - 1) / pieces + unit - 1) / unit * unit, blocks = tiles * pieces;
    double ns = 3000.0 + static_cast<double>((blocks + slots - 1) / slots) * (prompt ? 7000.0 + 14.1 * chunk : 6500.0 + 13.1 * chunk);
    if (pieces > 1) ns += 4000.0 + 2.0 * blocks * tile_rows * a.kv.d * sizeof(float) / 6800.0;
    if (pieces == 1) best.ns = ns;
    else if (ns < best.ns) best = {chunk, ns};
    if (chunk <= unit || blocks > 4 * slots) break;
  }
  return best;
}

// Up to 16 rows per sequence and key/value head the keys' bytes bound the call, and 8- or 16-row tiles of
// the warp-level kernel stream them; above, the 256-row tiles of the prompt kernel convert a key once for
// all of them.  Both sides of the limit, 32 / 8 heads, 4000 tokens: 12 and 16 rows, 16 sequences, 48 and 49
// us (floor 19); 20, 32 and 64 rows in 256-row tiles 91, 92 and 95 us, in 16-row tiles 74, 77 and 121; with
// 64 sequences 226, 226 and 228 against 220, 222 and 414 (floor 78).  The keys of a tile are cut so that
// the tiles of the largest batch the bounds allow fill the machine about twice, or four times where there
// are many tiles (many sequences, whose lengths differ), in pieces of at least 128 keys (a step of each
// warp; prompt kernel: 512).  A piece costs about 3 us beside its keys, the start and the join, so tiles
// that fill the machine by themselves are cut into 4096 keys or more (8-row tiles that fill it less than
// twice, whose last wave is far from full: 2304), and up to 1024 keys stay whole where tiles fill half of
// it.  Measured, 8 key/value heads of 128: two sequences of 131002 tokens 88 us (79 for the bytes at the
// copy rate; cut twice as fine 92), 64 ragged sequences up to 8101 tokens 83 us (66; in five pieces at
// most, in two 90, whole 116, in sixteen 88), one of 1030 tokens 6.1 us, 64 of 1001 tokens 28 us (cut in
// four 36), 100 of 4001 tokens 137 us (whole 151), 200 of 2501 tokens 162 us (cut in two 171); 16 x 5 rows
// of 40 full heads, window 2048, 41 us (30; cut in two 48).  Where all pieces are of one length they come
// in one wave: one sequence of 32001 tokens 20 us (two waves 24, 10 for its bytes), 4 drafted tokens behind
// 32000 24 us (31), 12 windows of 1000 tokens 10.6 us (12).  The host knows bounds, not lengths: that two
// sequences are about equally long is a guess (one of 32001 tokens beside one of 100: 25 us).
//
// Calls through sinks or behind a prefix (kv_attn's own calls keep their plans, and so their bits) choose between 16- and
// 256-row tiles up to 128 rows, and the pieces of both, by plan_pieces: 32 rows of 1, 16 and 64 sequences with 500 keys
// take 12, 18.5 and 59 us in 16-row tiles and 16, 18.5 and 67 in 256-row tiles, with 4000 keys 16, 62 and 237 and 18.5, 66
// and 245 (kv_attn's plans: 18.5, 51 and 67, 19.5, 106 and 245); 64 rows with 500 keys 14, 33 and 107 and 16, 18.5 and 67.
void plan_attn(AttnArgs& a, int sms) {
  const int64_t rows = static_cast<int64_t>(a.kv.max_rows) * a.group;
  const bool general = attn_general(a);
  a.tile_rows = rows <= 8 ? 8 : rows <= 16 ? 16 : kPromptRows;
  a.sink_pad = static_cast<int>((static_cast<int64_t>(a.sinks) + 15) & ~15);
  int64_t keys = a.kv.max_len > a.first ? a.kv.max_len - a.first : 0;
  // the keys that a tile of `tile_rows` rows may see
  auto in_window = [&](int tile_rows) {
    const int64_t tokens = general ? (tile_rows + a.group - 2) / a.group + 1 : tile_rows;
    const int64_t w = static_cast<int64_t>(a.window) + tokens + kKeyAlign + a.sink_pad;
    return a.window > 0 && w < keys ? w : keys;
  };
  Pieces cut{0, 0.0};
  if (general && rows > 8) {
    cut = plan_pieces(a, in_window(a.tile_rows), a.tile_rows, sms);
    if (rows > 16 && rows <= 128) {
      const Pieces small = plan_pieces(a, in_window(16), 16, sms);
      if (small.ns < cut.ns) cut = small, a.tile_rows = 16;
    }
  }
  const bool prompt = a.tile_rows == kPromptRows;
  a.row_tiles = static_cast<int>((rows + a.tile_rows - 1) / a.tile_rows);
  if (a.row_tiles < 1) a.row_tiles = 1;
  keys = in_window(a.tile_rows);
  const int64_t tiles = static_cast<int64_t>(a.kv.n_seqs) * a.kv.heads * a.row_tiles;
  const int64_t at_once = static_cast<int64_t>(sms) * (prompt ? 1 : a.tile_rows == 8 ? kPerSm : kPerSm / 2);
  const int64_t want = at_once * (prompt || 4 * tiles < at_once ? 2 : 4);
  const int64_t unit = 128;
  int64_t least = prompt ? 512 : 128;
  if (!prompt && tiles >= at_once) least = a.tile_rows == 8 && tiles < 2 * at_once ? 2304 : 4096;
  else if (!prompt && 2 * tiles >= at_once && keys <= 1024) least = 1024;
  int64_t chunk = (keys * tiles + want - 1) / want;
  // one or two sequences, or windows shorter than the sequences: pieces of equal length, so one wave of them
  if (!prompt && 2 * tiles <= at_once && (a.kv.n_seqs <= 2 || 2 * keys <= a.kv.max_len))
    chunk = (keys + at_once / tiles - 1) / (at_once / tiles);
  chunk = (chunk + unit - 1) / unit * unit;
  if (chunk < least) chunk = least;
  if (cut.chunk > 0) chunk = cut.chunk;
  const int64_t whole = (keys + unit) / unit * unit;         // with many tiles keys * tiles / want passes 32 bits
  if (chunk > whole || (prompt && cut.chunk == 0 && tiles >= want)) chunk = whole;
  a.chunk = static_cast<int>(chunk);
  const int64_t splits = (keys + chunk - 1) / chunk;
  a.splits = static_cast<int>(splits < 1 ? 1 : splits);
}

// Asked of the bound on one sequence's rows, whatever the others have: 63 single tokens beside one sequence of 32 rows, 4
// heads a key head, behind 16000 tokens 79 us, beside one of 33 rows, each over the prefix alone, 918.
bool shared_together(const AttnArgs& a) {
  return a.kv.n_seqs > 1 && static_cast<int64_t>(a.kv.max_rows) * a.group <= 128;
}

// A planned call in which every sequence goes over prefix and own keys: 8-row tiles take 9 us and their bytes at 5200 GB/s,
// the others what plan_pieces says.
double apart_ns(const AttnArgs& a, int sms) {
  const double keys = a.kv.max_len;
  if (a.tile_rows == 8) return 9000.0 + a.kv.n_seqs * keys * a.kv.heads * 2.0 * a.kv.d / 5200.0;
  return plan_pieces(a, a.kv.max_len, a.tile_rows, sms).ns;
}

// The bounds stand for what the sequences hold, and the constants, as plan_pieces', are of 8 heads of 128.  What own keys
// might take makes the prefix's pieces longer: 64 single tokens behind 16000 with up to 501 of their own 38 us under their
// own bound, 79 under 1.25 times it, 264 (one piece, a block a head) from twice it on; 16 x 5 rows behind 2000 27, 27 and 39.
// At most one wave of pieces: a piece costs its start and its join whatever its length.  Blocks of the prompt kernel have
// an SM to themselves, and the sequences' own keys (`own`, planned), which run beside them, what is left and then all: a
// piece takes 9 us and 2 us a tile of 128 keys; own keys, of an SM, 0.75 us a block and three quarters of their bound's
// bytes at the copy rate in 8-row tiles, 3.25 us and 6.5 ns a key in 16-row tiles, 7 us and 14.1 ns in 256-row tiles.  64 rows
// of 32 heads, 8 of them for keys, behind 16000 tokens, 500 of their own: 18 pieces 50 us, 15 41, 13 42, 10 48; 16 x 5
// rows of 40 heads behind 2000 tokens: three pieces 35 us, two 32, one 45.  Returns the call's time with launches and
// join, about 8 us and the parts' bytes.
double plan_prefix(AttnArgs& a, const AttnArgs& own, int sms) {
  const int64_t rows = a.kv.rows * a.group;
  a.tile_rows = rows <= 8 ? 8 : rows <= 32 ? 16 : kPromptRows;      // 48 rows behind 16000: 39 us in 16-row tiles, 64 in 256 34
  const bool prompt = a.tile_rows == kPromptRows;
  a.row_tiles = static_cast<int>((rows + a.tile_rows - 1) / a.tile_rows);
  if (a.row_tiles < 1) a.row_tiles = 1;
  const int64_t tiles = static_cast<int64_t>(a.kv.heads) * a.row_tiles;
  const int64_t at_once = static_cast<int64_t>(sms) * (prompt ? 1 : a.tile_rows == 8 ? kPerSm : kPerSm / 2);
  const int64_t most = tiles < at_once ? at_once / tiles : 1, unit = 128;
  auto chunk_of = [&](int64_t pieces) { return ((a.prefix + pieces - 1) / pieces + unit - 1) / unit * unit; };
  const double copy_rate = 6800.0;           // bytes a nanosecond, the machine
  const double keys = a.kv.max_len > a.prefix ? a.kv.max_len - a.prefix : 0, key_bytes = 2.0 * a.kv.d;
  const double own_ns = static_cast<double>(a.kv.n_seqs) * a.kv.heads * own.row_tiles *
                        (own.tile_rows == 8 ? 750.0 + 0.75 * keys * key_bytes / copy_rate * sms
                                            : own.tile_rows == 16 ? 3250.0 + 6.5 * keys : 7000.0 + 14.1 * keys);
  int64_t chunk = chunk_of(most);
  double best = 0.0;
  if (prompt) {
    for (int64_t pieces = most; pieces >= 1; --pieces) {
      const int64_t c = chunk_of(pieces), used = (a.prefix + c - 1) / c, waves = (used * tiles + sms - 1) / sms;
      const double mine = waves * (9000.0 + 2000.0 / unit * c), left = own_ns - mine * (sms * waves - used * tiles) / waves;
      const double all = mine + (left > 0.0 ? left / sms : 0.0);
      if (pieces == most || all < best) best = all, chunk = c;
      if (mine > best) break;
    }
  } else {
    const double bytes = a.prefix * key_bytes * a.kv.heads / 5200.0;
    best = a.tile_rows == 8 ? 4000.0 : 6500.0 + 13.1 * chunk;
    best = (best > bytes + 4000.0 ? best : bytes + 4000.0) + own_ns / sms;
  }
  a.chunk = static_cast<int>(chunk);
  a.splits = static_cast<int>((a.prefix + chunk - 1) / chunk);
  return best + 8000.0 + static_cast<double>(rows) * a.kv.heads * (a.splits + own.splits) * a.kv.d * sizeof(float) / copy_rate;
}

cudaError_t launch_kv_attn(const AttnArgs& a, cudaStream_t stream) {
  if (attn_general(a)) return a.kv.d == 128 ? launch<128, true>(a, stream) : launch<64, true>(a, stream);
  return a.kv.d == 128 ? launch<128, false>(a, stream) : launch<64, false>(a, stream);
}

cudaError_t launch_kv_attn_shared(const AttnArgs& prefix, const AttnArgs& own, cudaStream_t stream) {
  return own.kv.d == 128 ? launch_shared<128>(prefix, own, stream) : launch_shared<64>(prefix, own, stream);
}

}  // namespace lrqat
