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
template <int D, int NT>
__global__ void __launch_bounds__(32 * kWarps, NT == 1 ? kPerSm : kPerSm / 2) kv_attn_split_kernel(AttnArgs a) {
  using Sm = SplitSmem<D, NT>;
  constexpr int kC = D / 64;         // 64-dimension pieces of a token
  constexpr int kRows = 8 * NT;
  extern __shared__ __align__(16) uint8_t smem[];
  const int h = blockIdx.x % a.kv.heads, rt = blockIdx.x / a.kv.heads, b = blockIdx.y;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  Tile t;
  if (!attn_tile(a, b, rt, t)) return;
  // Whole pieces first, every tile's shorter one (or its piece number a.splits - 1) in the end, where it fills
  // gaps: 20 ragged sequences of up to 5000 tokens with 40 heads 103 -> 97 us, 90 of up to 3000 with 8 heads
  // 65 -> 60, 64 of up to 8100 no faster (82 -> 83).
  const int ns = tile_splits(a, t);
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
  auto block_of = [&](int key) { return key < k1 ? __ldg(table + (key >> a.kv.block_log2)) : -2; };
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
          off[u] = ((at << a.kv.block_log2) + ((key + 16 * u) & in_block)) * D + lane * 16;
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
    }
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
    const int key = first_key + i * kStep * kWarps, stage = i % kStages;
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
    const bool all = skip == 0 && key + kStep - 1 <= t.pos_lo && (a.window == 0 || key > t.pos_hi - a.window);
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
              if (k > pos[nt][j] || (a.window > 0 && k <= pos[nt][j] - a.window) || (skip >> u & 1))
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
  if (ns <= 1) {
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

// Joins the splits of one row per thread block: the warps take interleaved splits, each relative to its own
// maxima, and are then added in order.
constexpr int kJoinWarps = 8;
template <int D>
__global__ void __launch_bounds__(32 * kJoinWarps) kv_attn_join_kernel(AttnArgs a) {
  constexpr int kPer = D / 32;
  const int h = blockIdx.y % a.kv.heads, rt = blockIdx.y / a.kv.heads, b = blockIdx.z, row = blockIdx.x;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  Tile t;
  const bool in = attn_tile(a, b, rt, t);
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

template <int D, int NT>
cudaError_t launch_split(const AttnArgs& a, cudaStream_t stream) {
  using Sm = SplitSmem<D, NT>;
  const dim3 grid(a.kv.heads * a.row_tiles, a.kv.n_seqs, a.splits);
  static bool smem_set[kMaxDevices];
  const cudaError_t e = ensure_smem_attr(reinterpret_cast<const void*>(kv_attn_split_kernel<D, NT>), Sm::kBytes, smem_set);
  if (e != cudaSuccess) return e;
  kv_attn_split_kernel<D, NT><<<grid, 32 * kWarps, Sm::kBytes, stream>>>(a);
  return cudaGetLastError();
}

template <int D>
cudaError_t launch(const AttnArgs& a, cudaStream_t stream) {
  const cudaError_t e = a.tile_rows == kPromptRows ? launch_kv_prompt(a, stream)
                        : a.tile_rows == 8         ? launch_split<D, 1>(a, stream)
                                                   : launch_split<D, 2>(a, stream);
  if (e != cudaSuccess || a.splits <= 1) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(a.tile_rows, a.kv.heads * a.row_tiles, a.kv.n_seqs);
  cfg.blockDim = dim3(32 * (a.splits > 32 ? kJoinWarps : a.splits > 8 ? kJoinWarps / 2 : 2));   // at least D / 2 threads
  cfg.stream = stream;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;   // its blocks line up behind the last splits
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kv_attn_join_kernel<D>, a);
}

}  // namespace

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
void plan_attn(AttnArgs& a, int sms) {
  const int64_t rows = static_cast<int64_t>(a.kv.max_rows) * a.group;
  a.tile_rows = rows <= 8 ? 8 : rows <= 16 ? 16 : kPromptRows;
  const bool prompt = a.tile_rows == kPromptRows;
  a.row_tiles = static_cast<int>((rows + a.tile_rows - 1) / a.tile_rows);
  if (a.row_tiles < 1) a.row_tiles = 1;
  int64_t keys = a.kv.max_len;
  if (a.window > 0) {
    const int64_t w = static_cast<int64_t>(a.window) + a.tile_rows + kKeyAlign;
    keys = keys < w ? keys : w;
  }
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
  const int64_t whole = (keys + unit) / unit * unit;         // with many tiles keys * tiles / want passes 32 bits
  if (chunk > whole || (prompt && tiles >= want)) chunk = whole;
  a.chunk = static_cast<int>(chunk);
  const int64_t splits = (keys + chunk - 1) / chunk;
  a.splits = static_cast<int>(splits < 1 ? 1 : splits);
}

cudaError_t launch_kv_attn(const AttnArgs& a, cudaStream_t stream) {
  return a.kv.d == 128 ? launch<128>(a, stream) : launch<64>(a, stream);
}

}  // namespace lrqat
