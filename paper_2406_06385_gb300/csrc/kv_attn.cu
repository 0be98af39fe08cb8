// Attention of the newest tokens of each sequence over the paged 8-bit cache.
//
// With s_k, s_v the scales of a cache block and c_k, c_v its codes, query row q at position p:
//   z_j = scale s_k (q . c_k,j)   for the keys j <= p (and j > p - window),
//   o = sum_j e^{z_j} s_v c_v,j / sum_j e^{z_j},   0 for a row that sees no key.
// The kernels fold s_v into the exponent: with z'_j = z_j log2(e) + log2(s_v) and m their running
// maximum, P_j = 2^{z'_j - m} lies in [0, 1] and is what a key contributes to o, whatever the scales
// of the blocks are.  The denominator, the sum of P_j / s_v, is kept relative to a running
// maximum n of its own, that of z_j log2(e): scales of one sequence may lie as far apart as fp32 reaches.
// So P fits 11-bit half precision and the codes (|c| <= 128) are exact in it; a row of q is first divided by the power of two of its largest
// magnitude, which half precision also holds (exact but for elements below 2^-14 of the largest).
// Scores, maxima, sums and outputs are 32-bit.
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "serve.cuh"

namespace lrqat {
namespace {

constexpr int kRows = 16;          // (token, head) rows of one tile: the M of mma.m16n8k16
constexpr int kWarps = 4;
constexpr int kStep = 16;          // keys of one step of a warp

__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
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

__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.0f : m; }
// 2^up / l, 0 for a row that saw no key (l = 0); up = m - n is at most log2 of the largest scale.
__device__ __forceinline__ float out_factor(float l, float up) {
  const float half = ex2(0.5f * up);                   // 2^up itself may be subnormal
  return l == 0.0f ? 0.0f : half / l * half;
}

// The tile of kRows rows `rt` of (sequence, key/value head): row i is token (16 rt + i) / group of
// the sequence's rows and query head (16 rt + i) % group of the head's group.
struct Tile {
  SeqRows seq;
  int rows;            // rows of the sequence and head, all tiles
  int r0;              // first row of this tile
  int pos_lo, pos_hi;  // positions of the tile's first and last row
  int lo, hi;          // keys [lo, hi) that some row may see; lo a multiple of 16
};
__device__ __forceinline__ bool attn_tile(const AttnArgs& a, int b, int rt, Tile& t) {
  if (!seq_rows(a.kv, b, t.seq)) return false;
  t.rows = t.seq.n * a.group;
  t.r0 = rt * kRows;
  if (t.r0 >= t.rows) return false;
  const int last = min(t.r0 + kRows, t.rows) - 1;
  t.pos_lo = t.seq.first + t.r0 / a.group;
  t.pos_hi = t.seq.first + last / a.group;
  t.hi = max(t.pos_hi + 1, 0);
  t.lo = a.window > 0 ? max(t.pos_lo - a.window + 1, 0) & ~(kStep - 1) : 0;
  return true;
}

__device__ __forceinline__ int tile_splits(const AttnArgs& a, const Tile& t) {
  return t.hi > t.lo ? (t.hi - t.lo + a.chunk - 1) / a.chunk : 0;
}

// One thread block per (split, head and row tile, sequence).  A warp takes every fourth step of 16
// keys and keeps its own maximum, sum and outputs; the warps join at the end.  Keys and values go
// from global memory straight into the fragments of the matrix instructions: the order of the
// head's dimensions inside a product is free, so each lane takes 16 consecutive bytes of a token.
template <int D>
__global__ void __launch_bounds__(32 * kWarps) kv_attn_split_kernel(AttnArgs a) {
  constexpr int kC = D / 64;         // 64-dimension pieces of a token
  const int split = blockIdx.x, h = blockIdx.y % a.kv.heads, rt = blockIdx.y / a.kv.heads, b = blockIdx.z;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
  Tile t;
  if (!attn_tile(a, b, rt, t)) return;
  const int ns = tile_splits(a, t);
  if (split > 0 && split >= ns) return;
  const int k0 = t.lo + split * a.chunk, k1 = min(t.hi, k0 + a.chunk);

  // rows g and g + 8 of the tile: fragments of q, its power of two, positions
  uint32_t qf[4 * kC][4];
  float qs[2];
  int pos[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = t.r0 + g + 8 * i;
    const int tok = r / a.group;
    const bool in = r < t.rows;
    pos[i] = in ? t.seq.first + tok : -1;
    const uint16_t* q = a.Q + (t.seq.row0 + tok) * a.ldq + static_cast<int64_t>(h * a.group + r % a.group) * D;
    float x[kC][16], top = 0.0f;
#pragma unroll
    for (int c = 0; c < kC; ++c) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        float v[8];
        unpack8(in ? __ldg(reinterpret_cast<const uint4*>(q + 64 * c + 16 * t4) + u) : make_uint4(0u, 0u, 0u, 0u), v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[c][8 * u + e] = v[e];
          top = fmaxf(top, fabsf(v[e]));
        }
      }
    }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const uint32_t e = min(max(__float_as_uint(top) >> 23, 1u), 253u);   // exponent of a normal power of two
    qs[i] = __uint_as_float(e << 23);
    const float inv = __uint_as_float((254u - e) << 23);
#pragma unroll
    for (int c = 0; c < kC; ++c)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        qf[4 * c + u][i] = pack_half(x[c][4 * u] * inv, x[c][4 * u + 1] * inv);
        qf[4 * c + u][2 + i] = pack_half(x[c][4 * u + 2] * inv, x[c][4 * u + 3] * inv);
      }
  }

  float acc[D / 8][4];
#pragma unroll
  for (int j = 0; j < D / 8; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[j][e] = 0.0f;
  float m[2] = {-INFINITY, -INFINITY}, n[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};

  for (int key = k0 + kStep * warp; key < k1; key += kStep * kWarps) {
    const int blk = seq_block(a.kv, b, key);
    if (blk < 0) continue;
    const int64_t at = static_cast<int64_t>(blk) * a.kv.heads + h;
    const int64_t off = ((at << a.kv.block_log2) + (key & ((1 << a.kv.block_log2) - 1))) * D;
    const int8_t* kp = a.kv.codes[0] + off + g * D + 16 * t4;
    const int8_t* vp = a.kv.codes[1] + off + 2 * t4 * D + g * (D / 8);
    uint4 kw[2][kC];
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int c = 0; c < kC; ++c) kw[hf][c] = __ldg(reinterpret_cast<const uint4*>(kp + 8 * hf * D + 64 * c));
    uint32_t vw[4][D / 32];            // tokens 2t, 2t + 1, 2t + 8, 2t + 9
#pragma unroll
    for (int tk = 0; tk < 4; ++tk) {
      const int8_t* p = vp + ((tk & 1) + 8 * (tk >> 1)) * D;
      if constexpr (D == 128) {
        const uint4 w = __ldg(reinterpret_cast<const uint4*>(p));
        vw[tk][0] = w.x, vw[tk][1] = w.y, vw[tk][2] = w.z, vw[tk][3] = w.w;
      } else {
        const uint2 w = __ldg(reinterpret_cast<const uint2*>(p));
        vw[tk][0] = w.x, vw[tk][1] = w.y;
      }
    }
    const float sk = __ldg(a.kv.scale[0] + at), sv = __ldg(a.kv.scale[1] + at);

    float s[2][4] = {};
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int c = 0; c < kC; ++c) {
        const uint32_t w[4] = {kw[hf][c].x, kw[hf][c].y, kw[hf][c].z, kw[hf][c].w};
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const uint32_t x = w[u] ^ 0x80808080u;
          mma_16816(s[hf], qf[4 * c + u], half_codes<0x4140>(x), half_codes<0x4342>(x));
        }
      }

    const float coef = a.scale_log2 * sk, lsv = log2f(sv);
    const bool all = key + kStep - 1 <= t.pos_lo && (a.window == 0 || key > t.pos_hi - a.window);
    uint32_t p[4];
    float alpha[2];
    bool moved = false;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float ci = coef * qs[i];
      float mx = -INFINITY;
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float& x = s[hf][2 * i + e];
          x = fmaf(x, ci, lsv);
          if (!all) {
            const int j = key + 8 * hf + 2 * t4 + e;
            if (j > pos[i] || (a.window > 0 && j <= pos[i] - a.window)) x = -INFINITY;
          }
          mx = fmaxf(mx, x);
        }
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
      const float m1 = fmaxf(m[i], mx), n1 = fmaxf(n[i], mx - lsv);
      const float base = finite_max(m1), nbase = finite_max(n1);
      alpha[i] = ex2(m[i] - base);
      moved = moved || m1 != m[i];
      float sum = 0.0f;
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        const float p0 = ex2(s[hf][2 * i] - base), p1 = ex2(s[hf][2 * i + 1] - base);
        p[2 * hf + i] = pack_half(p0, p1);
        sum += p0 + p1;
      }
      // the step's part of the denominator, relative to 2^n1: its largest P is 2^{mx - m1}, so a step that
      // contributes next to nothing to o, for its tiny scale, sums its terms relative to its own maximum
      float to = base - lsv - nbase;
      if (mx - base < -64.0f && mx > -INFINITY) {
        sum = 0.0f;
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) sum += ex2(s[hf][2 * i] - mx) + ex2(s[hf][2 * i + 1] - mx);
        to = mx - lsv - nbase;
      }
      // a hidden block adds nothing, whatever its scale
      l[i] = fmaf(l[i], ex2(n[i] - nbase), sum == 0.0f ? 0.0f : sum * ex2(to));
      m[i] = m1;
      n[i] = n1;
    }
    if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
      for (int j = 0; j < D / 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[j][e] *= alpha[e >> 1];
    }
    // a fragment of P: rows g, g + 8 by keys 2t, 2t + 1 and 2t + 8, 2t + 9
    const uint32_t pa[4] = {p[0], p[1], p[2], p[3]};
#pragma unroll
    for (int w = 0; w < D / 32; ++w) {
      const uint32_t x0 = vw[0][w] ^ 0x80808080u, x1 = vw[1][w] ^ 0x80808080u;
      const uint32_t x2 = vw[2][w] ^ 0x80808080u, x3 = vw[3][w] ^ 0x80808080u;
      const uint32_t lo0 = __byte_perm(x0, x1, 0x5140), hi0 = __byte_perm(x0, x1, 0x7362);
      const uint32_t lo1 = __byte_perm(x2, x3, 0x5140), hi1 = __byte_perm(x2, x3, 0x7362);
      mma_16816(acc[4 * w], pa, half_codes<0x4140>(lo0), half_codes<0x4140>(lo1));
      mma_16816(acc[4 * w + 1], pa, half_codes<0x4342>(lo0), half_codes<0x4342>(lo1));
      mma_16816(acc[4 * w + 2], pa, half_codes<0x4140>(hi0), half_codes<0x4140>(hi1));
      mma_16816(acc[4 * w + 3], pa, half_codes<0x4342>(hi0), half_codes<0x4342>(hi1));
    }
  }

  // join the warps: accumulator j of lane (g, t4) holds dimensions 2 t4 D/8 + j and (2 t4 + 1) D/8 + j
  __shared__ float o_sm[kWarps][kRows][D + 4];
  __shared__ float stat_sm[kWarps][kRows][3];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
    l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
    if (t4 == 0) {
      stat_sm[warp][g + 8 * i][0] = m[i];
      stat_sm[warp][g + 8 * i][1] = n[i];
      stat_sm[warp][g + 8 * i][2] = l[i];
    }
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int j = 0; j < D / 8; j += 4)
        *reinterpret_cast<float4*>(&o_sm[warp][g + 8 * i][(2 * t4 + e) * (D / 8) + j]) =
            make_float4(acc[j][2 * i + e], acc[j + 1][2 * i + e], acc[j + 2][2 * i + e], acc[j + 3][2 * i + e]);
  }
  __syncthreads();
  constexpr int kPer = kRows * D / (32 * kWarps);            // 16 or 8 dimensions of one row a thread
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
    const float inv = out_factor(ll, base - nbase);
    uint16_t* out = a.O + (t.seq.row0 + r / a.group) * a.ldo + static_cast<int64_t>(h * a.group + r % a.group) * D + d0;
#pragma unroll
    for (int e = 0; e < kPer; e += 8) {
      const float v[8] = {o[e] * inv,     o[e + 1] * inv, o[e + 2] * inv, o[e + 3] * inv,
                          o[e + 4] * inv, o[e + 5] * inv, o[e + 6] * inv, o[e + 7] * inv};
      reinterpret_cast<uint4*>(out + e)[0] = pack8(v);
    }
    return;
  }
  const int64_t slot = ((((static_cast<int64_t>(b) * a.kv.heads + h) * a.row_tiles + rt) * a.splits + split) * kRows) + row;
#pragma unroll
  for (int e = 0; e < kPer; e += 4)
    *reinterpret_cast<float4*>(a.part + slot * D + d0 + e) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
  if (d0 == 0) *reinterpret_cast<float4*>(a.part_stat + slot * 4) = make_float4(mm, nn, ll, 0.0f);
}

// Joins the splits of a row, one warp per row, in the order of the splits.
template <int D>
__global__ void __launch_bounds__(32 * kRows) kv_attn_join_kernel(AttnArgs a) {
  constexpr int kPer = D / 32;
  const int h = blockIdx.x % a.kv.heads, rt = blockIdx.x / a.kv.heads, b = blockIdx.y;
  const int row = threadIdx.x >> 5, lane = threadIdx.x & 31;
  Tile t;
  if (!attn_tile(a, b, rt, t)) return;
  const int ns = tile_splits(a, t), r = t.r0 + row;
  if (ns <= 1 || r >= t.rows) return;
  const int64_t slot0 = (((static_cast<int64_t>(b) * a.kv.heads + h) * a.row_tiles + rt) * a.splits) * kRows + row;
  const float4* stat = reinterpret_cast<const float4*>(a.part_stat) + slot0;
  float m = -INFINITY, n = -INFINITY;
  for (int s = lane; s < ns; s += 32) {
    m = fmaxf(m, stat[s * kRows].x);
    n = fmaxf(n, stat[s * kRows].y);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    n = fmaxf(n, __shfl_xor_sync(0xffffffffu, n, o));
  }
  const float base = finite_max(m), nbase = finite_max(n);
  float acc[kPer] = {}, l = 0.0f;
#pragma unroll 4
  for (int s = 0; s < ns; ++s) {
    const float4 v = stat[s * kRows];
    const float f = ex2(v.x - base);
    const float* p = a.part + (slot0 + static_cast<int64_t>(s) * kRows) * D + lane * kPer;
    l = fmaf(v.z, ex2(v.y - nbase), l);
    if constexpr (kPer == 4) {
      const float4 x = *reinterpret_cast<const float4*>(p);
      acc[0] = fmaf(x.x, f, acc[0]), acc[1] = fmaf(x.y, f, acc[1]);
      acc[2] = fmaf(x.z, f, acc[2]), acc[3] = fmaf(x.w, f, acc[3]);
    } else {
      const float2 x = *reinterpret_cast<const float2*>(p);
      acc[0] = fmaf(x.x, f, acc[0]), acc[1] = fmaf(x.y, f, acc[1]);
    }
  }
  const float inv = out_factor(l, base - nbase);
  uint16_t* out = a.O + (t.seq.row0 + r / a.group) * a.ldo + static_cast<int64_t>(h * a.group + r % a.group) * D + lane * kPer;
  if constexpr (kPer == 4)
    *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16(acc[0] * inv, acc[1] * inv), pack_bf16(acc[2] * inv, acc[3] * inv));
  else
    *reinterpret_cast<uint32_t*>(out) = pack_bf16(acc[0] * inv, acc[1] * inv);
}

template <int D>
cudaError_t launch(const AttnArgs& a, cudaStream_t stream) {
  const dim3 grid(a.splits, a.kv.heads * a.row_tiles, a.kv.n_seqs);
  kv_attn_split_kernel<D><<<grid, 32 * kWarps, 0, stream>>>(a);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess || a.splits <= 1) return e;
  kv_attn_join_kernel<D><<<dim3(a.kv.heads * a.row_tiles, a.kv.n_seqs), 32 * kRows, 0, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace

// The keys are cut so that the tiles of the largest batch the bounds allow fill the machine about
// four times over (ragged sequences then even out), in pieces of at least 64 keys: one step of each warp.
void plan_attn(AttnArgs& a, int sms) {
  const int64_t rows = static_cast<int64_t>(a.kv.max_rows) * a.group;
  a.row_tiles = static_cast<int>((rows + kRows - 1) / kRows);
  if (a.row_tiles < 1) a.row_tiles = 1;
  int64_t keys = a.kv.max_len;
  if (a.window > 0) {
    const int64_t w = static_cast<int64_t>(a.window) + kRows + 2 * kStep;
    keys = keys < w ? keys : w;
  }
  const int64_t tiles = static_cast<int64_t>(a.kv.n_seqs) * a.kv.heads * a.row_tiles;
  const int64_t want = static_cast<int64_t>(sms) * 12;
  int64_t chunk = (keys * tiles + want - 1) / want;
  chunk = (chunk + 63) / 64 * 64;
  if (chunk < 64) chunk = 64;
  a.chunk = static_cast<int>(chunk);
  const int64_t splits = (keys + chunk - 1) / chunk;
  a.splits = static_cast<int>(splits < 1 ? 1 : splits);
}

cudaError_t launch_kv_attn(const AttnArgs& a, cudaStream_t stream) {
  return a.kv.d == 128 ? launch<128>(a, stream) : launch<64>(a, stream);
}

}  // namespace lrqat
