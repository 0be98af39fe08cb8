// Residual addition, root-mean-square norm and per-token 8-bit quantization in one pass, its
// gradient, and the values of stored 8-bit activations.
//
//   h = x + r,  n = h / sqrt(mean(h^2) + eps),  y = n gamma                    (rows of k)
//   s = max|y| / 127 (1 for a row of zeros),  c = round(y / s),  y_hat = s c
// Backward, the quantizer passed straight through (its scale is not differentiated), with
// g = dy gamma and R = 1 / sqrt(mean(h^2) + eps):
//   dx = dr = R (g - h R^2 mean(g h)) + dh,   dgamma = sum over rows of dy h R
#include <cuda_runtime.h>
#include <cstdint>

#include "kernels.h"
#include "serve.cuh"

namespace lrqat {
namespace {

// Threads of one row: `wpr` warps that hold V 16-byte words each; `rpb` rows per block.
struct RowShape {
  int wpr, rpb;
};
RowShape row_shape(int64_t k8, int V) {
  const int wpr = static_cast<int>((k8 + 32 * V - 1) / (32 * V));
  return {wpr, wpr >= 8 ? 1 : 8 / wpr};
}

__device__ __forceinline__ float2 warp_sum_max(float2 v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
    v.y = max_nan(v.y, __shfl_xor_sync(0xffffffffu, v.y, o));
  }
  return v;
}

// One pass over a row: the row stays in registers (as h gamma) between the load and the
// quantization, and one exchange between the warps carries both the sum of squares and
// max|h gamma|; rounding is monotone, so max|y| = fl(R max|h gamma|) exactly and no second
// exchange is needed.  Bound by memory: what counts is loads in flight, so the fewest threads a row
// (four words each) and as many rows at once as 64 registers a thread allow.  16384 rows of 5120 with
// residual: 99.5 us, 6.74 TB/s; with two words a thread 115 us, with one 150 us.
template <int V>
__global__ void __launch_bounds__(V == 1 ? 1024 : 512, V == 1 ? 1 : 2) add_rmsnorm_fwd_kernel(NormFwdArgs a, int wpr) {
  __shared__ float2 red[32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int wr = warp / wpr;                                   // row of this block
  const int sub = (warp - wr * wpr) * 32 + lane, nthr = wpr * 32;
  const int rpb = (blockDim.x >> 5) / wpr;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * rpb + wr;
  const int k8 = static_cast<int>(a.k / 8);
  const bool live = t < a.T;
  const int64_t base = (live ? t : 0) * k8;
  const uint4* X = reinterpret_cast<const uint4*>(a.X) + base;
  const uint4* R = reinterpret_cast<const uint4*>(a.R) + base;
  const uint4* G = reinterpret_cast<const uint4*>(a.gamma);
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  uint4 x[V], r[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int j = sub + nthr * i;
    const bool in = live && j < k8;
    x[i] = in ? X[j] : zero;
    r[i] = in && a.R ? R[j] : zero;
  }
  float hg[V][8];
  float2 sm = make_float2(0.0f, 0.0f);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int j = sub + nthr * i;
    const bool in = live && j < k8;
    float rr[8], gg[8];
    unpack8(in ? __ldg(G + j) : zero, gg);
    unpack8(x[i], hg[i]);
    unpack8(r[i], rr);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      hg[i][e] += rr[e];
      sm.x = fmaf(hg[i][e], hg[i][e], sm.x);
    }
    if (a.H && in) reinterpret_cast<uint4*>(a.H)[base + j] = pack8(hg[i]);
#pragma unroll
    for (int e = 0; e < 8; ++e) hg[i][e] *= gg[e];
#pragma unroll
    for (int e = 0; e < 8; e += 2) sm.y = max3_abs_nan(sm.y, hg[i][e], hg[i][e + 1]);
  }
  sm = warp_sum_max(sm);
  if (wpr > 1) {
    if (lane == 0) red[warp] = sm;
    __syncthreads();
    sm = make_float2(0.0f, 0.0f);
    for (int w = 0; w < wpr; ++w) {
      const float2 o = red[wr * wpr + w];
      sm.x += o.x;
      sm.y = max_nan(sm.y, o.y);
    }
  }
  if (!live) return;
  const float rstd = 1.0f / sqrtf(sm.x / static_cast<float>(a.k) + a.eps);
  if (!a.quant) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int j = sub + nthr * i;
#pragma unroll
      for (int e = 0; e < 8; ++e) hg[i][e] *= rstd;
      if (j < k8) reinterpret_cast<uint4*>(a.Y)[base + j] = pack8(hg[i]);
    }
    return;
  }
  // a NaN or an infinity in h (the sum is not finite) or in h gamma (the maximum, which keeps a NaN, is not)
  // makes the scale NaN, so that the codes, which cannot say so, read back as NaN
  const float top = sm.y * rstd;
  const float amax = isfinite(sm.x) && isfinite(top) ? top : __int_as_float(0x7FFFFFFF);
  const float s = amax == 0.0f ? 1.0f : __fdiv_rn(amax, 127.0f);
  const float inv = __frcp_rn(s);
  if (sub == 0 && a.s_y) a.s_y[t] = s;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int j = sub + nthr * i;
    if (j >= k8) break;
    float q[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) hg[i][e] *= rstd;
    round_div8<true>(hg[i], s, inv, q);
    if (a.Y_q) reinterpret_cast<uint2*>(a.Y_q)[base + j] = pack_codes8(q);
    if (a.Y) {
#pragma unroll
      for (int e = 0; e < 8; ++e) q[e] = (q[e] - kRoundMagic) * s;
      reinterpret_cast<uint4*>(a.Y)[base + j] = pack8(q);
    }
  }
}

__device__ __forceinline__ float2 warp_sum2(float2 v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    v = __fadd2_rn(v, make_float2(__shfl_xor_sync(0xffffffffu, v.x, o), __shfl_xor_sync(0xffffffffu, v.y, o)));
  return v;
}
__device__ __forceinline__ void unpack4x2(const uint4& v, float2 (&x)[4]) {
  x[0] = make_float2(bf16_lo(v.x), bf16_hi(v.x)), x[1] = make_float2(bf16_lo(v.y), bf16_hi(v.y));
  x[2] = make_float2(bf16_lo(v.z), bf16_hi(v.z)), x[3] = make_float2(bf16_lo(v.w), bf16_hi(v.w));
}

// A row group takes rows t, t + stride, ...; its threads keep the dgamma sums of their
// columns in registers over all of them and write them once, as one row of `part`.  mean(h^2)
// and mean(g h) are reduced together.  The next kBwdStages rows are on their way into shared memory
// meanwhile; a thread copies, waits for and reads its own words only, so no barrier guards them, and
// registers hold nothing but the sums.  What bounds it is the chain load, sums, exchange, gradient of a row
// against three blocks an SM, and its instructions (packed pairs and rsqrtf, within two units in the last
// place of 32 bits, count: 122 us with scalars and a division by the root): 16384 rows of 5120 with dH in
// 116 us, 5.8 TB/s, the sum of dgamma included (rows held in registers with the next one prefetched: 12 us
// more, without prefetch 7; three or four stages leave room for two blocks: 6, 47 more).
constexpr int kBwdStages = 2;
constexpr int kBwdSmem = 200 * 1024, kSmemPerSm = 220 * 1024;  // most shared memory of a block, of an SM's blocks
template <int V>
__global__ void __launch_bounds__(512, V == 4 ? 1 : 2) add_rmsnorm_bwd_kernel(NormBwdArgs a, int wpr) {
  extern __shared__ uint4 words[];                             // [stage][H, dY, dH][V][thread]
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // the sum of dgamma may line up
  __shared__ float2 red[2][16];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int wr = warp / wpr;
  const int sub = (warp - wr * wpr) * 32 + lane, nthr = wpr * 32;
  const int rpb = (blockDim.x >> 5) / wpr;
  const int k8 = static_cast<int>(a.k / 8);
  const int64_t group = static_cast<int64_t>(blockIdx.x) * rpb + wr;
  const int64_t stride = static_cast<int64_t>(gridDim.x) * rpb;
  const float inv_k = 1.0f / static_cast<float>(a.k);
  const uint4* G = reinterpret_cast<const uint4*>(a.gamma);
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  auto word = [&](int stage, int what, int i) { return words + ((stage * 3 + what) * V + i) * blockDim.x + threadIdx.x; };
  auto load = [&](int stage, int64_t t) {
    if (t < a.T) {
      const int64_t base = t * k8;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int j = sub + nthr * i;
        if (j >= k8) break;
        copy_async16(word(stage, 0, i), reinterpret_cast<const uint4*>(a.H) + base + j);
        copy_async16(word(stage, 1, i), reinterpret_cast<const uint4*>(a.dY) + base + j);
        if (a.dH) copy_async16(word(stage, 2, i), reinterpret_cast<const uint4*>(a.dH) + base + j);
      }
    }
    copy_commit();
  };
  float2 acc[V][4];
#pragma unroll
  for (int i = 0; i < V; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[i][e] = make_float2(0.0f, 0.0f);
#pragma unroll
  for (int i = 0; i < kBwdStages; ++i) load(i, group + i * stride);
  int turn = 0;
  // every row group of a block runs the same number of turns (they share the barrier)
  for (int64_t t0 = static_cast<int64_t>(blockIdx.x) * rpb; t0 < a.T; t0 += stride, ++turn) {
    const int64_t t = t0 + wr, base = t * k8;
    const int stage = turn % kBwdStages, ph = turn & 1;
    copy_wait<kBwdStages - 1>();
    float2 hh = make_float2(0.0f, 0.0f), gh = hh;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int j = sub + nthr * i;
      const bool in = t < a.T && j < k8;
      float2 h[4], y[4], g[4];
      unpack4x2(in ? *word(stage, 0, i) : zero, h);
      unpack4x2(in ? *word(stage, 1, i) : zero, y);
      unpack4x2(in ? __ldg(G + j) : zero, g);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        hh = __ffma2_rn(h[e], h[e], hh);
        gh = __ffma2_rn(__fmul2_rn(y[e], g[e]), h[e], gh);
      }
    }
    float2 sm = warp_sum2(make_float2(hh.x + hh.y, gh.x + gh.y));
    if (wpr > 1) {
      if (lane == 0) red[ph][warp] = sm;
      __syncthreads();
      sm = make_float2(0.0f, 0.0f);
#pragma unroll 4
      for (int w = 0; w < wpr; ++w) sm = __fadd2_rn(sm, red[ph][wr * wpr + w]);
    }
    if (t < a.T) {
      const float rstd = rsqrtf(sm.x * inv_k + a.eps);
      const float c = -rstd * (rstd * rstd * (sm.y * inv_k));
      const float2 rstd2 = make_float2(rstd, rstd), c2 = make_float2(c, c);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int j = sub + nthr * i;
        if (j >= k8) break;
        float2 h[4], y[4], g[4], d[4];
        unpack4x2(*word(stage, 0, i), h);
        unpack4x2(*word(stage, 1, i), y);
        unpack4x2(a.dH ? *word(stage, 2, i) : zero, d);
        unpack4x2(__ldg(G + j), g);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          acc[i][e] = __ffma2_rn(y[e], __fmul2_rn(h[e], rstd2), acc[i][e]);
          d[e] = __ffma2_rn(rstd2, __fmul2_rn(y[e], g[e]), __ffma2_rn(c2, h[e], d[e]));
        }
        reinterpret_cast<uint4*>(a.dX)[base + j] =
            make_uint4(pack_bf16(d[0].x, d[0].y), pack_bf16(d[1].x, d[1].y), pack_bf16(d[2].x, d[2].y),
                       pack_bf16(d[3].x, d[3].y));
      }
    }
    load(stage, t + kBwdStages * stride);
  }
  if (!a.dgamma) return;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int j = sub + nthr * i;
    if (j >= k8) break;
    float4* dst = reinterpret_cast<float4*>(a.part + group * a.k) + 2 * j;
    dst[0] = make_float4(acc[i][0].x, acc[i][0].y, acc[i][1].x, acc[i][1].y);
    dst[1] = make_float4(acc[i][2].x, acc[i][2].y, acc[i][3].x, acc[i][3].y);
  }
}

// dgamma[j] = sum of part[.][j] in a fixed order: a block owns 8 float4 columns, its 32 row lanes add
// interleaved rows and a fixed tree adds the lanes.
constexpr int kSumRows = 32;
__global__ void __launch_bounds__(8 * kSumRows) dgamma_sum_kernel(const float4* part, int64_t np, int64_t k4,
                                                                  float4* out, int accumulate) {
  __shared__ float4 red[kSumRows][8];
  asm volatile("griddepcontrol.wait;" ::: "memory");           // the partial sums are there
  const int row = threadIdx.x >> 3, col = threadIdx.x & 7;
  const int64_t j = static_cast<int64_t>(blockIdx.x) * 8 + col;
  float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  if (j < k4) {
#pragma unroll 8
    for (int64_t p = row; p < np; p += kSumRows) {
      const float4 v = __ldcg(part + p * k4 + j);               // written while this grid may already be waiting
      s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
    }
  }
  red[row][col] = s;
  __syncthreads();
  for (int h = kSumRows / 2; h > 0; h >>= 1) {
    if (row < h) {
      const float4 o = red[row + h][col];
      float4& m = red[row][col];
      m.x += o.x, m.y += o.y, m.z += o.z, m.w += o.w;
    }
    __syncthreads();
  }
  if (row == 0 && j < k4) {
    float4 m = red[0][col];
    if (accumulate) {
      const float4 o = out[j];
      m.x += o.x, m.y += o.y, m.z += o.z, m.w += o.w;
    }
    out[j] = m;
  }
}

// X_hat = bf16(s c): a thread takes 16 codes (two words of the result) at a time, or 8 where rows are an odd
// number of 8 codes and so only 8-byte aligned.
__device__ __forceinline__ uint4 dequant8(uint32_t w0, uint32_t w1, float s) {
  float lo[4], hi[4];
  codes4(w0, lo);
  codes4(w1, hi);
  return make_uint4(pack_bf16(lo[0] * s, lo[1] * s), pack_bf16(lo[2] * s, lo[3] * s), pack_bf16(hi[0] * s, hi[1] * s),
                    pack_bf16(hi[2] * s, hi[3] * s));
}
template <int W>
__global__ void __launch_bounds__(256) act_dequant_kernel(const int8_t* __restrict__ codes,
                                                          const float* __restrict__ scale, int64_t T, int kw, int wpr,
                                                          uint4* __restrict__ out) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int wr = warp / wpr, sub = (warp - wr * wpr) * 32 + lane;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * (8 / wpr) + wr;
  if (t >= T) return;
  const float s = __ldg(scale + t);
  for (int j = sub; j < kw; j += wpr * 32) {
    const int64_t i = t * kw + j;
    if constexpr (W == 2) {
      const uint4 w = __ldg(reinterpret_cast<const uint4*>(codes) + i);
      out[2 * i] = dequant8(w.x, w.y, s);
      out[2 * i + 1] = dequant8(w.z, w.w, s);
    } else {
      const uint2 w = __ldg(reinterpret_cast<const uint2*>(codes) + i);
      out[i] = dequant8(w.x, w.y, s);
    }
  }
}

// Words per thread of a row (k <= 16384).  A row that fills fewer than `most` words of a warp's lanes takes
// no more than it needs.
int words_per_thread(int64_t k8, int most) {
  int V = 1;
  while (V < most && k8 > 32 * V) V *= 2;
  return V;
}

}  // namespace

cudaError_t launch_add_rmsnorm_fwd(const NormFwdArgs& a, int sms, cudaStream_t stream) {
  const int64_t k8 = a.k / 8;
  // few rows: one word a thread, the shortest chain (k up to 8192: 1024 threads)
  const int V = words_per_thread(k8, a.T <= 2 * sms && k8 <= 1024 ? 1 : 4);
  const RowShape rs = row_shape(k8, V);
  const unsigned grid = static_cast<unsigned>((a.T + rs.rpb - 1) / rs.rpb);
  const int threads = 32 * rs.wpr * rs.rpb;
  switch (V) {
    case 1: add_rmsnorm_fwd_kernel<1><<<grid, threads, 0, stream>>>(a, rs.wpr); break;
    case 2: add_rmsnorm_fwd_kernel<2><<<grid, threads, 0, stream>>>(a, rs.wpr); break;
    default: add_rmsnorm_fwd_kernel<4><<<grid, threads, 0, stream>>>(a, rs.wpr); break;
  }
  return cudaGetLastError();
}

namespace {
struct BwdPlan {
  int V;
  RowShape rs;
  int smem;
  int64_t grid;
};
BwdPlan plan_bwd(int64_t T, int64_t k, int sms) {
  BwdPlan p;
  // the dgamma sums cost 8 registers a word: two words a thread (k above 8192: four)
  p.V = words_per_thread(k / 8, k > 8192 ? 4 : 2);
  p.rs = row_shape(k / 8, p.V);
  p.smem = kBwdStages * 3 * p.V * 32 * p.rs.wpr * p.rs.rpb * 16;
  const int64_t turns = (T + p.rs.rpb - 1) / p.rs.rpb;
  const int64_t by_smem = kSmemPerSm / p.smem, by_regs = 1024 / (32 * p.rs.wpr * p.rs.rpb);
  // a block writes a row of partial sums: four turns a block before an SM gets another one
  const int64_t by_turns = (turns + 4 * sms - 1) / (4 * sms);
  int64_t per_sm = by_smem < by_regs ? by_smem : by_regs;
  if (per_sm > by_turns) per_sm = by_turns;
  const int64_t most = sms * (per_sm < 1 ? 1 : per_sm);
  p.grid = turns < most ? turns : most;
  return p;
}
}  // namespace

namespace {
template <int V>
cudaError_t launch_bwd(const NormBwdArgs& a, int wpr, unsigned grid, int threads, int smem, cudaStream_t stream) {
  static bool smem_set[kMaxDevices];
  const cudaError_t e = ensure_smem_attr(reinterpret_cast<const void*>(add_rmsnorm_bwd_kernel<V>), kBwdSmem, smem_set);
  if (e != cudaSuccess) return e;
  add_rmsnorm_bwd_kernel<V><<<grid, threads, smem, stream>>>(a, wpr);
  return cudaGetLastError();
}
}  // namespace

int64_t norm_bwd_parts(int64_t T, int64_t k, int sms) {
  const BwdPlan p = plan_bwd(T, k, sms);
  return p.grid * p.rs.rpb;
}

cudaError_t launch_add_rmsnorm_bwd(const NormBwdArgs& a, int sms, cudaStream_t stream) {
  const BwdPlan p = plan_bwd(a.T, a.k, sms);
  const unsigned grid = static_cast<unsigned>(p.grid);
  const int threads = 32 * p.rs.wpr * p.rs.rpb;
  const cudaError_t e = p.V == 1   ? launch_bwd<1>(a, p.rs.wpr, grid, threads, p.smem, stream)
                        : p.V == 2 ? launch_bwd<2>(a, p.rs.wpr, grid, threads, p.smem, stream)
                                   : launch_bwd<4>(a, p.rs.wpr, grid, threads, p.smem, stream);
  if (e != cudaSuccess || !a.dgamma) return e;
  const int64_t k4 = a.k / 4;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>((k4 + 7) / 8));
  cfg.blockDim = dim3(8 * kSumRows);
  cfg.stream = stream;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, dgamma_sum_kernel, reinterpret_cast<const float4*>(a.part),
                            static_cast<int64_t>(p.grid * p.rs.rpb), k4, reinterpret_cast<float4*>(a.dgamma), a.accumulate);
}

cudaError_t launch_act_dequant(const int8_t* codes, const float* scale, int64_t T, int64_t k, uint16_t* x_hat,
                               cudaStream_t stream) {
  const int W = k % 16 == 0 ? 2 : 1, kw = static_cast<int>(k / (8 * W));
  int wpr = 1;
  while (wpr < 8 && wpr * 32 < kw) wpr *= 2;
  const int rpb = 8 / wpr;
  const unsigned grid = static_cast<unsigned>((T + rpb - 1) / rpb);
  if (W == 2) act_dequant_kernel<2><<<grid, 256, 0, stream>>>(codes, scale, T, kw, wpr, reinterpret_cast<uint4*>(x_hat));
  else act_dequant_kernel<1><<<grid, 256, 0, stream>>>(codes, scale, T, kw, wpr, reinterpret_cast<uint4*>(x_hat));
  return cudaGetLastError();
}

}  // namespace lrqat
