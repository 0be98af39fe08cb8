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
    v.y = fmaxf(v.y, __shfl_xor_sync(0xffffffffu, v.y, o));
  }
  return v;
}

// One pass over a row: the row stays in registers (as h gamma) between the load and the
// quantization, and one exchange between the warps carries both the sum of squares and
// max|h gamma|; rounding is monotone, so max|y| = fl(R max|h gamma|) exactly and no second
// exchange is needed.
template <int V>
__global__ void __launch_bounds__(V == 1 ? 1024 : 512) add_rmsnorm_fwd_kernel(NormFwdArgs a, int wpr) {
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
  uint4 x[V], r[V], g[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int j = sub + nthr * i;
    const bool in = live && j < k8;
    x[i] = in ? X[j] : zero;
    r[i] = in && a.R ? R[j] : zero;
    g[i] = in ? __ldg(G + j) : zero;
  }
  float hg[V][8];
  float2 sm = make_float2(0.0f, 0.0f);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int j = sub + nthr * i;
    float h[8], rr[8], gg[8];
    unpack8(x[i], h);
    unpack8(r[i], rr);
    unpack8(g[i], gg);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      h[e] += rr[e];
      sm.x = fmaf(h[e], h[e], sm.x);
      hg[i][e] = h[e] * gg[e];
      sm.y = fmaxf(sm.y, fabsf(hg[i][e]));
    }
    if (a.H && live && j < k8) reinterpret_cast<uint4*>(a.H)[base + j] = pack8(h);
  }
  sm = warp_sum_max(sm);
  if (wpr > 1) {
    if (lane == 0) red[warp] = sm;
    __syncthreads();
    sm = make_float2(0.0f, 0.0f);
    for (int w = 0; w < wpr; ++w) {
      const float2 o = red[wr * wpr + w];
      sm.x += o.x;
      sm.y = fmaxf(sm.y, o.y);
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
  // a row with a NaN or an infinity has rstd NaN or 0 and max|y| NaN: its scale is NaN
  const float amax = isfinite(sm.x) ? sm.y * rstd : __int_as_float(0x7FFFFFFF);
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
    round_div8(hg[i], s, inv, q);
    if (a.Y_q) reinterpret_cast<uint2*>(a.Y_q)[base + j] = pack_codes8(q);
    if (a.Y) {
#pragma unroll
      for (int e = 0; e < 8; ++e) q[e] *= s;
      reinterpret_cast<uint4*>(a.Y)[base + j] = pack8(q);
    }
  }
}

__device__ __forceinline__ float2 warp_sum2(float2 v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
    v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
  }
  return v;
}

// A row group takes rows t, t + stride, ...; its threads keep the dgamma sums of their
// columns in registers over all of them and write them once, as one row of `part`.  mean(h^2)
// and mean(g h) are reduced together.
template <int V>
__global__ void __launch_bounds__(V == 1 ? 1024 : 512) add_rmsnorm_bwd_kernel(NormBwdArgs a, int wpr) {
  __shared__ float2 red[2][32];
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
  float acc[V][8];
#pragma unroll
  for (int i = 0; i < V; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[i][e] = 0.0f;
  int ph = 0;
  // every row group of a block runs the same number of turns (they share the barrier)
  for (int64_t t0 = static_cast<int64_t>(blockIdx.x) * rpb; t0 < a.T; t0 += stride, ph ^= 1) {
    const int64_t t = t0 + wr;
    const bool live = t < a.T;
    const int64_t base = (live ? t : 0) * k8;
    uint4 h4[V], y4[V], d4[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int j = sub + nthr * i;
      const bool in = live && j < k8;
      h4[i] = in ? reinterpret_cast<const uint4*>(a.H)[base + j] : zero;
      y4[i] = in ? reinterpret_cast<const uint4*>(a.dY)[base + j] : zero;
      d4[i] = in && a.dH ? reinterpret_cast<const uint4*>(a.dH)[base + j] : zero;
    }
    float2 sm = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int j = sub + nthr * i;
      float h[8], y[8], g[8];
      unpack8(h4[i], h);
      unpack8(y4[i], y);
      unpack8(j < k8 ? __ldg(G + j) : zero, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        sm.x = fmaf(h[e], h[e], sm.x);
        sm.y = fmaf(y[e] * g[e], h[e], sm.y);
      }
    }
    sm = warp_sum2(sm);
    if (wpr > 1) {
      if (lane == 0) red[ph][warp] = sm;
      __syncthreads();
      sm = make_float2(0.0f, 0.0f);
      for (int w = 0; w < wpr; ++w) {
        const float2 o = red[ph][wr * wpr + w];
        sm.x += o.x;
        sm.y += o.y;
      }
    }
    if (!live) continue;
    const float rstd = 1.0f / sqrtf(sm.x * inv_k + a.eps);
    const float c = rstd * rstd * (sm.y * inv_k);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int j = sub + nthr * i;
      if (j >= k8) break;
      float h[8], y[8], g[8], d[8];
      unpack8(h4[i], h);
      unpack8(y4[i], y);
      unpack8(d4[i], d);
      unpack8(__ldg(G + j), g);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        acc[i][e] = fmaf(y[e], h[e] * rstd, acc[i][e]);
        d[e] = fmaf(rstd, y[e] * g[e] - h[e] * c, d[e]);
      }
      reinterpret_cast<uint4*>(a.dX)[base + j] = pack8(d);
    }
  }
  if (!a.dgamma) return;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int j = sub + nthr * i;
    if (j >= k8) break;
    float4* dst = reinterpret_cast<float4*>(a.part + group * a.k) + 2 * j;
    dst[0] = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
    dst[1] = make_float4(acc[i][4], acc[i][5], acc[i][6], acc[i][7]);
  }
}

// dgamma[j] = sum of part[.][j] in a fixed order: a block owns 32 float4 columns, its warps add
// interleaved rows and a fixed tree adds the warps.
constexpr int kSumWarps = 16;
__global__ void __launch_bounds__(32 * kSumWarps) dgamma_sum_kernel(const float4* __restrict__ part, int64_t np,
                                                                    int64_t k4, float4* __restrict__ out,
                                                                    int accumulate) {
  __shared__ float4 red[kSumWarps][32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t j = static_cast<int64_t>(blockIdx.x) * 32 + lane;
  float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  if (j < k4) {
#pragma unroll 4
    for (int64_t p = warp; p < np; p += kSumWarps) {
      const float4 v = part[p * k4 + j];
      s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
    }
  }
  red[warp][lane] = s;
  __syncthreads();
  for (int h = kSumWarps / 2; h > 0; h >>= 1) {
    if (warp < h) {
      const float4 o = red[warp + h][lane];
      float4& m = red[warp][lane];
      m.x += o.x, m.y += o.y, m.z += o.z, m.w += o.w;
    }
    __syncthreads();
  }
  if (warp == 0 && j < k4) {
    float4 m = red[0][lane];
    if (accumulate) {
      const float4 o = out[j];
      m.x += o.x, m.y += o.y, m.z += o.z, m.w += o.w;
    }
    out[j] = m;
  }
}

// X_hat = bf16(s c): 8 codes a thread, a row's threads in as many turns as it takes.
__global__ void __launch_bounds__(256) act_dequant_kernel(const uint2* __restrict__ codes,
                                                          const float* __restrict__ scale, int64_t T, int k8, int wpr,
                                                          uint4* __restrict__ out) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int wr = warp / wpr, sub = (warp - wr * wpr) * 32 + lane;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * (8 / wpr) + wr;
  if (t >= T) return;
  const float s = __ldg(scale + t);
  for (int j = sub; j < k8; j += wpr * 32) {
    const uint2 w = __ldg(codes + t * k8 + j);
    float lo[4], hi[4];
    codes4(w.x, lo);
    codes4(w.y, hi);
    out[t * k8 + j] = make_uint4(pack_bf16(lo[0] * s, lo[1] * s), pack_bf16(lo[2] * s, lo[3] * s),
                                 pack_bf16(hi[0] * s, hi[1] * s), pack_bf16(hi[2] * s, hi[3] * s));
  }
}

// Words per thread of a row (k <= 16384): few rows take one word a thread (the shortest chain
// of loads), many rows two; rows above 1024 words four, which 512 threads hold.
int words_per_thread(int64_t k8, int64_t T, int sms) {
  if (k8 > 1024) return 4;
  return T <= 2 * sms ? 1 : 2;
}

}  // namespace

cudaError_t launch_add_rmsnorm_fwd(const NormFwdArgs& a, int sms, cudaStream_t stream) {
  const int64_t k8 = a.k / 8;
  const int V = words_per_thread(k8, a.T, sms);
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
  int64_t grid;
};
BwdPlan plan_bwd(int64_t T, int64_t k, int sms) {
  BwdPlan p;
  p.V = words_per_thread(k / 8, T, sms);
  p.rs = row_shape(k / 8, p.V);
  const int64_t turns = (T + p.rs.rpb - 1) / p.rs.rpb;
  const int64_t per_sm = 1024 / (32 * p.rs.wpr * p.rs.rpb);
  const int64_t most = sms * (per_sm < 1 ? 1 : per_sm);
  p.grid = turns < most ? turns : most;
  return p;
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
  switch (p.V) {
    case 1: add_rmsnorm_bwd_kernel<1><<<grid, threads, 0, stream>>>(a, p.rs.wpr); break;
    case 2: add_rmsnorm_bwd_kernel<2><<<grid, threads, 0, stream>>>(a, p.rs.wpr); break;
    default: add_rmsnorm_bwd_kernel<4><<<grid, threads, 0, stream>>>(a, p.rs.wpr); break;
  }
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess || !a.dgamma) return e;
  const int64_t k4 = a.k / 4;
  dgamma_sum_kernel<<<static_cast<unsigned>((k4 + 31) / 32), 32 * kSumWarps, 0, stream>>>(
      reinterpret_cast<const float4*>(a.part), p.grid * p.rs.rpb, k4, reinterpret_cast<float4*>(a.dgamma),
      a.accumulate);
  return cudaGetLastError();
}

cudaError_t launch_act_dequant(const int8_t* codes, const float* scale, int64_t T, int64_t k, uint16_t* x_hat,
                               cudaStream_t stream) {
  const int k8 = static_cast<int>(k / 8);
  int wpr = 1;
  while (wpr < 8 && wpr * 64 < k8) wpr *= 2;   // up to two words a thread and turn
  const int rpb = 8 / wpr;
  act_dequant_kernel<<<static_cast<unsigned>((T + rpb - 1) / rpb), 256, 0, stream>>>(
      reinterpret_cast<const uint2*>(codes), scale, T, k8, wpr, reinterpret_cast<uint4*>(x_hat));
  return cudaGetLastError();
}

}  // namespace lrqat
