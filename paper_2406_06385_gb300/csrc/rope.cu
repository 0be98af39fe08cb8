// Norm of each head's queries and keys and their rotation by position in one pass, and its gradient.
//
// Per head x of d elements:  n = x / sqrt(mean(x^2) + eps) gamma (n = x without gamma), and of its first `rot`
// elements the pair (a, b) number i, elements (i, i + rot / 2) or (2 i, 2 i + 1), becomes
//   (a cos w - b sin w, a sin w + b cos w),  w = pos freq_i.
// Backward:  g = the gradient rotated by -w;  with r = 1 / sqrt(mean(x^2) + eps):
//   dx = r (g gamma - x r^2 mean(g gamma x)),  dgamma = sum over rows and heads of g x r.
//
// An angle is kept in turns, w / (2 pi), modulo 1 as a 64-bit fraction: pos times the 64-bit fraction of
// freq_i / (2 pi) wraps around by itself, so an angle is off by at most pos 2^-65 turns, 2^-34 at the farthest
// position, for one multiplication of whole numbers; the sine and cosine then see the fraction rounded to 24 bits.
#include <cuda_runtime.h>
#include <cstdint>

#include "serve.cuh"

namespace lrqat {
namespace {

constexpr int kRopeWarps = 8;
constexpr int kMostPairs = 128;              // head_dim <= 256

// How a warp lies over heads: L lanes a head, a lane two 16-byte words (16 elements: 8 pairs where they rotate).
// With pairs half a head apart those are words j and j + rot / 16, so that a lane holds whole pairs; lanes behind
// rot / 16 hold two neighbouring words that pass.
template <int L, bool kNeighbours>
struct HeadLane {
  int sub, w0, w1;                           // head of the warp's 32 / L; the lane's words
  bool holds, turns;
  __device__ __forceinline__ HeadLane(int lane, int d, int rot) {
    const int j = lane % L, half = rot / 16;
    sub = lane / L;
    holds = j < d / 16;
    turns = j < half;
    w0 = !kNeighbours && turns ? j : 2 * j;
    w1 = !kNeighbours && turns ? j + half : 2 * j + 1;
  }
  // sum over the lanes of a head
  static __device__ __forceinline__ float sum(float v) {
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
  }
  // (a, b) of pair e among the lane's 16 elements
  static __device__ __forceinline__ constexpr int a(int e) { return kNeighbours ? 2 * e : e; }
  static __device__ __forceinline__ constexpr int b(int e) { return kNeighbours ? 2 * e + 1 : 8 + e; }
};

// cos and sin of the position's angles, shared by the warp's lanes (and so by all heads)
__device__ __forceinline__ void warp_angles(float2* cs, const uint64_t* turns, int pairs, int lane, int pos) {
  for (int i = lane; i < pairs; i += 32) {
    const uint64_t w = static_cast<uint64_t>(static_cast<uint32_t>(pos)) * __ldg(turns + i);
    float s, c;
    sincospif(static_cast<float>(static_cast<int32_t>(w >> 32)) * 0x1p-31f, &s, &c);
    cs[i] = make_float2(c, s);
  }
  __syncwarp();
}
__device__ __forceinline__ void lane_angles(const float2* cs, int j, bool turns, float (&c)[8], float (&s)[8]) {
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const float4 v = turns ? *reinterpret_cast<const float4*>(cs + 8 * j + e) : make_float4(1.0f, 0.0f, 1.0f, 0.0f);
    c[e] = v.x, s[e] = v.y, c[e + 1] = v.z, s[e + 1] = v.w;
  }
}
__device__ __forceinline__ void unpack16(const uint4 (&w)[2], float (&x)[16]) {
  float lo[8], hi[8];
  unpack8(w[0], lo);
  unpack8(w[1], hi);
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = lo[e], x[8 + e] = hi[e];
}
__device__ __forceinline__ void pack16(const float (&x)[16], uint4 (&w)[2]) {
  float lo[8], hi[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) lo[e] = x[e], hi[e] = x[8 + e];
  w[0] = pack8(lo);
  w[1] = pack8(hi);
}

// A warp takes one token (or `per` of its groups of 32 / L heads), works its angles out once and walks over the
// heads, kAhead groups loaded before the first is stored (in place the loads may not move over the stores).
constexpr int kAhead = 4;
template <int L, bool kNeighbours>
__global__ void __launch_bounds__(32 * kRopeWarps) rope_fwd_kernel(RopeArgs a, int per, int parts) {
  using Lane = HeadLane<L, kNeighbours>;
  __shared__ __align__(16) float2 cs[kRopeWarps][kMostPairs];
  constexpr int kHeads = 32 / L;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t unit = static_cast<int64_t>(blockIdx.x) * kRopeWarps + warp, t = unit / parts;
  if (t >= a.T) return;
  const int pos = a.pos ? __ldg(a.pos + t) : static_cast<int>(t);
  if (pos < 0) return;
  const Lane my(lane, a.d, a.rot);
  warp_angles(cs[warp], a.turns, a.rot / 2, lane, pos);
  float c[8], s[8];
  lane_angles(cs[warp], lane % L, my.turns, c, s);
  uint4 gamma[2][2];
#pragma unroll
  for (int kind = 0; kind < 2; ++kind) {
    const uint4* g = reinterpret_cast<const uint4*>(a.gamma[kind]);
    gamma[kind][0] = g && my.holds ? __ldg(g + my.w0) : make_uint4(0u, 0u, 0u, 0u);
    gamma[kind][1] = g && my.holds ? __ldg(g + my.w1) : make_uint4(0u, 0u, 0u, 0u);
  }
  const int q_groups = (a.heads[0] + kHeads - 1) / kHeads, groups = q_groups + (a.heads[1] + kHeads - 1) / kHeads;
  const int first = static_cast<int>(unit % parts) * per, end = min(first + per, groups);
  const float inv_d = 1.0f / static_cast<float>(a.d);
  for (int g0 = first; g0 < end; g0 += kAhead) {
    uint4 w[kAhead][2];
    bool in[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int g = g0 + u, kind = g >= q_groups, h = (g - (kind ? q_groups : 0)) * kHeads + my.sub;
      in[u] = g < end && my.holds && h < (kind ? a.heads[1] : a.heads[0]);
      const uint4* x = reinterpret_cast<const uint4*>((kind ? a.X[1] : a.X[0]) + t * (kind ? a.ldx[1] : a.ldx[0]) +
                                                      static_cast<int64_t>(h) * a.d);
      w[u][0] = in[u] ? x[my.w0] : make_uint4(0u, 0u, 0u, 0u);
      w[u][1] = in[u] ? x[my.w1] : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int g = g0 + u, kind = g >= q_groups, h = (g - (kind ? q_groups : 0)) * kHeads + my.sub;
      if (g >= end) break;
      float x[16];
      unpack16(w[u], x);
      if (kind ? a.gamma[1] : a.gamma[0]) {
        float ss = 0.0f, gm[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) ss = fmaf(x[e], x[e], ss);
        const float r = 1.0f / sqrtf(Lane::sum(ss) * inv_d + a.eps);
        const uint4 gw[2] = {kind ? gamma[1][0] : gamma[0][0], kind ? gamma[1][1] : gamma[0][1]};
        unpack16(gw, gm);
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = x[e] * r * gm[e];
      }
      if (my.turns) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float p = x[Lane::a(e)], q = x[Lane::b(e)];
          x[Lane::a(e)] = p * c[e] - q * s[e];
          x[Lane::b(e)] = p * s[e] + q * c[e];
        }
      }
      if (!in[u]) continue;
      uint4 o[2];
      pack16(x, o);
      uint4* y = reinterpret_cast<uint4*>((kind ? a.Y[1] : a.Y[0]) + t * (kind ? a.ldy[1] : a.ldy[0]) +
                                          static_cast<int64_t>(h) * a.d);
      y[my.w0] = o[0];
      y[my.w1] = o[1];
    }
  }
}

// The same walk backwards, by blocks that stay: a lane keeps the sums of dgamma for its 16 elements of query and key
// heads in registers over all its tokens; heads, warps and blocks are added in a fixed order afterwards.
constexpr int kBwdAhead = 2;
template <int L, bool kNeighbours>
__global__ void __launch_bounds__(32 * kRopeWarps) rope_bwd_kernel(RopeBwdArgs a, int per, int parts) {
  using Lane = HeadLane<L, kNeighbours>;
  __shared__ __align__(16) float2 cs[kRopeWarps][kMostPairs];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // the sum of dgamma may line up
  constexpr int kHeads = 32 / L;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Lane my(lane, a.f.d, a.f.rot);
  const float inv_d = 1.0f / static_cast<float>(a.f.d);
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  uint4 gamma[2][2];
  float acc[2][16];
#pragma unroll
  for (int kind = 0; kind < 2; ++kind) {
    const uint4* g = reinterpret_cast<const uint4*>(a.f.gamma[kind]);
    gamma[kind][0] = g && my.holds ? __ldg(g + my.w0) : zero;
    gamma[kind][1] = g && my.holds ? __ldg(g + my.w1) : zero;
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[kind][e] = 0.0f;
  }
  const int n_groups[2] = {(a.f.heads[0] + kHeads - 1) / kHeads, (a.f.heads[1] + kHeads - 1) / kHeads};
  for (int64_t unit = static_cast<int64_t>(blockIdx.x) * kRopeWarps + warp; unit < a.f.T * parts;
       unit += static_cast<int64_t>(gridDim.x) * kRopeWarps) {
    const int64_t t = unit / parts;
    const int pos = a.f.pos ? __ldg(a.f.pos + t) : static_cast<int>(t);
    float c[8], s[8];
    __syncwarp();                            // the last token's angles have been read
    warp_angles(cs[warp], a.f.turns, a.f.rot / 2, lane, max(pos, 0));
    lane_angles(cs[warp], lane % L, my.turns, c, s);
    const int first = static_cast<int>(unit % parts) * per;
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
      const int before = kind ? n_groups[0] : 0;
      const int g_lo = max(first - before, 0), g_hi = min(first + per - before, n_groups[kind]);
      const bool norm = a.f.gamma[kind] != nullptr;
      for (int g0 = g_lo; g0 < g_hi; g0 += kBwdAhead) {
        uint4 wy[kBwdAhead][2], wx[kBwdAhead][2];
        bool in[kBwdAhead];
#pragma unroll
        for (int u = 0; u < kBwdAhead; ++u) {
          const int h = (g0 + u) * kHeads + my.sub;
          in[u] = g0 + u < g_hi && my.holds && h < a.f.heads[kind];
          const uint4* y = reinterpret_cast<const uint4*>(a.dY[kind] + t * a.lddy[kind] + static_cast<int64_t>(h) * a.f.d);
          const uint4* x = reinterpret_cast<const uint4*>(a.f.X[kind] + t * a.f.ldx[kind] + static_cast<int64_t>(h) * a.f.d);
          const bool live = in[u] && pos >= 0;
          wy[u][0] = live ? y[my.w0] : zero;
          wy[u][1] = live ? y[my.w1] : zero;
          wx[u][0] = live && norm ? x[my.w0] : zero;
          wx[u][1] = live && norm ? x[my.w1] : zero;
        }
#pragma unroll
        for (int u = 0; u < kBwdAhead; ++u) {
          if (g0 + u >= g_hi) break;
          const int h = (g0 + u) * kHeads + my.sub;
          float g[16];
          unpack16(wy[u], g);
          if (my.turns) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float p = g[Lane::a(e)], q = g[Lane::b(e)];
              g[Lane::a(e)] = p * c[e] + q * s[e];
              g[Lane::b(e)] = q * c[e] - p * s[e];
            }
          }
          if (norm) {
            float x[16], gm[16], ss = 0.0f, gx = 0.0f;
            unpack16(wx[u], x);
            unpack16(gamma[kind], gm);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              ss = fmaf(x[e], x[e], ss);
              gx = fmaf(g[e] * gm[e], x[e], gx);
            }
            const float r = 1.0f / sqrtf(Lane::sum(ss) * inv_d + a.f.eps);
            const float k = -r * (r * r * (Lane::sum(gx) * inv_d));
            if (pos >= 0) {                  // padding adds nothing, whatever eps is
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                if (in[u]) acc[kind][e] = fmaf(g[e], x[e] * r, acc[kind][e]);
                g[e] = fmaf(r, g[e] * gm[e], k * x[e]);
              }
            }
          }
          if (!in[u]) continue;
          uint4 o[2];
          pack16(g, o);
          uint4* dx = reinterpret_cast<uint4*>(a.f.Y[kind] + t * a.f.ldy[kind] + static_cast<int64_t>(h) * a.f.d);
          dx[my.w0] = o[0];
          dx[my.w1] = o[1];
        }
      }
    }
  }
  if (!a.part) return;
  // the warp's heads, then the block's warps in order
  float* red = reinterpret_cast<float*>(cs[warp]);                     // 256 floats: one kind at a time
#pragma unroll
  for (int kind = 0; kind < 2; ++kind) {
    __syncthreads();                         // angles, or the other kind's sums, have been read
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      float v = acc[kind][e];
#pragma unroll
      for (int o = L; o < 32; o *= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
      if (my.sub == 0 && my.holds) red[8 * (e < 8 ? my.w0 : my.w1) + e % 8] = v;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.f.d; i += blockDim.x) {
      float v = 0.0f;
#pragma unroll
      for (int w = 0; w < kRopeWarps; ++w) v += reinterpret_cast<const float*>(cs[w])[i];
      a.part[(static_cast<int64_t>(blockIdx.x) * 2 + kind) * a.f.d + i] = v;
    }
  }
}

// dgamma = the blocks' sums in a fixed order: 32 row lanes add interleaved rows, a fixed tree adds the lanes.
constexpr int kSumRows = 32, kSumCols = 16;
__global__ void __launch_bounds__(kSumRows* kSumCols) rope_dgamma_kernel(const float* part, int rows, int d, float* dq,
                                                                         float* dk, int accumulate) {
  __shared__ float red[kSumRows][kSumCols + 1];
  asm volatile("griddepcontrol.wait;" ::: "memory");         // the partial sums are there
  const int row = threadIdx.x / kSumCols, col = threadIdx.x % kSumCols, i = blockIdx.x * kSumCols + col;
  float v = 0.0f;
#pragma unroll 4
  for (int r = row; r < rows; r += kSumRows) v += __ldcg(part + static_cast<int64_t>(r) * 2 * d + i);
  red[row][col] = v;
  __syncthreads();
  for (int h = kSumRows / 2; h > 0; h >>= 1) {
    if (row < h) red[row][col] += red[row + h][col];
    __syncthreads();
  }
  float* out = i < d ? dq : dk;
  if (row == 0 && out) {
    out += i < d ? i : i - d;
    *out = red[0][col] + (accumulate ? *out : 0.0f);
  }
}

// Head groups of a token that one warp takes: all of them, or fewer where that many warps would not fill the machine.
struct RopePlan {
  int per, parts;
};
RopePlan plan_rope(const RopeArgs& a, int lanes, int ahead, int sms) {
  const int heads = 32 / lanes;
  const int groups = (a.heads[0] + heads - 1) / heads + (a.heads[1] + heads - 1) / heads;
  RopePlan p{groups, 1};
  const int64_t want = 16 * static_cast<int64_t>(sms);
  if (a.T < want) {
    const int64_t parts = (want + a.T - 1) / a.T;
    p.per = static_cast<int>((groups + parts - 1) / parts);
    if (p.per < ahead) p.per = groups < ahead ? groups : ahead;
    p.parts = (groups + p.per - 1) / p.per;
  }
  return p;
}
int head_lanes(int d) {
  int L = 2;
  while (16 * L < d) L *= 2;
  return L;
}
int64_t bwd_blocks(const RopeArgs& a, const RopePlan& p, int sms) {
  const int64_t units = a.T * p.parts, blocks = (units + kRopeWarps - 1) / kRopeWarps;
  return blocks < 2 * sms ? blocks : 2 * sms;
}

template <int L>
cudaError_t fwd(const RopeArgs& a, bool neighbours, int sms, cudaStream_t stream) {
  const RopePlan p = plan_rope(a, L, 1, sms);
  const unsigned grid = static_cast<unsigned>((a.T * p.parts + kRopeWarps - 1) / kRopeWarps);
  if (neighbours) rope_fwd_kernel<L, true><<<grid, 32 * kRopeWarps, 0, stream>>>(a, p.per, p.parts);
  else rope_fwd_kernel<L, false><<<grid, 32 * kRopeWarps, 0, stream>>>(a, p.per, p.parts);
  return cudaGetLastError();
}
template <int L>
cudaError_t bwd(const RopeBwdArgs& a, bool neighbours, int sms, cudaStream_t stream) {
  const RopePlan p = plan_rope(a.f, L, kBwdAhead, sms);
  const unsigned grid = static_cast<unsigned>(bwd_blocks(a.f, p, sms));
  if (neighbours) rope_bwd_kernel<L, true><<<grid, 32 * kRopeWarps, 0, stream>>>(a, p.per, p.parts);
  else rope_bwd_kernel<L, false><<<grid, 32 * kRopeWarps, 0, stream>>>(a, p.per, p.parts);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess || !a.part) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(2 * a.f.d / kSumCols));
  cfg.blockDim = dim3(kSumRows * kSumCols);
  cfg.stream = stream;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, rope_dgamma_kernel, static_cast<const float*>(a.part), static_cast<int>(grid), a.f.d,
                            a.dgamma[0], a.dgamma[1], a.accumulate);
}

}  // namespace

int64_t rope_bwd_parts(const RopeArgs& a, int sms) {
  return bwd_blocks(a, plan_rope(a, head_lanes(a.d), kBwdAhead, sms), sms);
}

cudaError_t launch_rope_fwd(const RopeArgs& a, bool neighbours, int sms, cudaStream_t stream) {
  switch (head_lanes(a.d)) {
    case 2: return fwd<2>(a, neighbours, sms, stream);
    case 4: return fwd<4>(a, neighbours, sms, stream);
    case 8: return fwd<8>(a, neighbours, sms, stream);
    default: return fwd<16>(a, neighbours, sms, stream);
  }
}
cudaError_t launch_rope_bwd(const RopeBwdArgs& a, bool neighbours, int sms, cudaStream_t stream) {
  switch (head_lanes(a.f.d)) {
    case 2: return bwd<2>(a, neighbours, sms, stream);
    case 4: return bwd<4>(a, neighbours, sms, stream);
    case 8: return bwd<8>(a, neighbours, sms, stream);
    default: return bwd<16>(a, neighbours, sms, stream);
  }
}

}  // namespace lrqat
