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
// position, for one multiplication of whole numbers.  The sine and cosine see its upper 32 bits (less than 2^-32 turns
// below it) rounded to 24 (up to 2^-26): fp32 angles could not tell more apart.
#include <cuda_runtime.h>
#include <cstdint>
#include <type_traits>

#include "kernels.h"
#include "serve.cuh"

namespace lrqat {
namespace {

constexpr int kRopeWarps = 8, kRopeThreads = 32 * kRopeWarps;
constexpr int kMostPairs = 128;              // head_dim <= 256
constexpr int kFwdPerSm = 2, kBwdPerSm = 2;  // thread blocks an SM holds

// How a warp lies over heads: L lanes a head, a lane two 16-byte words (16 elements: 8 pairs where they rotate).
// With pairs half a head apart those are words j and j + rot / 16, so that a lane holds whole pairs; lanes behind
// rot / 16 hold two neighbouring words that pass.  kFull: heads of 16 L elements that rotate whole.
template <int L, bool kNeighbours, bool kFull>
struct HeadLane {
  int sub, w0, w1;                           // head of the warp's 32 / L; the lane's words
  bool holds, turns;
  __device__ __forceinline__ HeadLane(int lane, int d, int rot) {
    const int j = lane % L, half = kFull ? L : rot / 16;
    sub = lane / L;
    holds = kFull || j < d / 16;
    turns = kFull || j < half;
    w0 = !kNeighbours && turns ? j : 2 * j;
    w1 = !kNeighbours && turns ? j + half : 2 * j + 1;
  }
  // 16-byte words from the lane's first to its second
  __device__ __forceinline__ int apart() const { return kFull ? (kNeighbours ? 1 : L) : w1 - w0; }
  // elements from one group of 32 / L heads to the next
  static __device__ __forceinline__ int group(int d) { return kFull ? 512 : 32 / L * d; }
  // sum over the lanes of a head
  static __device__ __forceinline__ float sum(float2 p) {
    float v = p.x + p.y;
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
  }
};

// cos and sin of the position's angles, shared by the warp's lanes (and so by all heads)
__device__ __forceinline__ void warp_angles(float2* cs, const uint64_t* turns, int pairs, int lane, int pos) {
  for (int i = lane; i < pairs; i += 32) {
    const uint64_t w = static_cast<uint64_t>(static_cast<uint32_t>(pos)) * __ldg(turns + i);
    float s, c;
    sincospif(static_cast<float>(static_cast<int32_t>(w >> 32)) * 0x1p-31f, &s, &c);
    cs[(i % 8 / 2 * (kMostPairs / 8) + i / 8) * 2 + i % 2] = make_float2(c, s);      // lanes read 16 bytes side by side
  }
  __syncwarp();
}
// The cosines and sines (negative ones to turn back) of a lane's 8 pairs, two to a register pair.
struct Angles {
  float2 c[4], s[4];
};
template <bool kBack>
__device__ __forceinline__ Angles lane_angles(const float2* cs, int j, bool turns) {
  Angles a;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float4 v = turns ? reinterpret_cast<const float4*>(cs)[e * (kMostPairs / 8) + j] : make_float4(1.0f, 0.0f, 1.0f, 0.0f);
    a.c[e] = make_float2(v.x, v.z);
    a.s[e] = kBack ? make_float2(-v.y, -v.w) : make_float2(v.y, v.w);
  }
  return a;
}
__device__ __forceinline__ float2 neg2(float2 v) { return make_float2(-v.x, -v.y); }
// Turns the lane's pairs: (x[i], x[4 + i]) are the first and second elements of pairs 2 i and 2 i + 1, or x[i] is pair i.
template <bool kNeighbours>
__device__ __forceinline__ void turn(float2 (&x)[8], const Angles& a) {
  if constexpr (kNeighbours) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float c = i & 1 ? a.c[i / 2].y : a.c[i / 2].x, s = i & 1 ? a.s[i / 2].y : a.s[i / 2].x;
      x[i] = __ffma2_rn(x[i], make_float2(c, c), __fmul2_rn(make_float2(x[i].y, x[i].x), make_float2(-s, s)));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 p = x[i], q = x[4 + i];
      x[i] = __ffma2_rn(p, a.c[i], neg2(__fmul2_rn(q, a.s[i])));
      x[4 + i] = __ffma2_rn(q, a.c[i], __fmul2_rn(p, a.s[i]));
    }
  }
}
__device__ __forceinline__ void unpack16(const uint4& lo, const uint4& hi, float2 (&x)[8]) {
  const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = make_float2(bf16_lo(w[e]), bf16_hi(w[e]));
}
__device__ __forceinline__ uint4 pack4x2(const float2* x) {
  return make_uint4(pack_bf16(x[0].x, x[0].y), pack_bf16(x[1].x, x[1].y), pack_bf16(x[2].x, x[2].y), pack_bf16(x[3].x, x[3].y));
}

// A warp takes one token, or `per` of its groups of 32 / L heads, works the angles out once and walks over the groups,
// the words of the next kAhead of them on their way: the first ones before the angles, each further one as soon as its
// registers are free.  In place an address is read by the lane that later writes it, and by nobody else.
constexpr int kAhead = 4;
template <int L, bool kNeighbours, bool kFull>
__global__ void __launch_bounds__(kRopeThreads, kFwdPerSm) rope_fwd_kernel(RopeArgs a, int per, int parts) {
  using Lane = HeadLane<L, kNeighbours, kFull>;
  __shared__ __align__(16) float2 cs[kRopeWarps][kMostPairs];
  constexpr int kHeads = 32 / L;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t unit = blockIdx.x * kRopeWarps + warp;
  const int64_t t = parts == 1 ? unit : unit / parts;
  if (t >= a.T) return;
  const int pos = a.pos ? __ldg(a.pos + t) : static_cast<int>(t);
  if (pos < 0) return;
  const Lane my(lane, a.d, a.rot);
  const int apart = my.apart();
  const int q_groups = (a.heads[0] + kHeads - 1) / kHeads, groups = q_groups + (a.heads[1] + kHeads - 1) / kHeads;
  const int first = parts == 1 ? 0 : static_cast<int>(unit - static_cast<uint32_t>(t) * parts) * per;
  const int end = min(first + per, groups);
  // of group 0 of each kind; groups are numbered through both
  const int64_t lane_at = static_cast<int64_t>(my.sub) * a.d + 8 * my.w0, k_off = static_cast<int64_t>(q_groups) * Lane::group(a.d);
  const uint16_t* xq = a.X[0] + t * a.ldx[0] + lane_at;
  const uint16_t* xk = a.X[1] + t * a.ldx[1] + lane_at - k_off;
  uint16_t* yq = a.Y[0] + t * a.ldy[0] + lane_at;
  uint16_t* yk = a.Y[1] + t * a.ldy[1] + lane_at - k_off;
  const int most_q = a.heads[0] - my.sub, most_k = a.heads[1] - my.sub + q_groups * kHeads;
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  uint4 w[kAhead][2];
  auto live = [&](int g) { return g < end && my.holds && g * kHeads < (g >= q_groups ? most_k : most_q); };
  auto load = [&](uint4 (&v)[2], int g) {
    const bool in = live(g);
    const uint4* x = reinterpret_cast<const uint4*>((g >= q_groups ? xk : xq) + static_cast<int64_t>(g) * Lane::group(a.d));
    v[0] = in ? x[0] : zero;
    v[1] = in ? x[apart] : zero;
  };
#pragma unroll
  for (int u = 0; u < kAhead; ++u) load(w[u], first + u);
  warp_angles(cs[warp], a.turns, a.rot / 2, lane, pos);
  const Angles angles = lane_angles<false>(cs[warp], lane % L, my.turns);
  const float inv_d = 1.0f / static_cast<float>(a.d);
  for (int g0 = first; g0 < end; g0 += kAhead) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int g = g0 + u;
      if (g >= end) break;
      float2 x[8];
      unpack16(w[u][0], w[u][1], x);
      load(w[u], g + kAhead);
      const uint16_t* gamma = g >= q_groups ? a.gamma[1] : a.gamma[0];
      if (gamma) {
        float2 ss = make_float2(0.0f, 0.0f), gm[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = __ffma2_rn(x[e], x[e], ss);
        const float r = 1.0f / sqrtf(Lane::sum(ss) * inv_d + a.eps);
        const uint4* gw = reinterpret_cast<const uint4*>(gamma) + my.w0;
        unpack16(my.holds ? __ldg(gw) : zero, my.holds ? __ldg(gw + apart) : zero, gm);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = __fmul2_rn(__fmul2_rn(x[e], make_float2(r, r)), gm[e]);
      }
      if (my.turns) turn<kNeighbours>(x, angles);
      if (live(g)) {
        uint4* y = reinterpret_cast<uint4*>((g >= q_groups ? yk : yq) + static_cast<int64_t>(g) * Lane::group(a.d));
        y[0] = pack4x2(x);
        y[apart] = pack4x2(x + 4);
      }
    }
  }
}

// The same walk backwards, by blocks that stay, first over all query heads, then over all key heads (the angles once
// more): a lane keeps the sums of dgamma for its 16 elements in registers over all its tokens, and gamma as well; heads,
// warps and blocks are added in a fixed order afterwards.  The words of the next kRing groups are on their way into
// shared memory, tokens' ends or not; a lane copies, waits for and reads its own words only, so nothing guards them.
// 128 registers a thread: heads that fill their lanes and rotate whole spill none, the others 8 to 48 bytes.
constexpr int kRing = 3;
template <int L, bool kNeighbours, bool kFull>
__global__ void __launch_bounds__(kRopeThreads, kBwdPerSm) rope_bwd_kernel(RopeBwdArgs a, int per) {
  using Lane = HeadLane<L, kNeighbours, kFull>;
  __shared__ __align__(16) float2 cs[kRopeWarps][kMostPairs];
  extern __shared__ uint4 words[];                                     // [ring][dy, x][2][thread]
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // the sum of dgamma may line up
  constexpr int kHeads = 32 / L;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Lane my(lane, a.f.d, a.f.rot);
  const int apart = my.apart();
  const float inv_d = 1.0f / static_cast<float>(a.f.d);
  const int64_t lane_at = static_cast<int64_t>(my.sub) * a.f.d + 8 * my.w0;
  const uint32_t tokens = static_cast<uint32_t>(a.f.T), stride = gridDim.x * kRopeWarps;
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll 1
  for (int kind = 0; kind < 2; ++kind) {
    const int heads = a.f.heads[kind], groups = (heads + kHeads - 1) / kHeads, most = heads - my.sub;
    if (groups == 0) continue;               // no such heads
    const int parts = per == 0 ? 1 : (groups + per - 1) / per, n = per == 0 ? groups : per;     // groups of a unit
    const uint16_t* gamma = a.f.gamma[kind];
    const uint16_t* dY = a.dY[kind] + lane_at;
    const uint16_t* X = gamma ? a.f.X[kind] + lane_at : nullptr;
    uint16_t* dX = a.f.Y[kind] + lane_at;
    const int64_t lddy = a.lddy[kind], ldx = a.f.ldx[kind], lddx = a.f.ldy[kind];
    float2 acc[8], gm[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = make_float2(0.0f, 0.0f);
    {
      const uint4* gw = reinterpret_cast<const uint4*>(gamma) + my.w0;
      const bool g = gamma && my.holds;
      unpack16(g ? __ldg(gw) : zero, g ? __ldg(gw + apart) : zero, gm);
    }
    auto token = [&](uint32_t unit) { return parts == 1 ? unit : unit / parts; };
    auto group0 = [&](uint32_t unit) { return parts == 1 ? 0 : static_cast<int>(unit % parts) * n; };
    auto position = [&](uint32_t t) { return t >= tokens ? -1 : a.f.pos ? __ldg(a.f.pos + t) : static_cast<int>(t); };
    // the cursor that runs ahead
    uint32_t unit2 = blockIdx.x * kRopeWarps + warp, t2 = token(unit2);
    int g2 = group0(unit2), left2 = n;
    auto word = [&](int stage, int i) { return words + (stage * 4 + i) * kRopeThreads + threadIdx.x; };
    auto issue = [&](int stage) {
      if (t2 < tokens) {
        if (my.holds && g2 * kHeads < most) {
          const int64_t at = static_cast<int64_t>(g2) * Lane::group(a.f.d);
          const uint4* y = reinterpret_cast<const uint4*>(dY + t2 * lddy + at);
          copy_async16(word(stage, 0), y);
          copy_async16(word(stage, 1), y + apart);
          if (X) {
            const uint4* x = reinterpret_cast<const uint4*>(X + t2 * ldx + at);
            copy_async16(word(stage, 2), x);
            copy_async16(word(stage, 3), x + apart);
          }
        }
        ++g2;
        if (--left2 == 0) {
          unit2 += stride;
          t2 = token(unit2), g2 = group0(unit2), left2 = n;
        }
      }
      copy_commit();
    };
#pragma unroll
    for (int i = 0; i < kRing; ++i) issue(i);
    int stage = 0, next_pos = position(token(blockIdx.x * kRopeWarps + warp));
    for (uint32_t unit = blockIdx.x * kRopeWarps + warp;; unit += stride) {
      const uint32_t t = token(unit);
      if (t >= tokens) break;
      const int pos = next_pos;
      next_pos = position(token(unit + stride));
      __syncwarp();                          // the last token's angles have been read
      warp_angles(cs[warp], a.f.turns, a.f.rot / 2, lane, max(pos, 0));
      // a unit's last groups may lie behind the token's: they hold nothing
      for (int g = group0(unit), end = g + n; g < end; ++g) {
        copy_wait<kRing - 1>();
        const bool live = my.holds && g * kHeads < most, reads = live && pos >= 0;     // what padding holds may be anything
        float2 y[8];
        unpack16(reads ? *word(stage, 0) : zero, reads ? *word(stage, 1) : zero, y);
        if (my.turns) turn<kNeighbours>(y, lane_angles<true>(cs[warp], lane % L, true));
        if (gamma) {
          float2 x[8], ss = make_float2(0.0f, 0.0f), gx = ss, yg[8];
          unpack16(reads ? *word(stage, 2) : zero, reads ? *word(stage, 3) : zero, x);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            ss = __ffma2_rn(x[e], x[e], ss);
            yg[e] = __fmul2_rn(y[e], gm[e]);
            gx = __ffma2_rn(yg[e], x[e], gx);
          }
          // over the head's lanes, both at a time: one after the other, and with a division, 51 us where this takes 48
          float x2 = ss.x + ss.y, xg = gx.x + gx.y;
#pragma unroll
          for (int o = L / 2; o > 0; o >>= 1) {
            const float other_x2 = __shfl_xor_sync(0xffffffffu, x2, o), other_xg = __shfl_xor_sync(0xffffffffu, xg, o);
            x2 += other_x2, xg += other_xg;
          }
          const float r = rsqrtf(x2 * inv_d + a.f.eps);
          const float c = -r * (r * r * (xg * inv_d));
          if (reads) {                       // eps may be 0: nothing of a head that is not there is added
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              acc[e] = __ffma2_rn(y[e], __fmul2_rn(x[e], make_float2(r, r)), acc[e]);
              y[e] = __ffma2_rn(make_float2(r, r), yg[e], __fmul2_rn(make_float2(c, c), x[e]));
            }
          }
        }
        issue(stage);
        stage = stage + 1 == kRing ? 0 : stage + 1;
        if (live) {
          uint4* dx = reinterpret_cast<uint4*>(dX + t * lddx + static_cast<int64_t>(g) * Lane::group(a.f.d));
          dx[0] = pack4x2(y);
          dx[apart] = pack4x2(y + 4);
        }
      }
    }
    copy_wait<0>();
    if (!a.part) continue;
    // the warp's heads, then the block's warps in order
    float* red = reinterpret_cast<float*>(cs[warp]);                   // 256 floats
    __syncwarp();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float2 v = acc[e];
#pragma unroll
      for (int o = L; o < 32; o *= 2)
        v = __fadd2_rn(v, make_float2(__shfl_xor_sync(0xffffffffu, v.x, o), __shfl_xor_sync(0xffffffffu, v.y, o)));
      if (my.sub == 0 && my.holds) *reinterpret_cast<float2*>(red + 8 * (e < 4 ? my.w0 : my.w1) + 2 * (e % 4)) = v;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.f.d; i += blockDim.x) {
      float v = 0.0f;
#pragma unroll
      for (int q = 0; q < kRopeWarps; ++q) v += reinterpret_cast<const float*>(cs[q])[i];
      a.part[(static_cast<int64_t>(blockIdx.x) * 2 + kind) * a.f.d + i] = v;
    }
    __syncthreads();                         // the sums have been read
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

// Head groups of a token that one warp takes: all of them, or as few as it takes to give every warp that the machine holds
// a unit.
int fwd_per(const RopeArgs& a, int groups, int sms) {
  const int64_t want = static_cast<int64_t>(kFwdPerSm) * sms * kRopeWarps, parts = (want + a.T - 1) / a.T;
  return static_cast<int>((groups + parts - 1) / parts);
}
int head_groups(int heads, int lanes) { return (heads + 32 / lanes - 1) / (32 / lanes); }
int head_lanes(int d) {
  int L = 2;
  while (16 * L < d) L *= 2;
  return L;
}
struct BwdPlan {
  int per;                                   // 0: all of a kind
  unsigned grid;
};
BwdPlan plan_bwd(const RopeArgs& a, int sms) {
  const int L = head_lanes(a.d), q = head_groups(a.heads[0], L), k = head_groups(a.heads[1], L), most_groups = q > k ? q : k;
  const int64_t most = static_cast<int64_t>(kBwdPerSm) * sms, want = most * kRopeWarps, parts = (want + a.T - 1) / a.T;
  BwdPlan p{0, 0};
  if (parts > 1) p.per = static_cast<int>((most_groups + parts - 1) / parts);
  const int64_t units = a.T * (p.per ? (most_groups + p.per - 1) / p.per : 1), blocks = (units + kRopeWarps - 1) / kRopeWarps;
  p.grid = static_cast<unsigned>(blocks < most ? blocks : most);
  return p;
}

template <int L, bool kNeighbours, bool kFull>
cudaError_t fwd(const RopeArgs& a, int sms, cudaStream_t stream) {
  const int groups = head_groups(a.heads[0], L) + head_groups(a.heads[1], L), per = fwd_per(a, groups, sms);
  const int parts = (groups + per - 1) / per;
  const unsigned grid = static_cast<unsigned>((a.T * parts + kRopeWarps - 1) / kRopeWarps);
  rope_fwd_kernel<L, kNeighbours, kFull><<<grid, kRopeThreads, 0, stream>>>(a, per, parts);
  return cudaGetLastError();
}
template <int L, bool kNeighbours, bool kFull>
cudaError_t bwd(const RopeBwdArgs& a, int sms, cudaStream_t stream) {
  const BwdPlan p = plan_bwd(a.f, sms);
  constexpr int bytes = kRing * 4 * kRopeThreads * 16;
  static bool smem_set[kMaxDevices];
  cudaError_t e = ensure_smem_attr(reinterpret_cast<const void*>(rope_bwd_kernel<L, kNeighbours, kFull>), bytes, smem_set);
  if (e != cudaSuccess) return e;
  rope_bwd_kernel<L, kNeighbours, kFull><<<p.grid, kRopeThreads, bytes, stream>>>(a, p.per);
  e = cudaGetLastError();
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
  return cudaLaunchKernelEx(&cfg, rope_dgamma_kernel, static_cast<const float*>(a.part), static_cast<int>(p.grid), a.f.d,
                            a.dgamma[0], a.dgamma[1], a.accumulate);
}
// The variant for a head: its lanes, how pairs lie, and whether heads fill their lanes and rotate whole.
template <template <int, bool, bool> class Launch, typename Args>
cudaError_t by_head(const Args& a, int d, int rot, bool neighbours, int sms, cudaStream_t stream) {
  const int L = head_lanes(d);
  const bool full = d == 16 * L && rot == d;
  auto pick = [&](auto lanes) {
    constexpr int kL = decltype(lanes)::value;
    if (neighbours) return full ? Launch<kL, true, true>::run(a, sms, stream) : Launch<kL, true, false>::run(a, sms, stream);
    return full ? Launch<kL, false, true>::run(a, sms, stream) : Launch<kL, false, false>::run(a, sms, stream);
  };
  switch (L) {
    case 2: return pick(std::integral_constant<int, 2>{});
    case 4: return pick(std::integral_constant<int, 4>{});
    case 8: return pick(std::integral_constant<int, 8>{});
    default: return pick(std::integral_constant<int, 16>{});
  }
}
template <int L, bool kNeighbours, bool kFull>
struct Fwd {
  static cudaError_t run(const RopeArgs& a, int sms, cudaStream_t stream) { return fwd<L, kNeighbours, kFull>(a, sms, stream); }
};
template <int L, bool kNeighbours, bool kFull>
struct Bwd {
  static cudaError_t run(const RopeBwdArgs& a, int sms, cudaStream_t stream) { return bwd<L, kNeighbours, kFull>(a, sms, stream); }
};

}  // namespace

int64_t rope_bwd_parts(const RopeArgs& a, int sms) { return plan_bwd(a, sms).grid; }

cudaError_t launch_rope_fwd(const RopeArgs& a, bool neighbours, int sms, cudaStream_t stream) {
  return by_head<Fwd>(a, a.d, a.rot, neighbours, sms, stream);
}
cudaError_t launch_rope_bwd(const RopeBwdArgs& a, bool neighbours, int sms, cudaStream_t stream) {
  return by_head<Bwd>(a, a.f.d, a.f.rot, neighbours, sms, stream);
}

}  // namespace lrqat
