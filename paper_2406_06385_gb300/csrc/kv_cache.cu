// Keys and values quantized into a paged 8-bit cache as they are written, and read back.
//
// A block holds `block` tokens of one key/value head as int8 codes with one fp32 scale s:
// value = s c.  Writing new tokens x into a block whose first e tokens are older:
//   a = max|x| over the block's new tokens;  s' = a / 127 (1 if a = 0) where e = 0 or the older
//   tokens are all zeros, else max(s, a / 127);  new codes round(x / s');  where s' > s the e older
//   codes become round(c (s / s')).
// A thread block owns one (cache block, head, key or value), so nothing is shared between
// thread blocks and the result does not depend on their order.  Everything is bound by memory: a
// thread keeps its words of the new tokens in registers between the maximum and the codes.
#include <cuda_runtime.h>
#include <cstdint>

#include "serve.cuh"

namespace lrqat {
namespace {


// Threads of a block.  With 64 tokens of 128 dimensions a block, 128 threads of 8 words write 29484 tokens of 40
// heads in 168 us (64 threads of 16 words 233, 256 of 4: 202) and read them back in 137 us (the bytes' floor: 134).
constexpr int kKvThreads = 128;

// The part of sequence b's new tokens that lies in its j-th touched block.
struct BlockPart {
  int64_t row0;        // batch row of the block's first new token
  int64_t at;          // cache block times heads plus head
  int old, end;        // slots [old, end) hold new tokens
};
__device__ __forceinline__ bool block_part(const KvArgs& a, int b, int j, int head, BlockPart& p) {
  SeqRows s;
  if (!seq_rows(a, b, s)) return false;
  const int first = s.first > 0 ? s.first : 0;
  // the batch's bounds may allow many more blocks than are left below 2^31 tokens
  const int64_t start = (static_cast<int64_t>(first >> a.block_log2) + j) << a.block_log2;
  if (start >= s.len || s.n == 0) return false;
  const int p0 = static_cast<int>(start);
  const int blk = seq_block(a, b, p0);
  if (blk < 0) return false;
  p.old = first > p0 ? first - p0 : 0;
  p.end = min(s.len - p0, 1 << a.block_log2);
  p.row0 = s.row0 + (p0 + p.old - s.first);
  p.at = static_cast<int64_t>(blk) * a.heads + head;
  return true;
}

// NV 16-byte words of bf16 a thread; word v of the block is slot v / (d / 8).
template <int NV>
__global__ void __launch_bounds__(kKvThreads) kv_write_kernel(KvArgs a, const uint16_t* __restrict__ K, int64_t ldk,
                                                              const uint16_t* __restrict__ V, int64_t ldv) {
  // heads run fastest: neighbouring thread blocks read (write) neighbouring parts of the same rows
  const int kvh = blockIdx.x % (2 * a.heads), kv = kvh >= a.heads, head = kv ? kvh - a.heads : kvh;
  BlockPart p;
  if (!block_part(a, blockIdx.y, blockIdx.x / (2 * a.heads), head, p)) return;
  const uint16_t* X = (kv ? V : K) + static_cast<int64_t>(head) * a.d;
  const int64_t ld = kv ? ldv : ldk;
  const int dlog = a.d == 64 ? 3 : 4;                       // 16-byte words of one token
  uint4 x[NV];
  uint32_t top = 0;                                         // |x| as bf16 bits orders like |x|, NaN above all
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int v = threadIdx.x + kKvThreads * i, slot = v >> dlog;
    x[i] = make_uint4(0u, 0u, 0u, 0u);
    if (slot >= p.old && slot < p.end)
      x[i] = __ldg(reinterpret_cast<const uint4*>(X + (p.row0 + slot - p.old) * ld) + (v & ((1 << dlog) - 1)));
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    top = __vmaxu2(top, __vmaxu2(x[i].x & 0x7FFF7FFFu, x[i].y & 0x7FFF7FFFu));
    top = __vmaxu2(top, __vmaxu2(x[i].z & 0x7FFF7FFFu, x[i].w & 0x7FFF7FFFu));
  }
  top = max(top >> 16, top & 0xFFFFu);
  top = __reduce_max_sync(0xffffffffu, top);
  __shared__ uint32_t red[kKvThreads / 32];
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = top;
  float* scale = (kv ? a.scale[1] : a.scale[0]) + p.at;
  const float was = p.old ? *scale : 0.0f;                  // read before thread 0 writes it
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kKvThreads / 32; ++w) top = max(top, red[w]);
  // infinities and NaN leave a NaN scale: the block then reads back as NaN
  const float amax = top < 0x7F80u ? __uint_as_float(top << 16) : __int_as_float(0x7FFFFFFF);
  const float fresh = __fdiv_rn(amax, 127.0f);
  uint2* codes = reinterpret_cast<uint2*>((kv ? a.codes[1] : a.codes[0]) + (p.at << a.block_log2) * a.d);
  // Older tokens that are all zeros (scale 1, the one a block of zeros takes, and codes 0; or scale 0) fix no scale: at
  // scale 1 small new ones would be lost.  The whole thread block takes the same branch.
  bool empty = p.old == 0 || was == 0.0f;
  if (p.old && was == 1.0f) {
    uint32_t any = 0;
    for (int v = threadIdx.x; v < p.old << dlog; v += kKvThreads) any |= codes[v].x | codes[v].y;
    empty = !__syncthreads_or(any != 0);
  }
  const float s = empty ? (amax == 0.0f ? 1.0f : fresh) : was >= fresh || was != was ? was : fresh;
  const float inv = __frcp_rn(s);
  if (threadIdx.x == 0) *scale = s;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int v = threadIdx.x + kKvThreads * i, slot = v >> dlog;
    if (slot >= p.old && slot < p.end) {
      float xf[8], q[8];
      unpack8(x[i], xf);
      round_div8<false>(xf, s, inv, q);
      codes[v] = pack_codes8(q);
    }
  }
  if (s > was && p.old) {
    const float ratio = __fdiv_rn(was, s);
    for (int v = threadIdx.x; v < p.old << dlog; v += kKvThreads) {
      const uint2 w = codes[v];
      float lo[4], hi[4], q[8];
      codes4(w.x, lo);
      codes4(w.y, hi);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        q[e] = __fadd_rn(__fmul_rn(lo[e], ratio), kRoundMagic);
        q[4 + e] = __fadd_rn(__fmul_rn(hi[e], ratio), kRoundMagic);
      }
      codes[v] = pack_codes8(q);
    }
  }
}

template <int NV>
__global__ void __launch_bounds__(kKvThreads) kv_read_kernel(KvArgs a, uint16_t* __restrict__ K, int64_t ldk,
                                                             uint16_t* __restrict__ V, int64_t ldv) {
  // heads run fastest: neighbouring thread blocks read (write) neighbouring parts of the same rows
  const int kvh = blockIdx.x % (2 * a.heads), kv = kvh >= a.heads, head = kv ? kvh - a.heads : kvh;
  BlockPart p;
  if (!block_part(a, blockIdx.y, blockIdx.x / (2 * a.heads), head, p)) return;
  uint16_t* X = (kv ? V : K) + static_cast<int64_t>(head) * a.d;
  const int64_t ld = kv ? ldv : ldk;
  const int dlog = a.d == 64 ? 3 : 4;
  const float s = __ldg((kv ? a.scale[1] : a.scale[0]) + p.at);
  const uint2* codes = reinterpret_cast<const uint2*>((kv ? a.codes[1] : a.codes[0]) + (p.at << a.block_log2) * a.d);
  uint2 w[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int v = threadIdx.x + kKvThreads * i, slot = v >> dlog;
    if (slot >= p.old && slot < p.end) w[i] = __ldg(codes + v);
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int v = threadIdx.x + kKvThreads * i, slot = v >> dlog;
    if (slot < p.old || slot >= p.end) continue;
    float lo[4], hi[4];
    codes4(w[i].x, lo);
    codes4(w[i].y, hi);
    reinterpret_cast<uint4*>(X + (p.row0 + slot - p.old) * ld)[v & ((1 << dlog) - 1)] =
        make_uint4(pack_bf16(lo[0] * s, lo[1] * s), pack_bf16(lo[2] * s, lo[3] * s),
                   pack_bf16(hi[0] * s, hi[1] * s), pack_bf16(hi[2] * s, hi[3] * s));
  }
}

}  // namespace

cudaError_t launch_kv_write(const KvArgs& a, const uint16_t* K, int64_t ldk, const uint16_t* V, int64_t ldv,
                            cudaStream_t stream) {
  const int touched = kv_touched_blocks(a);
  const dim3 grid(static_cast<unsigned>(touched) * 2 * a.heads, a.n_seqs);
  switch ((a.d << a.block_log2) / 1024) {
    case 1: kv_write_kernel<1><<<grid, kKvThreads, 0, stream>>>(a, K, ldk, V, ldv); break;
    case 2: kv_write_kernel<2><<<grid, kKvThreads, 0, stream>>>(a, K, ldk, V, ldv); break;
    case 4: kv_write_kernel<4><<<grid, kKvThreads, 0, stream>>>(a, K, ldk, V, ldv); break;
    case 8: kv_write_kernel<8><<<grid, kKvThreads, 0, stream>>>(a, K, ldk, V, ldv); break;
    default: kv_write_kernel<16><<<grid, kKvThreads, 0, stream>>>(a, K, ldk, V, ldv); break;
  }
  return cudaGetLastError();
}

cudaError_t launch_kv_read(const KvArgs& a, uint16_t* K, int64_t ldk, uint16_t* V, int64_t ldv, cudaStream_t stream) {
  const int touched = kv_touched_blocks(a);
  const dim3 grid(static_cast<unsigned>(touched) * 2 * a.heads, a.n_seqs);
  switch ((a.d << a.block_log2) / 1024) {
    case 1: kv_read_kernel<1><<<grid, kKvThreads, 0, stream>>>(a, K, ldk, V, ldv); break;
    case 2: kv_read_kernel<2><<<grid, kKvThreads, 0, stream>>>(a, K, ldk, V, ldv); break;
    case 4: kv_read_kernel<4><<<grid, kKvThreads, 0, stream>>>(a, K, ldk, V, ldv); break;
    case 8: kv_read_kernel<8><<<grid, kKvThreads, 0, stream>>>(a, K, ldk, V, ldv); break;
    default: kv_read_kernel<16><<<grid, kKvThreads, 0, stream>>>(a, K, ldk, V, ldv); break;
  }
  return cudaGetLastError();
}

}  // namespace lrqat
