// Attention over the 8-bit cache for many (token, head) rows per sequence: tiles of 2 x 128 rows on
// the fifth-generation tensor cores.
//
// The mathematics, and the folding of the value scales into the exponent, are those of kv_attn.cu.
// A thread block takes 256 rows of one sequence and key/value head (rows of a group are neighbours, so
// all heads of a group share the keys) and walks over tiles of 128 keys.  Per key tile:
//   producer warps   turn the int8 codes into halves (exact) in the swizzled layout of the matrix
//                    instructions: [keys][64 dimensions], K read K-major, V read MN-major;
//   one thread       issues S = Q K^T (128 x 128 per row half) and O += P V with P read from tensor
//                    memory, alternating the two row halves: while one half's softmax runs, the tensor
//                    cores work on the other;
//   softmax warps    one thread per row: maximum, P = 2^{z' - m} as halves back into tensor memory, over
//                    the scores they came from.  m moves only when a row's maximum has grown by more than
//                    2^8 (P <= 256 is exact enough in half precision and fits), so O is rarely rescaled.
// Scores and O live in tensor memory: 2 x 128 and 2 x d columns.
#include <cuda.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "attn.cuh"
#include "kernels.h"
#include "ptx.cuh"

namespace lrqat {
namespace {

constexpr int kTileKeys = 128;
constexpr int kGroups = kTileKeys / 16;      // a cache block holds a multiple of 16 tokens
constexpr int kStages = 2;
constexpr int kScaleSlots = 4;
constexpr int kSoftmaxWarps = 8, kProducerWarps = 4;
constexpr int kThreads = 32 * (kSoftmaxWarps + kProducerWarps + 1);
constexpr float kLazy = 8.0f;                // how far a maximum may run ahead of m
constexpr float kTame = 64.0f;               // spread of log2 of the value scales that one exponential serves

enum : int {
  B_QFULL = 0, B_KFULL = 2, B_VFULL = 4, B_KEMPTY = 6, B_VEMPTY = 8, B_SFULL = 10, B_PFULL = 12, B_OFULL = 14,
  B_SCALES = 16, B_DRAIN = 20, B_COUNT = 21
};

template <int D>
struct PromptSmem {
  static constexpr uint32_t kBox = 128 * 128;                  // 128 rows of 64 halves
  static constexpr uint32_t kOperand = kBox * (D / 64);        // 128 rows of one operand
  static constexpr uint32_t kQ = 0, kK = 2 * kOperand, kV = kK + kStages * kOperand;
  static constexpr uint32_t kScale = kV + kStages * kOperand;  // [slot][coef 8, log2 s_v 8]
  static constexpr uint32_t kBytes = kScale + kScaleSlots * 2 * kGroups * 4;
};

// D[tmem] (+)= A[tmem] B[smem], kind::f16: A's row r in lane r, two halves a column.
__device__ __forceinline__ void mma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc,
                                           uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Instruction descriptor, kind::f16: D fp32, A and B f16, A K-major.
__host__ __device__ constexpr uint32_t make_idesc_f16(int M, int N, int b_mn) {
  return (1u << 4) | (static_cast<uint32_t>(b_mn) << 16) | (static_cast<uint32_t>(N >> 3) << 17) |
         (static_cast<uint32_t>(M >> 4) << 24);
}
// 32 lanes x 32 bits, 16 consecutive columns per thread.
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
        "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ void drain(uint32_t bar, uint64_t timeout_ns) {
  const uint64_t t0 = global_timer_ns();
  while (!mbar_try_wait(bar, 0)) {
    if (global_timer_ns() - t0 > timeout_ns) break;
  }
}

// 16 codes as 16 halves: two 16-byte pieces.
__device__ __forceinline__ void store_codes(uint32_t box, uint32_t row, uint32_t piece, const uint4& w) {
  const uint32_t x[4] = {w.x ^ 0x80808080u, w.y ^ 0x80808080u, w.z ^ 0x80808080u, w.w ^ 0x80808080u};
#pragma unroll
  for (uint32_t i = 0; i < 2; ++i)
    st_shared_v4(box + swz_offset(row, 2 * piece + i, 128), half_codes<0x4140>(x[2 * i]), half_codes<0x4342>(x[2 * i]),
                 half_codes<0x4140>(x[2 * i + 1]), half_codes<0x4342>(x[2 * i + 1]));
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1) kv_prompt_kernel(AttnArgs a) {
  using Sm = PromptSmem<D>;
  constexpr uint32_t kBoxes = D / 64;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bars[B_COUNT];
  __shared__ uint32_t tmem_base_s;
  __shared__ volatile int abort_s;
  const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto bar = [&](int i) { return smem_u32(&bars[i]); };

  // the longest rows first: the last tile of every sequence and head, then the one before, ...
  const int split = blockIdx.x % a.splits, hb = blockIdx.x / a.splits, h = hb % a.kv.heads, b = hb / a.kv.heads;
  Tile t;
  if (!seq_rows(a.kv, b, t.seq)) return;
  const int rt = (t.seq.n * a.group + a.tile_rows - 1) / a.tile_rows - 1 - static_cast<int>(blockIdx.y);
  if (rt < 0 || !attn_tile(a, b, rt, t)) return;
  const int ns = tile_splits(a, t);
  if (split > 0 && split >= ns) return;
  const int k0 = t.lo + split * a.chunk, k1 = min(t.hi, k0 + a.chunk);
  const int tiles = k1 > k0 ? (k1 - k0 + kTileKeys - 1) / kTileKeys : 0;
  const int halves = t.rows - t.r0 > 128 ? 2 : 1;

  if (threadIdx.x == 0) {
    abort_s = 0;
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar(B_QFULL + i), 4);
      mbar_init(bar(B_KFULL + i), kProducerWarps);
      mbar_init(bar(B_VFULL + i), kProducerWarps);
      mbar_init(bar(B_KEMPTY + i), 1);
      mbar_init(bar(B_VEMPTY + i), 1);
      mbar_init(bar(B_SFULL + i), 1);
      mbar_init(bar(B_PFULL + i), 4);
      mbar_init(bar(B_OFULL + i), 1);
    }
    for (int i = 0; i < kScaleSlots; ++i) mbar_init(bar(B_SCALES + i), kProducerWarps);
    mbar_init(bar(B_DRAIN), 1);
    mbar_fence_init();
  }
  if (warp == kSoftmaxWarps + kProducerWarps) tmem_alloc(smem_u32(&tmem_base_s), 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_base_s;
  const WaitCtl ctl{&abort_s, a.kv.status, a.timeout_ns};

  if (warp < kSoftmaxWarps) {
    // ------------------------------------------------------------ one thread per row
    const int half = warp >> 2;
    if (half < halves) {
      const int r_in = threadIdx.x & 127, r = t.r0 + 128 * half + r_in, tok = r / a.group;
      const bool in = r < t.rows;
      const int pos = in ? t.seq.first + tok : -1;
      // rows of the two halves this one's keys are masked against
      const int h_lo = t.seq.first + (t.r0 + 128 * half) / a.group;
      const int h_hi = t.seq.first + (min(t.r0 + 128 * half + 128, t.rows) - 1) / a.group;
      float qs;
      {
        const uint4* q = reinterpret_cast<const uint4*>(a.Q + (t.seq.row0 + tok) * a.ldq +
                                                        static_cast<int64_t>(h * a.group + r % a.group) * D);
        uint4 w[D / 8];
        float top = 0.0f;
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
          w[i] = in ? __ldg(q + i) : make_uint4(0u, 0u, 0u, 0u);
          float x[8];
          unpack8(w[i], x);
#pragma unroll
          for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[e]));
        }
        const uint32_t ex = min(max(__float_as_uint(top) >> 23, 1u), 253u);   // exponent of a normal power of two
        qs = __uint_as_float(ex << 23);
        // a negative softmax scale moves into q, so that the scores' coefficients are >= 0
        const float inv = a.scale_log2 < 0.0f ? -__uint_as_float((254u - ex) << 23) : __uint_as_float((254u - ex) << 23);
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
          float x[8];
          unpack8(w[i], x);
          st_shared_v4(smem + Sm::kQ + half * Sm::kOperand + (i / 8) * Sm::kBox + swz_offset(r_in, i % 8, 128),
                       pack_half(x[0] * inv, x[1] * inv), pack_half(x[2] * inv, x[3] * inv),
                       pack_half(x[4] * inv, x[5] * inv), pack_half(x[6] * inv, x[7] * inv));
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(B_QFULL + half));

      const uint32_t lanes = static_cast<uint32_t>(32 * (warp & 3)) << 16;
      const uint32_t t_s = tmem + lanes + 128u * half, t_o = tmem + lanes + 256u + D * half;
      float m = -INFINITY, n = -INFINITY, l = 0.0f;
      float lv_min = INFINITY, lv_max = -INFINITY;       // log2 of the value scales so far
      bool ok = true;
      for (int j = 0; j < tiles; ++j) {
        ok = wait_bounded(bar(B_SCALES + j % kScaleSlots), (j / kScaleSlots) & 1u, ctl, 1) &&
             wait_bounded(bar(B_SFULL + half), j & 1u, ctl, 2);
        if (!__all_sync(0xffffffffu, ok)) break;
        tc_fence_after();
        float coef[kGroups], lsv[kGroups];
        float tile_min = INFINITY, tile_max = -INFINITY;
        const uint32_t slot = smem + Sm::kScale + (j % kScaleSlots) * 2 * kGroups * 4;
#pragma unroll
        for (int i = 0; i < kGroups; i += 4) {
          const uint4 c = ld_shared_v4(slot + 4 * i), v = ld_shared_v4(slot + 4 * (kGroups + i));
          const uint32_t cc[4] = {c.x, c.y, c.z, c.w}, vv[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            coef[i + e] = __uint_as_float(cc[e]) * qs;
            lsv[i + e] = __uint_as_float(vv[e]);
            tile_max = fmaxf(tile_max, lsv[i + e]);
            tile_min = fminf(tile_min, lsv[i + e] == -INFINITY ? INFINITY : lsv[i + e]);
          }
        }
        lv_min = fminf(lv_min, tile_min);
        lv_max = fmaxf(lv_max, tile_max);
        const bool tame = lv_max - lv_min < kTame;
        const int key = k0 + j * kTileKeys;
        const bool all = key + kTileKeys - 1 <= h_lo && (a.window == 0 || key > h_hi - a.window);
        const int c_hi = pos - key;                      // columns c_lo .. c_hi of this row are visible
        const int c_lo = a.window > 0 ? pos - a.window + 1 - key : 0;

        // the largest z' (and z) of the row
        float mx = -INFINITY, zx = -INFINITY;
#pragma unroll
        for (int c = 0; c < kTileKeys; c += 32) {
          float s[32];
          tmem_ld32(t_s + c, s);
          tmem_ld_wait();
          if (!all) {
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (c + e > c_hi || c + e < c_lo) s[e] = -INFINITY;
          }
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            float g = s[16 * u];
#pragma unroll
            for (int e = 1; e < 16; ++e) g = fmaxf(g, s[16 * u + e]);
            const float z = g * coef[c / 16 + u];
            zx = fmaxf(zx, z);
            mx = fmaxf(mx, z + lsv[c / 16 + u]);
          }
        }
        const float m1 = mx > m + kLazy || m == -INFINITY ? fmaxf(m, mx) : m;
        const float base = finite_max(m1);
        const float alpha = ex2(m - base);
        if (j > 0 && __any_sync(0xffffffffu, m1 != m)) {
          ok = wait_bounded(bar(B_OFULL + half), (j - 1) & 1u, ctl, 3);
          if (!__all_sync(0xffffffffu, ok)) break;
          tc_fence_after();
#pragma unroll 1
          for (int c = 0; c < D; c += 16) {
            float o[16];
            uint32_t w[16];
            tmem_ld16(t_o + c, o);
            tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 16; ++e) w[e] = __float_as_uint(o[e] * alpha);
            tmem_st16(t_o + c, w);
          }
        }
        m = m1;
        // the denominator relative to 2^n
        const float n1 = tame ? fmaxf(n, m1 - lv_min) : fmaxf(n, zx);
        const float nbase = finite_max(n1);
        l *= ex2(n - nbase);
        n = n1;
#pragma unroll
        for (int c = 0; c < kTileKeys; c += 32) {
          float s[32];
          uint32_t p[16];
          tmem_ld32(t_s + c, s);
          tmem_ld_wait();
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const float cu = coef[c / 16 + u], du = lsv[c / 16 + u] - base;
            float2 sum = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
              float2 x = __ffma2_rn(make_float2(s[16 * u + e], s[16 * u + e + 1]), make_float2(cu, cu), make_float2(du, du));
              if (!all) {
                const int k = c + 16 * u + e;
                if (k > c_hi || k < c_lo) x.x = -INFINITY;
                if (k + 1 > c_hi || k + 1 < c_lo) x.y = -INFINITY;
              }
              x.x = ex2(x.x);
              x.y = ex2(x.y);
              sum = __fadd2_rn(sum, x);
              p[8 * u + e / 2] = pack_half(x.x, x.y);
            }
            if (tame) {
              const float part = sum.x + sum.y;          // a hidden group adds nothing, whatever its scale
              l = part == 0.0f ? l : fmaf(part, ex2(base - lsv[c / 16 + u] - nbase), l);
            }
          }
          if (!tame) {
            // scales far apart: P may vanish where a term of the denominator does not
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              const bool seen = lsv[(c + e) / 16] != -INFINITY && (all || (c + e <= c_hi && c + e >= c_lo));
              l += seen ? ex2(fmaf(s[e], coef[(c + e) / 16], -nbase)) : 0.0f;
            }
          }
          tmem_st16(t_s + c / 2, p);
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(B_PFULL + half));
      }
      if (tiles > 0) {
        ok = ok && wait_bounded(bar(B_OFULL + half), (tiles - 1) & 1u, ctl, 4);
        ok = __all_sync(0xffffffffu, ok);
        tc_fence_after();
      }
      if (ok) {
        const int64_t slot = ((((static_cast<int64_t>(b) * a.kv.heads + h) * a.row_tiles + rt) * a.splits + split) * a.tile_rows) +
                             128 * half + r_in;
        const float f = ns <= 1 ? out_factor(l, finite_max(m) - finite_max(n)) : 1.0f;
        uint16_t* out = a.O + (t.seq.row0 + tok) * a.ldo + static_cast<int64_t>(h * a.group + r % a.group) * D;
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
          float o[32];
          if (tiles > 0) {
            tmem_ld32(t_o + c, o);
            tmem_ld_wait();
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = 0.0f;
          }
          if (!in) continue;
          if (ns <= 1) {
#pragma unroll
            for (int e = 0; e < 32; e += 8) {
              float v[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) v[i] = o[e + i] * f;
              *reinterpret_cast<uint4*>(out + c + e) = pack8(v);
            }
          } else {
#pragma unroll
            for (int e = 0; e < 32; e += 4)
              *reinterpret_cast<float4*>(a.part + slot * D + c + e) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
          }
        }
        if (ns > 1 && in) *reinterpret_cast<float4*>(a.part_stat + slot * 4) = make_float4(m, n, l, 0.0f);
      }
    }
  } else if (warp < kSoftmaxWarps + kProducerWarps) {
    // ------------------------------------------------------------ codes into operands
    // A warp has 32 tokens of the tile, two groups of 16.  A load instruction takes 64 bytes of 8
    // tokens: four lanes a token, so that the stores of 8 lanes (two rows) hit distinct banks.
    const int w = warp - kSoftmaxWarps;
    const uint32_t piece = lane & 3, sub = lane >> 2;
    const uint32_t in_block = (1u << a.kv.block_log2) - 1;
    const int32_t* table = a.kv.table + static_cast<int64_t>(b) * a.kv.max_blocks;
    // lanes 0 and 1: the cache block of the warp's group `lane` of a tile (-1: none, -2: past the keys)
    auto block_of = [&](int j) {
      const int key = k0 + j * kTileKeys + 32 * w + 16 * (lane & 1);
      if (j >= tiles || key >= k1) return -2;
      const int blk = __ldg(table + (key >> a.kv.block_log2));
      return static_cast<uint32_t>(blk) < static_cast<uint64_t>(a.kv.n_blocks) ? blk : -1;
    };
    uint4 kr[4 * kBoxes], vr[4 * kBoxes];
    auto load = [&](uint4 (&reg)[4 * kBoxes], const int8_t* codes, int j, int blk) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int bu = __shfl_sync(0xffffffffu, blk, u);
        const int key = k0 + j * kTileKeys + 32 * w + 16 * u;
        const int64_t at = static_cast<int64_t>(bu) * a.kv.heads + h;
        const int8_t* p = codes + ((at << a.kv.block_log2) + (key & in_block) + sub) * D + 16 * piece;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (uint32_t x = 0; x < kBoxes; ++x)
            reg[(2 * u + i) * kBoxes + x] =
                bu >= 0 ? __ldg(reinterpret_cast<const uint4*>(p + 8 * i * D + 64 * x)) : make_uint4(0u, 0u, 0u, 0u);
      }
    };
    auto store = [&](const uint4 (&reg)[4 * kBoxes], uint32_t operand) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (uint32_t x = 0; x < kBoxes; ++x)
          store_codes(operand + x * Sm::kBox, 32 * w + 8 * i + sub, piece, reg[i * kBoxes + x]);
    };
    auto scale_of = [&](const float* scale, int blk) {
      return lane < 2 && blk >= 0 ? __ldg(scale + static_cast<int64_t>(blk) * a.kv.heads + h) : 0.0f;
    };
    int blk = block_of(0), blk_next = block_of(1);
    float sk = scale_of(a.kv.scale[0], blk), sv = scale_of(a.kv.scale[1], blk);
    load(kr, a.kv.codes[0], 0, blk);
    load(vr, a.kv.codes[1], 0, blk);
    bool ok = true;
    for (int j = 0; j < tiles; ++j) {
      const uint32_t stage = j % kStages, par = ((j / kStages) & 1u) ^ 1u;
      // the scales' slot was last read four tiles ago: the scores of two tiles ago, which freed this stage,
      // were computed after the softmax of three tiles ago
      ok = wait_bounded(bar(B_KEMPTY + stage), par, ctl, 5);
      if (!__all_sync(0xffffffffu, ok)) break;
      if (lane < 2) {
        if (blk == -1) atomicOr(a.kv.status, kStatusRange);
        const uint32_t at = smem + Sm::kScale + (j % kScaleSlots) * 2 * kGroups * 4 + 4 * (2 * w + lane);
        const float c = blk >= 0 ? fabsf(a.scale_log2) * sk : 0.0f, v = blk >= 0 ? lg2(sv) : -INFINITY;
        asm volatile("st.shared.f32 [%0], %1;" ::"r"(at), "f"(c) : "memory");
        asm volatile("st.shared.f32 [%0], %1;" ::"r"(at + 4 * kGroups), "f"(v) : "memory");
      }
      const int cur_next = blk_next;
      store(kr, smem + Sm::kK + stage * Sm::kOperand);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(bar(B_SCALES + j % kScaleSlots));
        mbar_arrive(bar(B_KFULL + stage));
      }
      blk_next = block_of(j + 2);
      load(kr, a.kv.codes[0], j + 1, cur_next);
      sk = scale_of(a.kv.scale[0], cur_next);
      sv = scale_of(a.kv.scale[1], cur_next);
      blk = cur_next;
      ok = wait_bounded(bar(B_VEMPTY + stage), par, ctl, 6);
      if (!__all_sync(0xffffffffu, ok)) break;
      store(vr, smem + Sm::kV + stage * Sm::kOperand);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(B_VFULL + stage));
      load(vr, a.kv.codes[1], j + 1, cur_next);
    }
  } else if (lane == 0) {
    // ------------------------------------------------------------ MMA issuer
    const uint32_t idesc_s = make_idesc_f16(128, kTileKeys, 0), idesc_o = make_idesc_f16(128, D, 1);
    const uint64_t d_q = make_sdesc(smem + Sm::kQ, 16, 1024, SWZ_128B), d_k = make_sdesc(smem + Sm::kK, 16, 1024, SWZ_128B);
    const uint64_t d_v = make_sdesc(smem + Sm::kV, Sm::kBox, 1024, SWZ_128B);
    auto scores = [&](int half, uint32_t stage) {
#pragma unroll
      for (uint32_t ks = 0; ks < D / 16; ++ks) {
        const uint32_t off = (Sm::kBox * (ks >> 2) + 32u * (ks & 3)) >> 4;
        mma_bf16(tmem + 128u * half, d_q + half * (Sm::kOperand >> 4) + off, d_k + stage * (Sm::kOperand >> 4) + off,
                 idesc_s, ks > 0 ? 1u : 0u);
      }
      mma_commit(bar(B_SFULL + half));
    };
    bool ok = true;
    for (int half = 0; half < halves && ok && tiles > 0; ++half) {
      ok = wait_spin_bounded(bar(B_QFULL + half), 0, ctl, 7) && (half > 0 || wait_spin_bounded(bar(B_KFULL), 0, ctl, 8));
      if (!ok) break;
      tc_fence_after();
      scores(half, 0);
      if (half == halves - 1) mma_commit(bar(B_KEMPTY));
    }
    for (int j = 0; j < tiles && ok; ++j) {
      const uint32_t stage = j % kStages, next = (j + 1) % kStages;
      for (int half = 0; half < halves && ok; ++half) {
        ok = (half > 0 || wait_spin_bounded(bar(B_VFULL + stage), (j / kStages) & 1u, ctl, 9)) &&
             wait_spin_bounded(bar(B_PFULL + half), j & 1u, ctl, 10);
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (uint32_t ks = 0; ks < kTileKeys / 16; ++ks)
          mma_f16_ts(tmem + 256u + D * half, tmem + 128u * half + 8 * ks, d_v + stage * (Sm::kOperand >> 4) + 128 * ks,
                     idesc_o, j > 0 || ks > 0 ? 1u : 0u);
        mma_commit(bar(B_OFULL + half));
        if (half == halves - 1) mma_commit(bar(B_VEMPTY + stage));
        if (j + 1 < tiles) {
          ok = half > 0 || wait_spin_bounded(bar(B_KFULL + next), ((j + 1) / kStages) & 1u, ctl, 11);
          if (!ok) break;
          tc_fence_after();
          scores(half, next);                            // in order after the product that reads P from the same columns
          if (half == halves - 1) mma_commit(bar(B_KEMPTY + next));
        }
      }
    }
    // every matrix instruction has completed before the memories are released
    mma_commit(bar(B_DRAIN));
    drain(bar(B_DRAIN), a.timeout_ns);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kSoftmaxWarps + kProducerWarps) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

template <int D>
cudaError_t launch(const AttnArgs& a, cudaStream_t stream) {
  static bool smem_set[kMaxDevices];
  constexpr int bytes = PromptSmem<D>::kBytes + 1024;
  const cudaError_t e = ensure_smem_attr(reinterpret_cast<const void*>(kv_prompt_kernel<D>), bytes, smem_set);
  if (e != cudaSuccess) return e;
  const dim3 grid(static_cast<unsigned>(a.splits) * a.kv.heads * a.kv.n_seqs, a.row_tiles);
  kv_prompt_kernel<D><<<grid, kThreads, bytes, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_kv_prompt(const AttnArgs& a, cudaStream_t stream) {
  return a.kv.d == 128 ? launch<128>(a, stream) : launch<64>(a, stream);
}

}  // namespace lrqat
