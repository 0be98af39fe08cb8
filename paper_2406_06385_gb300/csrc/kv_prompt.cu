// Attention over the 8-bit cache for many (token, head) rows per sequence: tiles of 2 x 128 rows on
// the fifth-generation tensor cores.
//
// The mathematics, and the folding of the value scales into the exponent, are those of kv_attn.cu.
// A thread block takes 256 rows of one sequence and key/value head (rows of a group are neighbours, so
// all heads of a group share the keys) and walks over tiles of 128 keys.  Per key tile:
//   producer warps   turn the int8 codes into halves (exact) in the swizzled layout of the matrix
//                    instructions: [keys][64 dimensions], K read K-major, V read MN-major;
//   two threads      (one per half of the rows) issue S = Q K^T for 64 keys at a time and O += P V with P
//                    read from tensor memory.  A half has two score buffers: while its softmax works on
//                    one, the tensor cores fill the other;
//   softmax warps    one thread per row: maximum, P = 2^{z' - m} as halves back into tensor memory, over
//                    the scores they came from.  m is the maximum of the first keys a row sees; it moves (and O
//                    is rescaled) only when a sum of P has grown beyond what half precision holds, so that
//                    most steps look for no maximum at all.
// Scores and O live in tensor memory: 2 x 2 x 64 and 2 x d columns.
//
// Four prompts of up to 4000 tokens behind 500 older ones, 32 query and 8 key/value heads of 128: 513 us,
// 990 TFLOP/s, 53% of the rate of a plain product; behind a window of 1000 tokens and 4 sinks 319 us (floor 117: a block
// has 8.6 tiles of keys; 322 when the others below were measured).  A tile of 256 rows and 128 keys takes about 3700 cycles, its matrix instructions 2033, a step
// whose columns are masked one by one 900 more than another; the first scores come after 12600 cycles (arrays of the
// sequence 2400, barriers 1300, table and codes 3700, q and the keys turned into halves beside each other 3000), and
// behind the last the rows take 5000 to leave.  Of an earlier 524 us, without the softmax's arithmetic the call would
// take 407, without the producers' stores 479, without both 358, almost without matrix instructions still 505.
// Measured against it: two threads a row 686 of 524 (the exchange of their maxima), one 128-key score buffer 834, eight
// producer warps with 136 softmax registers 574; a row of q and of O a thread, not whole lines by the warp, 525 of 513;
// 184, 104 and 40 registers, with spills in the issuing threads, 330 of 322 behind the window (176, 104 and 56 spill none);
// blocks that stay and take over the grid positions of blocks not yet launched, q and keys of the next item brought in
// beside this one's last steps, 549 us where this takes 536 (one tile of long sequences) and 317 where it takes 322 (the
// window).
#include <cuda.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "attn.cuh"
#include "kernels.h"
#include "ptx.cuh"

namespace lrqat {
namespace {

constexpr int kTileKeys = 128;               // keys converted at a time
constexpr int kStepKeys = 64;                // keys of one softmax step: one of a half's two score buffers
constexpr int kGroups = kTileKeys / 16;      // a cache block holds a multiple of 16 tokens
constexpr int kStages = 2;
constexpr int kScaleSlots = 4;
constexpr int kSoftmaxWarps = 8, kProducerWarps = 4, kMmaWarp = kSoftmaxWarps + kProducerWarps;
constexpr int kThreads = 32 * (kMmaWarp + 4);                // four warpgroups; of the last, two warps work
// Registers a thread of each role: over the warpgroups their sum is what the block is launched with.
constexpr int kLaunchRegs = 128, kSoftmaxRegs = 176, kProducerRegs = 104, kMmaRegs = 56;
static_assert(2 * kSoftmaxRegs + kProducerRegs + kMmaRegs <= 4 * kLaunchRegs, "registers of the warpgroups");
constexpr float kMostP = 32768.0f;           // largest sum of 16 P before m follows the maximum
// How far log2 of the value scales may lie from the first one's for P to serve the denominator too.  Against m, which a
// key behind the largest of them may set, P of a key behind the smallest is 2^{-2 kTame} times its share e^z, and P is
// zero below 2^-126: 62 powers of two are left for the share, 31 for the number of keys and 31 for a sum's bits.
constexpr float kTame = 32.0f;

enum : int {
  B_QFULL = 0, B_KFULL = 2, B_VFULL = 4, B_KEMPTY = 6, B_VEMPTY = 8, B_SFULL = 10, B_PFULL = 14, B_OFULL = 18,
  B_SCALES = 20, B_DONE = 24, B_COUNT = 26
};

template <int D>
struct PromptSmem {
  static constexpr uint32_t kBox = 128 * 128;                  // 128 rows of 64 halves
  static constexpr uint32_t kOperand = kBox * (D / 64);        // 128 rows of one operand
  static constexpr uint32_t kQ = 0, kK = 2 * kOperand, kV = kK + kStages * kOperand;
  static constexpr uint32_t kScale = kV + kStages * kOperand;  // [slot][coefficient 8, log2 s_v 8, weight 8]
  static constexpr uint32_t kSlot = 3 * kGroups * 4;
  static constexpr uint32_t kBytes = kScale + kScaleSlots * kSlot + 16;     // and ref
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
// Uses of v stay behind this point, and so behind the wait for the load that fills v.
__device__ __forceinline__ void tmem_ready32(float (&v)[32]) {
#pragma unroll
  for (int i = 0; i < 32; i += 8)
    asm volatile("" : "+f"(v[i]), "+f"(v[i + 1]), "+f"(v[i + 2]), "+f"(v[i + 3]), "+f"(v[i + 4]), "+f"(v[i + 5]),
                      "+f"(v[i + 6]), "+f"(v[i + 7]));
}
__device__ __forceinline__ float ld_shared_f32(uint32_t at) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void st_shared_f32(uint32_t at, float v) {
  asm volatile("st.shared.f32 [%0], %1;" ::"r"(at), "f"(v) : "memory");
}
template <bool kValue>
struct Flag {
  static constexpr bool value = kValue;
};
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// True in one lane of a converged warp; unlike a test of the lane number it tells the compiler that one
// thread is left, whose operands can stay in uniform registers.
__device__ __forceinline__ bool elect_one() {
  uint32_t one;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
  return one != 0;
}
// The lowest n bits; none where n < 0, all where n > 32.
__device__ __forceinline__ uint32_t bits_below(int n) {
  uint32_t r;
  asm("bmsk.clamp.b32 %0, 0, %1;" : "=r"(r) : "r"(max(n, 0)));
  return r;
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ void drain(uint32_t bar, uint64_t timeout_ns) {
  const uint64_t t0 = global_timer_ns();
  while (!mbar_try_wait(bar, 0)) {
    if (global_timer_ns() - t0 > timeout_ns) break;
  }
}

// 16 codes as 16 halves, two 16-byte pieces at `at0` and `at1`.
__device__ __forceinline__ void store_codes(uint32_t at0, uint32_t at1, const uint4& w) {
  const uint32_t x0 = w.x ^ 0x80808080u, x1 = w.y ^ 0x80808080u, x2 = w.z ^ 0x80808080u, x3 = w.w ^ 0x80808080u;
  st_shared_v4(at0, half_codes<0x4140>(x0), half_codes<0x4342>(x0), half_codes<0x4140>(x1), half_codes<0x4342>(x1));
  st_shared_v4(at1, half_codes<0x4140>(x2), half_codes<0x4342>(x2), half_codes<0x4140>(x3), half_codes<0x4342>(x3));
}

template <int D, bool kGeneral>
__device__ __forceinline__ void prompt_block(const AttnArgs& a) {
  using Sm = PromptSmem<D>;
  constexpr uint32_t kBoxes = D / 64;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bars[B_COUNT];
  __shared__ uint32_t tmem_base_s;
  __shared__ volatile int abort_s;
  const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto bar = [&](int i) { return smem_u32(&bars[i]); };

  if (kGeneral && a.across) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // the rows' own keys run beside
  // the longest rows first: the last tile of every sequence and head, then the one before, ...
  const int split = blockIdx.x % a.splits, hb = blockIdx.x / a.splits, h = hb % a.kv.heads, b = hb / a.kv.heads;
  Tile t;
  int rt = blockIdx.y;
  if (!(kGeneral && a.across)) {
    if (!seq_rows(a.kv, b, t.seq)) return;
    rt = (t.seq.n * a.group + a.tile_rows - 1) / a.tile_rows - 1 - static_cast<int>(blockIdx.y);
  }
  if (rt < 0 || !attn_tile<kGeneral>(a, b, rt, t)) return;
  const int ns = tile_splits(a, t);
  if ((split > 0 || (kGeneral && a.keep_parts)) && split >= ns) return;
  const int k0 = t.lo + split * a.chunk, k1 = piece_end(a, t, k0);
  const int tiles = k1 > k0 ? (k1 - k0 + kTileKeys - 1) / kTileKeys : 0;
  const int halves = t.rows - t.r0 > 128 ? 2 : 1;

  if (threadIdx.x == 0) {
    abort_s = 0;
    for (int i = 0; i < 4; ++i) {
      mbar_init(bar(B_SFULL + i), 1);
      mbar_init(bar(B_PFULL + i), 4);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar(B_QFULL + i), 4);
      mbar_init(bar(B_KFULL + i), kProducerWarps);
      mbar_init(bar(B_VFULL + i), kProducerWarps);
      mbar_init(bar(B_KEMPTY + i), halves);
      mbar_init(bar(B_VEMPTY + i), halves);
      mbar_init(bar(B_OFULL + i), 1);
      mbar_init(bar(B_DONE + i), 1);
    }
    for (int i = 0; i < kScaleSlots; ++i) mbar_init(bar(B_SCALES + i), kProducerWarps);
    mbar_fence_init();
  }
  if (warp == kMmaWarp) tmem_alloc(smem_u32(&tmem_base_s), 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_base_s;
  const WaitCtl ctl{&abort_s, a.kv.status, a.timeout_ns};

  if (warp < kSoftmaxWarps) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
    // ------------------------------------------------------------ one thread per row
    const int half = warp >> 2;
    if (half < halves) {
      const int r_in = threadIdx.x & 127, r = t.r0 + 128 * half + r_in, tok = r / a.group;
      bool in = r < t.rows;
      int pos = in ? t.seq.first + tok : -1;
      // rows of the two halves this one's keys are masked against
      int h_lo = t.seq.first + (t.r0 + 128 * half) / a.group;
      const int h_hi = t.seq.first + (min(t.r0 + 128 * half + 128, t.rows) - 1) / a.group;
      float qs;
      {
        // A load takes whole rows, kLanes lanes each.  Every step of this is done for all of a lane's rows before the next, none
        // behind a branch: as a chain of one row after the other it took 9000 cycles of the block, where nothing else runs.
        constexpr int kLanes = D / 8, kTogether = 32 / kLanes;
        const int first = 32 * (warp & 3), sub = lane / kLanes, chunk = lane % kLanes;
        const int last = t.rows - 1 - (t.r0 + 128 * half + first);           // of the warp's rows, the last there is
        uint4 w[kLanes];
        {
          const uint16_t* base = a.Q + t.seq.row0 * a.ldq + static_cast<int64_t>(h) * a.group * D + 8 * chunk;
          int tk[kLanes];
#pragma unroll
          for (int i = 0; i < kLanes; ++i) tk[i] = __shfl_sync(0xffffffffu, tok, min(kTogether * i + sub, max(last, 0)));
#pragma unroll
          for (int i = 0; i < kLanes; ++i) {
            const int rr = t.r0 + 128 * half + first + min(kTogether * i + sub, last);
            w[i] = last < 0 ? make_uint4(0u, 0u, 0u, 0u)
                            : __ldg(reinterpret_cast<const uint4*>(base + tk[i] * a.ldq + (rr - tk[i] * a.group) * D));
          }
        }
        if (kGeneral && a.across) {          // while q is on its way; padding has no part
          pos = find_rows(a.kv, in ? tok : t.seq.n - 1).pos;
          in = in && pos >= 0;
          if (!in) pos = -1;
          h_lo = __reduce_min_sync(0xffffffffu, in ? pos : INT32_MAX);
        }
        const uint32_t rows_in = __ballot_sync(0xffffffffu, in);
        if (rows_in != 0xffffffffu) {
#pragma unroll
          for (int i = 0; i < kLanes; ++i)
            if (!(rows_in >> (kTogether * i + sub) & 1u)) w[i] = make_uint4(0u, 0u, 0u, 0u);
        }
        float top[kLanes];
#pragma unroll
        for (int i = 0; i < kLanes; ++i) {
          float x[8];
          unpack8(w[i], x);
          top[i] = fmaxf(max3(fabsf(x[0]), fabsf(x[1]), fabsf(x[2])), max3(fabsf(x[3]), fabsf(x[4]), fabsf(x[5])));
          top[i] = max3(top[i], fabsf(x[6]), fabsf(x[7]));
        }
        // over a row's lanes; each exchange halves the rows a lane still has, until lane x of them is left with row x
#pragma unroll
        for (int o = kLanes / 2; o > 0; o /= 2)
#pragma unroll
          for (int i = 0; i < o; ++i) {
            const bool up = lane & o;
            const float other = __shfl_xor_sync(0xffffffffu, up ? top[i] : top[i + o], o);
            top[i] = fmaxf(up ? top[i + o] : top[i], other);
          }
        const uint32_t ex = min(max(__float_as_uint(fmaxf(top[0], 0.0f)) >> 23, 1u), 253u);   // exponent of a normal power of two
        qs = __uint_as_float(__shfl_sync(0xffffffffu, ex, lane % kTogether * kLanes + lane / kTogether) << 23);
        // a negative softmax scale moves into q, so that the scores' coefficients are >= 0
        const float scale = a.scale_log2 < 0.0f ? -__uint_as_float((254u - ex) << 23) : __uint_as_float((254u - ex) << 23);
        float inv[kLanes];
#pragma unroll
        for (int i = 0; i < kLanes; ++i) inv[i] = __shfl_sync(0xffffffffu, scale, sub * kLanes + i);
        const uint32_t dst = smem + Sm::kQ + half * Sm::kOperand + (chunk / 8) * Sm::kBox;
        // without keys nothing reads them, and the outputs of a warp that is ahead may lie there by now
        if (tiles > 0) {
#pragma unroll
          for (int i = 0; i < kLanes; ++i) {
            float x[8];
            unpack8(w[i], x);
            st_shared_v4(dst + swz_offset(first + kTogether * i + sub, chunk % 8, 128),
                         pack_half(x[0] * inv[i], x[1] * inv[i]), pack_half(x[2] * inv[i], x[3] * inv[i]),
                         pack_half(x[4] * inv[i], x[5] * inv[i]), pack_half(x[6] * inv[i], x[7] * inv[i]));
          }
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(B_QFULL + half));

      const uint32_t lanes = static_cast<uint32_t>(32 * (warp & 3)) << 16;
      const uint32_t t_s = tmem + lanes + 128u * half, t_o = tmem + lanes + 256u + D * half;
      // The denominator is l 2^{m - ref} with ref = log2 of the first value scale: a group's P count with weight
      // 2^{ref - log2 s_v}, which the producers prepare.  Once a scale lies 2^kTame or more away from the first
      // (a weight of -1), P may vanish where a term of the denominator does not: from then on it is l 2^n, summed
      // from exponentials of its own relative to the running maximum n.
      float m = in ? -INFINITY : 0.0f, n = 0.0f, l = 0.0f;
      bool wild = false, ok = true;
      float s[2][32], coef[4], lsv[4], weight[4];
      // scores and scales of step i
      auto fetch = [&](int i) {
        const int j = i >> 1, sub = i & 1;
        ok = wait_bounded(bar(B_SFULL + 2 * half + sub), j & 1u, ctl, 2) &&
             (sub == 1 || wait_bounded(bar(B_SCALES + j % kScaleSlots), (j / kScaleSlots) & 1u, ctl, 1));
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) return;
        tc_fence_after();
        tmem_ld32(t_s + kStepKeys * sub, s[0]);
        tmem_ld32(t_s + kStepKeys * sub + 32, s[1]);
        const uint32_t slot = smem + Sm::kScale + (j % kScaleSlots) * Sm::kSlot + 16 * sub;
        const uint4 c = ld_shared_v4(slot), v = ld_shared_v4(slot + 4 * kGroups), w = ld_shared_v4(slot + 8 * kGroups);
        coef[0] = __uint_as_float(c.x) * qs, coef[1] = __uint_as_float(c.y) * qs;
        coef[2] = __uint_as_float(c.z) * qs, coef[3] = __uint_as_float(c.w) * qs;
        lsv[0] = __uint_as_float(v.x), lsv[1] = __uint_as_float(v.y), lsv[2] = __uint_as_float(v.z), lsv[3] = __uint_as_float(v.w);
        weight[0] = __uint_as_float(w.x), weight[1] = __uint_as_float(w.y);
        weight[2] = __uint_as_float(w.z), weight[3] = __uint_as_float(w.w);
        tmem_ld_wait();
        tmem_ready32(s[0]);
        tmem_ready32(s[1]);
      };
      if (tiles > 0) fetch(0);
      for (int i = 0; i < 2 * tiles && ok; ++i) {
        const int sub = i & 1;
        const uint32_t t_p = t_s + kStepKeys * sub;      // this step's scores and, over them, its P
        const int number = k0 + i * kStepKeys, key = kGeneral ? number + t.gap : number;
        const bool all = key + kStepKeys - 1 <= h_lo &&
                         (a.window == 0 || key > h_hi - a.window || (kGeneral && number + kStepKeys <= a.sinks));
        const int c_hi = pos - key;                      // columns c_lo .. c_hi of this row are visible
        const int c_lo = a.window > 0 ? c_hi - a.window + 1 : 0;
        const int c_sink = kGeneral ? a.sinks - number : 0;   // and those before c_sink
        uint32_t see[2] = {};                            // bit c of word u: column 32 u + c
        if (!all) {
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            see[u] = ~bits_below(c_lo - 32 * u);
            if (kGeneral) see[u] |= bits_below(c_sink - 32 * u);
            see[u] &= bits_below(c_hi + 1 - 32 * u);
#pragma unroll
            for (int c = 0; c < 32; ++c)
              if (!(see[u] >> c & 1u)) s[u][c] = -INFINITY;
          }
        }
        if (fminf(fminf(weight[0], weight[1]), fminf(weight[2], weight[3])) < 0.0f || wild) {
          const uint32_t slot = smem + Sm::kScale + ((i >> 1) % kScaleSlots) * Sm::kSlot + 16 * sub;
          const float was = wild ? n : finite_max(m) - ld_shared_f32(smem + Sm::kScale + kScaleSlots * Sm::kSlot);
          wild = true;
          float n1 = l == 0.0f ? -INFINITY : was;
#pragma unroll 1
          for (int turn = 0; turn < 2; ++turn) {         // the largest z, then the sum
#pragma unroll 1
            for (int u = 0; u < 4; ++u) {
              const float cu = ld_shared_f32(slot + 4 * u) * qs;
              const bool block = ld_shared_f32(slot + 8 * kGroups + 4 * u) != 0.0f;   // weight 0: no block
              float x[16];
              tmem_ld16(t_p + 16 * u, x);
              tmem_ld_wait();
#pragma unroll
              for (int e = 0; e < 16; ++e) {             // hidden keys and groups without a block add nothing
                const bool seen =
                    block && (all || (16 * u + e <= c_hi && (16 * u + e >= c_lo || (kGeneral && 16 * u + e < c_sink))));
                if (turn == 0) n1 = seen ? fmaxf(n1, x[e] * cu) : n1;
                else l += seen ? ex2(fmaf(x[e], cu, -n)) : 0.0f;
              }
            }
            if (turn == 0) {
              n = finite_max(n1);
              l = l == 0.0f ? 0.0f : l * ex2(was - n);
            }
          }
        }
        // P relative to the m so far.  The row's maximum is only looked for where there is none yet, or where a sum of
        // P shows that scores have outrun m beyond what half precision holds.
        float part[4], base;                             // a group's sum of P
        bool look = __any_sync(0xffffffffu, m == -INFINITY);
#pragma unroll 1
        for (int turn = 0; turn < 2; ++turn) {
          if (look) {
            float mx = -INFINITY;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              const float* v = &s[u / 2][16 * (u % 2)];
              float g0 = max3(v[0], v[1], v[2]), g1 = max3(v[3], v[4], v[5]);
              g0 = max3(g0, v[6], v[7]), g1 = max3(g1, v[8], v[9]);
              g0 = max3(g0, v[10], v[11]), g1 = max3(g1, v[12], v[13]);
              mx = fmaxf(mx, fmaf(max3(g0, g1, fmaxf(v[14], v[15])), coef[u], lsv[u]));
            }
            const float m1 = fmaxf(m, mx), alpha = ex2(m - finite_max(m1));
            if (!wild) l *= alpha;
            if (i > 0) {
              // of the products' phases only step i - 1's can be open: this step's scores have arrived, and they were
              // issued behind step i - 2's product
              ok = wait_bounded(bar(B_OFULL + half), (i - 1) & 1u, ctl, 3);
              ok = __all_sync(0xffffffffu, ok);
              if (!ok) break;
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
          }
          base = finite_max(m);
          auto weights = [&](auto masked) {
#pragma unroll
            for (int c = 0; c < kStepKeys; c += 32) {
              uint32_t p[16];
#pragma unroll
              for (int u = 0; u < 2; ++u) {
                const float cu = coef[c / 16 + u], du = lsv[c / 16 + u] - base;
                const float* v = &s[c / 32][16 * u];
                float2 sum = make_float2(0.0f, 0.0f);
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                  float2 x = __ffma2_rn(make_float2(v[e], v[e + 1]), make_float2(cu, cu), make_float2(du, du));
                  if (decltype(masked)::value) {         // a coefficient of 0 or NaN must not bring a hidden key back
                    x.x = see[c / 32] >> (16 * u + e) & 1u ? x.x : -INFINITY;
                    x.y = see[c / 32] >> (16 * u + e + 1) & 1u ? x.y : -INFINITY;
                  }
                  x.x = ex2(x.x);
                  x.y = ex2(x.y);
                  sum = __fadd2_rn(sum, x);
                  p[8 * u + e / 2] = pack_half(x.x, x.y);
                }
                part[c / 16 + u] = sum.x + sum.y;
              }
              tmem_st16(t_p + c / 2, p);
            }
          };
          if (all) weights(Flag<false>{});
          else weights(Flag<true>{});
          look = __any_sync(0xffffffffu, fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3])) > kMostP);
          if (!look) break;
        }
        if (!ok) break;
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(B_PFULL + 2 * half + sub));
        if (!wild) l += fmaf(part[0], weight[0], part[1] * weight[1]) + fmaf(part[2], weight[2], part[3] * weight[3]);
        if (i + 1 < 2 * tiles) fetch(i + 1);
      }
      if (!wild) n = m == -INFINITY ? 0.0f : m - ld_shared_f32(smem + Sm::kScale + kScaleSlots * Sm::kSlot);
      if (tiles > 0) {
        ok = ok && wait_bounded(bar(B_DONE + half), 0u, ctl, 4);
        ok = __all_sync(0xffffffffu, ok);
        tc_fence_after();
      }
      if (ok) {
        const int64_t slot = ((((static_cast<int64_t>(b) * a.kv.heads + h) * a.row_tiles + rt) * a.splits + split) * a.tile_rows) +
                             128 * half + r_in;
        const bool whole = ns <= 1 && !(kGeneral && a.keep_parts);
        const float f = whole ? out_factor(l, m - n) : 1.0f;
        const uint32_t rows_in = __ballot_sync(0xffffffffu, in);
        // A thread's row goes through the half's part of Q, which nothing reads any more, so that a store takes whole lines
        // of few rows; the 16-byte pieces of a row lie in an order of its own, for distinct banks.
        const uint32_t stage = smem + Sm::kQ + half * Sm::kOperand;
        auto out_row = [&](int c, float (&o)[32]) {
          if (tiles > 0) {
            tmem_ld32(t_o + c, o);
            tmem_ld_wait();
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = 0.0f;
          }
        };
        if (whole) {
          constexpr int kLanes = D / 8, kTogether = 32 / kLanes;
          const int sub = lane / kLanes, chunk = lane % kLanes;
#pragma unroll 1
          for (int c = 0; c < D; c += 32) {
            float o[32];
            out_row(c, o);
#pragma unroll
            for (int e = 0; e < 32; e += 8) {
              float v[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) v[i] = o[e + i] * f;
              const uint4 x = pack8(v);
              st_shared_v4(stage + r_in * (2 * D) + (((c + e) / 8) ^ (r_in & 7)) * 16, x.x, x.y, x.z, x.w);
            }
          }
          __syncwarp();
#pragma unroll 4
          for (int i = 0; i < kLanes; ++i) {
            const int k = kTogether * i + sub, row = r_in - lane + k, rr = r - lane + k;
            const int tk = __shfl_sync(0xffffffffu, tok, k);
            const uint4 x = ld_shared_v4(stage + row * (2 * D) + (chunk ^ (row & 7)) * 16);
            if (rows_in >> k & 1u)
              reinterpret_cast<uint4*>(a.O + (t.seq.row0 + tk) * a.ldo + static_cast<int64_t>(h * a.group + rr - tk * a.group) * D)[chunk] = x;
          }
        } else {
          float4* part = reinterpret_cast<float4*>(a.part + (slot - lane) * D);
#pragma unroll 1
          for (int c = 0; c < D; c += 32) {
            const uint32_t box = stage + c / 32 % 2 * Sm::kBox * (D / 128);
            float o[32];
            out_row(c, o);
            if (D == 64) __syncwarp();
#pragma unroll
            for (int e = 0; e < 8; ++e)
              st_shared_v4(box + r_in * 128 + (e ^ (r_in & 7)) * 16, __float_as_uint(o[4 * e]), __float_as_uint(o[4 * e + 1]),
                           __float_as_uint(o[4 * e + 2]), __float_as_uint(o[4 * e + 3]));
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int k = 4 * i + (lane >> 3), row = r_in - lane + k;
              const uint4 x = ld_shared_v4(box + row * 128 + ((lane & 7) ^ (row & 7)) * 16);
              if (rows_in >> k & 1u)
                part[k * (D / 4) + c / 4 + (lane & 7)] =
                    make_float4(__uint_as_float(x.x), __uint_as_float(x.y), __uint_as_float(x.z), __uint_as_float(x.w));
            }
          }
        }
        if (!whole && in)
          *reinterpret_cast<float4*>(a.part_stat + slot * 4) = make_float4(m, l == 0.0f ? -INFINITY : n, l, 0.0f);
      }
    }
  } else if (warp < kMmaWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kProducerRegs));
    // ------------------------------------------------------------ codes into operands
    // A warp has 32 tokens of the tile, two groups of 16.  A load instruction takes 64 bytes of 8 tokens:
    // four lanes a token, so that the stores of 8 lanes (two rows) hit distinct banks.
    const int w = warp - kSoftmaxWarps;
    const uint32_t piece = lane & 3, row = lane >> 2;
    const uint32_t in_block = (1u << a.kv.block_log2) - 1;
    const int32_t* table = a.kv.table + static_cast<int64_t>(b) * a.kv.max_blocks;
    // lanes 0 and 1: the cache block of the warp's group `lane` of a tile (-1: none, -2: past the keys)
    auto block_of = [&](int j) {
      const int key = k0 + j * kTileKeys + 32 * w + 16 * (lane & 1);
      if (j >= tiles || key >= k1) return -2;
      const int blk = group_block<kGeneral>(a, t, table, key);
      return static_cast<uint32_t>(blk) < static_cast<uint64_t>(a.kv.n_blocks) ? blk : -1;
    };
    uint4 kr[4 * kBoxes], vr[4 * kBoxes];
    auto load = [&](uint4 (&reg)[4 * kBoxes], const int8_t* codes, int j, int blk) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int bu = __shfl_sync(0xffffffffu, blk, u);
        const int key = key_at<kGeneral>(a, t, k0 + j * kTileKeys + 32 * w + 16 * u);
        const int64_t at = static_cast<int64_t>(bu) * a.kv.heads + h;
        const int8_t* p = codes + ((at << a.kv.block_log2) + (key & in_block) + row) * D + 16 * piece;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (uint32_t x = 0; x < kBoxes; ++x)
            reg[(2 * u + i) * kBoxes + x] =
                bu >= 0 ? __ldg(reinterpret_cast<const uint4*>(p + 8 * i * D + 64 * x)) : make_uint4(0u, 0u, 0u, 0u);
      }
    };
    // row 32 w + 8 i + row of a box: the swizzle depends on the row within 8 alone
    const uint32_t off0 = (32 * w + row) * 128 + ((2 * piece) ^ row) * 16, off1 = off0 ^ 16u;
    auto store = [&](const uint4 (&reg)[4 * kBoxes], uint32_t operand) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (uint32_t x = 0; x < kBoxes; ++x)
          store_codes(operand + off0 + (x * Sm::kBox + 1024 * i), operand + off1 + (x * Sm::kBox + 1024 * i),
                      reg[i * kBoxes + x]);
    };
    auto scale_of = [&](const float* scale, int blk) {
      return lane < 2 && blk >= 0 ? __ldg(scale + static_cast<int64_t>(blk) * a.kv.heads + h) : 0.0f;
    };
    int blk = block_of(0), blk_next = block_of(1);
    float sk = scale_of(a.kv.scale[0], blk), sv = scale_of(a.kv.scale[1], blk);
    load(kr, a.kv.codes[0], 0, blk);
    load(vr, a.kv.codes[1], 0, blk);
    // log2 of the value scale of the first key's block, 0 where that has none
    float ref = 0.0f;
    if (tiles > 0) {
      const int first = table_entry<kGeneral>(a, table, key_at<kGeneral>(a, t, k0));
      const float v = scale_of(a.kv.scale[1], static_cast<uint32_t>(first) < static_cast<uint64_t>(a.kv.n_blocks) ? first : -1);
      ref = v > 0.0f && v < INFINITY ? lg2(v) : 0.0f;
    }
    if (w == 0 && lane == 0) st_shared_f32(smem + Sm::kScale + kScaleSlots * Sm::kSlot, ref);
    bool ok = true;
    for (int j = 0; j < tiles; ++j) {
      const uint32_t stage = j % kStages, par = ((j / kStages) & 1u) ^ 1u;
      // the scales' slot was last read four tiles ago: the scores of two tiles ago, which freed this stage,
      // were computed after the softmax of three tiles ago
      ok = wait_bounded(bar(B_KEMPTY + stage), par, ctl, 5);
      if (!__all_sync(0xffffffffu, ok)) break;
      if (lane < 2) {
        if (blk == -1) atomicOr(a.kv.status, kStatusRange);
        const uint32_t at = smem + Sm::kScale + (j % kScaleSlots) * Sm::kSlot + 4 * (2 * w + lane);
        const float v = blk >= 0 ? lg2(sv) : -INFINITY, away = ref - v;
        st_shared_f32(at, blk >= 0 ? fabsf(a.scale_log2) * sk : 0.0f);
        st_shared_f32(at + 4 * kGroups, v);
        // 0: no block; NaN: its P are NaN themselves where they are seen; a value scale of 0 is an infinity away:
        // its keys add nothing to O and their share to the denominator
        st_shared_f32(at + 8 * kGroups, blk < 0 ? 0.0f : away != away ? 1.0f : fabsf(away) < kTame ? ex2(away) : -1.0f);
      }
      store(kr, smem + Sm::kK + stage * Sm::kOperand);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(bar(B_SCALES + j % kScaleSlots));
        mbar_arrive(bar(B_KFULL + stage));
      }
      blk = blk_next;
      blk_next = block_of(j + 2);
      load(kr, a.kv.codes[0], j + 1, blk);
      sk = scale_of(a.kv.scale[0], blk);
      sv = scale_of(a.kv.scale[1], blk);
      ok = wait_bounded(bar(B_VEMPTY + stage), par, ctl, 6);
      if (!__all_sync(0xffffffffu, ok)) break;
      store(vr, smem + Sm::kV + stage * Sm::kOperand);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(B_VFULL + stage));
      load(vr, a.kv.codes[1], j + 1, blk);
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kMmaRegs));
    // one thread per row half
    const int half = warp - kMmaWarp;
    if (half < halves && elect_one()) {
      const uint32_t idesc_s = make_idesc_f16(128, kStepKeys, 0), idesc_o = make_idesc_f16(128, D, 1);
      const uint64_t d_q = make_sdesc(smem + Sm::kQ + half * Sm::kOperand, 16, 1024, SWZ_128B);
      const uint64_t d_k = make_sdesc(smem + Sm::kK, 16, 1024, SWZ_128B);
      const uint64_t d_v = make_sdesc(smem + Sm::kV, Sm::kBox, 1024, SWZ_128B);
      const uint32_t t_s = tmem + 128u * half, t_o = tmem + 256u + D * half;
      auto scores = [&](uint32_t stage, uint32_t sub) {
#pragma unroll
        for (uint32_t ks = 0; ks < D / 16; ++ks) {
          const uint32_t off = (Sm::kBox * (ks >> 2) + 32u * (ks & 3)) >> 4;
          mma_bf16(t_s + kStepKeys * sub, d_q + off, d_k + stage * (Sm::kOperand >> 4) + sub * (kStepKeys * 128 >> 4) + off,
                   idesc_s, ks > 0 ? 1u : 0u);
        }
        mma_commit(bar(B_SFULL + 2 * half + sub));
      };
      bool ok = tiles > 0 && wait_bounded(bar(B_QFULL + half), 0, ctl, 7) && wait_bounded(bar(B_KFULL), 0, ctl, 8);
      if (ok) {
        tc_fence_after();
        scores(0, 0);
        scores(0, 1);
        mma_commit(bar(B_KEMPTY));
      }
      for (int j = 0; j < tiles && ok; ++j) {
        const uint32_t stage = j % kStages, next = (j + 1) % kStages;
        ok = wait_bounded(bar(B_VFULL + stage), (j / kStages) & 1u, ctl, 9);
        for (uint32_t sub = 0; sub < 2 && ok; ++sub) {
          if (!(ok = wait_bounded(bar(B_PFULL + 2 * half + sub), j & 1u, ctl, 10))) break;
          tc_fence_after();
#pragma unroll
          for (uint32_t ks = 0; ks < kStepKeys / 16; ++ks)
            mma_f16_ts(t_o, t_s + kStepKeys * sub + 8 * ks, d_v + stage * (Sm::kOperand >> 4) + 128 * (4 * sub + ks), idesc_o,
                       j > 0 || sub > 0 || ks > 0 ? 1u : 0u);
          mma_commit(bar(B_OFULL + half));
          if (sub == 1) mma_commit(bar(B_VEMPTY + stage));
          if (j + 1 < tiles) {
            if (sub == 0 && !(ok = wait_bounded(bar(B_KFULL + next), ((j + 1) / kStages) & 1u, ctl, 11))) break;
            tc_fence_after();
            scores(next, sub);                           // in order after the product that reads P from the same columns
            if (sub == 1) mma_commit(bar(B_KEMPTY + next));
          }
        }
      }
      // every matrix instruction has completed: O is read, and the memories are released
      mma_commit(bar(B_DONE + half));
      drain(bar(B_DONE + half), a.timeout_ns);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kMmaWarp) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

template <int D, bool kGeneral>
__global__ void __launch_bounds__(kThreads, 1) kv_prompt_kernel(AttnArgs a) {
  prompt_block<D, kGeneral>(a);
  if (kGeneral && a.keep_parts && blockIdx.x == 0 && blockIdx.y == 0) finish_behind();
}

template <int D, bool kGeneral>
cudaError_t launch(const AttnArgs& a, cudaStream_t stream) {
  static bool smem_set[kMaxDevices];
  constexpr int bytes = PromptSmem<D>::kBytes + 1024;
  const cudaError_t e = ensure_smem_attr(reinterpret_cast<const void*>(kv_prompt_kernel<D, kGeneral>), bytes, smem_set);
  if (e != cudaSuccess) return e;
  const dim3 grid(static_cast<unsigned>(a.splits) * a.kv.heads * attn_grid_seqs(a), a.row_tiles);
  return launch_lined_up(kv_prompt_kernel<D, kGeneral>, grid, kThreads, bytes, a.behind, stream, a);
}

}  // namespace

cudaError_t launch_kv_prompt(const AttnArgs& a, cudaStream_t stream) {
  if (attn_general(a)) return a.kv.d == 128 ? launch<128, true>(a, stream) : launch<64, true>(a, stream);
  return a.kv.d == 128 ? launch<128, false>(a, stream) : launch<64, false>(a, stream);
}

}  // namespace lrqat
