// 8-bit GEMM on the 5th-generation tensor cores, operands in e4m3 with a scale for each block of 128:
//   C[m, n] = act( sum_kb sA[m, kb] * sW[n / 128, kb] * (sum over the 128 columns of kb of A[m, k] W[n, k]) + bias[n] )
// with kb the blocks of 128 columns.  A has a scale per row and block, W one per 128 x 128 elements.
//
// The scales are any fp32 numbers, so a block's sum cannot simply go on in the tensor core's accumulator: the MMAs of one block
// (four steps of K = 32, one 128-byte swizzle row) write a TMEM buffer of their own, and the epilogue warps take it into fp32
// registers with one packed FMA per two sums, acc += (sA sW) * sum, while the MMAs of the next block fill the other buffer.  A
// scale is a block's maximum / 448, so what is summed inside a block is bounded by 128 * 448^2 and the sum over the blocks runs
// in fp32 registers, in the order of the blocks.
//
// Two kernels (launch_tc_gemm_fp8 says which runs when):
//  * fp8_pair_kernel for problems that fill the chip: persistent CTA pairs on 256-row tiles (cta_group::2);
//  * fp8_split_kernel for the others: one tile per CTA, the K loop cut over the CTAs of a cluster; with few rows of A the roles of
//    the operands are exchanged, so that a tile is 128 rows of W by 16 rows of A.
#include <cuda.h>

#include "fp8_common.cuh"
#include "hero_internal.h"
#include "tc_common.cuh"

namespace hero {

int make_tmap_bytes(CUtensorMap* m, const void* base, uint64_t rows, uint64_t cols, uint32_t box_rows, bool narrow);

namespace {
using namespace tc;

constexpr int kRows = 128;                       // rows of a tile (of the first operand) per CTA
constexpr int kStepK = kF8Block;                 // a K step is a block of scales: 128 bytes of a row
constexpr int kRowBytes = kRows * kStepK;        // 16 KB
constexpr size_t kAlignSlack = 1024, kBarrierBytes = 512;

enum { kOutF32 = HERO_DTYPE_FP32, kOutBf16 = HERO_DTYPE_BF16, kOutF8 = HERO_DTYPE_E4M3 };

// Everything about the operands' scales and the result that a kernel needs.
struct F8Gemm {
  const float* a_scale;          // [M, kb]
  const float* w_scale;          // [ceil(N / 128), kb]
  const __nv_bfloat16* bias;     // [N] or null
  void* c;                       // [M, N]
  float* c_scale;                // [M, ceil(N / 128)], for e4m3 results
  int M, N, K, act;
  int vec;                       // rows of C start on multiples of: 32, 16 or 0 (less) bytes
};

// GELU-tanh to fp32 accuracy, for every type of result: t (1 + tanh u) / 2 = t / (1 + exp(-2u)), u = sqrt(2 / pi) (t + 0.044715 t^3).
// Four values share one reciprocal, that of the product of their denominators, so that a value costs 1.25 special-function
// instructions; the exponential is cut off at 2^30 to keep that product finite and t at -16 where it multiplies.  Down to -5.5 a value is
// off by less than 100 * 2^-24 of itself (30 * 4 roundings of the exponent, and 14 besides); below, where GELU is smaller than
// 5.2e-9, it comes out between zero and -16 * 2^-30.  (The hardware's tanh, one special-function instruction, does not serve bf16
// results either: 1 + tanh u cancels below zero, so that its 2^-11 is 20 % of the result at t = -3, and minus infinity becomes NaN.
// Scalar arithmetic: packed, the constants take registers that the 128 sums need, and 8774 x 12288 x 3072 454 us for 417.)
__device__ __forceinline__ float gelu_denominator(float t) {
  const float x = t * fmaf(-0.10294324f, t * t, -2.3022082f);        // -2 u log2(e)
  float e;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(fminf(x, 30.f)));
  return 1.0f + e;
}
__device__ __forceinline__ float gelu_factor(float t) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(t), "f"(-16.f));
  return r;
}
__device__ __forceinline__ void gelu4(float2& a, float2& b) {
  const float d0 = gelu_denominator(a.x), d1 = gelu_denominator(a.y), d2 = gelu_denominator(b.x), d3 = gelu_denominator(b.y);
  const float d01 = d0 * d1, d23 = d2 * d3;
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(d01 * d23));
  const float r01 = r * d23, r23 = r * d01;
  a = make_float2(gelu_factor(a.x) * (r01 * d1), gelu_factor(a.y) * (r01 * d0));
  b = make_float2(gelu_factor(b.x) * (r23 * d3), gelu_factor(b.y) * (r23 * d2));
}
// Wait for columns asked for with tmem_ld.  The registers are named behind it, two at a time, so that nothing that uses them moves
// ahead of the wait.
template <int CH>
__device__ __forceinline__ void tmem_wait(uint32_t (&r)[CH]) {
  tmem_ld_wait();
#pragma unroll
  for (int i = 0; i < CH; i += 2) asm volatile("" : "+r"(r[i]), "+r"(r[i + 1]));
}
// acc += s * (NC columns of this thread's TMEM lane), CH columns on their way while CH are added.
template <int NC, int CH>
__device__ __forceinline__ void promote(float2 (&acc)[NC / 2], uint32_t taddr, float s) {
  uint32_t r[2][CH];
  const float2 s2 = make_float2(s, s);
  tmem_ld(taddr, r[0]);
#pragma unroll
  for (int c = 0; c < NC / CH; ++c) {
    tmem_wait(r[c & 1]);
    if (c + 1 < NC / CH) tmem_ld(taddr + (c + 1) * CH, r[(c + 1) & 1]);
#pragma unroll
    for (int i = 0; i < CH / 2; ++i) {
      float2& a = acc[c * (CH / 2) + i];
      a = __ffma2_rn(make_float2(__uint_as_float(r[c & 1][2 * i]), __uint_as_float(r[c & 1][2 * i + 1])), s2, a);
    }
  }
}
// The same for 16 columns with a factor each, that of column c being lane c's `s`.
__device__ __forceinline__ void promote_columns(float2 (&acc)[8], uint32_t taddr, float s) {
  uint32_t r[16];
  tmem_ld16(taddr, r);
  float2 f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = make_float2(__shfl_sync(0xFFFFFFFFu, s, 2 * i), __shfl_sync(0xFFFFFFFFu, s, 2 * i + 1));
  tmem_wait(r);
#pragma unroll
  for (int i = 0; i < 8; ++i)
    acc[i] = __ffma2_rn(make_float2(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1])), f[i], acc[i]);
}

// The scales of A that a warp needs, R rows by the next 16 K blocks, in shared memory of its own.  A row's scales lie side by side
// and the rows do not: 16 lanes fetch 16 blocks of one row (64 bytes) and put them down transposed, so that lane r then finds its
// row's scales block by block without bank conflicts.  A thread that loads its own row's scale, block by block, touches 32 lines a
// load: 8774 x 12288 x 3072 took 672 us when it asked one block ahead, and the loads alone kept the promotion from its pace
// when it asked seven ahead.  Two windows: one is filled while the other is used.
template <int R, int W>
struct ScaleWindow {
  static constexpr int kBlocks = W;
  static constexpr int kFloats = 2 * W * (R + 1);
  float* buf;
  const float* scale;            // of A
  int M, k_blocks, lane;
  // Rows row0.. (past the end: the last one's), blocks from kb0 on as far as they go below kb_end, into window w.
  __device__ __forceinline__ void fetch(uint32_t w, int row0, int kb0, int kb_end) const {
    const int c = lane & (W - 1), kb = kb0 + c;
    if (kb < kb_end) {
      const uint32_t to = smem_u32(buf + ((w & 1) * W + c) * (R + 1));
#pragma unroll
      for (int i = 0; i < R * W / 32; ++i) {
        const int r = i * (32 / W) + lane / W;
        const float* from = scale + (long long)min(row0 + r, M - 1) * k_blocks + kb;
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to + r * 4), "l"(from) : "memory");
      }
    }
  }
  // All that was asked for is there, for every lane of the warp.
  static __device__ __forceinline__ void arrived() {
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncwarp();
  }
  __device__ __forceinline__ float at(uint32_t w, int c, int r) const { return buf[((w & 1) * W + c) * (R + 1) + r]; }
};

// The same for a whole tile of 128 rows of A by 256 rows of W, filled by a warp that does nothing else: scale of row r at block c,
// and of the two blocks of W.
struct ScaleBlock {
  static constexpr int kBlocks = 16, kLd = kRows + 1;          // (a column more: the writer's lanes go to different banks)
  static constexpr int kFloats = kBlocks * kLd + 2 * kBlocks;
  static __device__ __forceinline__ int a_at(int c, int r) { return c * kLd + r; }
  static __device__ __forceinline__ int w_at(int c, int half) { return kBlocks * kLd + half * kBlocks + c; }
  // Rows and blocks past the end take the last one's scales (what they scale is not stored).
  static __device__ __forceinline__ void fetch(float* to, const F8Gemm& g, int row0, int n0, int kb0, int k_blocks, int lane) {
    const int c = lane & (kBlocks - 1), kb = kb0 + c;
    if (kb >= k_blocks) return;
    const uint32_t a = smem_u32(to + a_at(c, 0)), w = smem_u32(to + w_at(c, lane / kBlocks));
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(w),
                 "l"(g.w_scale + (long long)(min(n0 + lane / kBlocks * kF8Block, g.N - 1) / kF8Block) * k_blocks + kb) : "memory");
#pragma unroll 8
    for (int r = lane / kBlocks; r < kRows; r += 32 / kBlocks)
      asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(a + r * 4),
                   "l"(g.a_scale + (long long)min(row0 + r, g.M - 1) * k_blocks + kb) : "memory");
  }
};

// A warp puts NC bias values from column n0 on into its own piece of shared memory, in fp32; zeros past the end of the row and
// where there is no bias.
template <int NC>
__device__ __forceinline__ void stage_bias(float* s_bias, const __nv_bfloat16* bias, int n0, int N, int lane) {
  __syncwarp();                              // (all lanes are done with what is there)
#pragma unroll
  for (int i = lane; i < NC; i += 32) s_bias[i] = bias != nullptr && n0 + i < N ? __bfloat162float(__ldg(bias + n0 + i)) : 0.f;
  __syncwarp();
}

// One row's NC columns: bias and activation.
template <int NC>
__device__ __forceinline__ void finish_row(float2 (&acc)[NC / 2], const float* s_bias, int act) {
#pragma unroll
  for (int v = 0; v < NC / 4; ++v) {
    const float4 b4 = *reinterpret_cast<const float4*>(s_bias + v * 4);
    acc[2 * v] = __fadd2_rn(acc[2 * v], make_float2(b4.x, b4.y));
    acc[2 * v + 1] = __fadd2_rn(acc[2 * v + 1], make_float2(b4.z, b4.w));
  }
  if (act) {
#pragma unroll
    for (int i = 0; i < NC / 2; i += 2) gelu4(acc[i], acc[i + 1]);
  }
}
template <int NC>
__device__ __forceinline__ uint32_t row_amax(const float2 (&acc)[NC / 2]) {
  float m[2] = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < NC / 2; ++i) m[i & 1] = max_abs3(m[i & 1], acc[i].x, acc[i].y);
  return __float_as_uint(max_abs3(0.f, m[0], m[1]));
}
__device__ __forceinline__ uint32_t bf16x2(float2 f) {
  const __nv_bfloat162 p = __floats2bfloat162_rn(f.x, f.y);
  return *reinterpret_cast<const uint32_t*>(&p);
}
// 32 bytes of a row from column n on, as far as the row goes (it ends on a multiple of 16 bytes at least).
template <typename T>
__device__ __forceinline__ void store32(T* dst, const uint32_t (&w)[8], int n, int N, int vec) {
  constexpr int kPer = 32 / (int)sizeof(T);
  if (vec == 32) {
    if (n < N) st_global_v8(dst, w);
  } else {
    if (n < N) *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
    if (n + kPer / 2 < N) *reinterpret_cast<uint4*>(dst + kPer / 2) = make_uint4(w[4], w[5], w[6], w[7]);
  }
}
// A warp's 32 rows (from m0 on, one a lane) by NC columns where rows of C start anywhere: 32 columns at a time through shared memory
// of the warp's own (32 x 33 floats), so that a store writes 32 columns of one row and not one column of 32 rows (1753 x 1001 x 1040:
// 8.9 us fp32 so, 17.7 with a store per element; 8774 x 3001 x 3072 bf16 107 us for 333, and 92 with 3000 columns).
template <int NC, int OUT>
__device__ __forceinline__ void store_ragged(const float2 (&acc)[NC / 2], const F8Gemm& g, int m0, int n0, float* s_rows, int lane) {
#pragma unroll
  for (int c = 0; c < NC; c += 32) {
    if (n0 + c >= g.N) break;                  // warp-uniform
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s_rows[lane * 33 + 2 * i] = acc[c / 2 + i].x;
      s_rows[lane * 33 + 2 * i + 1] = acc[c / 2 + i].y;
    }
    __syncwarp();
    const int n = n0 + c + lane;
#pragma unroll 4
    for (int r = 0; r < 32; ++r) {
      const float v = s_rows[r * 33 + lane];
      if (m0 + r < g.M && n < g.N) {
        const long long at = (long long)(m0 + r) * g.N + n;
        if constexpr (OUT == kOutBf16) static_cast<__nv_bfloat16*>(g.c)[at] = __float2bfloat16_rn(v);
        else static_cast<float*>(g.c)[at] = v;
      }
    }
  }
}
// 32 bytes of results: columns [v * kPer, (v + 1) * kPer) of a row's NC.
template <int OUT>
constexpr int kPer32 = OUT == kOutF32 ? 8 : (OUT == kOutBf16 ? 16 : 32);
template <int NC, int OUT>
__device__ __forceinline__ void pack32(uint32_t (&w)[8], const float2 (&acc)[NC / 2], int v, float inv) {
  const float2* a = &acc[v * (kPer32<OUT> / 2)];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if constexpr (OUT == kOutF32) w[i] = __float_as_uint(i & 1 ? a[i / 2].y : a[i / 2].x);
    else if constexpr (OUT == kOutBf16) w[i] = bf16x2(a[i]);
    else w[i] = f8_pack4(a[2 * i].x * inv, a[2 * i].y * inv, a[2 * i + 1].x * inv, a[2 * i + 1].y * inv);
  }
}
template <int OUT>
struct OutType { typedef float T; };
template <>
struct OutType<kOutBf16> { typedef __nv_bfloat16 T; };
template <>
struct OutType<kOutF8> { typedef uint8_t T; };
template <int NC, int OUT>
__device__ __forceinline__ void store_row(const float2 (&acc)[NC / 2], const F8Gemm& g, int m, int n0, float inv) {
  typename OutType<OUT>::T* dst = static_cast<typename OutType<OUT>::T*>(g.c) + (long long)m * g.N + n0;
#pragma unroll
  for (int v = 0; v < NC / kPer32<OUT>; ++v) {
    uint32_t w[8];
    pack32<NC, OUT>(w, acc, v, inv);
    store32(dst + v * kPer32<OUT>, w, n0 + v * kPer32<OUT>, g.N, g.vec);
  }
}
// A warp's 32 rows (from m0 on, one a lane) by NC columns, 64 bytes of each at a time through two buffers of shared memory (2 KB each, the
// 64-byte swizzle of the tensor map) and TMA.  A lane's own 32-byte stores touch 32 lines an instruction: 8774 x 12288 x 3072 with bf16
// results 381 us so, 421 with them.
template <int NC, int OUT>
__device__ __forceinline__ void store_tma(const float2 (&acc)[NC / 2], const F8Gemm& g, const CUtensorMap* tm_c, int m0, int n0, float inv,
                                          uint32_t s_rows, int lane) {
  constexpr int kCols = 2 * kPer32<OUT>, kSize = (int)sizeof(typename OutType<OUT>::T);
#pragma unroll
  for (int q = 0; q < NC / kCols; ++q) {
    const uint32_t buf = s_rows + (q & 1) * 2048, to = buf + lane * 64, turn = (lane >> 1) & 3;
    if (lane == 0) tma_store_wait_read<1>();
    __syncwarp();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t w[8];
      pack32<NC, OUT>(w, acc, 2 * q + h, inv);
#pragma unroll
      for (int k = 0; k < 2; ++k)
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + (((2 * h + k) ^ turn) << 4)), "r"(w[4 * k]), "r"(w[4 * k + 1]),
                     "r"(w[4 * k + 2]), "r"(w[4 * k + 3])
                     : "memory");
    }
    proxy_fence_shared();
    __syncwarp();
    if (lane == 0) {
      const int n = n0 + q * kCols;
      if (m0 < g.M && n < g.N) tma_store_2d(tm_c, buf, n * kSize, m0);
      tma_store_commit();
    }
  }
}
// A block's scale from its largest magnitude, and the factor for its values.
__device__ __forceinline__ float put_scale(const F8Gemm& g, uint32_t amax, int m, int n0, bool mine) {
  const F8Scale s = f8_scale(amax);
  if (mine && m < g.M && n0 < g.N) g.c_scale[(long long)m * ((g.N + kF8Block - 1) / kF8Block) + n0 / kF8Block] = s.scale;
  return s.inv;
}
// Finish and store NC columns of a warp's 32 rows, m this lane's; s_rows: see store_ragged.  e4m3: the two warps that hold the halves
// of a block trade their maxima through `s_amax` (two words a row) and `meet`, a barrier of theirs for two arrivals, used once; the
// wait is bounded like every other.
template <int NC, int OUT>
__device__ __forceinline__ void emit_rows(float2 (&acc)[NC / 2], const F8Gemm& g, const float* s_bias, int m, int n0, float* s_rows,
                                          uint32_t* s_amax, uint64_t* meet, int which, volatile int* abort_flag) {
  const int lane = threadIdx.x & 31;
  finish_row<NC>(acc, s_bias, g.act);
  if constexpr (OUT == kOutF8) {
    static_assert(2 * NC == kF8Block, "two warps hold a block");
    uint32_t amax = row_amax<NC>(acc);
    s_amax[which * 32 + lane] = amax;
    __syncwarp();
    if (lane == 0) mbar_arrive(meet);
    if (!mbar_wait_warp(meet, 0, abort_flag)) return;
    amax = max(amax, s_amax[(which ^ 1) * 32 + lane]);
    const float inv = put_scale(g, amax, m, n0, which == 0);
    if (m < g.M) store_row<NC, OUT>(acc, g, m, n0, inv);
  } else if (g.vec) {
    if (m < g.M) store_row<NC, OUT>(acc, g, m, n0, 0.f);
  } else {
    store_ragged<NC, OUT>(acc, g, m - lane, n0, s_rows, lane);
  }
}
// The same for a whole block of columns a thread, through TMA where the rows allow it.
template <int OUT>
__device__ __forceinline__ void emit_block(float2 (&acc)[kF8Block / 2], const F8Gemm& g, const CUtensorMap* tm_c, const float* s_bias, int m,
                                           int n0, float* s_rows, int lane) {
  finish_row<kF8Block>(acc, s_bias, g.act);
  float inv = 0.f;
  if constexpr (OUT == kOutF8) inv = put_scale(g, row_amax<kF8Block>(acc), m, n0, true);
  if (OUT == kOutF8 || g.vec) store_tma<kF8Block, OUT>(acc, g, tm_c, m - lane, n0, inv, smem_u32(s_rows), lane);
  else if constexpr (OUT != kOutF8) store_ragged<kF8Block, OUT>(acc, g, m - lane, n0, s_rows, lane);
}

// ---------------------------------------------------------------------------------------------------------------
// One tile per CTA.  A tile is 128 rows of the first operand by BN of the second: of A by W, or (SWAP) of W by A, for
// few rows of A.  A cluster of `split` CTAs shares a tile, each taking a run of its K blocks; their partial sums meet through
// distributed shared memory: the CTA that finishes a row (a column, SWAP) adds the others' to its own in the order of their ranks, the
// same order in every call.
//   warp 0     TMA producer
//   warp 1     MMA issuer
//   warps 2..  promotion and epilogue: eight (two per TMEM quadrant, half of the columns each), SWAP: four
// ---------------------------------------------------------------------------------------------------------------
template <int BN, bool SWAP>
struct SplitCfg {
  static_assert(!SWAP || BN == 16, "promote_columns");
  static constexpr int kWarps = SWAP ? 4 : 8;
  static constexpr int kThreads = 64 + 32 * kWarps;
  static constexpr int kCols = SWAP ? BN : BN / 2;             // of a warp
  static constexpr int kStageBytes = kRowBytes + BN * kStepK;
  static constexpr int kStages = BN == 128 ? 4 : 5;
  static constexpr int kTmemCols = 2 * BN;                     // (a power of two, at least 32)
  static constexpr int kMaxSplit = SWAP ? 8 : 4;
  static constexpr size_t kBiasBytes = SWAP ? 0 : (size_t)kWarps * kCols * 4;
  static constexpr size_t kAmaxBytes = SWAP ? (size_t)4 * BN * 4 : (size_t)2 * kRows * 4;
  static constexpr int kScaleRows = SWAP ? BN : 32;            // rows of A whose scales a warp needs
  static constexpr size_t kScaleBytes = (size_t)kWarps * ScaleWindow<kScaleRows, 16>::kFloats * 4;
  static constexpr size_t part_bytes(int split) {              // columns of A's rows, or 128 / split rows, from each of the others
    return SWAP ? (size_t)(split - 1) * (BN / split) * kRows * 4 : (size_t)(split - 1) * (kRows / split) * BN * 4;
  }
  static constexpr size_t smem(int split) {
    return kAlignSlack + (size_t)kStages * kStageBytes + kBiasBytes + kAmaxBytes + kScaleBytes + kBarrierBytes + part_bytes(split);
  }
};

template <int BN, bool SWAP, int OUT>
__global__ void __launch_bounds__(SplitCfg<BN, SWAP>::kThreads)
fp8_split_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_w, const F8Gemm g, int split,
                 int* __restrict__ status) {
  using Cfg = SplitCfg<BN, SWAP>;
  constexpr int kStages = Cfg::kStages, kCols = Cfg::kCols;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  float* s_bias_all = reinterpret_cast<float*>(smem + (size_t)kStages * Cfg::kStageBytes);
  uint32_t* s_amax = reinterpret_cast<uint32_t*>(reinterpret_cast<uint8_t*>(s_bias_all) + Cfg::kBiasBytes);
  float* s_scale = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(s_amax) + Cfg::kAmaxBytes);
  uint64_t* bars = reinterpret_cast<uint64_t*>(reinterpret_cast<uint8_t*>(s_scale) + Cfg::kScaleBytes);
  uint64_t* full = bars;                    // [kStages] TMA -> MMA
  uint64_t* empty = bars + kStages;         // [kStages] MMA -> TMA
  uint64_t* acc_full = bars + 2 * kStages;  // [2] MMA -> promotion
  uint64_t* acc_empty = acc_full + 2;       // [2] promotion -> MMA
  uint64_t* meet = acc_empty + 2;           // [4] the two warps of a quadrant (e4m3 results)
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(meet + 4);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  float* s_part = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(bars) + kBarrierBytes);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = split > 1 ? (int)cluster_rank() : 0;
  const int tile = blockIdx.x / split;
  const int m_tile = SWAP ? BN : kRows, n_tile = SWAP ? kRows : BN;
  const int m_tiles = (g.M - 1) / m_tile + 1;
  const int m0 = (tile % m_tiles) * m_tile, n0 = (tile / m_tiles) * n_tile;
  const int k_blocks = (g.K - 1) / kStepK + 1;
  const int kb0 = (int)((long long)k_blocks * rank / split), kb1 = (int)((long long)k_blocks * (rank + 1) / split);

  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&acc_full[i], 1); mbar_init(&acc_empty[i], Cfg::kWarps); }
    for (int i = 0; i < 4; ++i) mbar_init(&meet[i], 2);
    *abort_flag = 0;
    mbar_fence_init();
  }
  if (warp == 0 && lane == 0) { tma_prefetch_desc(&tm_a); tma_prefetch_desc(&tm_w); }
  if (warp == 1) { tmem_alloc(tmem_slot, Cfg::kTmemCols); tmem_relinquish(); }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (split > 1) cluster_arrive();           // waited for before anything is sent to another CTA
  const uint32_t tmem_base = *tmem_slot;
  stream_order();

  float2 acc[kCols / 2];
  bool ok = true;
  const int quad = warp & 3;                 // TMEM lane quadrant this warp may read
  const int half = SWAP ? 0 : (warp - 2) >> 2;
  const int tile_row = quad * 32 + lane;
  float* s_bias = s_bias_all + (SWAP || warp < 2 ? 0 : (size_t)(warp - 2) * kCols);

  if (warp == 0) {
    // ------------------------------------------------------------ TMA producer
    if (lane == 0) {
      int stage = 0; uint32_t phase = 0;
      for (int kb = kb0; kb < kb1; ++kb) {
        uint8_t* first = smem + (size_t)stage * Cfg::kStageBytes;
        uint8_t* second = first + kRowBytes;
        if (!mbar_wait(&empty[stage], phase ^ 1, abort_flag)) break;
        mbar_expect_tx(&full[stage], Cfg::kStageBytes);
        tma_load_2d(SWAP ? first : second, &tm_w, &full[stage], kb * kStepK, n0);
        tma_load_2d(SWAP ? second : first, &tm_a, &full[stage], kb * kStepK, m0);
        if (++stage == kStages) { stage = 0; phase ^= 1; }
      }
      for (int i = 0; i < kStages; ++i) {      // all armed stages consumed before the CTA retires
        if (!mbar_wait(&empty[stage], phase ^ 1, abort_flag)) break;
        if (++stage == kStages) { stage = 0; phase ^= 1; }
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMA issuer
    const bool leader = elect_one();
    constexpr uint32_t idesc = idesc_e4m3(kRows, BN);
    int stage = 0; uint32_t phase = 0;
    for (int kb = kb0; kb < kb1; ++kb) {
      const int j = kb - kb0, buf = j & 1;
      if (!mbar_wait_warp(&acc_empty[buf], ((j >> 1) & 1) ^ 1, abort_flag)) break;
      if (!mbar_wait_warp(&full[stage], phase, abort_flag)) break;
      tc_fence_after();
      const uint32_t sa = smem_u32(smem + (size_t)stage * Cfg::kStageBytes);
      const uint64_t da = smem_desc_sw128(sa, 1024), db = smem_desc_sw128(sa + kRowBytes, 1024);
      if (leader) {
#pragma unroll
        for (int k = 0; k < kStepK / 32; ++k)   // +32 bytes (encoded >>4) per K step of 32 inside the swizzle atom
          mma_f8_ss(tmem_base + buf * BN, da + 2 * k, db + 2 * k, idesc, k != 0);
        mma_commit(&empty[stage]);
        mma_commit(&acc_full[buf]);
      }
      if (++stage == kStages) { stage = 0; phase ^= 1; }
    }
  } else {
    // ------------------------------------------------------------ promotion
    const uint32_t t_row = tmem_base + ((uint32_t)(quad * 32) << 16) + (uint32_t)(half * kCols);
    if constexpr (!SWAP) stage_bias<kCols>(s_bias, g.bias, n0 + half * kCols, g.N, lane);
#pragma unroll
    for (int i = 0; i < kCols / 2; ++i) acc[i] = make_float2(0.f, 0.f);
    using Window = ScaleWindow<Cfg::kScaleRows, 16>;
    constexpr int kWindow = Window::kBlocks;
    const Window window = {s_scale + (size_t)(warp - 2) * Window::kFloats, g.a_scale, g.M, k_blocks, lane};
    const float* sw = g.w_scale + (long long)(n0 / kF8Block) * k_blocks;
    const int row0 = SWAP ? m0 : m0 + quad * 32, mine = SWAP ? lane & (BN - 1) : lane;
    float w16 = 0.f, w16_next = 0.f;           // W's scales of a window, lane c that of block c
    auto fetch = [&](uint32_t w, int kb) {
      window.fetch(w, row0, kb, kb1);
      if (lane < kWindow && kb + lane < kb1) w16_next = __ldg(sw + kb + lane);
    };
    fetch(0, kb0);
    for (int kb = kb0; kb < kb1; ++kb) {
      const int j = kb - kb0, buf = j & 1, c = j & (kWindow - 1);
      const uint32_t w = (uint32_t)j / kWindow;
      if (c == 0) {
        Window::arrived();
        w16 = w16_next;
        fetch(w + 1, kb + kWindow);
      }
      const float f = window.at(w, c, mine) * __shfl_sync(0xFFFFFFFFu, w16, c);
      if (!(ok = mbar_wait_warp(&acc_full[buf], (j >> 1) & 1, abort_flag))) break;
      tc_fence_after();
      if constexpr (SWAP) promote_columns(acc, t_row + buf * BN, f);
      else promote<kCols, 16>(acc, t_row + buf * BN, f);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&acc_empty[buf]);
    }
    Window::arrived();
  }

  // ---------------------------------------------------------------- partial sums
  // A CTA finishes 128 / split rows (whole TMEM quadrants), or (SWAP) every split-th column.
  const int shift = split == 8 ? 3 : (split == 4 ? 2 : (split == 2 ? 1 : 0));
  const int owner = (quad << shift) >> 2;
  const int rows_own = kRows >> shift, own_row = tile_row - owner * rows_own;
  const int columns = SWAP ? min(BN, g.M - m0) : BN;           // that exist
  if (split > 1) {
    __syncwarp();
    cluster_wait();                          // the other CTAs have started (long since)
    if (warp >= 2 && ok) {
      if constexpr (SWAP) {
#pragma unroll
        for (int c = 0; c < BN; ++c) {
          const int to = c & (split - 1);
          if (c < columns && to != rank) {   // (warp-uniform)
            const int slot = rank < to ? rank : rank - 1;
            const float v = c & 1 ? acc[c / 2].y : acc[c / 2].x;
            st_cluster_f32(cluster_map(smem_u32(s_part + ((size_t)slot * (BN >> shift) + (c >> shift)) * kRows + tile_row), (uint32_t)to), v);
          }
        }
      } else if (owner != rank) {
        const int slot = rank < owner ? rank : rank - 1;
        const uint32_t base = cluster_map(smem_u32(s_part + (((size_t)slot * (BN / 4) + half * (kCols / 4)) * rows_own + own_row) * 4), (uint32_t)owner);
#pragma unroll
        for (int v = 0; v < kCols / 4; ++v)
          st_cluster_v4(base + v * rows_own * 16, acc[2 * v].x, acc[2 * v].y, acc[2 * v + 1].x, acc[2 * v + 1].y);
      }
    }
    __syncwarp();
    cluster_sync();                          // every wait above is bounded, so everybody gets here
    if (warp >= 2 && ok) {
      for (int s = 0; s < split - 1; ++s) {
        if constexpr (SWAP) {
#pragma unroll
          for (int c = 0; c < BN; ++c)
            if (c < columns && (c & (split - 1)) == rank) {
              const float v = s_part[((size_t)s * (BN >> shift) + (c >> shift)) * kRows + tile_row];
              if (c & 1) acc[c / 2].y += v; else acc[c / 2].x += v;
            }
        } else if (owner == rank) {
          const float4* part = reinterpret_cast<const float4*>(s_part) + ((size_t)s * (BN / 4) + half * (kCols / 4)) * rows_own + own_row;
#pragma unroll
          for (int v = 0; v < kCols / 4; ++v) {
            const float4 p = part[v * rows_own];
            acc[2 * v].x += p.x; acc[2 * v].y += p.y; acc[2 * v + 1].x += p.z; acc[2 * v + 1].y += p.w;
          }
        }
      }
    }
  }

  // ---------------------------------------------------------------- epilogue
  if (warp >= 2) {
    if constexpr (!SWAP) {
      if (owner == rank && ok)
        emit_rows<kCols, OUT>(acc, g, s_bias, m0 + tile_row, n0 + half * kCols, reinterpret_cast<float*>(smem) + (warp - 2) * 32 * 33,
                              s_amax + quad * 64, meet + quad, half, abort_flag);      // (the operands' stages are free by now)
    } else {
      const int n = n0 + tile_row;
      const float b = g.bias != nullptr && n < g.N ? __bfloat162float(__ldg(g.bias + n)) : 0.f;
#pragma unroll
      for (int i = 0; i < BN / 2; ++i) acc[i] = __fadd2_rn(acc[i], make_float2(b, b));
      if (g.act) {
#pragma unroll
        for (int i = 0; i < BN / 2; i += 2) gelu4(acc[i], acc[i + 1]);
      }
      F8Scale sc = {};
      if constexpr (OUT == kOutF8) {         // the 128 rows of W are a block: a column's maximum over the four warps
#pragma unroll
        for (int c = 0; c < BN; ++c) {
          const uint32_t amax = __reduce_max_sync(0xFFFFFFFFu, abs_bits(c & 1 ? acc[c / 2].y : acc[c / 2].x));
          if (lane == 0) s_amax[quad * BN + c] = amax;
        }
        asm volatile("bar.sync 1, 128;" ::: "memory");
      }
#pragma unroll
      for (int c = 0; c < BN; ++c) {
        if (ok && c < columns && (c & (split - 1)) == rank) {  // (warp-uniform)
          const float v = c & 1 ? acc[c / 2].y : acc[c / 2].x;
          const long long at = (long long)(m0 + c) * g.N + n;
          if constexpr (OUT == kOutF8) {
            sc = f8_scale(max(max(s_amax[c], s_amax[BN + c]), max(s_amax[2 * BN + c], s_amax[3 * BN + c])));
            if (n < g.N) static_cast<uint8_t*>(g.c)[at] = (uint8_t)f8_pack4(v * sc.inv, 0.f, 0.f, 0.f);
            if (tile_row == 0) g.c_scale[(long long)(m0 + c) * ((g.N + kF8Block - 1) / kF8Block) + n0 / kF8Block] = sc.scale;
          } else if (n < g.N) {
            if constexpr (OUT == kOutBf16) static_cast<__nv_bfloat16*>(g.c)[at] = __float2bfloat16_rn(v);
            else static_cast<float*>(g.c)[at] = v;
          }
        }
      }
    }
  }

  // ---------------------------------------------------------------- teardown
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag) atomicExch(status, 1);
  if (warp == 1) { tc_fence_after(); tmem_dealloc(tmem_base, Cfg::kTmemCols); }
}

// ---------------------------------------------------------------------------------------------------------------
// Persistent clusters of two CTAs, one per pair of SMs, on tiles of 256 x 256: each CTA fetches its own 128 rows of A and half
// of the tile's rows of W, a K step of 128 costs an SM 32 KB from L2 for the 8.4 MFLOP it computes.
//   warp 0       TMA producer (both CTAs, each its own operand rows; all bytes reported to the even CTA's barrier)
//   warp 1       MMA issuer (even CTA only): 4 x tcgen05.mma M256 N256 K32 per block into one of two TMEM buffers; the commits free
//                both CTAs' stage and hand the buffer to both CTAs' promotion
//   warp 2       nothing
//   warp 3       tensor memory; then the scales, 16 K blocks at a time
//   warps 4..11  promotion and epilogue (both CTAs, each its own 128 rows): a warpgroup for each half of the columns
// ---------------------------------------------------------------------------------------------------------------
struct PairCfg {
  static constexpr int kBN = 256, kCols = 128;                 // of a tile, of a warp
  static constexpr int kWarps = 8, kThreads = 384;
  static constexpr int kStageBytes = kRowBytes + kBN / 2 * kStepK;
  static constexpr int kStages = 5;                            // 160 KB
  static constexpr int kTmemCols = 512;
  static constexpr size_t kBiasBytes = (size_t)kWarps * kCols * 4;
  static constexpr size_t kScaleBytes = 2 * ScaleBlock::kFloats * 4;
  static constexpr size_t kRowsBytes = (size_t)kWarps * 32 * 33 * 4;     // store_ragged
  static constexpr size_t kSmem = kAlignSlack + (size_t)kStages * kStageBytes + kBiasBytes + kScaleBytes + kRowsBytes + kBarrierBytes;
  // Registers: 384 threads start with 168 each; the first warpgroup gives up what the other two, with 128 sums a thread, take
  // (128 * 40 + 256 * 232 = 384 * 168).  20 bytes a thread are spilled, 28 with fp32 results.
  static constexpr int kFewRegs = 40, kManyRegs = 232;
  static constexpr int kPromote = 32;                          // columns a TMEM read
};

template <int OUT>
__global__ void __launch_bounds__(PairCfg::kThreads, 1)
fp8_pair_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_w,
                const __grid_constant__ CUtensorMap tm_c, const F8Gemm g,
                int* __restrict__ status) {
  using Cfg = PairCfg;
  constexpr int kStages = Cfg::kStages, kCols = Cfg::kCols, BN = Cfg::kBN, kPromote = Cfg::kPromote, kWindow = ScaleBlock::kBlocks;
  extern __shared__ uint8_t smem_raw[];
  // The dynamic shared memory starts at the same offset in both CTAs, and so does everything carved from it: a
  // descriptor or a barrier offset means the same place in either.
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  float* s_rows_all = reinterpret_cast<float*>(smem + (size_t)kStages * Cfg::kStageBytes);      // (on a multiple of 1024 bytes)
  float* s_bias_all = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(s_rows_all) + Cfg::kRowsBytes);
  float* s_scale = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(s_bias_all) + Cfg::kBiasBytes);
  uint64_t* bars = reinterpret_cast<uint64_t*>(reinterpret_cast<uint8_t*>(s_scale) + Cfg::kScaleBytes);
  uint64_t* full = bars;                    // [kStages] both CTAs' TMA -> MMA (the even CTA's is the one in use)
  uint64_t* empty = bars + kStages;         // [kStages] MMA -> TMA (each CTA its own)
  uint64_t* acc_full = bars + 2 * kStages;  // [2] MMA -> promotion (each CTA its own)
  uint64_t* acc_empty = acc_full + 2;       // [2] both CTAs' promotion -> MMA (the even CTA's)
  uint64_t* sc_full = acc_empty + 2;        // [2] scales -> promotion
  uint64_t* sc_empty = sc_full + 2;         // [2] promotion -> scales
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(sc_empty + 2);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
  const int m_tiles = (g.M - 1) / (2 * kRows) + 1, n_tiles = (g.N - 1) / BN + 1;
  const int n_tiles_total = m_tiles * n_tiles;
  const int k_blocks = (g.K - 1) / kStepK + 1;

  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&acc_full[i], 1); mbar_init(&acc_empty[i], 2 * Cfg::kWarps); }
    for (int i = 0; i < 2; ++i) { mbar_init(&sc_full[i], 32); mbar_init(&sc_empty[i], Cfg::kWarps); }
    *abort_flag = 0;
    mbar_fence_init();
  }
  if (warp == 0 && lane == 0) { tma_prefetch_desc(&tm_a); tma_prefetch_desc(&tm_w); if (OUT == kOutF8 || g.vec) tma_prefetch_desc(&tm_c); }
  if (warp == 3) tmem_alloc_pair(tmem_slot, Cfg::kTmemCols);
  tc_fence_before();
  __syncwarp();
  cluster_sync();                           // both CTAs' barriers exist before anybody signals across
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  stream_order();

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Cfg::kFewRegs));
    if (warp == 0 && lane == 0) {
      // ------------------------------------------------------------ TMA producer
      int stage = 0; uint32_t phase = 0;
      bool ok = true;
      for (int tile = pair; tile < n_tiles_total && ok; tile += n_pairs) {
        int mt, nt;
        tile_coords(tile, m_tiles, n_tiles, mt, nt);
        const int row_a = (2 * mt + (int)rank) * kRows, row_w = nt * BN + (int)rank * kCols;
        for (int kb = 0; kb < k_blocks; ++kb) {
          if (!(ok = mbar_wait(&empty[stage], phase ^ 1, abort_flag))) break;
          // The even CTA's barrier counts the bytes of both CTAs.  The odd CTA's may land before it is armed: its
          // phase cannot complete before the arrival that arms it.
          if (rank == 0) mbar_expect_tx(&full[stage], 2 * Cfg::kStageBytes);
          const uint32_t sa = smem_u32(smem + (size_t)stage * Cfg::kStageBytes), bar = cluster_map(smem_u32(&full[stage]), 0);
          tma_load_2d_pair(sa, &tm_a, bar, kb * kStepK, row_a);
          tma_load_2d_pair(sa + kRowBytes, &tm_w, bar, kb * kStepK, row_w);
          if (++stage == kStages) { stage = 0; phase ^= 1; }
        }
      }
      // On the way out make sure every stage that was armed has been consumed (bounded): the CTA must
      // not retire with bulk copies still writing its shared memory.
      for (int i = 0; i < kStages; ++i) {
        if (!mbar_wait(&empty[stage], phase ^ 1, abort_flag)) break;
        if (++stage == kStages) { stage = 0; phase ^= 1; }
      }
    } else if (warp == 1 && rank == 0) {
      // ------------------------------------------------------------ MMA issuer (even CTA)
      const bool leader = elect_one();
      constexpr uint32_t idesc = idesc_e4m3(2 * kRows, BN);
      int stage = 0; uint32_t phase = 0;
      bool ok = true;
      uint32_t j = 0;                        // K blocks so far
      for (int tile = pair; tile < n_tiles_total && ok; tile += n_pairs) {
        for (int kb = 0; kb < k_blocks; ++kb, ++j) {
          const uint32_t buf = j & 1;
          if (!(ok = mbar_wait_warp(&full[stage], phase, abort_flag))) break;
          if (!(ok = mbar_wait_warp(&acc_empty[buf], ((j >> 1) & 1) ^ 1, abort_flag))) break;
          tc_fence_after();
          const uint32_t sa = smem_u32(smem + (size_t)stage * Cfg::kStageBytes);
          const uint64_t da = smem_desc_sw128(sa, 1024), db = smem_desc_sw128(sa + kRowBytes, 1024);
          if (leader) {
#pragma unroll
            for (int k = 0; k < kStepK / 32; ++k)
              mma_f8_ss_pair(tmem_base + buf * BN, da + 2 * k, db + 2 * k, idesc, k != 0);
            mma_commit_pair(&empty[stage]);
            mma_commit_pair(&acc_full[buf]);
          }
          if (++stage == kStages) { stage = 0; phase ^= 1; }
        }
      }
    } else if (warp == 3) {
      // ------------------------------------------------------------ scales
      uint32_t w = 0;                        // windows so far
      bool ok = true;
      for (int tile = pair; tile < n_tiles_total && ok; tile += n_pairs) {
        int mt, nt;
        tile_coords(tile, m_tiles, n_tiles, mt, nt);
        for (int kb = 0; kb < k_blocks; kb += kWindow, ++w) {
          if (!(ok = mbar_wait_warp(&sc_empty[w & 1], ((w >> 1) & 1) ^ 1, abort_flag))) break;
          ScaleBlock::fetch(s_scale + (w & 1) * ScaleBlock::kFloats, g, (2 * mt + (int)rank) * kRows, nt * BN, kb, k_blocks, lane);
          asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&sc_full[w & 1])) : "memory");
        }
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
    }
  } else {
    // ------------------------------------------------------------ promotion and epilogue (warps 4..11)
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(Cfg::kManyRegs));
    const int quad = warp & 3;                 // TMEM lane quadrant this warp may read
    const int half = (warp - 4) >> 2;          // which half of the tile's columns it has
    float* s_bias = s_bias_all + (size_t)(warp - 4) * kCols;
    // (a warp's rows lie 4224 bytes apart for store_ragged and 4096 for TMA, which wants the alignment)
    float* s_rows = s_rows_all + (warp - 4) * (OUT == kOutF8 || g.vec ? 1024 : 32 * 33);
    const uint32_t t_row = tmem_base + ((uint32_t)(quad * 32) << 16) + (uint32_t)(half * kCols);
    const uint32_t full_bar = smem_u32(acc_full), empty_bar = cluster_map(smem_u32(acc_empty), 0);
    uint32_t w = 0;                            // windows of scales so far
    bool ok = true;
    uint32_t j = 0;
    for (int tile = pair; tile < n_tiles_total && ok; tile += n_pairs) {
      int mt, nt;
      tile_coords(tile, m_tiles, n_tiles, mt, nt);
      const int m = (2 * mt + (int)rank) * kRows + quad * 32 + lane, n_first = nt * BN + half * kCols;
      // the bias is asked for now and put into shared memory two blocks later
      float bias[kCols / 32];
#pragma unroll
      for (int i = 0; i < kCols / 32; ++i) {
        const int n = n_first + i * 32 + lane;
        bias[i] = g.bias != nullptr && n < g.N ? __bfloat162float(__ldg(g.bias + n)) : 0.f;
      }
      float2 acc[kCols / 2];
#pragma unroll
      for (int i = 0; i < kCols / 2; ++i) acc[i] = make_float2(0.f, 0.f);
      // The promotion of a block reaches into the next, so that little latency is left between two packed FMAs: the next block's
      // scales are read while the first columns are added; once the last columns are in registers the buffer goes back and the
      // first of the next block are asked for.
      uint32_t r[2][kPromote];
      const float* scales = s_scale;
      auto turn = [&]() {                      // into the next window, handing back the last
        if (w > 0) {
          __syncwarp();
          if (lane == 0) mbar_arrive(&sc_empty[(w - 1) & 1]);
        }
        mbar_wait_lane(smem_u32(&sc_full[w & 1]), (w >> 1) & 1, abort_flag);
        scales = s_scale + (w & 1) * ScaleBlock::kFloats;
        ++w;
      };
      turn();
      float a_next = scales[ScaleBlock::a_at(0, quad * 32 + lane)], w_next = scales[ScaleBlock::w_at(0, half)];
      mbar_wait_lane(full_bar + (j & 1) * 8, (j >> 1) & 1, abort_flag);
      __syncwarp();
      tc_fence_after();
      tmem_ld(t_row + (j & 1) * BN, r[0]);
      for (int kb = 0; kb < k_blocks; ++kb) {
        const uint32_t taddr = t_row + (j & 1) * BN;
        const float f = a_next * w_next;
        const float2 s2 = make_float2(f, f);
        const bool more = kb + 1 < k_blocks;
        const int c = (kb + 1) & (kWindow - 1);
        if (more && c == 0) turn();
        a_next = scales[ScaleBlock::a_at(c, quad * 32 + lane)];
        w_next = scales[ScaleBlock::w_at(c, half)];
        constexpr int kPieces = kCols / kPromote;
#pragma unroll
        for (int q = 0; q < kPieces; ++q) {
          tmem_wait(r[q & 1]);
          if (q + 1 < kPieces) {
            tmem_ld(taddr + (q + 1) * kPromote, r[(q + 1) & 1]);
          } else {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster_relaxed(empty_bar + (j & 1) * 8);
            ++j;
            if (more) mbar_wait_lane(full_bar + (j & 1) * 8, (j >> 1) & 1, abort_flag);
            __syncwarp();
            tc_fence_after();
            tmem_ld(t_row + (j & 1) * BN, r[0]);       // (behind the last block whatever is there: with a condition the 32
                                                          // registers were copied from turn to turn)
          }
#pragma unroll
          for (int i = 0; i < kPromote / 2; ++i) {
            float2& a = acc[q * (kPromote / 2) + i];
            a = __ffma2_rn(make_float2(__uint_as_float(r[q & 1][2 * i]), __uint_as_float(r[q & 1][2 * i + 1])), s2, a);
          }
        }
        if (kb == 0) {                         // (the bias has arrived by now)
          __syncwarp();                        // (all lanes are done with what is there)
#pragma unroll
          for (int i = 0; i < kCols / 32; ++i) s_bias[i * 32 + lane] = bias[i];
          __syncwarp();
        }
      }
      tmem_wait(r[0]);
      ok = __all_sync(0xFFFFFFFFu, *abort_flag == 0);
      if (ok) emit_block<OUT>(acc, g, &tm_c, s_bias, m, n_first, s_rows, lane);
    }
    if (lane == 0) tma_store_wait_all();       // (nothing is in flight from shared memory when the CTA ends)
  }

  // ---------------------------------------------------------------- teardown
  tc_fence_before();
  __syncwarp();
  cluster_sync();                            // neither CTA leaves while the other may still reach into it
  if (threadIdx.x == 0 && *abort_flag) atomicExch(status, 1);
  if (warp == 3) { tc_fence_after(); tmem_dealloc_pair(tmem_base, Cfg::kTmemCols); }
}

template <int OUT>
int launch_pair(const CUtensorMap& tm_a, const CUtensorMap& tm_w, const CUtensorMap& tm_c, const F8Gemm& g, int* d_status, cudaStream_t s) {
  static PerDeviceOnce attr_once;            // the opt-in is a property of the kernel ON a device
  HERO_TRY(per_device_once(attr_once, [](int) {
    HERO_CUDA_TRY(cudaFuncSetAttribute(fp8_pair_kernel<OUT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)PairCfg::kSmem));
    return HERO_OK;
  }));
  const long long tiles = (long long)((g.M - 1) / (2 * kRows) + 1) * ((g.N - 1) / PairCfg::kBN + 1);
  if (tiles > 0x3FFFFFFF) return HERO_ERR_ARG;
  const int pairs = tiles < num_sms() / 2 ? (int)tiles : num_sms() / 2;
  return launch_kernel(fp8_pair_kernel<OUT>, (unsigned)(2 * pairs), PairCfg::kThreads, PairCfg::kSmem, s, 2, tm_a, tm_w, tm_c, g, d_status);
}

template <int BN, bool SWAP, int OUT>
int launch_split(const CUtensorMap& tm_a, const CUtensorMap& tm_w, const F8Gemm& g, int split, int* d_status, cudaStream_t s) {
  using Cfg = SplitCfg<BN, SWAP>;
  static PerDeviceOnce attr_once;
  HERO_TRY(per_device_once(attr_once, [](int) {
    HERO_CUDA_TRY(cudaFuncSetAttribute(fp8_split_kernel<BN, SWAP, OUT>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       (int)Cfg::smem(Cfg::kMaxSplit)));
    return HERO_OK;
  }));
  const int m_tile = SWAP ? BN : kRows, n_tile = SWAP ? kRows : BN;
  const long long ctas = (long long)((g.M - 1) / m_tile + 1) * ((g.N - 1) / n_tile + 1) * split;
  if (ctas > 0x7FFFFFFF) return HERO_ERR_ARG;
  return launch_kernel(fp8_split_kernel<BN, SWAP, OUT>, (unsigned)ctas, Cfg::kThreads, Cfg::smem(split), s, (unsigned)split, tm_a, tm_w,
                       g, split, d_status);
}

template <int OUT>
int launch_out(const TcGemmF8Plan& plan, const CUtensorMap& tm_a, const CUtensorMap& tm_w, const CUtensorMap& tm_c, const F8Gemm& g, int* d_status, cudaStream_t s) {
  if (plan.split == 0) return launch_pair<OUT>(tm_a, tm_w, tm_c, g, d_status, s);
  if (plan.swap) return launch_split<16, true, OUT>(tm_a, tm_w, g, plan.split, d_status, s);
  if constexpr (OUT != kOutF8)
    if (plan.bn == 64) return launch_split<64, false, OUT>(tm_a, tm_w, g, plan.split, d_status, s);
  return launch_split<128, false, OUT>(tm_a, tm_w, g, plan.split, d_status, s);
}

}  // namespace

// ---------------------------------------------------------------------------------------------------------------
// Which kernel, which tile, how many CTAs per tile.  The estimate is in nanoseconds: rounds of tiles times (K blocks times the
// time of a block, plus what a tile costs besides) plus what a launch costs, and for a split tile the exchange.  Fitted to 127
// problems (1 to 3510 rows, 256 to 12288 columns, K 512 to 12288), each timed with every kernel in launches in a row; on them
// the rule's choice takes 0.3 % longer than the best on average and 12 % at worst.  Some of them (us; 16 exchanged over 1 / 2 / 4,
// 128 over 1 / 2 / 4, 64 over 1 / 2 / 4, pair):
//   1 x 12288 x 3072     10.7 / 10.6 / 16.5 | 17.3 / 21.1 / 27.9 | 24.0 / 28.1 / 43.5 | 18.0
//   1 x 3072 x 12288     30.2 / 17.7 / 12.4 | 40.2 / 23.1 / 15.8 | 35.0 / 24.2 / 25.1 | 41.8
//   16 x 2304 x 768      4.3 / 4.5 / 5.1 | 4.8 / 5.1 / 6.0 | 4.3 / 4.2 / 8.9 | 6.3
//   48 x 12288 x 3072    11.8 / 20.0 / 39.4 | 13.2 / 19.1 / 25.9 | 21.8 / 23.9 / 39.6 | 15.6
//   64 x 3072 x 3072     10.3 / 8.8 / 15.1 | 12.5 / 9.3 / 8.4 | 11.2 / 8.0 / 12.8 | 14.6
//   200 x 1280 x 5120    - / - / - | 18.9 / 12.4 / 9.8 | 16.5 / 10.7 / 15.0 | 21.6
//   614 x 3072 x 3072    - / - / - | 13.1 / 19.3 / 33.5 | 21.8 / 31.7 / 51.8 | 15.8
//   1394 x 3072 x 3072   - / - / - | 25.7 / 38.7 / 68.2 | 43.3 / 63.0 / 107.7 | 16.7
//   1394 x 2304 x 768    - / - / - | 11.4 / 18.9 / 40.7 | 14.5 / 30.5 / 63.2 | 9.2
//   3510 x 768 x 3072    - / - / - | 25.2 / 28.4 / 48.1 | 32.1 / 39.5 / 70.2 | 16.7
// ---------------------------------------------------------------------------------------------------------------
TcGemmF8Plan plan_tc_gemm_fp8(int M, int Nout, int K, bool f8_out, int sms) {
  const long long kb = ((long long)K + kStepK - 1) / kStepK;
  auto ceil_div = [](long long a, long long b) { return (a + b - 1) / b; };
  TcGemmF8Plan best = {PairCfg::kBN, 0, false};
  const long long pairs = sms < 2 ? 1 : sms / 2;
  long long best_t = ceil_div(ceil_div(M, 2 * kRows) * ceil_div(Nout, PairCfg::kBN), pairs) * (kb * 500 + 2420) + 1230;
  auto consider = [&](int bn, int split, bool swap, long long t) {
    if (t < best_t) { best_t = t; best = {bn, split, swap}; }
  };
  for (int split = 1; split <= 8 && split <= kb; split *= 2) {     // two CTAs an SM; the weights' bandwidth is shared by all
    const long long ctas = ceil_div(Nout, kRows) * ceil_div(M, 16) * split, room = 2ll * sms;
    if (ctas > 0x7FFFFFFFll) break;
    const long long shared = 19 * (ctas < room ? ctas : room) / 10, exchange = split == 1 ? 0 : 763 + 366 * (split - 2) + 9 * ctas;
    consider(16, split, true, ceil_div(ctas, room) * (ceil_div(kb, split) * (shared > 263 ? shared : 263) + 214) + 2440 + exchange);
  }
  struct { int bn, step, step_full, tile, launch, two, four, crowd; } const one[] = {{128, 337, 184, 1393, 1451, 1468, 2117, 1194},
                                                                                      {64, 227, 204, 770, 2070, 810, 948, 975}};
  for (const auto& o : one) {
    if (f8_out && o.bn < kF8Block) continue;           // (an e4m3 result's blocks of 128 columns stay in one tile)
    for (int split = 1; split <= 4 && split <= kb; split *= 2) {
      const long long ctas = ceil_div(M, kRows) * ceil_div(Nout, o.bn) * split;
      if (ctas > 0x7FFFFFFFll) break;
      // (clusters of four do not fill the chip: they need four free SMs of one processing cluster)
      const long long room = split < 4 ? sms : (sms < 8 ? sms : sms * 7 / 8), step = o.step + o.step_full * (ctas < sms ? ctas : sms) / sms;
      const long long exchange = split == 1 ? 0 : (split == 2 ? o.two : o.four + (ctas > 60 ? o.crowd * (ctas - 60) / 60 : 0));
      consider(o.bn, split, false, ceil_div(ctas, room) * (ceil_div(kb, split) * step + o.tile) + o.launch + exchange);
    }
  }
  return best;
}

int launch_tc_gemm_fp8(const void* a, const float* a_scale, const void* w, const float* w_scale, const void* bias, void* c,
                       float* c_scale, int M, int Nout, int K, int act, int out_dtype, int* d_status, cudaStream_t s) {
  const TcGemmF8Plan plan = plan_tc_gemm_fp8(M, Nout, K, out_dtype == HERO_DTYPE_E4M3, num_sms());
  F8Gemm g = {a_scale, w_scale, static_cast<const __nv_bfloat16*>(bias), c, c_scale, M, Nout, K, act, 0};
  const int size = out_dtype == HERO_DTYPE_FP32 ? 4 : (out_dtype == HERO_DTYPE_BF16 ? 2 : 1);
  const unsigned long long low = (unsigned long long)reinterpret_cast<uintptr_t>(c) | (unsigned long long)Nout * size;
  g.vec = low % 32 == 0 ? 32 : (low % 16 == 0 ? 16 : 0);
  CUtensorMap tm_a, tm_w, tm_c = {};
  HERO_TRY(make_tmap_bytes(&tm_a, a, (uint64_t)M, (uint64_t)K, plan.swap ? plan.bn : kRows, false));
  HERO_TRY(make_tmap_bytes(&tm_w, w, (uint64_t)Nout, (uint64_t)K, plan.split == 0 ? PairCfg::kCols : (plan.swap ? kRows : plan.bn), false));
  if (plan.split == 0 && g.vec) HERO_TRY(make_tmap_bytes(&tm_c, c, (uint64_t)M, (uint64_t)Nout * size, 32, true));
  switch (out_dtype) {
    case HERO_DTYPE_FP32: return launch_out<kOutF32>(plan, tm_a, tm_w, tm_c, g, d_status, s);
    case HERO_DTYPE_BF16: return launch_out<kOutBf16>(plan, tm_a, tm_w, tm_c, g, d_status, s);
    default: return launch_out<kOutF8>(plan, tm_a, tm_w, tm_c, g, d_status, s);
  }
}

}  // namespace hero
