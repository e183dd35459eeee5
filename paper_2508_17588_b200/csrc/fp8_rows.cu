// Kernels that write 8-bit operands with a scale per block, and the root-mean-square norm: one pass over the data each,
// bound by HBM.
//
//  * gather_ln_f8_kernel: the refresh prologue (gather, LayerNorm, modulation) in e4m3 with a scale per 128 columns.
//  * rms_norm_kernel: h = x + add (kept in the run dtype if asked for), y = h / sqrt(mean(h^2) + eps) * gain, y in the run dtype or
//    in e4m3 with a scale per 128 columns.
//  * quantize_rows_kernel / quantize_tiles_kernel: a matrix to e4m3 with a scale per 1 x 128 or 128 x 128 elements.
#include "fp8_common.cuh"
#include "hero_internal.h"

namespace hero {
namespace {

// ------------------------------------------------------------------ 16 bytes of a lane
template <typename T>
struct Pack;
template <>
struct Pack<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const uint4& r, float2 (&f)[2]) {
    f[0] = make_float2(__uint_as_float(r.x), __uint_as_float(r.y)); f[1] = make_float2(__uint_as_float(r.z), __uint_as_float(r.w));
  }
};
template <>
struct Pack<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const uint4& r, float2 (&f)[4]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
  }
};

// A packet to e4m3 (`to`: where it goes).
template <typename T>
__device__ __forceinline__ void store_f8(uint8_t* to, const float2 (&f)[Pack<T>::N / 2], float inv) {
  constexpr int N = Pack<T>::N;
  const float2 i2 = make_float2(inv, inv);
  uint32_t w[N / 4];
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    const float2 a = __fmul2_rn(f[2 * i], i2), b = __fmul2_rn(f[2 * i + 1], i2);
    w[i] = f8_pack4(a.x, a.y, b.x, b.y);
  }
  if constexpr (N == 8) __stcs(reinterpret_cast<uint2*>(to), make_uint2(w[0], w[1]));
  else __stcs(reinterpret_cast<uint32_t*>(to), w[0]);
}

// Scales of a row's blocks from the magnitudes' bits m[c] that a lane has in its chunk c of 32 lanes (zeros past the end of the row), blocks
// being LANES lanes that stand side by side: factors for the lane's values, scales to `row_scale`.  The maxima of all chunks go through
// the shuffles together, and of a block's lanes each works out another chunk's scale, so that a warp divides once a row and not
// once a chunk.  v0: place of the lane's chunk 0 in the row, step: from a chunk to the next, n: places in the row.
template <int LANES, int V>
__device__ __forceinline__ void row_scales(uint32_t (&m)[V], float (&inv)[V], float* row_scale, int v0, int step, int n) {
  static_assert(V <= LANES, "a lane for every chunk of a block");
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1)
#pragma unroll
    for (int c = 0; c < V; ++c) m[c] = max(m[c], __shfl_xor_sync(0xFFFFFFFFu, m[c], o));
  const int lane = threadIdx.x & 31, mine = lane & (LANES - 1);
  uint32_t pick = m[0];
#pragma unroll
  for (int c = 1; c < V; ++c) pick = mine == c ? m[c] : pick;
  const F8Scale s = f8_scale(pick);
  const int first = v0 - mine + mine * step;           // first place of the block that this lane did
  if (mine < V && first < n) row_scale[first / LANES] = s.scale;
#pragma unroll
  for (int c = 0; c < V; ++c) inv[c] = V == 1 ? s.inv : __shfl_sync(0xFFFFFFFFu, s.inv, (lane & ~(LANES - 1)) | c);
}

// What was made of `r` so far is made again where it is needed next and not kept in registers meanwhile.
__device__ __forceinline__ void again(uint4& r) { asm volatile("" : "+r"(r.x), "+r"(r.y), "+r"(r.z), "+r"(r.w)); }

// ------------------------------------------------------------------ 32 bytes of a lane
// A lane's piece of a row: two packets of 16 bytes, N elements as pairs; kLanes of them are a block of 128 columns.
template <typename T>
struct Piece {
  static constexpr int N = 32 / (int)sizeof(T), kLanes = kF8Block / N, kPacket = N / 2;
};
__device__ __forceinline__ void unpack(const uint4 (&r)[2], float2 (&f)[4], float) {
  f[0] = make_float2(__uint_as_float(r[0].x), __uint_as_float(r[0].y)); f[1] = make_float2(__uint_as_float(r[0].z), __uint_as_float(r[0].w));
  f[2] = make_float2(__uint_as_float(r[1].x), __uint_as_float(r[1].y)); f[3] = make_float2(__uint_as_float(r[1].z), __uint_as_float(r[1].w));
}
__device__ __forceinline__ void unpack(const uint4 (&r)[2], float2 (&f)[8], __nv_bfloat16) {
  const uint32_t w[8] = {r[0].x, r[0].y, r[0].z, r[0].w, r[1].x, r[1].y, r[1].z, r[1].w};
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
}
__device__ __forceinline__ void pack(uint4 (&r)[2], const float2 (&f)[4], float) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
    r[h] = make_uint4(__float_as_uint(f[2 * h].x), __float_as_uint(f[2 * h].y), __float_as_uint(f[2 * h + 1].x), __float_as_uint(f[2 * h + 1].y));
}
__device__ __forceinline__ void pack(uint4 (&r)[2], const float2 (&f)[8], __nv_bfloat16) {
  uint32_t w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(f[i].x, f[i].y);
    w[i] = *reinterpret_cast<const uint32_t*>(&p);
  }
  r[0] = make_uint4(w[0], w[1], w[2], w[3]);
  r[1] = make_uint4(w[4], w[5], w[6], w[7]);
}
// Packets 2v and 2v + 1 of a row that has `packets` (zeros past its end).
template <bool STREAM>
__device__ __forceinline__ void load_piece(uint4 (&r)[2], const void* row, int v, int packets) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint4* from = static_cast<const uint4*>(row) + 2 * v + h;
    r[h] = 2 * v + h < packets ? (STREAM ? __ldcs(from) : __ldg(from)) : make_uint4(0, 0, 0, 0);
  }
}
__device__ __forceinline__ void store_piece(void* row, const uint4 (&r)[2], int v, int packets) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
    if (2 * v + h < packets) __stcs(static_cast<uint4*>(row) + 2 * v + h, r[h]);
}
template <typename T>
__device__ __forceinline__ uint32_t piece_amax(const float2 (&f)[Piece<T>::N / 2]) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < Piece<T>::N / 2; ++i) m = max_abs3(m, f[i].x, f[i].y);
  return __float_as_uint(m);
}
// Piece v of a row to e4m3 (`row`: the row's bytes).
template <typename T>
__device__ __forceinline__ void store_f8(uint8_t* row, const float2 (&f)[Piece<T>::N / 2], float inv, int v) {
  constexpr int N = Piece<T>::N;
  uint32_t w[N / 4];
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    const float2 a = __fmul2_rn(f[2 * i], make_float2(inv, inv)), b = __fmul2_rn(f[2 * i + 1], make_float2(inv, inv));
    w[i] = f8_pack4(a.x, a.y, b.x, b.y);
  }
  if constexpr (N == 16) __stcs(reinterpret_cast<uint4*>(row) + v, make_uint4(w[0], w[1], w[2], w[3]));
  else __stcs(reinterpret_cast<uint2*>(row) + v, make_uint2(w[0], w[1]));
}

// ------------------------------------------------------------------ rows in registers
// G warps hold a row, V pieces a lane (the last predicated), G growing with the row so that a lane never holds more than three: all
// its loads are in flight at once, and enough rows are resident.  One row and done: CTAs that stay and fetch the next row ahead took
// 122 us for 35552 rows of 3072 where these take 114.  Beside the bytes the kernel costs instructions, about as long as the bytes where a
// row is read once and written in 8 bits: 8774 rows of 3072 bf16 through the norm alone take 17 us with packed arithmetic, a scale
// a warp and no division by the row's length, 20.4 without.
__host__ __device__ constexpr int rows_threads(int g) { return g == 1 ? 256 : 32 * g; }
template <int G>
struct RowThreads {
  int lane, warp, t;             // t: among the row's threads
  long long row;
  __device__ __forceinline__ RowThreads()
      : lane(threadIdx.x & 31), warp(threadIdx.x >> 5), t(G == 1 ? threadIdx.x & 31 : threadIdx.x),
        row(G == 1 ? (long long)blockIdx.x * 8 + (threadIdx.x >> 5) : blockIdx.x) {}
  // Sum over a row; `part` [G] is used once.
  __device__ __forceinline__ float total(float v, float* part) const {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    if constexpr (G > 1) {
      if (lane == 0) part[warp] = v;
      __syncthreads();
      v = 0.f;
#pragma unroll
      for (int w = 0; w < G; ++w) v += part[w];
    }
    return v;
  }
};
// x, and add where there is one, as fp32 pairs.
template <typename T, int G, int V>
__device__ __forceinline__ void load_rows(float2 (&f)[V][Piece<T>::N / 2], const T* x, const T* add, int t, int packets) {
  uint4 vx[V][2], va[V][2];
#pragma unroll
  for (int c = 0; c < V; ++c) load_piece<true>(vx[c], x, c * 32 * G + t, packets);
  if (add) {
#pragma unroll
    for (int c = 0; c < V; ++c) load_piece<true>(va[c], add, c * 32 * G + t, packets);
  }
#pragma unroll
  for (int c = 0; c < V; ++c) {
    unpack(vx[c], f[c], T());
    if (add) {
      float2 g[Piece<T>::N / 2];
      unpack(va[c], g, T());
#pragma unroll
      for (int i = 0; i < Piece<T>::N / 2; ++i) f[c][i] = __fadd2_rn(f[c][i], g[i]);
    }
  }
}

// ------------------------------------------------------------------ root-mean-square norm
// A thread reads and writes the same packets of a row, so `sum` (or, in the run dtype, `out`) may be x or add.
// Bound by HBM: 35552 x 3072 bf16 with add and sum, e4m3 out, 114 us (6.7 TB/s).
template <typename T, int G, int V, bool Q8>
__global__ void __launch_bounds__(rows_threads(G))
rms_norm_kernel(const T* x, const T* add, const T* __restrict__ gain, T* sum, void* out, float* __restrict__ out_scale,
                int rows, int D, float inv_d, float eps) {
  stream_order();
  constexpr int N = Piece<T>::N;
  __shared__ float s_part[G];
  const RowThreads<G> w;
  if (G == 1 && w.row >= rows) return;
  const int packets = D / Piece<T>::kPacket;
  const long long at = w.row * D;
  float2 f[V][N / 2];
  load_rows<T, G, V>(f, x + at, add ? add + at : nullptr, w.t, packets);
  float2 sq = make_float2(0.f, 0.f);
#pragma unroll
  for (int c = 0; c < V; ++c) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) sq = __ffma2_rn(f[c][i], f[c][i], sq);
    if (sum) {
      uint4 r[2];
      pack(r, f[c], T());
      store_piece(sum + at, r, c * 32 * G + w.t, packets);
    }
  }
  const float rstd = rsqrtf(fmaf(w.total(sq.x + sq.y, s_part), inv_d, eps));
  uint32_t m[V];
#pragma unroll
  for (int c = 0; c < V; ++c) {
    const int v = c * 32 * G + w.t;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) f[c][i] = __fmul2_rn(f[c][i], make_float2(rstd, rstd));
    if (gain) {
      uint4 r[2];
      float2 g[N / 2];
      load_piece<false>(r, gain, v, packets);
      unpack(r, g, T());
#pragma unroll
      for (int i = 0; i < N / 2; ++i) f[c][i] = __fmul2_rn(f[c][i], g[i]);
    }
    if constexpr (Q8) {
      m[c] = piece_amax<T>(f[c]);
    } else {
      uint4 r[2];
      pack(r, f[c], T());
      store_piece(static_cast<T*>(out) + at, r, v, packets);
    }
  }
  if constexpr (Q8) {
    float inv[V];
    row_scales<Piece<T>::kLanes, V>(m, inv, out_scale + w.row * ((D + kF8Block - 1) / kF8Block), w.t, 32 * G, packets / 2);
#pragma unroll
    for (int c = 0; c < V; ++c) {
      const int v = c * 32 * G + w.t;
      if (2 * v < packets) store_f8<T>(static_cast<uint8_t*>(out) + at, f[c], inv[c], v);
    }
  }
}

// ------------------------------------------------------------------ gather + LayerNorm + modulate
// G warps take the rows of ONE batch item one after the other, a lane V packets of 16 bytes of each, and with them the item's
// (1 + scale) and shift of those columns: a thread puts the ones that it needs into shared memory, side by side with its neighbours'
// (no bank conflicts, and nobody else reads them, so no barrier).  The next row is on its way while this one is reduced (mean, then
// squared differences from it) and stored, and the list is read 32 turns at a time, an entry a lane.  8774 rows of 3072 with a second row
// to add, from two items: 26.1 us (5.2 TB/s); 31.7 with an entry of the list asked for every turn, for which, or for something that shares its
// scoreboard, a warp then waited; 33 and 39 (both so) with the vectors read from L1 for every row and with them in registers, which leaves
// 12 warps an SM.  Bound by instructions, 450 a warp for 24 elements a lane, and the chain of two reductions and a maximum a row.
__host__ __device__ constexpr int ln_threads(int g) { return g == 1 ? 256 : 32 * g; }
constexpr int ln_smem(int g, int v, int n) { return v * 2 * n * 4 * ln_threads(g); }
constexpr int ln_ctas_per_sm(int g, int v, int n) {            // n elements a packet; registers: the row, the next two packets and the rest
  const int regs = (g > 1 && v < 3 ? 32 : 40) + v * (n + 8), warps = ln_threads(g) / 32, by_regs = 64 * 1024 / (32 * warps * ((regs + 7) / 8 * 8));
  const int by_smem = 220 * 1024 / (ln_smem(g, v, n) + 1024), by_warps = 64 / warps;
  const int least = by_regs < by_smem ? (by_regs < by_warps ? by_regs : by_warps) : (by_smem < by_warps ? by_smem : by_warps);
  return least < 1 ? 1 : least;
}
template <typename T, int G, int V>
__global__ void __launch_bounds__(ln_threads(G), ln_ctas_per_sm(G, V, Pack<T>::N))
gather_ln_f8_kernel(const T* __restrict__ x, const T* __restrict__ add, const int* __restrict__ idx, const float* __restrict__ shift,
                    const float* __restrict__ scale, int mod_ld, int vec, uint8_t* __restrict__ out, float* __restrict__ out_scale,
                    int n_rows, int n_sel, int B, int D, float inv_d, float eps) {
  stream_order();
  using P = Pack<T>;
  constexpr int N = P::N, kLanes = kF8Block / N, kThreads = ln_threads(G);
  extern __shared__ float4 s_mod[];              // [V][1 + scale, shift][N / 4][threads]
  __shared__ float s_part[2][G];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, t = G == 1 ? lane : (int)threadIdx.x;
  const int b = blockIdx.x % B, packets = D / N, blocks = (D + kF8Block - 1) / kF8Block;
  const long long first = G == 1 ? (long long)(blockIdx.x / B) * 8 + warp : blockIdx.x / B, step = (long long)(gridDim.x / B) * (G == 1 ? 8 : 1);
  uint4 vx[V], va[V];
  int listed = 0;                                // entries of the list for the next 32 turns, a lane each
  auto look = [&](long long i) {
    const long long mine = i + lane * step;
    if (mine < n_sel) listed = idx ? __ldg(idx + mine) : (int)mine;
  };
  auto fetch = [&](long long i, int turn) {
    if (i >= n_sel) return;
    const int entry = __shfl_sync(0xFFFFFFFFu, listed, turn & 31);
    const long long from = ((long long)b * n_rows + entry) * D;
    const uint4* xr = reinterpret_cast<const uint4*>(x + from);
    const uint4* ar = reinterpret_cast<const uint4*>(add + from);
#pragma unroll
    for (int c = 0; c < V; ++c) {
      const int v = c * 32 * G + t;
      vx[c] = v < packets ? __ldcs(xr + v) : make_uint4(0, 0, 0, 0);
      if (add) va[c] = v < packets ? __ldcs(ar + v) : make_uint4(0, 0, 0, 0);
    }
  };
  auto total = [&](float2 p, float* part) {      // over the row
    float v = p.x + p.y;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    if constexpr (G > 1) {
      if (lane == 0) part[warp] = v;
      __syncthreads();
      v = 0.f;
#pragma unroll
      for (int w = 0; w < G; ++w) v += part[w];
    }
    return v;
  };
  look(first);
  fetch(first, 0);
  const float* sc = scale + (long long)b * mod_ld;
  const float* sh = shift + (long long)b * mod_ld;
#pragma unroll
  for (int c = 0; c < V; ++c) {
    const int v = c * 32 * G + t;
    if (v < packets) {
#pragma unroll
      for (int q = 0; q < N / 4; ++q) {
        float4 s4, h4;
        if (vec) {
          s4 = __ldg(reinterpret_cast<const float4*>(sc) + v * (N / 4) + q);
          h4 = __ldg(reinterpret_cast<const float4*>(sh) + v * (N / 4) + q);
        } else {
          const float *a = sc + v * N + 4 * q, *e = sh + v * N + 4 * q;
          s4 = make_float4(__ldg(a), __ldg(a + 1), __ldg(a + 2), __ldg(a + 3));
          h4 = make_float4(__ldg(e), __ldg(e + 1), __ldg(e + 2), __ldg(e + 3));
        }
        s_mod[((c * 2) * (N / 4) + q) * kThreads + threadIdx.x] = make_float4(1.0f + s4.x, 1.0f + s4.y, 1.0f + s4.z, 1.0f + s4.w);
        s_mod[((c * 2 + 1) * (N / 4) + q) * kThreads + threadIdx.x] = h4;
      }
    }
  }
  int turn = 0;
  for (long long i = first; i < n_sel; i += step) {            // (the same turns for a row's threads)
    float2 f[V][N / 2];
    float2 sum = make_float2(0.f, 0.f), sq = make_float2(0.f, 0.f);
#pragma unroll
    for (int c = 0; c < V; ++c) {
      P::unpack(vx[c], f[c]);
      if (add) {
        float2 a[N / 2];
        P::unpack(va[c], a);
#pragma unroll
        for (int q = 0; q < N / 2; ++q) f[c][q] = __fadd2_rn(f[c][q], a[q]);
      }
#pragma unroll
      for (int q = 0; q < N / 2; ++q) sum = __fadd2_rn(sum, f[c][q]);
    }
    if ((++turn & 31) == 0) look(i + step);
    fetch(i + step, turn);
    const float mean = total(sum, s_part[0]) * inv_d;
    const float2 neg = make_float2(-mean, -mean);
#pragma unroll
    for (int c = 0; c < V; ++c)
      if (c * 32 * G + t < packets) {            // (absent packets stay zeros)
#pragma unroll
        for (int q = 0; q < N / 2; ++q) {
          f[c][q] = __fadd2_rn(f[c][q], neg);
          sq = __ffma2_rn(f[c][q], f[c][q], sq);
        }
      }
    const float rstd = rsqrtf(fmaf(total(sq, s_part[1]), inv_d, eps));
    const float2 rstd2 = make_float2(rstd, rstd);
    uint32_t m[V];
#pragma unroll
    for (int c = 0; c < V; ++c) {
      float most = 0.f;
      if (c * 32 * G + t < packets) {
#pragma unroll
        for (int q = 0; q < N / 4; ++q) {
          const float4 s4 = s_mod[((c * 2) * (N / 4) + q) * kThreads + threadIdx.x], h4 = s_mod[((c * 2 + 1) * (N / 4) + q) * kThreads + threadIdx.x];
          float2* u = &f[c][2 * q];
          u[0] = __ffma2_rn(__fmul2_rn(u[0], rstd2), make_float2(s4.x, s4.y), make_float2(h4.x, h4.y));
          u[1] = __ffma2_rn(__fmul2_rn(u[1], rstd2), make_float2(s4.z, s4.w), make_float2(h4.z, h4.w));
          most = max_abs3(max_abs3(most, u[0].x, u[0].y), u[1].x, u[1].y);
        }
      }
      m[c] = __float_as_uint(most);
    }
    const long long row = (long long)b * n_sel + i;
    float inv[V];
    row_scales<kLanes, V>(m, inv, out_scale + row * blocks, t, 32 * G, packets);
#pragma unroll
    for (int c = 0; c < V; ++c) {
      const int v = c * 32 * G + t;
      if (v < packets) store_f8<T>(out + row * D + (long long)v * N, f[c], inv[c]);
    }
  }
}

// The smallest G warps a row and V pieces (or packets) a lane that hold a row of `chunks` times 32 of them.
#define HERO_ROWS_CASE(G, V, LAUNCH) \
  if (chunks <= G * V) { LAUNCH(G, V); }
#define HERO_ROWS(LAUNCH)                                                              \
  HERO_ROWS_CASE(1, 1, LAUNCH) HERO_ROWS_CASE(1, 2, LAUNCH) HERO_ROWS_CASE(1, 3, LAUNCH)  \
  HERO_ROWS_CASE(2, 2, LAUNCH) HERO_ROWS_CASE(2, 3, LAUNCH)                              \
  HERO_ROWS_CASE(4, 2, LAUNCH) HERO_ROWS_CASE(4, 3, LAUNCH)                              \
  HERO_ROWS_CASE(8, 2, LAUNCH) HERO_ROWS_CASE(8, 3, LAUNCH)
#define HERO_ROWS_16(LAUNCH) HERO_ROWS_CASE(16, 2, LAUNCH) HERO_ROWS_CASE(16, 3, LAUNCH)
static inline int row_chunks(int D, int piece) { return (D - 1) / (32 * piece) + 1; }
static inline long long row_ctas(int g, long long rows) { return g == 1 ? (rows + 7) / 8 : rows; }
// (All of these kernels are placed early, also those of more blocks than fit the chip: they are waited for by nobody while they wait, and a
// call among others saves the launch, 16.4 -> 14.5 us for the quantiser on 8774 x 3072 bf16.)

template <typename T>
int gather_ln_f8_dispatch(const void* x, const void* add, const int* idx, const float* shift, const float* scale, int mod_ld, void* out,
                          float* out_scale, int B, int N, int n_sel, int D, float eps, cudaStream_t s) {
  const int chunks = row_chunks(D, Pack<T>::N);
  const int vec = mod_ld % 4 == 0 && aligned16(shift) && aligned16(scale);       // the vectors may be read 16 bytes at a time
  // the same number of CTAs for every batch item, at most as many as stay resident
  auto ctas = [&](int g, int per_sm) {
    const long long need = g == 1 ? (n_sel - 1) / 8 + 1 : n_sel, most = ((long long)num_sms() * per_sm + B - 1) / B;
    return (unsigned)((need < most ? need : most) * B);
  };
#define HERO_LN_F8(G, V)                                                                                                              \
  constexpr int smem = ln_smem(G, V, Pack<T>::N);                                                                                     \
  if (smem > 47 * 1024) {                                                                                                             \
    static PerDeviceOnce once;                                                                                                        \
    HERO_TRY(per_device_once(once, [](int) {                                                                                          \
      HERO_CUDA_TRY(cudaFuncSetAttribute(gather_ln_f8_kernel<T, G, V>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));           \
      return HERO_OK;                                                                                                                 \
    }));                                                                                                                              \
  }                                                                                                                                   \
  return launch_kernel(gather_ln_f8_kernel<T, G, V>, ctas(G, ln_ctas_per_sm(G, V, Pack<T>::N)), ln_threads(G), smem, s, 1, (const T*)x, \
                       (const T*)add, idx, shift, scale, mod_ld, vec, (uint8_t*)out, out_scale, N, n_sel, B, D, 1.0f / (float)D, eps)
  HERO_ROWS(HERO_LN_F8)
  HERO_ROWS_16(HERO_LN_F8)
  if constexpr (sizeof(T) == 4) { HERO_ROWS_CASE(16, 6, HERO_LN_F8) }            // rows of more than 6144
#undef HERO_LN_F8
  return HERO_ERR_ARG;
}

template <typename T, bool Q8>
int rms_norm_dispatch(const void* x, const void* add, const void* gain, void* sum, void* out, float* out_scale, int rows, int D,
                      float eps, cudaStream_t s) {
  const int chunks = row_chunks(D, Piece<T>::N);
#define HERO_RMS(G, V)                                                                                                          \
  return launch_kernel(rms_norm_kernel<T, G, V, Q8>, (unsigned)row_ctas(G, rows), rows_threads(G), 0, s, 1, (const T*)x, (const T*)add,         \
                          (const T*)gain, (T*)sum, out, out_scale, rows, D, 1.0f / (float)D, eps)
  HERO_ROWS(HERO_RMS)
  if constexpr (sizeof(T) == 4) { HERO_ROWS_16(HERO_RMS) }                       // (12288 columns of bf16 are 8 warps' three pieces)
#undef HERO_RMS
  return HERO_ERR_ARG;
}

// ------------------------------------------------------------------ blocks of 1 x 128
// A warp takes 512 columns of bf16 or 256 of fp32 of a row and nothing else: the more warps, the better the loads of some overlap the
// stores of others (8774 x 3072 bf16: 14.4 us with one piece a lane, 15.6 with two, 16.6 with four; 19.0 with four of 16 bytes).
template <typename T>
__global__ void __launch_bounds__(256)
quantize_rows_kernel(const T* __restrict__ x, uint8_t* __restrict__ out, float* __restrict__ scale, int cols, int per_row,
                     long long pieces) {
  stream_order();
  const long long piece = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (piece >= pieces) return;                                 // warp-uniform
  const long long row = piece / per_row;
  const int v = (int)(piece - row * per_row) * 32 + (threadIdx.x & 31), packets = cols / Piece<T>::kPacket;
  uint4 raw[2];
  load_piece<true>(raw, x + row * cols, v, packets);
  uint32_t m[1];
  {
    float2 f[Piece<T>::N / 2];
    unpack(raw, f, T());
    m[0] = piece_amax<T>(f);
  }
  float inv[1];
  row_scales<Piece<T>::kLanes, 1>(m, inv, scale + row * ((cols + kF8Block - 1) / kF8Block), v, 0, packets / 2);
  again(raw[0]);               // (31 registers and all warps resident: 14.4 us for 15.5)
  again(raw[1]);
  float2 f[Piece<T>::N / 2];
  unpack(raw, f, T());
  if (2 * v < packets) store_f8<T>(out + row * cols, f, inv[0], v);
}

// ------------------------------------------------------------------ blocks of 128 x 128
// One CTA a block, held in registers between the maximum and the rounding.
template <typename T>
__global__ void __launch_bounds__(256)
quantize_tiles_kernel(const T* __restrict__ x, uint8_t* __restrict__ out, float* __restrict__ scale, int rows, int cols,
                      int col_blocks) {
  stream_order();
  using P = Pack<T>;
  constexpr int kLanes = kF8Block / P::N, kStep = 256 / kLanes, kVec = kF8Block / kStep;
  __shared__ uint32_t s_max[8];
  const int rb = blockIdx.x / col_blocks, cb = blockIdx.x - rb * col_blocks;
  const int col = cb * kF8Block + (threadIdx.x % kLanes) * P::N;
  const int r0 = rb * kF8Block + threadIdx.x / kLanes;
  uint4 raw[kVec];
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    raw[i] = make_uint4(0, 0, 0, 0);
    const int r = r0 + i * kStep;
    if (r < rows && col < cols) raw[i] = __ldcs(reinterpret_cast<const uint4*>(x + (long long)r * cols + col));
  }
  float m[2] = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    float2 f[P::N / 2];
    P::unpack(raw[i], f);
#pragma unroll
    for (int q = 0; q < P::N / 2; ++q) m[i & 1] = max_abs3(m[i & 1], f[q].x, f[q].y);
  }
  uint32_t bits = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(max_abs3(0.f, m[0], m[1])));
  if ((threadIdx.x & 31) == 0) s_max[threadIdx.x >> 5] = bits;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 8; ++w) bits = max(bits, s_max[w]);
  const F8Scale s = f8_scale(bits);
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    const int r = r0 + i * kStep;
    if (r < rows && col < cols) {
      float2 f[P::N / 2];
      again(raw[i]);           // (12288 x 3072 bf16: 19.4 us, and 22 with the 64 values kept)
      P::unpack(raw[i], f);
      store_f8<T>(out + (long long)r * cols + col, f, s.inv);
    }
  }
  if (threadIdx.x == 0) scale[blockIdx.x] = s.scale;
}

template <typename T>
int quantize_t(const void* x, void* q, float* scale, int rows, int cols, int block_rows, cudaStream_t s) {
  const int col_blocks = (cols - 1) / kF8Block + 1;
  if (block_rows == 1) {
    const int per_row = row_chunks(cols, Piece<T>::N);
    const long long pieces = (long long)rows * per_row, blocks = (pieces + 7) / 8;
    if (blocks > 0x7FFFFFFFll) return HERO_ERR_ARG;
    return launch_kernel(quantize_rows_kernel<T>, (unsigned)blocks, 256, 0, s, 1, (const T*)x, (uint8_t*)q, scale, cols, per_row, pieces);
  }
  const long long blocks = (long long)((rows + (long long)kF8Block - 1) / kF8Block) * col_blocks;
  if (blocks > 0x7FFFFFFFll) return HERO_ERR_ARG;
  return launch_kernel(quantize_tiles_kernel<T>, (unsigned)blocks, 256, 0, s, 1, (const T*)x, (uint8_t*)q, scale, rows, cols, col_blocks);
}

}  // namespace

int launch_quantize_fp8(const void* x, void* q, float* scale, int rows, int cols, int block_rows, int dtype, cudaStream_t s) {
  return dtype == HERO_DTYPE_BF16 ? quantize_t<__nv_bfloat16>(x, q, scale, rows, cols, block_rows, s)
                                  : quantize_t<float>(x, q, scale, rows, cols, block_rows, s);
}

int launch_gather_ln_modulate_fp8(const void* x, const void* add, const int* idx, const float* shift, const float* scale, int mod_ld,
                                  void* out, float* out_scale, int B, int N, int n_sel, int D, float eps, int dtype, cudaStream_t s) {
  return dtype == HERO_DTYPE_BF16
             ? gather_ln_f8_dispatch<__nv_bfloat16>(x, add, idx, shift, scale, mod_ld, out, out_scale, B, N, n_sel, D, eps, s)
             : gather_ln_f8_dispatch<float>(x, add, idx, shift, scale, mod_ld, out, out_scale, B, N, n_sel, D, eps, s);
}

int launch_rms_norm(const void* x, const void* add, const void* gain, void* sum, void* out, float* out_scale, int rows, int D,
                    float eps, int dtype, cudaStream_t s) {
  if (dtype == HERO_DTYPE_BF16)
    return out_scale ? rms_norm_dispatch<__nv_bfloat16, true>(x, add, gain, sum, out, out_scale, rows, D, eps, s)
                     : rms_norm_dispatch<__nv_bfloat16, false>(x, add, gain, sum, out, out_scale, rows, D, eps, s);
  return out_scale ? rms_norm_dispatch<float, true>(x, add, gain, sum, out, out_scale, rows, D, eps, s)
                   : rms_norm_dispatch<float, false>(x, add, gain, sum, out, out_scale, rows, D, eps, s);
}

}  // namespace hero
