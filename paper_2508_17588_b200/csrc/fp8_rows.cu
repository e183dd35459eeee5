// Kernels that write 8-bit operands with a scale per block, and the root-mean-square norm: one pass over the data each,
// bound by HBM.
//
//  * rms_norm_kernel: h = x + add (kept in the run dtype if asked for), y = h / sqrt(mean(h^2) + eps) * gain, y in the run dtype or
//    in e4m3 with a scale per 128 columns.
//  * quantize_rows_kernel / quantize_tiles_kernel: a matrix to e4m3 with a scale per 1 x 128 or 128 x 128 elements.
#include "fp8_common.cuh"
#include "hero_internal.h"

namespace hero {
namespace {

// ------------------------------------------------------------------ 16-byte packets
template <typename T>
struct Pack;
template <>
struct Pack<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const uint4& r, float (&f)[4]) {
    f[0] = __uint_as_float(r.x); f[1] = __uint_as_float(r.y); f[2] = __uint_as_float(r.z); f[3] = __uint_as_float(r.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
};
template <>
struct Pack<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const uint4& r, float (&f)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 p = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&p);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// The lanes that hold a block's 128 columns: 16 of bf16 packets, 32 of fp32 ones.
template <typename T>
__device__ __forceinline__ uint32_t block_amax(const float (&f)[Pack<T>::N]) {
  uint32_t m = 0;
#pragma unroll
  for (int q = 0; q < Pack<T>::N; ++q) m = max(m, abs_bits(f[q]));
#pragma unroll
  for (int o = kF8Block / Pack<T>::N / 2; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
  return m;
}
// A packet's worth of e4m3 to `q` (N bytes).
template <typename T>
__device__ __forceinline__ void store_f8(uint8_t* q, const float (&f)[Pack<T>::N], float inv) {
  const uint32_t a = f8_pack4(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv);
  if constexpr (Pack<T>::N == 8) {
    const uint32_t b = f8_pack4(f[4] * inv, f[5] * inv, f[6] * inv, f[7] * inv);
    __stcs(reinterpret_cast<uint2*>(q), make_uint2(a, b));
  } else {
    __stcs(reinterpret_cast<unsigned int*>(q), a);
  }
}

// ------------------------------------------------------------------ root-mean-square norm
// G warps hold a row in registers, VPL packets of 16 bytes a lane (the last predicated): x and add are read once, the sum of
// squares is reduced by shuffles (and, over several warps, through shared memory), everything is written from the registers.
// G grows with the row so that a lane never holds more than six packets and all its loads are in flight at once.
// A thread reads and writes the same packets, so `sum` may be x or add.
constexpr int rms_threads(int g) { return g == 1 ? 256 : 32 * g; }
template <typename T, int G, int VPL, bool Q8>
__global__ void __launch_bounds__(rms_threads(G))
rms_norm_kernel(const T* x, const T* add, const T* __restrict__ gain, T* sum, void* out, float* __restrict__ out_scale,
                int rows, int D, float eps) {
  stream_order();
  using P = Pack<T>;
  constexpr int kRows = G == 1 ? 8 : 1;
  __shared__ float s_part[G == 1 ? 1 : G];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long row = (long long)blockIdx.x * kRows + (G == 1 ? warp : 0);
  if (G == 1 && row >= rows) return;
  const int t = G == 1 ? lane : (int)threadIdx.x;
  const int packets = D / P::N;
  const uint4* xr = reinterpret_cast<const uint4*>(x + row * D);
  const uint4* ar = reinterpret_cast<const uint4*>(add + row * D);
  uint4 vx[VPL], va[VPL];
#pragma unroll
  for (int c = 0; c < VPL; ++c) {
    const int v = c * 32 * G + t;
    vx[c] = va[c] = make_uint4(0, 0, 0, 0);
    if (v < packets) {
      vx[c] = __ldcs(xr + v);
      if (add) va[c] = __ldcs(ar + v);
    }
  }
  float f[VPL][P::N];
  float sq = 0.f;
#pragma unroll
  for (int c = 0; c < VPL; ++c) {
    P::unpack(vx[c], f[c]);
    if (add) {
      float g[P::N];
      P::unpack(va[c], g);
#pragma unroll
      for (int q = 0; q < P::N; ++q) f[c][q] += g[q];
    }
#pragma unroll
    for (int q = 0; q < P::N; ++q) sq = fmaf(f[c][q], f[c][q], sq);
    const int v = c * 32 * G + t;
    if (sum && v < packets) __stcs(reinterpret_cast<uint4*>(sum + row * D) + v, P::pack(f[c]));
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sq += __shfl_xor_sync(0xFFFFFFFFu, sq, o);
  if constexpr (G > 1) {
    if (lane == 0) s_part[warp] = sq;
    __syncthreads();
    sq = 0.f;
#pragma unroll
    for (int w = 0; w < G; ++w) sq += s_part[w];
  }
  const float rstd = 1.0f / sqrtf(sq / (float)D + eps);
#pragma unroll
  for (int c = 0; c < VPL; ++c) {
    const int v = c * 32 * G + t;
#pragma unroll
    for (int q = 0; q < P::N; ++q) f[c][q] *= rstd;
    if (gain && v < packets) {
      float g[P::N];
      P::unpack(__ldg(reinterpret_cast<const uint4*>(gain) + v), g);
#pragma unroll
      for (int q = 0; q < P::N; ++q) f[c][q] *= g[q];
    }
    if constexpr (Q8) {
      constexpr int kLanes = kF8Block / P::N;        // lanes of a block
      const F8Scale s = f8_scale(block_amax<T>(f[c]));
      if (v < packets) {
        store_f8<T>(static_cast<uint8_t*>(out) + row * D + (long long)v * P::N, f[c], s.inv);
        if (v % kLanes == 0) out_scale[row * ((D + kF8Block - 1) / kF8Block) + v / kLanes] = s.scale;
      }
    } else if (v < packets) {
      __stcs(reinterpret_cast<uint4*>(static_cast<T*>(out) + row * D) + v, P::pack(f[c]));
    }
  }
}

template <typename T, bool Q8>
int rms_norm_dispatch(const void* x, const void* add, const void* gain, void* sum, void* out, float* out_scale, int rows, int D,
                      float eps, cudaStream_t s) {
  const int chunks = (D / Pack<T>::N + 31) / 32;       // of 32 packets
#define HERO_RMS(G, V)                                                                                                      \
  if (chunks <= G * V)                                                                                                      \
  return launch_streaming(rms_norm_kernel<T, G, V, Q8>, G == 1 ? ((long long)rows + 7) / 8 : (long long)rows, rms_threads(G), s, \
                          (const T*)x, (const T*)add, (const T*)gain, (T*)sum, out, out_scale, rows, D, eps)
  HERO_RMS(1, 1); HERO_RMS(1, 2); HERO_RMS(1, 4);
  HERO_RMS(4, 2); HERO_RMS(4, 3); HERO_RMS(4, 4);
  HERO_RMS(8, 3); HERO_RMS(8, 4); HERO_RMS(8, 6);
  HERO_RMS(16, 4); HERO_RMS(16, 6);
#undef HERO_RMS
  return HERO_ERR_ARG;
}

// ------------------------------------------------------------------ blocks of 1 x 128
// A warp takes 32 packets of a row (256 columns of bf16, 128 of fp32) at a time, kPieces of them in flight.
constexpr int kQuantPieces = 4;
template <typename T>
__global__ void __launch_bounds__(256)
quantize_rows_kernel(const T* __restrict__ x, uint8_t* __restrict__ out, float* __restrict__ scale, int cols, int per_row,
                     long long pieces) {
  stream_order();
  using P = Pack<T>;
  constexpr int kLanes = kF8Block / P::N;
  const int lane = threadIdx.x & 31;
  const int packets = cols / P::N, blocks = (cols + kF8Block - 1) / kF8Block;
  const long long first = ((long long)blockIdx.x * 8 + (threadIdx.x >> 5)) * kQuantPieces;
  uint4 raw[kQuantPieces];
  long long row[kQuantPieces];
  int v[kQuantPieces];
#pragma unroll
  for (int i = 0; i < kQuantPieces; ++i) {
    const long long p = first + i;
    row[i] = p / per_row;
    v[i] = (int)(p - row[i] * per_row) * 32 + lane;
    if (p >= pieces) v[i] = packets;
    raw[i] = make_uint4(0, 0, 0, 0);
    if (v[i] < packets) raw[i] = __ldcs(reinterpret_cast<const uint4*>(x + row[i] * cols) + v[i]);
  }
#pragma unroll
  for (int i = 0; i < kQuantPieces; ++i) {
    float f[P::N];
    P::unpack(raw[i], f);
    const F8Scale s = f8_scale(block_amax<T>(f));
    if (v[i] < packets) {
      store_f8<T>(out + row[i] * cols + (long long)v[i] * P::N, f, s.inv);
      if (v[i] % kLanes == 0) scale[row[i] * blocks + v[i] / kLanes] = s.scale;
    }
  }
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
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    float f[P::N];
    P::unpack(raw[i], f);
#pragma unroll
    for (int q = 0; q < P::N; ++q) m = max(m, abs_bits(f[q]));
  }
  m = __reduce_max_sync(0xFFFFFFFFu, m);
  if ((threadIdx.x & 31) == 0) s_max[threadIdx.x >> 5] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 8; ++w) m = max(m, s_max[w]);
  const F8Scale s = f8_scale(m);
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    const int r = r0 + i * kStep;
    if (r < rows && col < cols) {
      float f[P::N];
      P::unpack(raw[i], f);
      store_f8<T>(out + (long long)r * cols + col, f, s.inv);
    }
  }
  if (threadIdx.x == 0) scale[blockIdx.x] = s.scale;
}

template <typename T>
int quantize_t(const void* x, void* q, float* scale, int rows, int cols, int block_rows, cudaStream_t s) {
  const int col_blocks = (cols + kF8Block - 1) / kF8Block;
  if (block_rows == 1) {
    const int per_row = (cols / Pack<T>::N + 31) / 32;
    const long long pieces = (long long)rows * per_row, blocks = (pieces + 8 * kQuantPieces - 1) / (8 * kQuantPieces);
    if (blocks > 0x7FFFFFFFll) return HERO_ERR_ARG;
    return launch_streaming(quantize_rows_kernel<T>, blocks, 256, s, (const T*)x, (uint8_t*)q, scale, cols, per_row, pieces);
  }
  const long long blocks = (long long)((rows + (long long)kF8Block - 1) / kF8Block) * col_blocks;
  if (blocks > 0x7FFFFFFFll) return HERO_ERR_ARG;
  return launch_streaming(quantize_tiles_kernel<T>, blocks, 256, s, (const T*)x, (uint8_t*)q, scale, rows, cols, col_blocks);
}

}  // namespace

int launch_quantize_fp8(const void* x, void* q, float* scale, int rows, int cols, int block_rows, int dtype, cudaStream_t s) {
  return dtype == HERO_DTYPE_BF16 ? quantize_t<__nv_bfloat16>(x, q, scale, rows, cols, block_rows, s)
                                  : quantize_t<float>(x, q, scale, rows, cols, block_rows, s);
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
