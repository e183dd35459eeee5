// e4m3 numbers with a scale per block: what the quantising kernels and epilogues share.
//
// A block of values v is stored as q = e4m3(v * inv) with inv = 1 / scale and scale = max(amax / 448, 2^-126), 448 being the
// largest e4m3: the block's largest magnitude uses the whole range, a block of zeros keeps a scale that can be inverted.  Scale
// and inverse are fp32, each rounded once; q is rounded once from an fp32 product (to nearest, ties to even).  A block that holds
// an infinity or a NaN has no such scale: its scale and all its values are NaN, so that what reads it sees NaN, not zeros.
#pragma once

#include <cuda_fp8.h>
#include <stdint.h>

namespace hero {

constexpr int kF8Block = 128;                    // columns (and, for weights, rows) of a block
constexpr float kF8InvMax = 1.0f / 448.0f;
constexpr float kF8ScaleFloor = 1.17549435e-38f; // 2^-126

// Magnitudes as their bits: ordered like the numbers, infinity above every number and NaN above infinity, so that an integer
// maximum carries both through.
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// The largest of m and the magnitudes of a and b, NaN if one of them is NaN (whose bits are then above infinity's): one
// instruction for two values where the integer maximum takes four (35552 x 3072 bf16 to e4m3 50.9 us for 52.2).
__device__ __forceinline__ float max_abs3(float m, float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(m), "f"(fabsf(a)), "f"(fabsf(b)));
  return r;
}

struct F8Scale { float scale, inv; };
__device__ __forceinline__ F8Scale f8_scale(uint32_t amax_bits) {
  F8Scale r;
  r.scale = fmaxf(__uint_as_float(amax_bits) * kF8InvMax, kF8ScaleFloor);
  r.inv = 1.0f / r.scale;
  if (amax_bits > 0x7F7FFFFFu) r.scale = r.inv = __uint_as_float(0x7FC00000u);
  return r;
}
// Four values to four e4m3 bytes, the first in the lowest.  (|v| is at most 448 and a rounding: nothing saturates.)
__device__ __forceinline__ uint32_t f8_pack4(float a, float b, float c, float d) {
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
  return lo | (hi << 16);
}

}  // namespace hero
