// Numbers in 8 bits with a power of two as scale for each block of 128: scales, rounding and widening.
//
// A block's scale is 2^e with the smallest e >= kLowest that takes the largest finite magnitude of the block to at most the
// format's largest number, which is 0.875 * 2^9 (e4m3) or 0.875 * 2^16 (e5m2); e = 0 for a block without any.  Dividing by
// it is exact, so that the one rounding is the one to 8 bits.  Infinities and NaN become NaN and have no part in the scale.
// e is stored as the byte e + 127, what the matrix instructions of sm_100a take as a scale.
#pragma once

#include "sgdb_rows.cuh"

namespace sgdb {

constexpr int kBlock = 128;    // elements that share a scale
constexpr int kLowest = -110;  // every value that is stored times its scale is then zero or a normal fp32 (and bf16) number

__host__ __device__ constexpr int blocks_of(long long n) { return static_cast<int>((n + kBlock - 1) / kBlock); }

// The scale's exponent for the largest finite magnitude of a block.
__device__ __forceinline__ int scale_exponent(float largest, int format) {
  const uint32_t top = __float_as_uint(largest);
  if (top == 0) return 0;
  const int e = static_cast<int>(top >> 23) - 126 - (format == SGDB_E4M3 ? 9 : 16) + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
  return e < kLowest ? kLowest : e;
}
__device__ __forceinline__ bool is_infinite(float x) { return fabsf(x) == INFINITY; }
// 2^e for e in [-126, 127]
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }
// 2^(byte - 127); byte 255 stands for NaN, and 0, which no call of this library writes, for a subnormal number
__device__ __forceinline__ float scale_value(uint32_t byte) {
  return byte == 255 ? __uint_as_float(0x7fffffffu) : byte == 0 ? __uint_as_float(0x00400000u) : __uint_as_float(byte << 23);
}

// Four numbers over their scale, to nearest even; the first in the lowest byte.  None is infinite; NaN stays NaN.
__device__ __forceinline__ uint32_t pack_f8(float a, float b, float c, float d, float inverse, int format) {
  const Pair by = pair(inverse);
  const float2 ab = split(mul2(pair(a, b), by)), cd = split(mul2(pair(c, d), by));
  a = ab.x, b = ab.y, c = cd.x, d = cd.y;
  uint16_t lo, hi;
  if (format == SGDB_E4M3) {
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
  } else {
    asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
  }
  return static_cast<uint32_t>(lo) | static_cast<uint32_t>(hi) << 16;
}

// Two numbers of 8 bits, not scaled: exact.
__device__ __forceinline__ float2 widen_f8x2(uint16_t two, int format) {
  uint32_t h;
  if (format == SGDB_E4M3)
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(two));
  else
    asm("cvt.rn.f16x2.e5m2x2 %0, %1;" : "=r"(h) : "h"(two));
  float2 v;
  asm("{\n"
      "  .reg .f16 lo, hi;\n"
      "  mov.b32 {lo, hi}, %2;\n"
      "  cvt.f32.f16 %0, lo;\n"
      "  cvt.f32.f16 %1, hi;\n"
      "}\n"
      : "=f"(v.x), "=f"(v.y)
      : "r"(h));
  return v;
}

}  // namespace sgdb
