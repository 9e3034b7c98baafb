// Values of 8-bit pages: x8 s with x8 of 1 sign, 4 exponent and 3 mantissa bits (largest 448, smallest step 2^-9,
// no infinities) and a scale s = 2^e for each page, key/value head and K or V. A float wants no finer scale than a
// power of two: its relative steps are the same wherever its range lies, and with such a scale a value is put in
// units of it, and taken out again, exactly. e is the least in -60 .. 60 that brings the page's largest value to
// 448 or below, so that 2^-17 of it still has all bits. Values that are not finite, or above 448 2^60, are NaN in 8
// bits and have no part in the scale.
#pragma once

#include <cuda_fp16.h>

#include <cstdint>

namespace mot {
namespace {

constexpr float kLargest8 = 448.f * 1152921504606846976.f;   // 448 2^60
constexpr uint32_t kNaN8 = 0x7Fu;

__device__ __forceinline__ bool held8(float x) { return fabsf(x) <= kLargest8; }   // false for NaN

// The scale for a largest value `top`, finite and not negative: 448 is 1.75 2^8.
__device__ __forceinline__ float scale8(float top) {
  const uint32_t u = __float_as_uint(top);
  const int e = int(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u);
  return __uint_as_float(uint32_t(min(max(e, -60), 60) + 127) << 23);
}

// A page's scale x as it lay in memory: a caller may have written it. What is not a power of two in range is taken as the
// one below (the end of the range beyond it), by every call alike, and reported. The question waits for the load: asked
// beside it, 64 decoding steps of 100 to 16,384 positions took 58.1 us for 54.6.
__device__ __forceinline__ bool is_scale8(float x) {
  const uint32_t u = __float_as_uint(x);
  return (u & 0x7FFFFFu) == 0 && u - (67u << 23) <= 120u << 23;
}
__device__ __forceinline__ float scale_of_page(float x, int32_t* status) {
  if (is_scale8(x)) return x;
  atomicOr(status, kStatusPageUse);
  return __uint_as_float(min(max(__float_as_uint(x) >> 23 & 255u, 67u), 187u) << 23);
}

// Four values in units of the scale to 8 bits, to the nearest, ties to the even one; the first in the lowest byte.
__device__ __forceinline__ uint32_t pack8(float a, float b, float c, float d) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
  return uint32_t(lo) | uint32_t(hi) << 16;
}
// The same of values in their own units, inv = 1 / scale: what 8 bits do not hold becomes NaN.
__device__ __forceinline__ float unit8(float x, float inv) { return held8(x) ? x * inv : __uint_as_float(0x7FC00000u); }

// Which of a word's four values are NaN, as bit 7 of each.
__device__ __forceinline__ uint32_t nan8(uint32_t u) { return ((u & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u; }

// Two 8-bit values (of the lower or the upper half of a word) as fp16, exactly; NaN stays NaN.
__device__ __forceinline__ uint32_t half2_of8(uint32_t pair) {
  uint32_t y;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(y) : "h"(static_cast<uint16_t>(pair)));
  return y;
}

__device__ __forceinline__ float2 float2_of8(uint32_t pair) {
  const uint32_t h = half2_of8(pair);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// A query's row in two 8-bit parts, q = (hi + lo) 2^-up: put by a power of two so that its largest value is at 2^7,
// each part takes 4 of the 8 bits that a bf16 has. That is exact from 2^-9 of the row's largest on, and off by 2^-17
// of that below (or by 2^-130, which no key makes count: the power is 2^120 at most).
// Two products with 8-bit keys take as long as one of 16 bits, and no key is converted.
struct Split8 {
  float by;       // 2^up
  float factor;   // 2^-up; NaN for a row that holds an infinity or NaN
  // top: the largest magnitude of the row as the bits of a bf16
  __device__ __forceinline__ explicit Split8(uint32_t top) {
    const int up = min(7 + 127 - int(top >> 7), top ? 120 : 60);   // a row of zeros: any
    by = __uint_as_float(uint32_t(up + 127) << 23);
    factor = top >= 0x7F80u ? __uint_as_float(0x7FC00000u) : __uint_as_float(uint32_t(127 - up) << 23);
  }
  // Four bf16 in two words.
  __device__ __forceinline__ void operator()(uint32_t w0, uint32_t w1, uint32_t& hi, uint32_t& lo) const {
    const float a = __uint_as_float(w0 << 16) * by, b = __uint_as_float(w0 & 0xFFFF0000u) * by;
    const float c = __uint_as_float(w1 << 16) * by, d = __uint_as_float(w1 & 0xFFFF0000u) * by;
    hi = pack8(a, b, c, d);
    const float2 x = float2_of8(hi), y = float2_of8(hi >> 16);
    lo = pack8(a - x.x, b - x.y, c - y.x, d - y.y);
  }
};
// A row's factor times a key scale, held to fp32's normal range: from 2^-126 up, so that nothing masked by -inf is
// multiplied by 0 (scores below 2^-100 then, which make no weight), and finite, so that a score of 0 stays 0. NaN stays.
__device__ __forceinline__ float factor8(float row, float key_scale) {
  float x = row * key_scale;
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(x) : "f"(0x1p-126f));
  asm("min.NaN.f32 %0, %0, %1;" : "+f"(x) : "f"(0x1.fffffep127f));
  return x;
}
// The largest magnitude among eight bf16 and `top`, in each half: magnitudes of bf16 are ordered as integers.
__device__ __forceinline__ uint32_t top_bf16x2(uint32_t top, const uint4& u) {
  return __vmaxu2(top, __vmaxu2(__vmaxu2(u.x & 0x7FFF7FFFu, u.y & 0x7FFF7FFFu),
                                __vmaxu2(u.z & 0x7FFF7FFFu, u.w & 0x7FFF7FFFu)));
}

// n values (a multiple of 4) in units of a scale that grows, by n_threads threads: `ratio` is the old one over the
// new one, and what it pushes below the smallest steps is rounded again.
__device__ __forceinline__ void rescale8(uint8_t* x, int n, float ratio, int t, int n_threads) {
  uint32_t* p = reinterpret_cast<uint32_t*>(x);
  for (int k = t; k < n / 4; k += n_threads) {
    const uint32_t u = p[k];
    const float2 a = float2_of8(u), b = float2_of8(u >> 16);
    p[k] = pack8(a.x * ratio, a.y * ratio, b.x * ratio, b.y * ratio);
  }
}

}  // namespace
}  // namespace mot
