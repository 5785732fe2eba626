// The 8-bit cache's numbers (decode_q8.hip).  A value is 2^k times an e4m3 number (4 significant bits, largest 448, smallest
// 2^-9, no infinity); k belongs to a block of Q8_BLOCK rows of a segment, of K and of V apart, and is the smallest with
// all of the block's finite magnitudes <= 448 * 2^k, within [Q8_LOW, Q8_HIGH].
//
// Why a power of two: e4m3 is a floating-point format, so another factor would not make the relative error of a value
// smaller, and multiplying by it is exact.  So quantising rounds once, and a block whose k has to grow for an appended
// row keeps its rows' values but for those that fall below 2^-6 of the new scale's unit.
// Why the limits: weights are cut into bf16 parts down to 2^-24 of a weight, and 2^-60 leaves room for these above the
// end of the fp32 range; 448 * 2^100 leaves it for sums of a segment's rows.
#pragma once

#include "common.h"

namespace adakv {
namespace {

constexpr int Q8_BLOCK = ADAKV_Q8_BLOCK;
constexpr int Q8_LOW = -60, Q8_HIGH = 100;
constexpr float Q8_TOP = 448.0f;

__device__ __forceinline__ float pow2(int k) { return __builtin_bit_cast(float, (unsigned)(k + 127) << 23); }
__device__ __forceinline__ int exponent_of(float scale) { return (int)(__builtin_bit_cast(unsigned, scale) >> 23) - 127; }

// The exponent for magnitudes up to m (finite, >= 0): m = f 2^e with 1 <= f < 2 fits 448 * 2^k = 1.75 * 2^(k + 8)
// with k = e - 8 up to f = 1.75, whose 23 bits of fraction are 0x600000; adding what they lack to all ones carries beyond.
__device__ __forceinline__ int exponent_for(float m) {
  const int k = (int)((__builtin_bit_cast(unsigned, m) + 0x1fffffu) >> 23) - (127 + 8);
  return min(max(k, Q8_LOW), Q8_HIGH);
}

__device__ __forceinline__ float magnitude(float x) {
  const float a = __builtin_fabsf(x);
  return a < INFINITY ? a : 0.0f;
}

// x / 2^k, inv = 2^-k, as an operand of the conversion: saturating, and NaN for what is no finite number.
__device__ __forceinline__ float to_range(float x, float inv) {
  const float y = fminf(fmaxf(x * inv, -Q8_TOP), Q8_TOP);
  return __builtin_fabsf(x) < INFINITY ? y : __builtin_nanf("");
}
// Four values into a word of four codes, rounded to nearest, halves to even.
__device__ __forceinline__ unsigned to_codes(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// Where the scale of a segment's first block is, the segment's first row being `row` of the cache: segments before it
// fill row / Q8_BLOCK blocks at most, and one more each that is not full.
__device__ __forceinline__ long long first_scale(long long row, int s) { return row / Q8_BLOCK + s; }

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) x = fmaxf(x, __shfl_xor(x, o));
  return x;
}

}  // namespace
}  // namespace adakv
