// Rows in registers, 16 bytes a lane (decode.hip, rotary.hip): sums over the lanes that share a row, and a row's elements in 32 bits.
#pragma once

#include "common.h"

namespace adakv {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

template <int CTRL>
__device__ __forceinline__ float dpp_add(float x) {
  const int y = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, false);
  return x + __builtin_bit_cast(float, y);
}

// Sum over the LPR neighbouring lanes that share a row; every one of them gets the sum.
template <int LPR>
__device__ __forceinline__ float row_sum(float x) {
  x = dpp_add<0xB1>(x);                       // quad_perm [1,0,3,2]
  x = dpp_add<0x4E>(x);                       // quad_perm [2,3,0,1]
  if (LPR >= 8) x = dpp_add<0x141>(x);        // row_half_mirror: lane i <-> 7-i
  if (LPR >= 16) x = dpp_add<0x140>(x);       // row_mirror: lane i <-> 15-i
  if (LPR >= 32) x += __shfl_xor(x, 16);
  return x;
}

struct f16_t { unsigned short bits; };        // IEEE half: tag type (bf16: unsigned short)
template <typename T> struct Elem;
template <> struct Elem<float> {
  static constexpr int EPL = 4;
  static __device__ __forceinline__ void widen(u32x4 v, float (&f)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned int word = v[i];          // a copy: bit_cast of the vector element itself
      f[i] = __builtin_bit_cast(float, word);  // reads element 0 for every i
    }
  }
};

template <> struct Elem<unsigned short> {     // bf16
  static constexpr int EPL = 8;
  static __device__ __forceinline__ void widen(u32x4 v, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned int word = v[i];
      f[2 * i] = __builtin_bit_cast(float, word << 16);
      f[2 * i + 1] = __builtin_bit_cast(float, word & 0xffff0000u);
    }
  }
};
template <> struct Elem<f16_t> {
  static constexpr int EPL = 8;
  static __device__ __forceinline__ void widen(u32x4 v, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned int word = v[i];
      f[2 * i] = (float)__builtin_bit_cast(_Float16, (unsigned short)(word & 0xffffu));
      f[2 * i + 1] = (float)__builtin_bit_cast(_Float16, (unsigned short)(word >> 16));
    }
  }
};

}  // namespace
}  // namespace adakv
