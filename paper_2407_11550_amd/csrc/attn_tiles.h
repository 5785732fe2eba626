// What the attention kernels with many queries share (window_attn.hip, decode_prefix.hip): tiles of keys and values in LDS and the
// matrix instructions' operands from them.  S^T = K Q^T and O^T += V^T P^T, with the keys along the registers of a lane and a query
// per lane: what a lane holds of P is the second product's operand as it is (the contraction runs in the order in which the lanes hold
// the keys, and V^T is read from LDS in that order).
#pragma once

#include "common.h"

namespace adakv {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16 f16x8;
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float floatx16;

struct BF16 { static constexpr int SIZE = 2; };
struct FP16 { static constexpr int SIZE = 2; };
struct FP32 { static constexpr int SIZE = 4; };
template <typename T> constexpr bool is_f16 = false;
template <> constexpr bool is_f16<FP16> = true;
template <typename T> constexpr bool is_f32 = T::SIZE == 4;

template <typename T> __device__ __forceinline__ float half_of(unsigned u) {
  if constexpr (is_f16<T>) return (float)__builtin_bit_cast(_Float16, (unsigned short)u);
  else return __builtin_bit_cast(float, u << 16);
}
template <typename T> constexpr unsigned EXPONENT = is_f16<T> ? 0x7c00u : 0x7f80u;     // all ones: infinite or NaN
template <typename T> __device__ __forceinline__ floatx16 product(const u32x4 &a, const u32x4 &b, const floatx16 &c) {
  if constexpr (is_f16<T>)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// The value of the lane 32 further on.
__device__ __forceinline__ float other_half(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}

// 64 x 16 bytes from base + at + the lane's off, straight into 1 KB of LDS, behind the compiler's back: the tiles take
// turns in LDS, and it would wait for every load before it reads any.  (In front of the load stand the wait states that
// follow a write of m0, one, and a scalar register's write by the vector unit, five.)
// The next tile's loads do not run beside the whole of this tile's work, though: the compiler keeps the waits for the queries,
// which are loaded in front of the loop and first used in it, between the first products of every tile, and by then they are
// waits for the loads just asked for.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"        // m0 among the clobbers
__device__ __forceinline__ void load_to_lds(const char *base, unsigned off, unsigned at, const u32x4 *dst) {
  const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(base), 0, 0x7fffffff, 0x00027000);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(
                   (unsigned)(size_t)(__attribute__((address_space(3))) const void *)dst),
               "v"(off), "s"(rs), "s"(at)
               : "memory", "m0");
}
#pragma clang diagnostic pop
// What this wavefront has asked for is in LDS, it has read what it read, and so has every other wavefront.
__device__ __forceinline__ void meet() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
__device__ __forceinline__ const char *scalar_address(const char *p) {
  const unsigned long long a = (unsigned long long)p;
  const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)a), hi = __builtin_amdgcn_readfirstlane((unsigned)(a >> 32));
  return (const char *)((unsigned long long)hi << 32 | lo);
}

// Tiles in LDS: KT rows of CH 16-byte words, of which the words of a row change places with the row so that the lanes of a
// read fall on different banks.  Keys: 32 lanes read a word each of neighbouring rows.  Values, 16 bits: 32 lanes read 32
// columns of four rows; 32 bits: 32 lanes read 32 columns of a row and the others those of the row four further on.
template <typename T, int D, int KS> struct Tile {
  static constexpr int ROWB = D * T::SIZE, CH = ROWB / 16;
  static constexpr int KT = KS > 1 ? 32 * KS : T::SIZE == 4 ? 32 : 64;
  static constexpr int WORDS = KT * CH;
  static constexpr int TURNS = 4 * WORDS * 16 <= 160 * 1024 ? 2 : 1;      // tiles of each tensor in LDS at a time
  static constexpr int RPI = 64 / CH;                          // rows per load instruction
  static constexpr int LOADS = WORDS / 256;                    // load instructions per wavefront and tensor
  static __device__ __forceinline__ int swz_k(int row) { return CH == 8 ? (row >> 1) & 7 : row & 15; }
  static __device__ __forceinline__ int swz_v(int row) {
    return T::SIZE == 4 ? 8 * ((row >> 2) & 1) : CH == 16 ? 4 * (row & 3) : 4 * ((row >> 1) & 1);
  }
};

// Two values rounded to the layer's 16-bit type, x0 in the lower half.
template <typename T> __device__ __forceinline__ unsigned round2(float x0, float x1) {
  if constexpr (is_f16<T>) return __builtin_bit_cast(unsigned, __builtin_convertvector(floatx2{x0, x1}, f16x2));
  return __builtin_bit_cast(unsigned, __builtin_convertvector(floatx2{x0, x1}, bf16x2));
}

// 32 keys of a tile times 32 queries, a query per lane (twice: the halves of the wavefront hold different keys, lane `half` of a
// query those numbered 8 (i / 4) + 4 half + i % 4).  In 32 bits a logit is one chain of D / 2 products, or the sum of `CHAINS` shorter ones.
template <typename T, typename TL, int CHAINS = 1>
__device__ __forceinline__ floatx16 tile_logits(const u32x4 *tk, const u32x4 (&qf)[TL::CH / 2], int l32, int half) {
  constexpr int CH = TL::CH;
  static_assert(CHAINS == 1 || (CHAINS == 2 && is_f32<T>), "chains");
  floatx16 sc[CHAINS];
#pragma unroll
  for (int i = 0; i < CHAINS; ++i) sc[i] = floatx16{0};
#pragma unroll
  for (int s = 0; s < CH / 2; ++s) {
    const u32x4 kw = tk[l32 * CH + ((2 * s + half) ^ TL::swz_k(l32))];
    if constexpr (is_f32<T>) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const unsigned ka = kw[e], qa = qf[s][e];
        sc[e % CHAINS] = __builtin_amdgcn_mfma_f32_32x32x2f32(__builtin_bit_cast(float, ka), __builtin_bit_cast(float, qa), sc[e % CHAINS], 0, 0, 0);
      }
    } else {
      sc[0] = product<T>(kw, qf[s], sc[0]);
    }
  }
  if constexpr (CHAINS == 2) return sc[0] + sc[1];
  else return sc[0];
}

}  // namespace
}  // namespace adakv
