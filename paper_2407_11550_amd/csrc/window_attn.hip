// Causal attention over a prompt, limited to a window and a few first tokens (the sinks): the softmax of Section 3.1 over
// all rows of a sequence, in one pass over the keys with a running maximum and sum, and the log-sum-exp of the
// last w rows, which the scoring call takes.
//
// Both products run on the matrix cores, S^T = K Q^T and O^T += V^T P^T, with the keys along the registers of a lane and
// a query per lane: the maximum and the sum of a row take one exchange between the two halves of a wavefront, the
// correction of O^T none, and what a lane holds of P is the second product's operand as it is (the contraction
// runs in the order in which the lanes hold the keys, and V^T is read from LDS in that order).
//
// 4 d flops per visible pair: bound by the matrix instructions, whose operands a wavefront of 32 rows reads from LDS at nearly the
// rate that LDS has (1 KB a matrix instruction: 124 of 128 bytes a clock when those follow one another), with much vector work
// beside them and, in every tile, a wait for the next one's loads (load_to_lds).  16384 tokens, all visible, 32 heads over 8,
// d = 128, bf16: 2.09 to 2.14 ms in a row, 1030 to 1050 TFLOP/s, 2.25 on average with pauses (a library product of 8192^3 1130 to 1400);
// without reading operands it would be 1.64 ms, without loading tiles 1.77, without either 1.26.  64 rows a wavefront read half as
// much, but leave one wavefront per SIMD: 2.6 ms.  d = 64: vector work and the same wait, 620 TFLOP/s.
#include <math.h>

#include <type_traits>

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

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float M_INIT = -1.0e30f;             // finite "no key seen yet"

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

// Weights are taken against a kept reference, which costs no search for a maximum: it is moved, to the maximum of all so far,
// only where the sum of a lane's 16 weights of a tile is beyond MOST (which holds for the first tile, whose reference lies
// below every number).  fp16 weights travel 2^7 times larger, so that the smallest of full precision is 2^-21 of the reference;
// none is beyond the type's range.
constexpr float MOST = 0x1p15f;
template <typename T> constexpr float BIAS = is_f16<T> ? 7.0f : 0.0f;

struct Shape {
  int h_q, h_kv, g, w, window, sinks;
  float c_log2;
  long long q_tok, q_head, k_tok, k_head, v_tok, v_head;     // bytes
};

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

// What a wavefront does with 32 keys, a query per lane (twice: the halves of the wavefront hold different keys, lane `half`
// of a query those numbered 8 (i / 4) + 4 half + i % 4).
template <typename T, int D, int KS> struct Step {
  typedef Tile<T, D, KS> TL;
  static constexpr int CH = TL::CH, CB = D / 32;
  static constexpr int PW = is_f32<T> ? 16 : 8;                // registers of a tile's weights
  typedef unsigned Weights __attribute__((ext_vector_type(PW)));
  typedef floatx16 Sums[CB];

  static __device__ __forceinline__ floatx16 logits(const u32x4 *tk, const u32x4 (&qf)[CH / 2], int l32, int half) {
    floatx16 sc = floatx16{0};
#pragma unroll
    for (int s = 0; s < CH / 2; ++s) {
      const u32x4 kw = tk[l32 * CH + ((2 * s + half) ^ TL::swz_k(l32))];
      if constexpr (is_f32<T>) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const unsigned ka = kw[e], qa = qf[s][e];
          sc = __builtin_amdgcn_mfma_f32_32x32x2f32(__builtin_bit_cast(float, ka), __builtin_bit_cast(float, qa), sc, 0, 0, 0);
        }
      } else {
        sc = product<T>(kw, qf[s], sc);
      }
    }
    return sc;
  }

  // Weights against the reference m, and their sum; all of them times `by`.
  static __device__ __forceinline__ Weights weights(const floatx16 &sc, float c_log2, float m, float &sum, float by = 1.0f) {
    float p[16], part[4];                      // (four sums: one after the other would be a chain of 16 additions)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      p[i] = __builtin_amdgcn_exp2f(fmaf(sc[i], c_log2, BIAS<T> - m)) * by;
      part[i % 4] = i < 4 ? p[i] : part[i % 4] + p[i];
    }
    sum = (part[0] + part[1]) + (part[2] + part[3]);
    Weights w;
#pragma unroll
    for (int i = 0; i < PW; ++i) {
      if constexpr (is_f32<T>) w[i] = __builtin_bit_cast(unsigned, p[i]);
      else w[i] = round2<T>(p[2 * i], p[2 * i + 1]);
    }
    return w;
  }

  // A weight as the matrix units get it.
  static __device__ __forceinline__ float weight(const Weights &w, int i) {
    if constexpr (is_f32<T>) return __builtin_bit_cast(float, (unsigned)w[i]);
    else return half_of<T>(i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu);
  }

  // o += the products of 32 keys' weights and the values of columns 32 cb on.  FINITE: infinities and NaN count as 0.
  template <bool FINITE> static __device__ __forceinline__ void add_block(floatx16 &o, const u32x4 *tv, const Weights &w, int lane, int ks, int cb) {
    const int l32 = lane & 31, half = lane >> 5;
    if constexpr (is_f32<T>) {
      const float *vt = reinterpret_cast<const float *>(tv);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int row = 8 * (2 * ks + i / 4) + 4 * half + i % 4;
        float va = vt[row * D + ((8 * cb + l32 / 4) ^ TL::swz_v(row)) * 4 + l32 % 4];
        if (FINITE) va = __builtin_fabsf(va) < INFINITY ? va : 0.0f;
        const unsigned pa = w[8 * ks + i];
        o = __builtin_amdgcn_mfma_f32_32x32x2f32(va, __builtin_bit_cast(float, pa), o, 0, 0, 0);
      }
    } else {
      typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
      typedef __attribute__((address_space(3))) char lds_char;
      const int sub = lane & 15, row4 = 4 * half + sub / 4, col16 = (lane >> 4) & 1;
      s16x4 v2[2];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        // 4 rows x 16 columns by 16 lanes: a lane gets a column of them
        const int row = 16 * ks + 8 * y + row4, ch = 4 * cb + 2 * col16 + (sub % 4) / 2;
        const int at = (row * CH + (ch ^ TL::swz_v(row))) * 16 + 8 * (sub % 2);
        v2[y] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)((const lds_char *)tv + at));
      }
      const uint2 a0 = __builtin_bit_cast(uint2, v2[0]), a1 = __builtin_bit_cast(uint2, v2[1]);
      u32x4 va = {a0.x, a0.y, a1.x, a1.y};
      if constexpr (FINITE) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const unsigned u = va[i], top = EXPONENT<T>;
          va[i] = ((u & top) == top ? 0u : u & 0xffffu) | ((u >> 16 & top) == top ? 0u : u & 0xffff0000u);
        }
      }
      o = product<T>(va, u32x4{w[4 * ks], w[4 * ks + 1], w[4 * ks + 2], w[4 * ks + 3]}, o);
    }
  }
  static __device__ __forceinline__ void add_values(floatx16 (&acc)[CB], const u32x4 *tv, const Weights &w, int lane) {
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) add_block<false>(acc[cb], tv, w, lane, ks, cb);
  }

  // The infinities and NaN that add_block<true> left out, for the rows that see them.
  template <typename Sees> static __device__ __forceinline__ void add_seen(floatx16 &o, const u32x4 *tv, const Weights &w, int lane, int cb, Sees &&sees) {
#pragma nounroll
    for (int row = 0; row < 32; ++row) {
      asm volatile("" : "+v"(lane));                           // (addresses are made here, not kept in registers for this rare loop)
      const int l32 = lane & 31, half = lane >> 5;
      const int reg = 4 * (row / 8) + row % 4, there = l32 + 32 * (row / 4 % 2);       // where the row's weights are
      float p = 0.0f;
#pragma unroll
      for (int i = 0; i < 16; ++i) p = i == reg ? weight(w, i) : p;
      p = __shfl(p, there);
      const bool seen = sees(row);
      const char *bytes = reinterpret_cast<const char *>(tv) + row * TL::ROWB;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int col = 32 * cb + 8 * (i / 4) + 4 * half + i % 4;
        const char *at = bytes + (col * T::SIZE / 16 ^ TL::swz_v(row)) * 16 + col * T::SIZE % 16;
        float v;
        if constexpr (is_f32<T>) v = *reinterpret_cast<const float *>(at);
        else v = half_of<T>(*reinterpret_cast<const unsigned short *>(at));
        o[i] += seen && !(__builtin_fabsf(v) < INFINITY) ? p * v : 0.0f;
        __builtin_amdgcn_sched_barrier(0);                     // (one at a time: this is rare)
      }
    }
  }
};

// KS wavefronts share 32 rows and take 32 keys of a tile each: 1, four times 32 rows in a workgroup; 2 or 4, a half or a quarter of
// the rows and as much of the way, and the sums meet at the end.
template <typename T, int D, int KS>
__global__ __launch_bounds__(256, D == 128 ? (KS == 4 || (KS == 2 && T::SIZE == 4) ? 1 : 2) : KS == 4 ? 2 : T::SIZE == 4 ? 3 : 4) void window_attn_kernel(
    SeqTab st, ChunkTab ct, Shape sh, const char *__restrict__ q, const char *__restrict__ K, const char *__restrict__ V,
    char *__restrict__ out, float *__restrict__ row_lse) {
  typedef Tile<T, D, KS> TL;
  typedef Step<T, D, KS> S;
  constexpr int ROWS = 128 / KS;                          // query rows of the workgroup
  constexpr int ROWB = TL::ROWB, CH = TL::CH, KT = TL::KT, KB = KT / 32 / KS;
  constexpr int CB = D / 32;                                   // column blocks of O^T
  __shared__ __align__(16) u32x4 shK[TL::TURNS][TL::WORDS], shV[TL::TURNS][TL::WORDS];
  __shared__ int sh_bad[4];

  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, half = lane >> 5;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);

  // ---- which rows of which head ------------------------------------------------------------------------------
  const int item = blockIdx.x, hh = item % sh.h_q, rank = item / sh.h_q;
  const int c = hh % sh.h_kv, hq = c * sh.g + hh / sh.h_kv;
  const int b = find_seq(ct, st.batch, rank);
  const int n = st.n[b] + sh.w;
  const int q0 = (ct.off[b + 1] - 1 - rank) * ROWS;            // the longest rows first
  const char *Kh = K + st.tok_off[b] * sh.k_tok + c * sh.k_head, *Vh = V + st.tok_off[b] * sh.v_tok + c * sh.v_head;
  const char *Qh = q + st.tok_off[b] * sh.q_tok + hq * sh.q_head;
  const int w0 = q0 + 32 * (wv / KS), r = min(w0 + l32, n - 1);        // the wavefront's first row, this lane's

  u32x4 qf[CH / 2];
#pragma unroll
  for (int s = 0; s < CH / 2; ++s) qf[s] = *reinterpret_cast<const u32x4 *>(Qh + r * sh.q_tok + (2 * s + half) * 16);

  const int last = min(q0 + ROWS, n) - 1;                      // the workgroup's last row
  const int lo = max(0, q0 - sh.window + 1) / KT, hi = last / KT;
  const int firsts = min((int)(((long long)sh.sinks + KT - 1) / KT), lo), tiles = firsts + hi - lo + 1;
  // the wavefront's share of a tile: rows on (wv * LOADS + i) * RPI + lane / CH
  auto at_k = [&](int row, int lane) { return row * (unsigned)sh.k_tok + ((lane % CH) ^ TL::swz_k(row)) * 16; };
  auto at_v = [&](int row, int lane) { return row * (unsigned)sh.v_tok + ((lane % CH) ^ TL::swz_v(row)) * 16; };
  unsigned off_k[TL::LOADS], off_v[TL::LOADS];
#pragma unroll
  for (int i = 0; i < TL::LOADS; ++i) {
    const int row = (wv * TL::LOADS + i) * TL::RPI + lane / CH;
    off_k[i] = at_k(row, lane);
    off_v[i] = at_v(row, lane);
  }
  auto first_key = [&](int t) { return (t < firsts ? t : lo + t - firsts) * KT; };
  auto load = [&](int t) __attribute__((always_inline)) {
    const int j0 = first_key(t);
    const char *kb = scalar_address(Kh + j0 * sh.k_tok), *vb = scalar_address(Vh + j0 * sh.v_tok);
    const u32x4 *dk = shK[t % TL::TURNS] + wv * TL::LOADS * 64, *dv = shV[t % TL::TURNS] + wv * TL::LOADS * 64;
    if (TL::LOADS > 8) {                                       // (so many places do not fit in registers)
      int here = lane;
      asm volatile("" : "+v"(here));
      const int end = n - 1 - j0;                              // rows past the sequence's end repeat its last one
#pragma unroll
      for (int i = 0; i < TL::LOADS; ++i) {
        const int row = (wv * TL::LOADS + i) * TL::RPI + here / CH, back = max(row - end, 0);
        load_to_lds(kb, at_k(row, here) - back * (unsigned)sh.k_tok, 0u, dk + i * 64);
        load_to_lds(vb, at_v(row, here) - back * (unsigned)sh.v_tok, 0u, dv + i * 64);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else if (j0 + KT <= n) {
#pragma unroll
      for (int i = 0; i < TL::LOADS; ++i) load_to_lds(kb, off_k[i], 0u, dk + i * 64);
#pragma unroll
      for (int i = 0; i < TL::LOADS; ++i) load_to_lds(vb, off_v[i], 0u, dv + i * 64);
    } else {
#pragma unroll
      for (int i = 0; i < TL::LOADS; ++i) {
        const int row = (wv * TL::LOADS + i) * TL::RPI + lane / CH, back = max(row - (n - 1 - j0), 0);
        load_to_lds(kb, off_k[i] - back * (unsigned)sh.k_tok, 0u, dk + i * 64);
        load_to_lds(vb, off_v[i] - back * (unsigned)sh.v_tok, 0u, dv + i * 64);
      }
    }
  };
  // tile t is there, and the next one on its way where it has a place of its own
  auto await = [&](int t) __attribute__((always_inline)) {
    if constexpr (TL::TURNS == 2) {
      meet();
      if (t + 1 < tiles) load(t + 1);
    } else {
      if (t > 0) {
        meet();
        load(t);
      }
      meet();
    }
  };

  floatx16 acc[CB];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) acc[cb] = floatx16{0};
  float m = M_INIT, l = 0.0f;
  // Logits of 32 keys, hidden ones -inf where there are any, and their weights against the running reference; where that has to
  // move, `move` multiplies what was summed against it.
  auto hide = [&](floatx16 &sc, int first, int half) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int j = first + 8 * (i / 4) + 4 * half + i % 4;
      const bool hidden = (j > r) | ((j <= r - sh.window) & (j >= sh.sinks));
      sc[i] = hidden ? -INFINITY : sc[i];
    }
  };
  auto weigh = [&](const floatx16 &sc, auto &&move) {
    float sum;
    typename S::Weights w = S::weights(sc, sh.c_log2, m, sum);
    if (__builtin_expect(__any(!(sum <= MOST)), 0)) {          // too far above the reference (or no number): a new one
      float top = sc[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) top = fmaxf(top, sc[i]);
      const float mn = fmaxf(m, fmaxf(top, other_half(top)) * sh.c_log2), corr = __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= corr;
      move(corr);
      w = S::weights(sc, sh.c_log2, m, sum);
    }
    l += sum;
    return w;
  };
  // whether none of the wavefront's rows sees a key of the tile, and whether some see only some
  auto unseen = [&](int j0) { return j0 > w0 + 31 || (j0 >= sh.sinks && j0 + KT - 1 <= w0 - sh.window); };
  auto edge = [&](int j0) { return j0 + KT - 1 > w0 || !(j0 > w0 + 31 - sh.window || j0 + KT - 1 < sh.sinks); };

  load(0);
  for (int t = 0; t < tiles; ++t) {
    const int j0 = first_key(t);
    const u32x4 *tk = shK[t % TL::TURNS], *tv = shV[t % TL::TURNS];
    await(t);
    if (unseen(j0)) continue;
    const int kb0 = wv % KS;                                   // this wavefront's keys of the tile
    floatx16 sc[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) sc[kb] = S::logits(tk + (kb0 + kb) * 32 * CH, qf, l32, half);
    if (edge(j0)) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) hide(sc[kb], j0 + 32 * (kb0 + kb), half);
    }
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const typename S::Weights w = weigh(sc[kb], [&](float corr) {
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) acc[cb] *= corr;
      });
      S::add_values(acc, tv + (kb0 + kb) * 32 * CH, w, lane);
    }
  }

  float *lse = row_lse ? row_lse + ((long long)b * sh.h_q + hq) * sh.w - st.n[b] : nullptr;     // of row 0
  char *dst = out + (st.tok_off[b] * sh.h_q + hq) * ROWB + r * ((long long)sh.h_q * ROWB);
  auto store = [&](const floatx16 &o, int cb, float inv) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int col = 32 * cb + 8 * k + 4 * half;
      const float x0 = o[4 * k] * inv, x1 = o[4 * k + 1] * inv, x2 = o[4 * k + 2] * inv, x3 = o[4 * k + 3] * inv;
      if constexpr (is_f32<T>) *reinterpret_cast<float4 *>(dst + col * 4) = make_float4(x0, x1, x2, x3);
      else *reinterpret_cast<uint2 *>(dst + col * 2) = make_uint2(round2<T>(x0, x1), round2<T>(x2, x3));
    }
  };
  auto store_lse = [&]() {
    if (lse && r >= st.n[b] && half == 0) lse[r] = (m - BIAS<T> + log2f(l)) * LN2;
  };

  l += other_half(l);

  // Where something came out infinite or as NaN, a value that none should have seen may be the reason (a weight of 0 does not
  // cancel it), or values so large that their sum against the kept reference is beyond the type: once more, 32 columns at a
  // time, with a look at every value of the tiles that hold hidden keys.  (In the others every row sees every key.)  The maximum
  // and the sum of a row's weights are known by now and hold, so the weights are taken by their sum's power of two less: what is
  // summed stays below the largest value.  (Not in fp16, whose values cannot sum up to the end of fp32 and whose weights would lose bits.)
  float worst = l * 0.0f;
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int i = 0; i < 16; ++i) worst = fmaf(acc[cb][i] * KS, 0.0f, worst);     // (KS such sums are added up below)
  const bool bad = __any(!(worst == 0.0f));
  if (lane == 0) sh_bad[wv] = bad;
  __syncthreads();
  if (sh_bad[0] | sh_bad[1] | sh_bad[2] | sh_bad[3]) {
    if constexpr (KS > 1) {
      float2(*ml)[64] = reinterpret_cast<float2(*)[64]>(&shV[0][0]);
      ml[wv][lane] = make_float2(m, l);
      __syncthreads();
      const float own = m;
#pragma unroll
      for (int k = 0; k < KS; ++k) m = fmaxf(m, ml[wv / KS * KS + k][lane].x);
      l *= __builtin_amdgcn_exp2f(own - m);
#pragma unroll
      for (int k = 1; k < KS; ++k) {
        const float2 other = ml[wv / KS * KS + (wv + k) % KS][lane];
        l += other.y * __builtin_amdgcn_exp2f(other.x - m);
      }
    }
    const float by = is_f16<T> ? 1.0f : ldexpf(1.0f, -__builtin_amdgcn_frexp_expf(l)), inv = 1.0f / (l * by);
    if (wv % KS == 0 && w0 + l32 < n) store_lse();
#pragma nounroll
    for (int cb = 0; cb < CB; ++cb) {
      floatx16 o = floatx16{0};
      __syncthreads();
      load(0);
#pragma nounroll
      for (int t = 0; t < tiles; ++t) {
        const int j0 = first_key(t);
        await(t);
        if (wv % KS || unseen(j0)) continue;                   // (one wavefront for all of its rows' keys)
#pragma nounroll
        for (int kb = 0; kb < KT / 32; ++kb) {
          int here = lane;
          asm volatile("" : "+v"(here));                       // (as in add_seen)
          const int first = j0 + 32 * kb;
          const u32x4 *values = shV[t % TL::TURNS] + kb * 32 * CH;
          floatx16 sc = S::logits(shK[t % TL::TURNS] + kb * 32 * CH, qf, here & 31, here >> 5);
          hide(sc, first, here >> 5);
          float sum;
          const typename S::Weights w = S::weights(sc, sh.c_log2, m, sum, by);
          if (edge(j0)) {
            S::template add_block<true>(o, values, w, here, 0, cb);
            S::template add_block<true>(o, values, w, here, 1, cb);
            S::add_seen(o, values, w, here, cb, [&](int row) {
              const int j = first + row;
              return (j <= r) & ((j > r - sh.window) | (j < sh.sinks));
            });
          } else {
            S::template add_block<false>(o, values, w, here, 0, cb);
            S::template add_block<false>(o, values, w, here, 1, cb);
          }
        }
      }
      if (wv % KS == 0 && w0 + l32 < n) store(o, cb, inv);
    }
    return;
  }

  if constexpr (KS > 1) {
    // the first of those that share their rows takes the others' sums, through the tiles' place
    typedef float Shared[CB * 16][64];
    static_assert((4 - 4 / KS) * sizeof(Shared) <= sizeof(shK), "the sums have room");
    Shared *sums = reinterpret_cast<Shared *>(&shK[0][0]);
    float2(*ml)[64] = reinterpret_cast<float2(*)[64]>(&shV[0][0]);
    const int place = wv / KS * (KS - 1) - 1;                  // + 1 .. KS - 1
    meet();
    if (wv % KS) {
#pragma unroll
      for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int i = 0; i < 16; ++i) sums[place + wv % KS][cb * 16 + i][lane] = acc[cb][i];
      ml[place + wv % KS][lane] = make_float2(m, l);
    }
    __syncthreads();
    if (wv % KS) return;
#pragma unroll
    for (int k = 1; k < KS; ++k) {
      const float2 other = ml[place + k][lane];
      const float mn = fmaxf(m, other.x), f0 = __builtin_amdgcn_exp2f(m - mn), f1 = __builtin_amdgcn_exp2f(other.x - mn);
      m = mn;
      l = l * f0 + other.y * f1;
#pragma unroll
      for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[cb][i] = acc[cb][i] * f0 + sums[place + k][cb * 16 + i][lane] * f1;
    }
  }

  if (w0 + l32 >= n) return;
  const float inv = 1.0f / l;                                  // (a row sees itself: l is 0 where all its logits are -inf, 0 / 0)
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) store(acc[cb], cb, inv);
  store_lse();
}

}  // namespace

hipError_t launch_window_attn(const SeqTab &st, const Dims &dm, int dtype, const void *q, long long q_tok, long long q_head,
                              const void *K, const void *V, int window, int sinks, void *out, float *row_lse, hipStream_t s) {
  const long long e = dtype == ADAKV_FP32 ? 4 : 2;
  const Shape sh = {dm.h_q, dm.h_kv, dm.g, dm.w, window, sinks, dm.scale * LOG2E, q_tok * e, q_head * e, dm.k_stride_tok * e,
                    dm.k_stride_head * e, dm.v_stride_tok * e, dm.v_stride_head * e};
  const auto chunks = [&](int rows) {
    ChunkTab ct;
    ct.off[0] = 0;
    for (int b = 0; b < st.batch; ++b) ct.off[b + 1] = ct.off[b] + (st.n[b] + dm.w + rows - 1) / rows;
    for (int b = st.batch + 1; b <= ADAKV_MAX_BATCH; ++b) ct.off[b] = ct.off[st.batch];
    return ct;
  };
  // A wavefront takes 0.9 us for 32 keys whatever else there is to do, so with few workgroups (two of 128 or 64 rows fit on each
  // of 256 compute units, one of 32; at d = 64 twice as many of those that share) wavefronts share rows.  us, 128 | 64 | 32 rows a
  // workgroup, by the number that 128 rows make; all keys visible, d = 128: 4 workgroups, 64 keys 6.0 | 6.6 | 7.6, 100 keys
  // 8.6 | 6.8 | 7.4; 64, 256 keys 10.6 | 9.7 | 8.8; 96, 1500 keys 37.7 | 24.6 | 21.1; 128, 2048 keys 43.5 | 31.0 | 28.9; 160, 541
  // keys 17.1 | 14.7 | 22.0; 192, 3000 keys 69 | 49 | 60; 256, 1024 keys 27.3 | 22.8 | 40.0; 384, 1500 keys 42 | 35 | 70; 512, 2043
  // keys 54.9 | 53.2; 512, 8192 keys 191 | 173; 1024, 4096 keys 159 | 182; d = 64: 192, 729 keys 18.2 | 13.0 | 14.3, 3000 keys
  // 52 | 34 | 26; 384, 1500 keys 32 | 23 | 31.  Where a window makes most rows' ways equally short there is no longest one to shorten;
  // 60 and 500 keys, d = 128: 48 workgroups 12.8 | 9.4 | 10.5 and 23.0 | 15.5 | 13.9, 96 13.1 | 9.7 | 19.4 and 23.6 | 16.0 | 21.9,
  // 192 13.7 | 12.5 | 28.5 and 24.1 | 21.4 | 38.9, 376 17.8 | 21.1 | 57.0 and 33.1 | 35.2 | 77.6; d = 64: 96 10.8 | 7.5 | 9.0 and
  // 18.8 | 11.9 | 12.4, 384 14.4 | 11.6 | 21.8 and 20.7 | 16.7 | 27.3.
  ChunkTab ct = chunks(128);
  const long long wgs = (long long)ct.off[st.batch] * dm.h_q;
  long long longest = 0;
  for (int b = 0; b < st.batch; ++b) longest = st.n[b] + dm.w > longest ? st.n[b] + dm.w : longest;
  const long long reach = (long long)window + sinks < longest ? (long long)window + sinks : longest;   // keys that the last rows see
  const bool even = reach < longest / 2;       // most rows have ways of the same length
  const int by_d = 128 / dm.d;
  const long long four = even ? (reach > 128 ? 64 : 0) : by_d == 2 && reach >= 1024 ? 192 : 128;
  const long long two = !even && reach >= 1024 ? 512 : 256 * by_d;
  int share = longest <= 64 ? 1 : wgs <= four ? 4 : wgs <= two ? 2 : 1;
  // fp32: 32 keys take 1.7 us at d = 64 and 3.4 at d = 128, so sharing pays from the second 32 on.  d = 128: 4 workgroups, 40
  // keys 13.1 | 9.8 | 11.6, 100 keys 22.8 | 14.4 | 12.0; 24, 729 keys 101 | 57 | 38; 96, 1500 keys 201 | 110 | 72; 192, 1500 keys
  // 203 | 115 | 129; 384, 1500 keys 250 | 194 | 231; 768, 1500 keys 342 | 356 | 454; a window of 200 of 1500 keys: 48 workgroups 59
  // | 34 | 31, 96 58 | 35 | 59, 192 59 | 67 | 86.  d = 64, where two of the workgroups of half the rows fit on a unit: 768, 3000 keys
  // 381 | 317 | 416, a window of 200: 384 56 | 51 | 91, 768 79 | 95 | 165.
  if (dtype == ADAKV_FP32)
    share = reach <= 64 ? (wgs <= 256 ? 2 : 1) : wgs <= (even ? 64 : 128) ? 4 : wgs <= (even ? 192 : 384) * by_d ? 2 : 1;
  if (share > 1) ct = chunks(128 / share);
  const dim3 grid((unsigned)((long long)ct.off[st.batch] * dm.h_q));
  // (a trace's name tells how many wavefronts share rows)
#define ADAKV_WINDOW_KS(T, D, KS)                                                                                           \
  ADAKV_LAUNCH(KS == 1 ? "window_attn" : KS == 2 ? "window_attn_2" : "window_attn_4", (window_attn_kernel<T, D, KS>), grid,   \
               dim3(256), s, st, ct, sh, (const char *)q, (const char *)K, (const char *)V, (char *)out, row_lse)
#define ADAKV_WINDOW(T, D)                                                                                                  \
  do {                                                                                                                      \
    if (share == 4) ADAKV_WINDOW_KS(T, D, 4);                                                                               \
    else if (share == 2) ADAKV_WINDOW_KS(T, D, 2);                                                                          \
    else ADAKV_WINDOW_KS(T, D, 1);                                                                                          \
  } while (0)
  if (dtype == ADAKV_BF16) { if (dm.d == 64) ADAKV_WINDOW(BF16, 64); else ADAKV_WINDOW(BF16, 128); }
  else if (dtype == ADAKV_FP16) { if (dm.d == 64) ADAKV_WINDOW(FP16, 64); else ADAKV_WINDOW(FP16, 128); }
  else { if (dm.d == 64) ADAKV_WINDOW(FP32, 64); else ADAKV_WINDOW(FP32, 128); }
#undef ADAKV_WINDOW
#undef ADAKV_WINDOW_KS
  return hipGetLastError();
}

}  // namespace adakv
