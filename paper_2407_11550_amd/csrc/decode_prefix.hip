// A decoding step of a batch whose sequences share caches (Section 3.5's flattened layout twice): every query head attends over a
// segment of a shared cache and over its own, which is one softmax over the rows of both.
//
// With M = g query heads of all the sequences that share a segment, its rows are read once for M rows of queries: 4 d M flops for
// 4 d bytes (16 bits).  Both products run on the matrix cores as the prompt's do (attn_tiles.h), S^T = K Q^T and O^T += V^T P^T, a
// query per lane, tiles of the segment in LDS.  Weights stay in 32 bits, as in the other decoding steps: what is added up is an fp32
// result.  bf16: a weight is cut into three bf16 parts whose sum it is to 2^-24, which share one operand of V and
// one sum.  fp16: two fp16 parts, the lower one times 2^11 with a sum of its own, 22 bits for weights down to 2^-24 of the largest and
// 2^-45 of it beyond.  fp32: the fp32 matrix instruction.
//
// A segment is split into parts as in decode.hip; a workgroup takes a part for 128, 64 or 32 rows of queries (1, 2 or 4 wavefronts
// share 32 of them) and files the sums, and a last kernel merges, for each query head, the parts of its own segment and of the shared one.
#include <math.h>

#include "attn_tiles.h"
#include "decode_prefix.h"

namespace adakv {
namespace {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float M_INIT = -1.0e30f;             // finite "no row seen yet"

// Weights are taken against a kept reference, 2^BIAS times, and the reference is moved, to the maximum of all so far, only where the
// sum of a lane's 16 weights of a tile is beyond MOST.  Moved, the largest weight is 2^BIAS, so 16 of them are below MOST.  32 bits and bf16: none
// is above 1, so that no sum is larger than the values times the rows.  fp16: none beyond the type.
template <typename T> constexpr float BIAS = is_f16<T> ? 10.0f : -15.0f;
template <typename T> constexpr float MOST = is_f16<T> ? 0x1p15f : 1.0f;
constexpr float LOW_UP = 0x1p11f, LOW_DOWN = 0x1p-11f;         // of an fp16 weight's lower part

// V^T of 32 columns from 32 cb on: what a lane takes of keys 16 ks .. 16 ks + 15, 32 bits (the i-th of its eight) and 16 bits.
template <int D, typename TL>
__device__ __forceinline__ float tile_value(const u32x4 *tv, int l32, int half, int ks, int cb, int i) {
  const float *vt = reinterpret_cast<const float *>(tv);
  const int row = 8 * (2 * ks + i / 4) + 4 * half + i % 4;
  return vt[row * D + ((8 * cb + l32 / 4) ^ TL::swz_v(row)) * 4 + l32 % 4];
}
template <typename TL> __device__ __forceinline__ u32x4 tile_values(const u32x4 *tv, int lane, int ks, int cb) {
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  typedef __attribute__((address_space(3))) char lds_char;
  const int sub = lane & 15, row4 = 4 * (lane >> 5) + sub / 4, col16 = (lane >> 4) & 1;
  s16x4 v2[2];
#pragma unroll
  for (int y = 0; y < 2; ++y) {
    // 4 rows x 16 columns by 16 lanes: a lane gets a column of them
    const int row = 16 * ks + 8 * y + row4, ch = 4 * cb + 2 * col16 + (sub % 4) / 2;
    const int at = (row * TL::CH + (ch ^ TL::swz_v(row))) * 16 + 8 * (sub % 2);
    v2[y] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)((const lds_char *)tv + at));
  }
  const uint2 a0 = __builtin_bit_cast(uint2, v2[0]), a1 = __builtin_bit_cast(uint2, v2[1]);
  return u32x4{a0.x, a0.y, a1.x, a1.y};
}

__device__ __forceinline__ float cut(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }
// x0 and x1 cut to bf16, x0 in the lower half of the word.
__device__ __forceinline__ unsigned pack(float x0, float x1) {
  return __builtin_amdgcn_perm(__float_as_uint(x1), __float_as_uint(x0), 0x07060302u);
}

// The weights of 32 keys and their products with values.
template <typename T, int D, typename TL> struct Weights {
  static constexpr int CB = D / 32;
  static constexpr int PARTS = is_f32<T> ? 1 : is_f16<T> ? 2 : 3;
  static constexpr int SUMS = is_f16<T> ? 2 : 1;               // sets of sums
  unsigned w[PARTS][is_f32<T> ? 16 : 8];

  // p: their values; `first` alone: what is needed to know where a product is no finite number
  __device__ __forceinline__ void set(const float (&p)[16], bool first = false) {
    if constexpr (is_f32<T>) {
#pragma unroll
      for (int i = 0; i < 16; ++i) w[0][i] = __float_as_uint(p[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float x0 = p[2 * i], x1 = p[2 * i + 1];
        if constexpr (is_f16<T>) {
          w[0][i] = round2<T>(x0, x1);
          x0 = (x0 - half_of<T>(w[0][i] & 0xffffu)) * LOW_UP;
          x1 = (x1 - half_of<T>(w[0][i] >> 16)) * LOW_UP;
          w[1][i] = round2<T>(x0, x1);
        } else {
          w[0][i] = pack(x0, x1);
          x0 -= cut(x0);
          x1 -= cut(x1);
          w[1][i] = pack(x0, x1);
          x0 -= cut(x0);
          x1 -= cut(x1);
          w[2][i] = pack(x0, x1);
        }
      }
    }
  }
  __device__ __forceinline__ u32x4 operand(int part, int ks) const {
    return {w[part][4 * ks], w[part][4 * ks + 1], w[part][4 * ks + 2], w[part][4 * ks + 3]};
  }
  __device__ __forceinline__ void add_values(floatx16 (&acc)[SUMS][CB], const u32x4 *tv, int lane) const {
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      if constexpr (is_f32<T>) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int cb = 0; cb < CB; ++cb)
            acc[0][cb] = __builtin_amdgcn_mfma_f32_32x32x2f32(tile_value<D, TL>(tv, lane & 31, lane >> 5, ks, cb, i), __uint_as_float(w[0][8 * ks + i]),
                                                             acc[0][cb], 0, 0, 0);
      } else {
        u32x4 va[CB];
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) va[cb] = tile_values<TL>(tv, lane, ks, cb);
#pragma unroll
        for (int part = 0; part < PARTS; ++part)
#pragma unroll
          for (int cb = 0; cb < CB; ++cb) acc[SUMS == 2 ? part : 0][cb] = product<T>(va[cb], operand(part, ks), acc[SUMS == 2 ? part : 0][cb]);
      }
    }
  }
  // The first parts alone, columns 32 cb on.
  __device__ __forceinline__ void add_first(floatx16 &o, const u32x4 *tv, int lane, int cb) const {
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      if constexpr (is_f32<T>) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          o = __builtin_amdgcn_mfma_f32_32x32x2f32(tile_value<D, TL>(tv, lane & 31, lane >> 5, ks, cb, i), __uint_as_float(w[0][8 * ks + i]), o, 0, 0, 0);
      } else {
        o = product<T>(tile_values<TL>(tv, lane, ks, cb), operand(0, ks), o);
      }
    }
  }
};

// What a workgroup works on: part `j` of segment s of the shared caches, rows r0 .. r1 - 1, and query rows from `row` on.
struct Part {
  int s, j, row, rows, parts, first_row;
};

// Finds it, as find_work does in decode_parts.h: from a prefix sum, over the segments, of the workgroups that their lengths make.  A segment's
// workgroups for the same part lie a multiple of 8 apart, so that one of the chip's 8 caches has the rows for all of them.
template <int RB>
__device__ __forceinline__ bool find_part(const Sharing &sh, int split, int headroom, const int *cu, const int *seg_len, int4 *tab, Part &pt) {
  const int nseg = sh.groups * sh.h, lane = threadIdx.x & 63, blk = (int)blockIdx.x;
  int base = 0;
  bool found = false;
  for (int s0 = 0; s0 < nseg; s0 += 64) {
    const int s = min(s0 + lane, nseg - 1), p = s / sh.h;
    const int from = cu[s], cap = cu[s + 1] - from + headroom;
    const int len = min(max(seg_len[s], 0), cap);              // (a corrupt length can never leave the segment)
    const int many = sh.first[p + 1] - sh.first[p], blocks = (many * sh.g + RB - 1) / RB;
    const int parts = (len + split - 1) / split, step = blocks > 1 ? (parts + 7) / 8 * 8 : parts;
    const int n = s0 + lane < nseg ? blocks * step : 0;
    const int upto = wave_scan_incl(n) + base, first = upto - n;
    if (s0 + lane == blk && blk < nseg && threadIdx.x < 64) tab[s] = make_int4(first, parts, step, len);
    const unsigned long long here = __ballot(blk >= first && blk < upto);
    if (here != 0 && !found) {
      const int L = __ffsll(here) - 1, at = blk - __builtin_amdgcn_readlane(first, L), st = __builtin_amdgcn_readlane(step, L);
      pt.s = s0 + L;
      pt.j = at % st;
      pt.row = at / st * RB;
      pt.rows = __builtin_amdgcn_readlane(len, L);
      pt.parts = __builtin_amdgcn_readlane(parts, L);
      pt.first_row = __builtin_amdgcn_readlane(from, L);
      found = pt.j < pt.parts;
    }
    base = __builtin_amdgcn_readlane(upto, 63);
    if (found && blk < s0 + 64) break;                         // (a later round may have the entry that this workgroup files)
  }
  return found;
}

template <typename T, int D, int KS>
__global__ __launch_bounds__(256, KS == 4 || (D == 128 && KS == 2 && T::SIZE == 4) ? 1 : 2) void prefix_attn_kernel(
    Sharing sh, int split, int headroom, float c_log2, const char *__restrict__ q, const int *__restrict__ cu,
    const int *__restrict__ seg_len, const char *__restrict__ Kc, const char *__restrict__ Vc, float *__restrict__ part_acc,
    float2 *__restrict__ part_ml, int4 *__restrict__ tab) {
  typedef Tile<T, D, KS> TL;
  typedef Weights<T, D, TL> W;
  constexpr int RB = 128 / KS;                                 // query rows of the workgroup
  constexpr int ROWB = TL::ROWB, CH = TL::CH, KT = TL::KT, KB = KT / 32 / KS, CB = D / 32;
  __shared__ __align__(16) u32x4 shK[TL::TURNS][TL::WORDS], shV[TL::TURNS][TL::WORDS];
  __shared__ int sh_bad[4];

  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, half = lane >> 5;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  Part pt;
  if (!find_part<RB>(sh, split, headroom, cu, seg_len, tab, pt)) return;
  const int p = pt.s / sh.h, c = pt.s % sh.h;
  const int M = (sh.first[p + 1] - sh.first[p]) * sh.g;
  // (equal parts, in whole tiles; none is empty)
  const int rows = min(split, ((pt.rows + pt.parts - 1) / pt.parts + KT - 1) / KT * KT);
  const int r0 = pt.j * rows, n = min(pt.rows - r0, rows);     // keys of this part
  const char *Kh = Kc + ((long long)pt.first_row + (long long)pt.s * headroom + r0) * ROWB;
  const char *Vh = Vc + ((long long)pt.first_row + (long long)pt.s * headroom + r0) * ROWB;

  const int w0 = pt.row + 32 * (wv / KS), m_row = min(w0 + l32, M - 1);         // the wavefront's first query row, this lane's
  const bool idle = w0 >= M;
  const int b = sh.order[sh.first[p] + m_row / sh.g];
  const char *Qh = q + ((long long)(b * sh.h + c) * sh.g + m_row % sh.g) * ROWB;
  u32x4 qf[CH / 2];
#pragma unroll
  for (int s = 0; s < CH / 2; ++s) qf[s] = *reinterpret_cast<const u32x4 *>(Qh + (2 * s + half) * 16);

  const int tiles = (n + KT - 1) / KT;
  // the wavefront's share of a tile: rows on (wv * LOADS + i) * RPI + lane / CH; rows past the end repeat the last one
  auto load = [&](int t) __attribute__((always_inline)) {
    const char *kb = scalar_address(Kh + (long long)t * KT * ROWB), *vb = scalar_address(Vh + (long long)t * KT * ROWB);
    const u32x4 *dk = shK[t % TL::TURNS] + wv * TL::LOADS * 64, *dv = shV[t % TL::TURNS] + wv * TL::LOADS * 64;
    const int end = n - 1 - t * KT;
#pragma unroll
    for (int i = 0; i < TL::LOADS; ++i) {
      const int row = (wv * TL::LOADS + i) * TL::RPI + lane / CH;
      load_to_lds(kb, (unsigned)min(row, end) * ROWB + ((lane % CH) ^ TL::swz_k(row)) * 16, 0u, dk + i * 64);
    }
#pragma unroll
    for (int i = 0; i < TL::LOADS; ++i) {
      const int row = (wv * TL::LOADS + i) * TL::RPI + lane / CH;
      load_to_lds(vb, (unsigned)min(row, end) * ROWB + ((lane % CH) ^ TL::swz_v(row)) * 16, 0u, dv + i * 64);
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

  floatx16 acc[W::SUMS][CB];
#pragma unroll
  for (int i = 0; i < W::SUMS; ++i)
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) acc[i][cb] = floatx16{0};
  float m = M_INIT, l = 0.0f;
  // Weights of 32 keys against the reference m, and their sum.
  auto weigh = [&](const floatx16 &sc, float (&pr)[16]) {
    float part[4];                             // (four sums: one after the other would be a chain of 16 additions)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      pr[i] = __builtin_amdgcn_exp2f(fmaf(sc[i], c_log2, BIAS<T> - m));
      part[i % 4] = i < 4 ? pr[i] : part[i % 4] + pr[i];
    }
    return (part[0] + part[1]) + (part[2] + part[3]);
  };

  load(0);
  for (int t = 0; t < tiles; ++t) {
    await(t);
    if (idle) continue;
    const u32x4 *tk = shK[t % TL::TURNS], *tv = shV[t % TL::TURNS];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const int kk = wv % KS * KB + kb, left = n - t * KT - 32 * kk;           // this wavefront's 32 keys of the tile; how many are
      if (left <= 0) break;
      floatx16 sc = tile_logits<T, TL>(tk + kk * 32 * CH, qf, l32, half);
      if (left < 32) {
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[i] = 8 * (i / 4) + 4 * half + i % 4 < left ? sc[i] : -INFINITY;
      }
      float pr[16];
      float sum = weigh(sc, pr);
      if (__builtin_expect(__any(!(sum <= MOST<T>)), 0)) {     // too far above the reference (or no number): a new one
        float top = sc[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, sc[i]);
        const float mn = fmaxf(m, fmaxf(top, other_half(top)) * c_log2), corr = __builtin_amdgcn_exp2f(m - mn);
        m = mn;
        l *= corr;
#pragma unroll
        for (int i = 0; i < W::SUMS; ++i)
#pragma unroll
          for (int cb = 0; cb < CB; ++cb) acc[i][cb] *= corr;
        sum = weigh(sc, pr);
      }
      l += sum;
      W w;
      w.set(pr);
      w.add_values(acc, tv + kk * 32 * CH, lane);
    }
  }
  l += other_half(l);
  if constexpr (W::SUMS == 2) {
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) acc[0][cb] += acc[1][cb] * LOW_DOWN;
  }

  // Where a sum is infinite or NaN, a value that is none may have met a weight's lower part of 0, or of the other sign, or a
  // weight of 0 of the rows past the end: once more with the upper parts alone, which say what it is.
  float worst = 0.0f;
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int i = 0; i < 16; ++i) worst = fmaf(acc[0][cb][i], 0.0f, worst);
  const bool bad = __any(!(worst == 0.0f));
  if (lane == 0) sh_bad[wv] = bad;
  __syncthreads();
  if (sh_bad[0] | sh_bad[1] | sh_bad[2] | sh_bad[3]) {
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      floatx16 o = floatx16{0};
      __syncthreads();
      load(0);
#pragma nounroll
      for (int t = 0; t < tiles; ++t) {
        await(t);
        if (idle) continue;
#pragma nounroll
        for (int kb = 0; kb < KB; ++kb) {
          const int kk = wv % KS * KB + kb;
          if (n - t * KT - 32 * kk <= 0) break;
          // (the rows past the end repeat the last one, so their weights may stay)
          const floatx16 sc = tile_logits<T, TL>(shK[t % TL::TURNS] + kk * 32 * CH, qf, l32, half);
          float pr[16];
          weigh(sc, pr);
          if constexpr (is_f16<T>) {                           // (none is too small for the type)
#pragma unroll
            for (int i = 0; i < 16; ++i) pr[i] = pr[i] > 0.0f ? fmaxf(pr[i], 0x1p-24f) : pr[i];
          }
          W w;
          w.set(pr);
          w.add_first(o, shV[t % TL::TURNS] + kk * 32 * CH, lane, cb);
        }
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[0][cb][i] = __builtin_fabsf(acc[0][cb][i]) < INFINITY ? acc[0][cb][i] : o[i];
    }
  }
  m -= BIAS<T>;

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
        for (int i = 0; i < 16; ++i) sums[place + wv % KS][cb * 16 + i][lane] = acc[0][cb][i];
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
        for (int i = 0; i < 16; ++i) acc[0][cb][i] = acc[0][cb][i] * f0 + sums[place + k][cb * 16 + i][lane] * f1;
    }
  }

  if (w0 + l32 >= M) return;
  const long long place = (long long)blockIdx.x * RB + w0 - pt.row + l32;
  float *dst = part_acc + place * D + 4 * half;
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int k = 0; k < 4; ++k)
      *reinterpret_cast<float4 *>(dst + 32 * cb + 8 * k) = make_float4(acc[0][cb][4 * k], acc[0][cb][4 * k + 1], acc[0][cb][4 * k + 2], acc[0][cb][4 * k + 3]);
  if (half == 0) part_ml[place] = make_float2(m, l);
}

// One workgroup per (own segment, query head of its group) merges the parts of the head's own segment and of the shared one, which are two lists of partial
// results, and normalises.  Parts are merged NSLOT side by side, each by D/4 lanes, then across slots.
template <int D>
__global__ __launch_bounds__(256) void prefix_combine_kernel(Sharing sh, int rb, const int4 *__restrict__ seg_tab, int *__restrict__ seg_len,
                                                             int *__restrict__ overflow, const float *__restrict__ own_acc,
                                                             const float2 *__restrict__ own_ml, const int4 *__restrict__ tab,
                                                             const float *__restrict__ part_acc, const float2 *__restrict__ part_ml,
                                                             float *__restrict__ out, float *__restrict__ lse) {
  constexpr int LPE = D / 4, NSLOT = 256 / LPE, UC = 4;
  __shared__ float sh_a[NSLOT][D];
  __shared__ float sh_m[NSLOT], sh_l[NSLOT];
  const int tid = threadIdx.x, s = blockIdx.x, gi = blockIdx.y, b = s / sh.h, c = s % sh.h;
  const int4 own = seg_tab[s];                 // first partial, partials, rows now, 1 if a row was appended
  if (seg_len && gi == 0 && tid == 0) {        // the call appended: the new lengths become visible
    if (own.w) seg_len[s] = own.z;
    else if (overflow) *overflow = 1;          // the segment was full, its new row was dropped
  }
  int cnt = own.y;
  long long first = 0, step = 0;
  const int p = sh.group[b];
  if (p != Sharing::NONE) {
    const int4 e = tab[p * sh.h + c];          // first workgroup, parts, workgroups from one block of rows to the next
    const int row = sh.place[b] * sh.g + gi;
    cnt += e.y;
    first = ((long long)e.x + row / rb * e.z) * rb + row % rb;
    step = rb;
  }
  const int e4 = tid % LPE, slot = tid / LPE;
  float m = M_INIT, l = 0.0f;
  float4 a = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  for (int i0 = slot; i0 < cnt; i0 += NSLOT * UC) {
    float2 ml[UC];
    float4 pa[UC];
#pragma unroll
    for (int u = 0; u < UC; ++u) {
      const int i = i0 + u * NSLOT, ii = i < cnt ? i : i0;
      const bool mine = ii < own.y;
      const long long at = mine ? (long long)(own.x + ii) * sh.g + gi : first + (ii - own.y) * step;
      ml[u] = (mine ? own_ml : part_ml)[at];
      pa[u] = *reinterpret_cast<const float4 *>((mine ? own_acc : part_acc) + at * D + e4 * 4);
      if (i >= cnt) { ml[u] = make_float2(M_INIT, 0.0f); pa[u] = make_float4(0.0f, 0.0f, 0.0f, 0.0f); }
    }
#pragma unroll
    for (int u = 0; u < UC; ++u) {
      const float mn = fmaxf(m, ml[u].x);
      const float fo = __builtin_amdgcn_exp2f(m - mn), fn = __builtin_amdgcn_exp2f(ml[u].x - mn);
      l = l * fo + ml[u].y * fn;
      a.x = a.x * fo + pa[u].x * fn; a.y = a.y * fo + pa[u].y * fn;
      a.z = a.z * fo + pa[u].z * fn; a.w = a.w * fo + pa[u].w * fn;
      m = mn;
    }
  }
  const int live = cnt < NSLOT ? cnt : NSLOT;  // slots that had partials
  if (slot < live) {
    *reinterpret_cast<float4 *>(&sh_a[slot][e4 * 4]) = a;
    if (e4 == 0) { sh_m[slot] = m; sh_l[slot] = l; }
  }
  __syncthreads();
  if (tid < D) {
    float M = M_INIT, acc = 0.0f, ll = 0.0f;
    for (int k = 0; k < live; ++k) M = fmaxf(M, sh_m[k]);
    for (int k = 0; k < live; ++k) {
      const float f = __builtin_amdgcn_exp2f(sh_m[k] - M);
      acc = fmaf(sh_a[k][tid], f, acc);
      ll = fmaf(sh_l[k], f, ll);
    }
    const long long row = (long long)s * sh.g + gi;
    out[row * D + tid] = cnt > 0 ? acc / ll : 0.0f;
    if (lse && tid == 0) lse[row] = (M + log2f(ll)) * LN2;
  }
}

template <typename T, int D> void run_parts(const Sharing &sh, const PrefixPlan &pl, const SharedCache &sc, float c_log2, const void *q, char *ws, hipStream_t s) {
#define ADAKV_PREFIX(KS)                                                                                                          \
  ADAKV_LAUNCH(KS == 1 ? "prefix_attn" : KS == 2 ? "prefix_attn_2" : "prefix_attn_4", (prefix_attn_kernel<T, D, KS>),              \
               dim3(pl.nblk), dim3(256), s, sh, pl.split, sc.headroom, c_log2, (const char *)q, sc.cu, sc.seg_len, (const char *)sc.K, \
               (const char *)sc.V, (float *)(ws + pl.part_acc), (float2 *)(ws + pl.part_ml), (int4 *)(ws + pl.tab))
  if (pl.rb == 128) ADAKV_PREFIX(1);
  else if (pl.rb == 64) ADAKV_PREFIX(2);
  else ADAKV_PREFIX(4);
#undef ADAKV_PREFIX
}

}  // namespace

Sharing share(const SeqTab &st, const Dims &dm, int groups, const int *of) {
  Sharing sh = {};
  sh.groups = groups;
  sh.h = dm.h_kv;
  sh.g = dm.g;
  int at = 0;
  for (int b = 0; b < st.batch; ++b) sh.group[b] = Sharing::NONE;
  for (int p = 0; p < groups; ++p) {
    sh.first[p] = (unsigned char)at;
    for (int b = 0; b < st.batch; ++b)
      if (of[b] == p) {
        sh.group[b] = (unsigned char)p;
        sh.place[b] = (unsigned char)(at - sh.first[p]);
        sh.order[at++] = (unsigned char)b;
      }
  }
  sh.first[groups] = (unsigned char)at;
  return sh;
}

PrefixPlan plan_prefix(const SeqTab &st, const Dims &dm, int dtype, int headroom, const Sharing &sh, const SeqTab &shared, int shared_headroom) {
  PrefixPlan pl = {};
  pl.own = plan_decode(st, dm, dtype, headroom);
  pl.own.whole = false;                        // (partial results, for the merge)
  pl.part_acc = align_up(pl.own.total, 256);
  const auto rows_of = [&](int p) { return (sh.first[p + 1] - sh.first[p]) * sh.g; };
  int most = 0;
  for (int p = 0; p < sh.groups; ++p) most = rows_of(p) > most ? rows_of(p) : most;
  pl.rb = most <= 32 ? 32 : most <= 64 ? 64 : 128;
  const auto blocks_of = [&](int p) { return (rows_of(p) + pl.rb - 1) / pl.rb; };
  const auto cap_of = [&](int p) { return (long long)shared.out_off[p + 1] - shared.out_off[p] + (long long)dm.h_kv * shared_headroom; };
  long long all = 0, least = 0;                // rows times workgroups that read them; workgroups at least
  for (int p = 0; p < sh.groups; ++p) {
    all += cap_of(p) * blocks_of(p);
    least += (long long)blocks_of(p) * dm.h_kv;
  }
  const long long round_wgs = pl.rb == 32 ? 256 : 512, room = round_wgs - least;
  long long want = room > 64 ? (all + room - 1) / room : all / 512;
  if (want < 128) want = 128;
  pl.split = (int)((want + 127) / 128 * 128);
  long long nblk = 0;
  for (int p = 0; p < sh.groups; ++p) {
    const long long blocks = blocks_of(p);
    // parts of a segment: at most capacity / split + 1; with several blocks of rows up to 7 more places each
    nblk += blocks * (cap_of(p) / pl.split + dm.h_kv * (blocks > 1 ? 8 : 1));
  }
  const long long nseg = (long long)sh.groups * dm.h_kv;
  pl.nblk = (int)(nblk > nseg ? nblk : nseg);  // (workgroup s files the entry of segment s)
  pl.part_ml = pl.part_acc + align_up((size_t)pl.nblk * pl.rb * dm.d * sizeof(float), 256);
  pl.tab = pl.part_ml + align_up((size_t)pl.nblk * pl.rb * sizeof(float2), 256);
  pl.total = pl.tab + align_up((size_t)nseg * sizeof(int4), 256);
  return pl;
}

hipError_t launch_decode_prefix(const SeqTab &st, const Dims &dm, int dtype, int headroom, const PrefixPlan &pl, const Sharing &sh,
                                const SharedCache &sc, const void *q, const void *k_new, const void *v_new, const int *cu, void *Kc,
                                void *Vc, int *seg_len, int *overflow, float *out, float *lse, char *ws, hipStream_t s) {
  hipError_t e = launch_decode_parts(st, dm, dtype, headroom, pl.own, q, k_new, v_new, cu, Kc, Vc, seg_len, ws, s);
  if (e != hipSuccess) return e;
  const float c_log2 = dm.scale * LOG2E;
  if (sh.first[sh.groups] > 0) {
    if (dtype == ADAKV_BF16) dm.d == 64 ? run_parts<BF16, 64>(sh, pl, sc, c_log2, q, ws, s) : run_parts<BF16, 128>(sh, pl, sc, c_log2, q, ws, s);
    else if (dtype == ADAKV_FP16) dm.d == 64 ? run_parts<FP16, 64>(sh, pl, sc, c_log2, q, ws, s) : run_parts<FP16, 128>(sh, pl, sc, c_log2, q, ws, s);
    else dm.d == 64 ? run_parts<FP32, 64>(sh, pl, sc, c_log2, q, ws, s) : run_parts<FP32, 128>(sh, pl, sc, c_log2, q, ws, s);
  }
  const dim3 grid(st.batch * dm.h_kv, dm.g);
#define ADAKV_PREFIX_COMBINE(D)                                                                                                      \
  ADAKV_LAUNCH("prefix_combine", prefix_combine_kernel<D>, grid, dim3(256), s, sh, pl.rb, (const int4 *)(ws + pl.own.seg_tab),        \
               k_new ? seg_len : nullptr, overflow, (const float *)(ws + pl.own.part_acc), (const float2 *)(ws + pl.own.part_ml),     \
               (const int4 *)(ws + pl.tab), (const float *)(ws + pl.part_acc), (const float2 *)(ws + pl.part_ml), out, lse)
  if (dm.d == 64) ADAKV_PREFIX_COMBINE(64);
  else ADAKV_PREFIX_COMBINE(128);
#undef ADAKV_PREFIX_COMBINE
  return hipGetLastError();
}

}  // namespace adakv
