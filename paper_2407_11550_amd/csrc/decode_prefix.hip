// A decoding step of a batch whose sequences share caches (Section 3.5's flattened layout twice): every query head attends over a
// segment of a shared cache and over its own, which is one softmax over the rows of both.
//
// With M = g query heads of all the sequences that share a segment, its rows are read once for M rows of queries: 4 d M flops for
// 4 d bytes (16 bits).  Own segments are the same with the g heads of one sequence.  Both products run on the matrix cores as the prompt's do
// (attn_tiles.h), S^T = K Q^T and O^T += V^T P^T, a query per lane, tiles of the segment in LDS.  Weights stay in 32 bits, as in the other
// decoding steps: what is added up is an fp32 result.  bf16: a weight is cut into three bf16 parts whose sum it is to 2^-24, which share one
// operand of V and one sum.  fp16: two fp16 parts, the lower one times 2^11 with a sum of its own, 22 bits for weights down to 2^-23
// of the largest and 2^-45 of it beyond.  fp32: the fp32 matrix instruction.
//
// A segment is split into parts as in decode.hip; a workgroup takes a part for 128, 64 or 32 rows of queries (1, 2 or 4 wavefronts
// share 32 of them; 16 rows in 32 bits) and files the sums.  A second kernel merges, for each query head, the parts of its own segment and of the shared one, and
// the row that the call appends, which it also puts into the cache.
//
// Bound by HBM while few sequences share a cache (8 sequences with 700 to 900 own rows over 3 caches of 16384 rows, 64 query heads: attention 34 us, 5.7
// TB/s), by matrix and vector instructions that take turns where many do (64 over one cache of 32768 rows, 8 heads of 128, g = 4, bf16: 86 us and, when the clock falls, up to 119; 70 GFLOP of
// matrix work with the three parts of the weights; matrix units busy for 39 %, vector units for 39 %, both for 15 %), and by its two launches and a workgroup's start where there is
// little to do (2 over 541 rows: 7.3 us and 5.0).
#include <math.h>

#include "attn_tiles.h"
#include "decode_parts.h"
#include "decode_prefix.h"
#include "row_parts.h"

namespace adakv {
namespace {

// Weights are taken against a kept reference, 2^BIAS times, and the reference is moved, to the maximum of all so far, only where the
// sum of a lane's 16 or 32 weights is beyond MOST.  Moved, the largest weight is 2^BIAS, so 32 of them are no more than MOST.  32 bits and bf16: none
// is above 1, so that no sum is larger than the values times the rows.  fp16: none beyond the type.
template <typename T> constexpr float BIAS = is_f16<T> ? 9.0f : -15.0f;
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

// The weights of 32 keys and their products with values.
template <typename T, int D, typename TL> struct Weights {
  static constexpr int CB = D / 32;
  static constexpr int PARTS = is_f32<T> ? 1 : is_f16<T> ? 2 : 3;
  static constexpr int SUMS = is_f16<T> ? 2 : 1;               // sets of sums
  unsigned w[PARTS][is_f32<T> ? 16 : 8];

  __device__ __forceinline__ void set(const float (&p)[16]) {
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
          x0 -= cut(x0, true);
          x1 -= cut(x1, true);
          w[1][i] = pack(x0, x1);
          x0 -= cut(x0, true);
          x1 -= cut(x1, true);
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
  // The first parts alone, columns 32 cb on (16 bits).
  __device__ __forceinline__ void add_first(floatx16 &o, const u32x4 *tv, int lane, int cb) const {
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) o = product<T>(tile_values<TL>(tv, lane, ks, cb), operand(0, ks), o);
  }
};

// Elements 4 e .. 4 e + 3 of a row as they are in memory.
template <typename T> struct Four {
  typedef unsigned Words __attribute__((ext_vector_type(is_f32<T> ? 4 : 2)));
  Words w;
  __device__ __forceinline__ void load(const char *row, int e) { w = reinterpret_cast<const Words *>(row)[e]; }
  __device__ __forceinline__ void store(char *row, int e) const { reinterpret_cast<Words *>(row)[e] = w; }
  __device__ __forceinline__ void widen(float (&f)[4]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned word = w[is_f32<T> ? i : i / 2];
      if constexpr (is_f32<T>) f[i] = __uint_as_float(word);
      else f[i] = half_of<T>(i % 2 ? word >> 16 : word & 0xffffu);
    }
  }
};

// What a workgroup works on: n keys from row `first_row` of the cache on, of segment s, for query rows from `row` on of the M that look at it.
struct Part {
  long long first_row;
  int s, c, row, M, n;                         // (c: the segment's head)
  int out, first;                              // where its sums go; the segment's first sequence in Sharing::order, or its only one
  bool own;
};
// a / b of numbers whose quotient is below 2^22: the reciprocal is off by 2^-22 of it at most, which is less than one.  (The compiler's divisions took 0.4 us
// of the search below.)
__device__ __forceinline__ int quotient(int a, int b) {
  const int q = (int)((float)a * __builtin_amdgcn_rcpf((float)b)), r = a - q * b;
  return q + (r >= b) - (r < 0);
}
__device__ __forceinline__ int quotient_up(int a, int b) { return quotient(a + b - 1, b); }

// Tiles of a part: at most `spare` parts and one for each segment, which is what the call takes at once; and no fewer than pay for the sums that a part
// leaves for the merge.  With P tiles a part the call takes P tiles' time and that of all / P parts' sums, least for P^2 = all * sums_cost (the
// time of a part's sums over a tile's).  us a call with parts of 1 | 2 | 4 tiles, bf16, d = 128, 8 KV heads, g = 4, 100 own rows: 24 sequences over 2000
// rows a head (all = 250) 22.5 | 17.9 | 19.3, 48 over 2000 (500) 26.2 | 26.1 | 22.2, 48 over 541 (136) 22.5 | 17.9 | 18.4, 24 over 541 (68) 14.6 |
// 15.4 | 16.4, 16 over 2000 (250) 17.8 | 15.4 | 16.2, 8 over 541 (68) 11.5 | 12.1 | 13.1.
__device__ __forceinline__ int tiles_a_part(int all, int spare, float sums_cost) {
  return max(max(1, quotient_up(all, spare)), (int)(__builtin_amdgcn_sqrtf((float)all * sums_cost) + 0.5f));
}

// Finds a part of a shared segment, as find_work does in decode_parts.h from a prefix sum, over the segments, of the parts that their lengths make; but
// a part is as long as it has to be for all of them to be `spare` and one for each segment at most, whatever the capacities are: the
// call lasts as long as its longest part.
// With several blocks of query rows a shared cache's workgroups come in groups of 8 parts, 8 for each block of rows, so that those for one part lie
// a multiple of 8 apart and one of the chip's 8 caches has the rows for all of them.  There are none without work in between: a workgroup that ends at
// once makes the next ones come two to a compute unit where another has room (512 parts with 50 of those among them: 98 us, behind them 71).
// The first part's workgroup files the segment's entry.
template <int TILE, int RB>
__device__ __forceinline__ bool find_shared(const Sharing &sh, int blk, int spare, float sums_cost, int headroom, const int *cu, const int *seg_len, int4 *tab, Part &pt) {
  const int h = sh.h, groups = sh.groups, nseg = groups * h, lane = threadIdx.x & 63;
  const int my_first = sh.first[lane], my_many = lane < groups ? sh.first[lane + 1] - my_first : 0;    // of shared cache `lane`
  const int my_blocks = ((my_many << sh.log_g) + RB - 1) / RB;
  int from, len;
  auto look = [&](int s) {                     // at a segment
    from = cu[s];
    len = min(max(seg_len[s], 0), cu[s + 1] - from + headroom);                // (a corrupt length can never leave the segment)
    return (len + TILE - 1) / TILE;
  };
  // tiles of each shared cache, one a lane, and all of them as often as they are read (less than 2^31 / TILE rows, times 16 blocks)
  const bool few = nseg <= 64;                 // a segment a lane
  int tiles = 0, split, my_parts = 0, upto = 0;
  if (few) {
    tiles = look(min(lane, nseg - 1));
    const int blocks = __shfl(my_blocks, quotient(min(lane, nseg - 1), h));             // (of all lanes: one that is off has nothing to give)
    const int all = wave_sum(lane < nseg ? tiles * blocks : 0);
    split = tiles_a_part(all, spare, sums_cost);
    // Segments' last parts are shorter than the others, so that there may be up to one part more for each segment and block of rows; and where one
    // compute unit gets two workgroups because of them, the call lasts as long as these take side by side.  So longer parts, twice at most.  us,
    // uneven heads, one part more | as many as fit: 64 sequences over 32768 rows a head, g = 8, bf16 199 | 138, 28 over 16000, fp32 237 | 166, 48 over 8000, g = 4
    // 30.5 | 27.9.
    int parts = 0;
#pragma nounroll
    for (int turn = 0; turn < 3; ++turn) {
      parts = lane < nseg && blocks > 0 ? quotient_up(tiles, split) : 0;
      const int over = turn < 2 ? wave_sum(parts * blocks) - spare : 0;
      if (over <= 0) break;
      split += max(1, (int)((float)split * (float)over * __builtin_amdgcn_rcpf((float)spare) + 0.999f));
    }
    upto = wave_scan_incl(parts);
    const int last = __shfl(upto, min(lane * h + h - 1, 63)), before = __shfl(upto, max(min(lane * h, 64) - 1, 0));
    my_parts = lane < groups ? last - (lane ? before : 0) : 0;
  } else {                                     // (not so here: each turn would look at every segment again)
    int mine = 0;
#pragma unroll 4
    for (int c = 0; c < h; ++c) mine += look(min(lane, groups - 1) * h + c);
    const int all = wave_sum(mine * my_blocks);
    split = tiles_a_part(all, spare, sums_cost);
#pragma unroll 4
    for (int c = 0; c < h; ++c) my_parts += quotient_up(look(min(lane, groups - 1) * h + c), split);
    my_parts = my_blocks > 0 ? my_parts : 0;
  }
  const int size = my_blocks > 1 ? my_blocks * ((my_parts + 7) / 8 * 8) : my_parts, end = wave_scan_incl(size);
  const unsigned long long here = __ballot(blk >= end - size && blk < end);
  if (here == 0) return false;
  const int p = __ffsll(here) - 1, base = __builtin_amdgcn_readlane(end - size, p), blocks = __builtin_amdgcn_readlane(my_blocks, p);
  const int count = __builtin_amdgcn_readlane(my_parts, p), at = blk - base;
  const int eights = blocks > 1 ? quotient(at / 8, blocks) : 0;
  const int i = blocks > 1 ? eights * 8 + at % 8 : at, block = blocks > 1 ? at / 8 - eights * blocks : 0;    // which part of the cache's
  if (i >= count) return false;
  int before;                                  // parts in front of the segment's, in its cache
  if (few) {
    const int shift = p ? __builtin_amdgcn_readlane(upto, p * h - 1) : 0;
    const int L = __ffsll(__ballot(upto - shift > i)) - 1;
    pt.s = L;
    before = (L ? __builtin_amdgcn_readlane(upto, L - 1) : 0) - shift;
  } else {
    tiles = look(p * h + min(lane, h - 1));
    upto = wave_scan_incl(lane < h ? quotient_up(tiles, split) : 0);
    const int L = __ffsll(__ballot(upto > i)) - 1;
    pt.s = p * h + L;
    before = L ? __builtin_amdgcn_readlane(upto, L - 1) : 0;
  }
  const int L = few ? pt.s : pt.s - p * h, j = i - before, all = __builtin_amdgcn_readlane(tiles, L), parts = quotient_up(all, split);
  const int rows = quotient_up(all, parts) * TILE, held = __builtin_amdgcn_readlane(len, L);       // equal parts, none of them empty
  pt.first_row = (long long)__builtin_amdgcn_readlane(from, L) + (long long)pt.s * headroom + (long long)j * rows;
  pt.n = min(held - j * rows, rows);
  pt.row = block * RB;
  pt.out = base + block * count + i;
  pt.first = __builtin_amdgcn_readlane(my_first, p);
  pt.M = __builtin_amdgcn_readlane(my_many, p) << sh.log_g;
  pt.c = pt.s - p * h;
  pt.own = false;
  if (j == 0 && block == 0 && threadIdx.x == 0) tab[pt.s] = make_int4(base + before, parts, count, held);
  return true;
}

// A tile of a workgroup whose wavefronts share 32 query rows `KS` at a time: 64 rows, 128 of 128 bytes, 32 of 512 where each wavefront takes all of them.  With
// tiles of 64 KB of keys and values two workgroups fit on a compute unit.
template <typename T, int D, int KS> using Rows = Tile<T, D, D * T::SIZE == 512 && KS == 1 ? 1 : D * T::SIZE == 128 ? 4 : 2>;
// Tiles in LDS: the keys of one or two of them, and behind these the values.
template <typename TL, int TURNS> struct Place {
  static constexpr int BYTES = 2 * TURNS * TL::WORDS * 16;
  u32x4 *lds;
  __device__ __forceinline__ u32x4 *keys(int t) const { return lds + t % TURNS * TL::WORDS; }
  __device__ __forceinline__ u32x4 *values(int t) const { return lds + (TURNS + t % TURNS) * TL::WORDS; }
};

// A wavefront's share of tile t of n rows: rows on (wv * LOADS + i) * RPI + lane / CH; rows past the end repeat the last one.
template <typename TL, int TURNS>
__device__ __forceinline__ void load_tile(const char *Kh, const char *Vh, int n, int t, int wv, int lane, const Place<TL, TURNS> &place) {
  constexpr int ROWB = TL::ROWB, CH = TL::CH, KT = TL::KT;
  const char *kb = scalar_address(Kh + (long long)t * KT * ROWB), *vb = scalar_address(Vh + (long long)t * KT * ROWB);
  const u32x4 *dk = place.keys(t) + wv * TL::LOADS * 64, *dv = place.values(t) + wv * TL::LOADS * 64;
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
}
// Tile t is there, and the next one on its way if it has a place; tile 0 has been asked for.
template <int TURNS, typename Load> __device__ __forceinline__ void await_tile(int t, int tiles, Load &&load) {
  if constexpr (TURNS == 2) {
    meet();
    if (t + 1 < tiles) load(t + 1);
  } else {
    if (t) {
      meet();                                  // (what was there has been read)
      load(t);
    }
    meet();
  }
}

// Sums of a part, `KS` wavefronts to 32 query rows.
template <typename T, int D, int KS>
__device__ __forceinline__ void sum_part(const Sharing &sh, const Part &pt, int order, float c_log2, const char *q, const Segments &seg, float *part_acc, float2 *part_ml,
                                         int stride, u32x4 *lds, int (&sh_bad)[4]) {
  typedef Rows<T, D, KS> TL;
  const Place<TL, 2> place_of{lds};
  typedef Weights<T, D, TL> W;
  constexpr int ROWB = TL::ROWB, CH = TL::CH, KT = TL::KT, CB = D / 32;
  // 32 keys at a time, or two times 32 where a wavefront has so many of a tile (fp16, d = 128: its two sets of sums leave no registers for the logits of two)
  constexpr int PAIR = 2 * KS <= KT / 32 && !(is_f16<T> && D == 128) ? 2 : 1;
  // The rounding of a logit is what an fp32 result's error against 64 bits consists of.  One chain | two | four, 28 sequences over 16000 rows, g = 8, d = 128: 1.3e-6 | 8.5e-7 |
  // 7.1e-7 in 161 | 161 | 165 us; 40 over 8000, g = 4, d = 64: 9.2e-7 | 6.5e-7 | 5.7e-7 in 49.8 | 49.9 | 50.2.
  constexpr int CHAINS = is_f32<T> ? 2 : 1;
  constexpr bool TIGHT = D == 128 && KS == 1;                 // addresses are made where they are used, not kept in registers
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, half = lane >> 5;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const char *Kh = seg.K + pt.first_row * ROWB, *Vh = seg.V + pt.first_row * ROWB;
  const int c = pt.c, n = pt.n;

  const int w0 = pt.row + 32 * (wv / KS), m_row = min(w0 + l32, pt.M - 1);      // the wavefront's first query row, this lane's
  const bool idle = w0 >= pt.M;
  const int b = pt.own ? pt.first : __shfl(order, pt.first + (m_row >> sh.log_g));
  const char *Qh = q + (((long long)(b * sh.h + c) << sh.log_g) + (m_row & ((1 << sh.log_g) - 1))) * ROWB;
  u32x4 qf[CH / 2];
#pragma unroll
  for (int s = 0; s < CH / 2; ++s) qf[s] = *reinterpret_cast<const u32x4 *>(Qh + (2 * s + half) * 16);

  const int tiles = (n + KT - 1) / KT;
  auto load = [&](int t) __attribute__((always_inline)) {
    int here = lane;
    if (TIGHT) asm volatile("" : "+v"(here));
    load_tile(Kh, Vh, n, t, wv, here, place_of);
  };
  // tile t is there, and the next one on its way
  auto await = [&](int t) __attribute__((always_inline)) { await_tile<2>(t, tiles, load); };

  load(0);
  // (the wait for the queries stands here, once, and not in front of the first products of every tile, where it would be one for the next tile's loads)
#pragma unroll
  for (int s = 0; s < CH / 2; ++s) asm volatile("" : "+v"(qf[s]));

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
  // 32 keys of tile t, or two times 32: all the logits, all the weights, then the sums, with nothing but the rare move of
  // the reference in between, so that the matrix instructions of one run beside the vector instructions of another.
  auto add_keys = [&](int t, int kk) __attribute__((always_inline)) {
    constexpr int N = PAIR, apart = KS;
    int here = lane;
    if (TIGHT) asm volatile("" : "+v"(here));
    const u32x4 *tk = place_of.keys(t), *tv = place_of.values(t);
    floatx16 sc[N];
#pragma unroll
    for (int k = 0; k < N; ++k) sc[k] = tile_logits<T, TL, CHAINS>(tk + (kk + k * apart) * 32 * CH, qf, here & 31, here >> 5);
    const int left = n - t * KT - 32 * kk;     // keys from the first on
    if (left < 32 * ((N - 1) * apart + 1)) {
#pragma unroll
      for (int k = 0; k < N; ++k)
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[k][i] = 8 * (i / 4) + 4 * half + i % 4 < left - 32 * k * apart ? sc[k][i] : -INFINITY;
    }
    float pr[N][16], sum = 0.0f;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float one = weigh(sc[k], pr[k]);
      sum = k ? sum + one : one;
    }
    if (__builtin_expect(__any(!(sum <= MOST<T>)), 0)) {       // too far above the reference (or no number): a new one
      float top = sc[0][0];
#pragma unroll
      for (int k = 0; k < N; ++k)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[k][i]);
      const float mn = fmaxf(m, fmaxf(top, other_half(top)) * c_log2), corr = __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= corr;
#pragma unroll
      for (int i = 0; i < W::SUMS; ++i)
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) acc[i][cb] *= corr;
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float one = weigh(sc[k], pr[k]);
        sum = k ? sum + one : one;
      }
    }
    l += sum;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      W w;
      w.set(pr[k]);
      w.add_values(acc, tv + (kk + k * apart) * 32 * CH, here);
    }
  };

  for (int t = 0; t < tiles; ++t) {
    await(t);
    if (is_f32<T> && n - t * KT < KT) {        // (the last tile: values past the end are cleared, as their weights are 0 and they may be no numbers)
      for (int i = (n - t * KT) * CH + tid; i < KT * CH; i += 256) place_of.values(t)[i] = u32x4{0, 0, 0, 0};
      __syncthreads();
    }
    if (idle) continue;
    // (this wavefront's 32 keys of the tile are every KS-th 32)
#pragma unroll
    for (int k = 0; k < KT / 32; k += PAIR * KS)
      if (n - t * KT - 32 * (wv % KS + k) > 0) add_keys(t, wv % KS + k);
  }
  l += other_half(l);
  if constexpr (W::SUMS == 2) {
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) acc[0][cb] += acc[1][cb] * LOW_DOWN;
  }

  // Where a sum is infinite or NaN, a value that is none may have met a weight's lower part of 0, or of the other sign, or a
  // weight of 0 of the rows past the end: once more with the upper parts alone, which say what it is.  (32 bits: a weight has no parts, and
  // there are no values past the end.)
  if constexpr (!is_f32<T>) {
    float worst[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int i = 0; i < 16; ++i) worst[i % 4] = fmaf(acc[0][cb][i], 0.0f, worst[i % 4]);
    const bool bad = __any(!((worst[0] + worst[1]) + (worst[2] + worst[3]) == 0.0f));
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
          for (int kk = wv % KS; kk < KT / 32; kk += KS) {
            if (n - t * KT - 32 * kk <= 0) break;
            // (the rows past the end repeat the last one, so their weights may stay)
            const floatx16 sc = tile_logits<T, TL>(place_of.keys(t) + kk * 32 * CH, qf, l32, half);
            float pr[16];
            weigh(sc, pr);
            if constexpr (is_f16<T>) {                           // (none is too small for the type)
#pragma unroll
              for (int i = 0; i < 16; ++i) pr[i] = pr[i] > 0.0f ? fmaxf(pr[i], 0x1p-24f) : pr[i];
            }
            W w;
            w.set(pr);
            w.add_first(o, place_of.values(t) + kk * 32 * CH, lane, cb);
          }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[0][cb][i] = __builtin_fabsf(acc[0][cb][i]) < INFINITY ? acc[0][cb][i] : o[i];
      }
    }
  }
  m -= BIAS<T>;

  if constexpr (KS > 1) {
    // the first of those that share their rows takes the others' sums, through the tiles' place
    typedef float4 Shared[CB * 4][64];
    static_assert((4 - 4 / KS) * (sizeof(Shared) + 64 * sizeof(float2)) <= Place<TL, 2>::BYTES, "the sums have room");
    Shared *others = reinterpret_cast<Shared *>(lds);
    float2(*ml)[64] = reinterpret_cast<float2(*)[64]>(others + 4 - 4 / KS);
    const int place = wv / KS * (KS - 1) - 1;                  // + 1 .. KS - 1
    meet();
    if (wv % KS) {
#pragma unroll
      for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          others[place + wv % KS][cb * 4 + k][lane] = make_float4(acc[0][cb][4 * k], acc[0][cb][4 * k + 1], acc[0][cb][4 * k + 2], acc[0][cb][4 * k + 3]);
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
        for (int x = 0; x < 4; ++x) {
          const float4 o = others[place + k][cb * 4 + x][lane];
          const float four[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[0][cb][4 * x + i] = acc[0][cb][4 * x + i] * f0 + four[i] * f1;
        }
    }
  }

  if (w0 + l32 >= pt.M) return;
  const long long place = (long long)pt.out * stride + w0 - pt.row + l32;
  float *dst = part_acc + place * D + 4 * half;
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int k = 0; k < 4; ++k)
      *reinterpret_cast<float4 *>(dst + 32 * cb + 8 * k) = make_float4(acc[0][cb][4 * k], acc[0][cb][4 * k + 1], acc[0][cb][4 * k + 2], acc[0][cb][4 * k + 3]);
  if (half == 0) part_ml[place] = make_float2(m, l);
}

// The same in 32 bits for no more than 16 query rows, each wavefront on 16 keys of a tile (32 keys of two wavefronts times 32 query rows, of which half
// or more are none: 64 sequences of 500 own rows, 8 heads of 128, g = 4 100 us, now 54, 4.9 TB/s).  A lane has query lane % 16, of the logits those of keys 4 (lane / 16)
// on, and of each value row 16 bytes: what they add to are columns 4 apart, so that what a lane has of a query in the end are 16 bytes again.
template <int D, int TURNS>
__device__ __forceinline__ void sum_few(const Sharing &sh, const Part &pt, int order, float c_log2, const char *q, const Segments &seg, float *part_acc, float2 *part_ml,
                                        int stride, u32x4 *lds) {
  typedef Rows<FP32, D, 8> TL;
  const Place<TL, TURNS> place_of{lds};
  typedef float floatx4 __attribute__((ext_vector_type(4)));
  constexpr int ROWB = TL::ROWB, CH = TL::CH, VB = D / 64;
  static_assert(TL::KT == 64, "16 keys a wavefront");
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, quad = lane >> 4;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const char *Kh = seg.K + pt.first_row * ROWB, *Vh = seg.V + pt.first_row * ROWB;
  const int n = pt.n, m_row = min(pt.row + l16, pt.M - 1);
  const int b = pt.own ? pt.first : __shfl(order, pt.first + (m_row >> sh.log_g));
  const char *Qh = q + (((long long)(b * sh.h + pt.c) << sh.log_g) + (m_row & ((1 << sh.log_g) - 1))) * ROWB;
  u32x4 qf[CH / 4];
#pragma unroll
  for (int s = 0; s < CH / 4; ++s) qf[s] = *reinterpret_cast<const u32x4 *>(Qh + (4 * s + quad) * 16);
  const int tiles = (n + TL::KT - 1) / TL::KT;
  auto load = [&](int t) __attribute__((always_inline)) { load_tile(Kh, Vh, n, t, wv, lane, place_of); };
  load(0);
#pragma unroll
  for (int s = 0; s < CH / 4; ++s) asm volatile("" : "+v"(qf[s]));             // (as above)

  floatx4 acc[VB][4];
#pragma unroll
  for (int c = 0; c < VB; ++c)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[c][e] = floatx4{0};
  float m = M_INIT, l = 0.0f;
  const int row = 16 * wv + l16;
  for (int t = 0; t < tiles; ++t) {
    await_tile<TURNS>(t, tiles, load);
    const int left = n - t * TL::KT - 16 * wv;
    if (left <= 0) continue;
    const u32x4 *tk = place_of.keys(t), *tv = place_of.values(t);
    // (four sums and then a tree, as above; 64 sequences of 500 own rows 8.4e-7 in one chain, 5.0e-7 now, 2 over 20000 shared ones 1.3e-6 and 4.8e-7, in the same time)
    floatx4 four[4] = {floatx4{0}, floatx4{0}, floatx4{0}, floatx4{0}};
#pragma unroll
    for (int s = 0; s < CH / 4; ++s) {
      const u32x4 kw = tk[row * CH + ((4 * s + quad) ^ TL::swz_k(row))];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const unsigned ka = kw[e], qa = qf[s][e];
        four[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(ka), __uint_as_float(qa), four[e], 0, 0, 0);
      }
    }
    floatx4 sc = (four[0] + four[1]) + (four[2] + four[3]);
    if (left < 16) {
#pragma unroll
      for (int i = 0; i < 4; ++i) sc[i] = 4 * quad + i < left ? sc[i] : -INFINITY;
    }
    float pr[4];
    auto weigh = [&]() {
#pragma unroll
      for (int i = 0; i < 4; ++i) pr[i] = __builtin_amdgcn_exp2f(fmaf(sc[i], c_log2, BIAS<FP32> - m));
      return (pr[0] + pr[1]) + (pr[2] + pr[3]);
    };
    float sum = weigh();
    if (__builtin_expect(__any(!(sum <= MOST<FP32>)), 0)) {
      float top = fmaxf(fmaxf(sc[0], sc[1]), fmaxf(sc[2], sc[3]));
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float mn = fmaxf(m, top * c_log2), corr = __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= corr;
#pragma unroll
      for (int c = 0; c < VB; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[c][e] *= corr;
      sum = weigh();
    }
    l += sum;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int key = 4 * quad + i, at = 16 * wv + key;
#pragma unroll
      for (int c = 0; c < VB; ++c) {
        u32x4 vw = tv[at * CH + ((16 * c + l16) ^ TL::swz_v(at))];
        if (left < 16) {                       // (what repeats the last row has no part in the sums, whatever it is)
#pragma unroll
          for (int e = 0; e < 4; ++e) vw[e] = key < left ? vw[e] : 0u;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const unsigned va = vw[e];
          acc[c][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(va), pr[i], acc[c][e], 0, 0, 0);
        }
      }
    }
  }
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  m -= BIAS<FP32>;

  typedef floatx4 Shared[VB * 4][64];
  static_assert(3 * (sizeof(Shared) + 64 * sizeof(float2)) <= Place<TL, TURNS>::BYTES, "the sums have room");
  Shared *others = reinterpret_cast<Shared *>(lds);
  float2(*ml)[64] = reinterpret_cast<float2(*)[64]>(others + 3);
  meet();
  if (wv) {
#pragma unroll
    for (int x = 0; x < VB * 4; ++x) others[wv - 1][x][lane] = acc[x / 4][x % 4];
    ml[wv - 1][lane] = make_float2(m, l);
  }
  __syncthreads();
  if (wv) return;
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const float2 other = ml[k][lane];
    const float mn = fmaxf(m, other.x), f0 = __builtin_amdgcn_exp2f(m - mn), f1 = __builtin_amdgcn_exp2f(other.x - mn);
    m = mn;
    l = l * f0 + other.y * f1;
#pragma unroll
    for (int x = 0; x < VB * 4; ++x) acc[x / 4][x % 4] = acc[x / 4][x % 4] * f0 + others[k][x][lane] * f1;
  }
  if (pt.row + l16 >= pt.M) return;
  const long long place = (long long)pt.out * stride + l16;
  float *dst = part_acc + place * D + 16 * quad;
#pragma unroll
  for (int c = 0; c < VB; ++c)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      *reinterpret_cast<float4 *>(dst + 64 * c + 4 * r) = make_float4(acc[c][0][r], acc[c][1][r], acc[c][2][r], acc[c][3][r]);
  if (quad == 0) part_ml[place] = make_float2(m, l);
}

// Workgroups on a compute unit.
template <typename T, int D, int KS> constexpr int AT_ONCE = Place<Rows<T, D, KS>, 2>::BYTES > 64 * 1024 ? 1 : 2;

template <typename T, int D, int KS>
__global__ __launch_bounds__(256, (AT_ONCE<T, D, KS>)) void prefix_attn_kernel(
    Sharing sh, PrefixSplit sp, float c_log2, const char *__restrict__ q, Segments shared, Segments own, PrefixSums sums) {
  typedef Rows<T, D, KS> TL;
  typedef Rows<T, D, D * T::SIZE == 128 ? 4 : 2> OL;           // of own segments, which have up to 8 query rows
  constexpr int OWN_TURNS = Place<OL, 2>::BYTES > Place<TL, 2>::BYTES ? 1 : 2;
  static_assert(Place<OL, OWN_TURNS>::BYTES <= Place<TL, 2>::BYTES, "own segments' tiles have room");
  __shared__ __align__(16) u32x4 lds[Place<TL, 2>::BYTES / 16];
  __shared__ int sh_bad[4], sh_scan[24];
  const int order = sh.order[threadIdx.x & 63];
  Part pt;
  if ((int)blockIdx.x < sp.shared_blocks) {
    if (!find_shared<TL::KT, 128 / KS>(sh, (int)blockIdx.x, sp.spare, sp.sums_cost, shared.headroom, shared.cu, shared.seg_len, sums.shared_tab, pt)) return;
    if constexpr (KS == 8) sum_few<D, 2>(sh, pt, order, c_log2, q, shared, sums.shared_acc, sums.shared_ml, 16, lds);
    else sum_part<T, D, KS>(sh, pt, order, c_log2, q, shared, sums.shared_acc, sums.shared_ml, 128 / KS, lds, sh_bad);
  } else {
    Work wk;
    if (!find_work<4, false>(sp.own_segments, sp.own_per, sp.own_split, own.headroom, 0, own.cu, own.seg_len, sh_scan, sums.own_tab, wk, {}, sp.shared_blocks))
      return;
    const int rows = min(sp.own_split, (quotient_up(wk.rows, wk.parts) + OL::KT - 1) / OL::KT * OL::KT);       // (as above)
    const int b = quotient(wk.s, sh.h), g = 1 << sh.log_g;
    pt = {(long long)wk.first_row + (long long)wk.s * own.headroom + wk.j * rows, wk.s, wk.s - b * sh.h, 0, g, min(wk.rows - wk.j * rows, rows),
          (int)blockIdx.x - sp.shared_blocks, b, true};
    if constexpr (is_f32<T>) sum_few<D, OWN_TURNS>(sh, pt, order, c_log2, q, own, sums.own_acc, sums.own_ml, g, lds);
    else sum_part<T, D, OL::KT / 32>(sh, pt, order, c_log2, q, own, sums.own_acc, sums.own_ml, g, lds, sh_bad);
  }
}

// One workgroup per (own segment, query head of its group) merges the parts of the head's own segment, of the shared one and the row that the call
// appends, which are one list of partial results, and normalises.  They are merged NSLOT side by side, each by D/4 lanes, then across slots.  The
// first head's workgroup puts the row into the cache.
template <typename T, int D>
__global__ __launch_bounds__(256) void prefix_combine_kernel(Sharing sh, int log_rb, float c_log2, const char *__restrict__ q, const char *__restrict__ k_new,
                                                             const char *__restrict__ v_new, Segments shared, Segments own, int *new_len,
                                                             int *__restrict__ overflow, PrefixSums sums, float *__restrict__ out,
                                                             float *__restrict__ lse) {
  constexpr int LPE = D / 4, NSLOT = 256 / LPE, UC = 4, ROWB = D * T::SIZE;
  __shared__ float sh_a[NSLOT][D];
  __shared__ float sh_m[NSLOT], sh_l[NSLOT];
  const int tid = threadIdx.x, s = blockIdx.x, gi = blockIdx.y, b = quotient(s, sh.h), c = s - b * sh.h;
  const int e4 = tid % LPE, slot = tid / LPE, rb = 1 << log_rb;
  const long long row = ((long long)s << sh.log_g) + gi;
  // everything that follows from the workgroup's number alone is asked for at once: one wait after the other is what the kernel's time is
  const int whose = sh.whose[b], from = own.cu[s], to = own.cu[s + 1];
  const int4 mine = sums.own_tab[s];           // first partial, partials, rows
  Four<T> q4, k4, v4;
  if (k_new) {
    q4.load(q + row * ROWB, e4);
    k4.load(k_new + (long long)s * ROWB, e4);
    v4.load(v_new + (long long)s * ROWB, e4);
  }
  int cnt = mine.y;
  long long first = 0, step = 0;
  if (whose >= 0) {
    const int t = (whose & 255) * sh.h + c, len = shared.seg_len[t], cap = shared.cu[t + 1] - shared.cu[t] + shared.headroom;
    const int4 e = sums.shared_tab[t];         // first partial of the first block of rows, parts, from one block to the next
    const int r = ((whose >> 8) << sh.log_g) + gi;
    if (len > 0 && cap > 0) {                  // (a shared segment without rows has no entry)
      cnt += e.y;
      first = ((long long)e.x + (r >> log_rb) * e.z << log_rb) + (r & (rb - 1));
      step = rb;
    }
  }
  float m = M_INIT, l = 0.0f;
  float4 a = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  // sums taken against the reference om = z * by, of which only the exponent's difference is made from both, so that an om too large to be
  // one fp32 number loses nothing
  auto add = [&](float z, float by, float ol, const float4 &oa) {
    const float mn = fmaxf(m, z * by), fo = fast_exp2(m - mn), fn = fast_exp2(fmaf(z, by, -mn));
    l = l * fo + ol * fn;
    a.x = a.x * fo + oa.x * fn; a.y = a.y * fo + oa.y * fn;
    a.z = a.z * fo + oa.z * fn; a.w = a.w * fo + oa.w * fn;
    m = mn;
  };
  for (int i0 = slot; i0 < cnt; i0 += NSLOT * UC) {
    float2 ml[UC];
    float4 pa[UC];
#pragma unroll
    for (int u = 0; u < UC; ++u) {
      const int i = i0 + u * NSLOT, ii = i < cnt ? i : i0;
      const bool of_own = ii < mine.y;
      const long long at = of_own ? ((long long)(mine.x + ii) << sh.log_g) + gi : first + (ii - mine.y) * step;
      ml[u] = (of_own ? sums.own_ml : sums.shared_ml)[at];
      pa[u] = *reinterpret_cast<const float4 *>((of_own ? sums.own_acc : sums.shared_acc) + at * D + e4 * 4);
      if (i >= cnt) { ml[u] = make_float2(M_INIT, 0.0f); pa[u] = make_float4(0.0f, 0.0f, 0.0f, 0.0f); }
    }
#pragma unroll
    for (int u = 0; u < UC; ++u) add(ml[u].x, 1.0f, ml[u].y, pa[u]);
  }
  // (the length is what the other kernel saw: this one writes the new one)
  const bool room = k_new && mine.z < to - from + own.headroom;
  if (room && slot == cnt % NSLOT) {           // the appended row: one of weight 1 at its logit
    float x[4], k[4], v[4];
    q4.widen(x);
    k4.widen(k);
    v4.widen(v);
    float dot = fmaf(x[0], k[0], x[1] * k[1]) + fmaf(x[2], k[2], x[3] * k[3]);
#pragma unroll
    for (int o = 1; o < LPE; o <<= 1) dot += __shfl_xor(dot, o);
    add(dot, c_log2, 1.0f, make_float4(v[0], v[1], v[2], v[3]));
  }
  if (k_new && gi == 0) {
    const long long at = ((long long)from + (long long)s * own.headroom + mine.z) * ROWB;
    if (room && slot == 0) k4.store(const_cast<char *>(own.K) + at, e4);
    if (room && slot == 1) v4.store(const_cast<char *>(own.V) + at, e4);
    if (tid == 0) {
      if (room) new_len[s] = mine.z + 1;
      else if (overflow) *overflow = 1;        // the segment was full, its new row was dropped
    }
  }
  const int all = cnt + room, live = all < NSLOT ? all : NSLOT;                // slots that had any
  if (slot < live) {
    *reinterpret_cast<float4 *>(&sh_a[slot][e4 * 4]) = a;
    if (e4 == 0) { sh_m[slot] = m; sh_l[slot] = l; }
  }
  __syncthreads();
  if (tid < D) {
    float M = M_INIT, acc = 0.0f, ll = 0.0f;
    for (int k = 0; k < live; ++k) M = fmaxf(M, sh_m[k]);
    for (int k = 0; k < live; ++k) {
      const float f = fast_exp2(sh_m[k] - M);
      acc = fmaf(sh_a[k][tid], f, acc);
      ll = fmaf(sh_l[k], f, ll);
    }
    out[row * D + tid] = all > 0 ? acc / ll : 0.0f;
    if (lse && tid == 0) lse[row] = (M + log2f(ll)) * LN2;
  }
}

template <typename T, int D>
void run_prefix(const Sharing &sh, const PrefixPlan &pl, float c_log2, const void *q, const void *k_new, const void *v_new, const Segments &shared,
                const Segments &own, int *seg_len, int *overflow, float *out, float *lse, char *ws, hipStream_t s) {
  const PrefixSums sums = {(float *)(ws + pl.shared_acc), (float *)(ws + pl.own_acc), (float2 *)(ws + pl.shared_ml), (float2 *)(ws + pl.own_ml),
                           (int4 *)(ws + pl.shared_tab), (int4 *)(ws + pl.own_tab)};
#define ADAKV_PREFIX(KS)                                                                                                              \
  ADAKV_LAUNCH(KS == 1 ? "prefix_attn" : KS == 2 ? "prefix_attn_2" : KS == 4 ? "prefix_attn_4" : "prefix_attn_8", (prefix_attn_kernel<T, D, KS>),                  \
               dim3(pl.split.shared_blocks + pl.own_blocks), dim3(256), s, sh, pl.split, c_log2, (const char *)q, shared, own, sums)
  if (pl.split.rb == 128) ADAKV_PREFIX(1);
  else if (pl.split.rb == 64) ADAKV_PREFIX(2);
  else if constexpr (is_f32<T>) ADAKV_PREFIX(8);               // (16 rows: plan_prefix)
  else if constexpr (D == 64) ADAKV_PREFIX(4);   // (32)
#undef ADAKV_PREFIX
  ADAKV_LAUNCH("prefix_combine", (prefix_combine_kernel<T, D>), dim3(pl.split.own_segments, 1 << sh.log_g), dim3(256), s, sh,
               pl.split.rb == 128 ? 7 : pl.split.rb == 64 ? 6 : pl.split.rb == 32 ? 5 : 4, c_log2,
               (const char *)q, (const char *)k_new, (const char *)v_new, shared, own, seg_len, overflow, sums, out, lse);
}

}  // namespace

Sharing share(const SeqTab &st, const Dims &dm, int groups, const int *of) {
  Sharing sh = {};
  sh.groups = groups;
  sh.h = dm.h_kv;
  sh.log_g = dm.g == 8 ? 3 : dm.g / 2;
  int at = 0;
  for (int b = 0; b < st.batch; ++b) sh.whose[b] = -1;
  for (int p = 0; p < groups; ++p) {
    sh.first[p] = (unsigned char)at;
    for (int b = 0; b < st.batch; ++b)
      if (of[b] == p) {
        sh.whose[b] = p | (at - sh.first[p]) << 8;
        sh.order[at++] = (unsigned char)b;
      }
  }
  sh.first[groups] = (unsigned char)at;
  return sh;
}

PrefixPlan plan_prefix(const SeqTab &st, const Dims &dm, int dtype, int headroom, const Sharing &sh) {
  PrefixPlan pl = {};
  const auto rows_of = [&](int p) { return (sh.first[p + 1] - sh.first[p]) << sh.log_g; };
  int most = 0;
  for (int p = 0; p < sh.groups; ++p) most = rows_of(p) > most ? rows_of(p) : most;
  // Query rows of a workgroup: as many as the longest shared list has, but then fewer, so that its wavefronts all have some.  us a call, 8 KV heads, g = 4, 60
  // to 100 own rows.  fp32, d = 128, 16 | 64: 8 sequences over 2000 rows a head 19.4 | 21.7, over 20000 56.5 | 62.5, 12 over 8000 48.7 | 38.8.
  // 16 bits, 32 | 64, d = 64: 8 over 2000 10.5 | 11.1, 2 over 20000 14.5 | 15.8.  64 | 128, bf16, d = 128: 18 over 2000 20.4 | 21.7, over 32768 48.9 |
  // 44.0, 48 over 8192 34.3 | 30.3.
  const bool wide = dtype == ADAKV_FP32;
  const int rb = pl.split.rb = wide && most <= 32 ? 16 : !wide && dm.d == 64 && most <= 32 ? 32 : most <= 64 ? 64 : 128;
  const auto blocks_of = [&](int p) { return (rows_of(p) + rb - 1) / rb; };
  long long n = 0, padding = 0;                // workgroups at least, one for each segment and block of rows; places that groups of 8 take
  for (int p = 0; p < sh.groups; ++p) {
    n += (long long)blocks_of(p) * dm.h_kv;
    if (blocks_of(p) > 1) padding += 7ll * blocks_of(p);
  }
  // A workgroup for each compute unit: own segments run beside them, and more of them only begin later.  us, 256 parts | twice as many, bf16, d = 128, g = 4:
  // 64 sequences over 32768 rows with 500 own rows 85.7 | 99.5, with none 82.7 | 77.5; 8 over 32768 29.3 | 34.5 (320 parts), and with 192 33.7.
  const long long want = 256;
  pl.split.spare = (int)(want > n / 2 + 1 ? want : n / 2 + 1);
  // sums of a block's rows, written and read at 5 TB/s, over a tile's time in a workgroup (Rows)
  const int sum_rows = most < rb ? most : rb;
  const float tile_us = !wide ? 1.0f : (dm.d == 64 || rb == 128 ? 3.0f : 6.0f) * (rb == 16 ? 0.25f : 1.0f);
  pl.split.sums_cost = sum_rows * (dm.d + 2) * 8.0f / 5.0e6f / tile_us;
  pl.split.shared_blocks = (int)(n ? pl.split.spare + n + padding : 0);
  const int tile = dm.d == 64 && !wide ? 128 : 64;
  const long long nseg = (long long)sh.groups * dm.h_kv, own = (long long)st.batch * dm.h_kv;
  const long long own_cap = (long long)st.out_off[st.batch] + own * headroom, a_part = (own_cap + 511) / 512;
  pl.split.own_segments = (int)own;
  pl.split.own_per = (int)((own + 255) / 256);
  pl.split.own_split = (int)((a_part < tile ? tile : a_part) + tile - 1) / tile * tile;
  long long longest = 0;                       // an own segment's capacity at most
  for (int b = 0; b < st.batch; ++b) {
    const long long most_kept = st.Bp[b] < st.n[b] ? st.Bp[b] : st.n[b];
    longest = most_kept + dm.w + headroom > longest ? most_kept + dm.w + headroom : longest;
  }
  pl.own_blocks = (int)(longest <= pl.split.own_split ? own : own_cap / pl.split.own_split + own);
  size_t at = 0;
  const auto take = [&](size_t bytes) {
    const size_t here = at;
    at += align_up(bytes, 256);
    return here;
  };
  pl.shared_acc = take((size_t)pl.split.shared_blocks * rb * dm.d * sizeof(float));
  pl.own_acc = take((size_t)pl.own_blocks * dm.g * dm.d * sizeof(float));
  pl.shared_ml = take((size_t)pl.split.shared_blocks * rb * sizeof(float2));
  pl.own_ml = take((size_t)pl.own_blocks * dm.g * sizeof(float2));
  pl.shared_tab = take((size_t)nseg * sizeof(int4));
  pl.own_tab = take((size_t)own * sizeof(int4));
  pl.total = at;
  return pl;
}

hipError_t launch_decode_prefix(const Dims &dm, int dtype, const PrefixPlan &pl, const Sharing &sh, const Segments &shared, const Segments &own,
                                const void *q, const void *k_new, const void *v_new, int *seg_len, int *overflow, float *out, float *lse,
                                char *ws, hipStream_t s) {
#define ADAKV_PREFIX(T)                                                                                                                     \
  (dm.d == 64 ? run_prefix<T, 64>(sh, pl, dm.scale * LOG2E, q, k_new, v_new, shared, own, seg_len, overflow, out, lse, ws, s)               \
              : run_prefix<T, 128>(sh, pl, dm.scale * LOG2E, q, k_new, v_new, shared, own, seg_len, overflow, out, lse, ws, s))
  if (dtype == ADAKV_BF16) ADAKV_PREFIX(BF16);
  else if (dtype == ADAKV_FP16) ADAKV_PREFIX(FP16);
  else ADAKV_PREFIX(FP32);
#undef ADAKV_PREFIX
  return hipGetLastError();
}

}  // namespace adakv
