// What the kernels of a decoding step share (decode.hip, decode_q8.hip): how a workgroup finds the rows it works on,
// the matrix instructions and the parts that a softmax weight is cut into for them.
#pragma once

#include "common.h"

namespace adakv {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
constexpr float M_INIT = -1.0e30f;    // finite "no row seen yet" maximum: exp2(-inf - M_INIT) = 0

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// Rows of segment s this call works on: the rows held, plus the row the call itself appends
// (`grow` = 1) if the segment has room for it.
__device__ __forceinline__ int rows_held(const int *cu, const int *seg_len, int s, int headroom,
                                         int grow) {
  const int cap = cu[s + 1] - cu[s] + headroom;
  const int held = min(max(seg_len[s], 0), cap);   // a corrupt length can never leave the segment
  return held + (held < cap ? grow : 0);
}

// What a workgroup works on: part `j` of the `parts` that the `rows` rows of segment s are split into.
struct Work {
  int s, j, parts, rows, first_row;
  bool appended;                               // the last row is the one the call appends
  int hidden;                                  // rows between the sinks and the window, which `rows` leaves out
};

// A call that looks at a segment's first `sinks` rows and its last ones alone: at most `limit` rows, sinks included.
// Rows are then numbered without those in between, `hidden` of them.
struct Window {
  int limit, sinks;
};
template <bool WIN> __device__ __forceinline__ int seen_rows(int now, Window win) { return WIN ? min(now, win.limit) : now; }
template <bool WIN> __device__ __forceinline__ int place_of(int r, int hidden, Window win) {
  return r + (WIN && r >= win.sinks ? hidden : 0);
}

// Finds it from a prefix sum, over the segments, of the parts that their lengths make (blocks of `split` rows).  The
// same in all lanes.  `before_us`: workgroups of the launch in front of these.  False: the workgroup has nothing to do (the launch is an upper bound).  The merge kernel finds a
// segment's partial results through seg_tab; the launch has at least one workgroup per segment, and workgroup s
// files the entry of segment s.
//
// Up to 64 segments every wavefront does it for itself, a segment a lane, without LDS or a barrier (by the other way a
// workgroup knew its rows 1.5 us after it had started; the kernel over 8 segments of 512 rows 5.4 -> 4.8 us, over 64 of
// 1500 13.3 -> 12.6).  Beyond, thread t of
// the workgroup takes segments t*per .. t*per+per-1 and the result goes through sh[0..21].
template <int NWV = 4, bool WIN = false>
__device__ __forceinline__ bool find_work(int nseg, int per, int split, int headroom, int grow, const int *cu,
                                          const int *seg_len, int *sh, int4 *seg_tab, Work &wk, Window win = {}, int before_us = 0) {
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, blk = (int)blockIdx.x - before_us;
  if (nseg <= 64) {
    const int s = min(lane, nseg - 1);
    const int from = cu[s], cap = cu[s + 1] - from + headroom;
    const int held = min(max(seg_len[s], 0), cap);       // (as in rows_held)
    const int now = held + (held < cap ? grow : 0);
    const int nb = lane < nseg ? (seen_rows<WIN>(now, win) + split - 1) / split : 0;
    const int upto = wave_scan_incl(nb), first = upto - nb;
    if (lane == blk && lane < nseg && wv == 0) seg_tab[s] = make_int4(first, nb, now, now - held);
    const unsigned long long here = __ballot(blk >= first && blk < upto);
    if (here == 0) return false;
    const int L = __ffsll(here) - 1;
    wk.s = L;
    wk.j = blk - __builtin_amdgcn_readlane(first, L);
    wk.parts = __builtin_amdgcn_readlane(nb, L);
    const int all = __builtin_amdgcn_readlane(now, L);
    wk.rows = seen_rows<WIN>(all, win);
    wk.hidden = all - wk.rows;
    wk.first_row = __builtin_amdgcn_readlane(from, L);
    wk.appended = __builtin_amdgcn_readlane(now - held, L) != 0;
    return true;
  }
  int mine = 0;
  for (int i = 0; i < per; ++i) {
    const int s = tid * per + i;
    if (s < nseg) mine += (seen_rows<WIN>(rows_held(cu, seg_len, s, headroom, grow), win) + split - 1) / split;
  }
  const int inc = wave_scan_incl(mine);
  if (lane == 63) sh[wv] = inc;
  __syncthreads();
  int before = 0, total = 0;
#pragma unroll
  for (int i = 0; i < NWV; ++i) {
    const int v = sh[i];
    if (i < wv) before += v;
    total += v;
  }
  int first = before + inc - mine;
  for (int i = 0; i < per; ++i) {
    const int s = tid * per + i;
    if (s >= nseg) break;
    const int now = rows_held(cu, seg_len, s, headroom, grow);
    const int appended = now - rows_held(cu, seg_len, s, headroom, 0);
    const int nb = (seen_rows<WIN>(now, win) + split - 1) / split;
    if (blk >= first && blk < first + nb) {
      sh[16] = s;
      sh[17] = blk - first;
      sh[18] = now;
      sh[19] = cu[s];
      sh[20] = appended;
      sh[21] = nb;
    }
    if (s == blk) seg_tab[s] = make_int4(first, nb, now, appended);
    first += nb;
  }
  if (blk >= total) return false;
  __syncthreads();
  wk.s = __builtin_amdgcn_readfirstlane(sh[16]);
  wk.j = __builtin_amdgcn_readfirstlane(sh[17]);
  const int all = __builtin_amdgcn_readfirstlane(sh[18]);
  wk.rows = seen_rows<WIN>(all, win);
  wk.hidden = all - wk.rows;
  wk.first_row = __builtin_amdgcn_readfirstlane(sh[19]);
  wk.appended = __builtin_amdgcn_readfirstlane(sh[20]) != 0;
  wk.parts = __builtin_amdgcn_readfirstlane(sh[21]);
  return true;
}

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16 f16x8;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float floatx4;

template <bool F16>
__device__ __forceinline__ floatx4 mfma16(u32x4 a, u32x4 b, floatx4 c) {
  if constexpr (F16)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

constexpr float LOW_MAX = 1024.0f;             // above the lower 3 bits of any finite fp16 value

// The bf16 value that x is cut to, back in 32 bits, where `on`; 0 elsewhere.
__device__ __forceinline__ float cut(float x, bool on) {
  return __builtin_bit_cast(float, __builtin_bit_cast(unsigned, x) & (on ? 0xffff0000u : 0u));
}
// x0 and x1 cut to bf16, x0 in the lower half of the word.
__device__ __forceinline__ unsigned pack(float x0, float x1) {
  return __builtin_amdgcn_perm(__builtin_bit_cast(unsigned, x1), __builtin_bit_cast(unsigned, x0), 0x07060302u);
}
// The upper (odd) or lower half of a word of two fp16 values.
__device__ __forceinline__ float half_of(unsigned w, bool odd) {
  return (float)__builtin_bit_cast(_Float16, (unsigned short)(odd ? w >> 16 : w & 0xffffu));
}
// What the cut leaves of an fp16 value in 32 bits.  Of an infinity (whose difference is a NaN) some
// finite number: the upper part alone makes the product infinite.
__device__ __forceinline__ float low_part(float x) { return fminf(x - cut(x, true), LOW_MAX); }

// Where a workgroup's result goes: partial results for the merge kernel, or (WHOLE, one workgroup per
// segment) straight to the caller.  Only a segment of no rows has zeros for a result: a sum of weights that is no
// number, or 0 because every logit is -inf, makes it NaN.
struct DecodeOut {
  float *part_acc, *part_ml;
  int4 *seg_tab;
  float *out, *lse;
  int *new_len, *overflow;                     // null unless the call appends
};

}  // namespace
}  // namespace adakv
