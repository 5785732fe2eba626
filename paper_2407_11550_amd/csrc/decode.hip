// Decode side of the flattened per-head cache (Section 3.5): the cache update of Eq. (1) and
// one decoding step of Eq. (2) per query head over segments of different lengths.
//
// Layout: segment s = b*h_kv + c starts at row cu[s] + s*headroom of K_cache / V_cache and holds
// seg_len[s] rows of ROWB = d*sizeof(T) bytes, so a segment is one contiguous byte range.
//
// Attention: HBM-bound (every cached K and V row is read once, 2*ROWB bytes for 4*g*d flops).
// 16-bit caches run both products on the matrix cores (decode_mfma_kernel); fp32 caches, and 16-bit ones
// with so few query heads per KV head that the matrix instructions stay empty, run on the vector ALUs
// (decode_attn_kernel): there a row is read by LPR = ROWB/16 neighbouring lanes, 16 bytes each: every load
// instruction of a wavefront fetches 64/LPR whole rows = 1 KB of consecutive memory.
// Segment lengths live on the device, so the host launches an upper bound of workgroups
// (capacity / split + segments); each workgroup finds its segment and its part of it from a prefix sum
// of the lengths, writes partial (max, sum, weighted value sum) per query head, and a second kernel
// merges the parts of each segment.  Where no segment of a layer can be long, one workgroup takes each
// segment (WHOLE: decode_mfma_kernel, and decode_attn_kernel for fp32 windows) and writes the result itself: no
// prefix sum, no merge.
//
// A call with a window looks at a segment's first rows (the sinks) and its last ones alone: the kernels number the
// rows it sees and leave a gap where the sinks end (WIN).  Those instantiations are built as a translation unit of
// their own (ADAKV_DECODE_PART = 2), beside the others and everything else (1).
#include <limits.h>
#include <math.h>

#include <type_traits>

#include "decode_parts.h"
#include "row_parts.h"

#ifndef ADAKV_DECODE_PART
#define ADAKV_DECODE_PART 1
#endif

namespace adakv {
namespace {

constexpr bool WIN_PART = ADAKV_DECODE_PART == 2;

// ---------------------------------------------------------------------------------------------
// Query heads one wavefront carries: at most four (queries and accumulators take 2*GW*EPL
// registers).  A larger group is split over NGRP sets of four wavefronts that read the
// same rows at the same time (the second read of a row is a cache hit).
template <typename T, int G> struct HeadSplit {
  static constexpr int GW = G > 4 ? 4 : G;
  static constexpr int NGRP = G / GW;
};

// WHOLE: one workgroup of 16 wavefronts takes a segment and writes the result itself (fp32 windows).
template <typename T, int D, int G, bool WHOLE, bool WIN>
__global__ __launch_bounds__((WHOLE ? 1024 : 256 * HeadSplit<T, G>::NGRP)) void decode_attn_kernel(
    int nseg, int h, int per, int split, int headroom, float c_log2, const T *__restrict__ q,
    const char *__restrict__ k_new, const char *__restrict__ v_new, const int *__restrict__ cu,
    const int *seg_len, char *Kc, char *Vc, DecodeOut res, Window win) {
  constexpr int EPL = Elem<T>::EPL;
  constexpr int ROWB = D * (int)sizeof(T);
  constexpr int LPR = ROWB / 16;               // lanes per row
  constexpr int RPW = 64 / LPR;                // rows per wavefront load
  constexpr int GW = HeadSplit<T, G>::GW, NGRP = HeadSplit<T, G>::NGRP;
  constexpr int NW = WHOLE ? 16 / NGRP : 4;    // wavefronts that share the rows of a split
  constexpr int NT = 64 * NW * NGRP;
  constexpr int U = 4;                         // row loads in flight per lane, for K and for V

  __shared__ int sh_scan[24];                  // [0..15] the prefix sum's wavefront totals, [16..21] results
  __shared__ float sh_acc[NW][G][D];
  __shared__ float sh_m[NW][G], sh_l[NW][G];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wv_all = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int grp = wv_all / NW, wv = wv_all % NW; // head set, and place among the set's wavefronts
  const int col = lane % LPR, slot = lane / LPR;

  // ---- which (segment, split) is this workgroup? -------------------------------------------
  // With k_new/v_new the call appends one row per segment (Eq. 1) and attends over it as well:
  // the row is taken from k_new/v_new by the lanes it falls to, which also store it in the cache.
  const int grow = k_new != nullptr ? 1 : 0;
  int s, len, hidden, cu_s, new_row, r0, r1;
  if constexpr (WHOLE) {
    s = blockIdx.x;
    cu_s = cu[s];
    const int now = rows_held(cu, seg_len, s, headroom, grow);
    len = seen_rows<WIN>(now, win);
    hidden = now - len;
    new_row = now > rows_held(cu, seg_len, s, headroom, 0) ? len - 1 : -1;
    r0 = 0;
    r1 = len;
  } else {
    Work wk;
    if (!find_work<NW * NGRP, WIN>(nseg, per, split, headroom, grow, cu, seg_len, sh_scan, res.seg_tab, wk, win)) return;
    s = wk.s;
    len = wk.rows;
    hidden = wk.hidden;
    cu_s = wk.first_row;
    new_row = wk.appended ? len - 1 : -1;
    // (equal parts of the segment, as in decode_mfma_kernel, in multiples of the split's own unit)
    const int part = ((len + wk.parts - 1) / wk.parts + 63) / 64 * 64;
    r0 = wk.j * part;
    r1 = min(len, r0 + part);
  }
  const int b = s / h, c = s % h;
  const long long seg_byte = ((long long)cu_s + (long long)s * headroom) * ROWB + col * 16;
  char *Kb = Kc + seg_byte;
  char *Vb = Vc + seg_byte;
  const long long new_byte = (long long)s * ROWB + col * 16;

  // ---- the g query rows of this KV head, pre-scaled so that exp() becomes exp2() --------------
  float qf[GW][EPL];
#pragma unroll
  for (int gi = 0; gi < GW; ++gi) {
    const T *qp = q + ((long long)(b * h + c) * G + grp * GW + gi) * D + col * EPL;
    Elem<T>::widen(*reinterpret_cast<const u32x4 *>(qp), qf[gi]);
#pragma unroll
    for (int e = 0; e < EPL; ++e) qf[gi][e] *= c_log2;
  }

  float m[GW], l[GW], acc[GW][EPL];
#pragma unroll
  for (int gi = 0; gi < GW; ++gi) {
    m[gi] = M_INIT; l[gi] = 0.0f;
#pragma unroll
    for (int e = 0; e < EPL; ++e) acc[gi][e] = 0.0f;
  }

  const int rows = r1 - r0;
  const int iters = (rows + U * NW * RPW - 1) / (U * NW * RPW);
  for (int it = 0; it < iters; ++it) {
    u32x4 kk[U], vv[U];
    bool ok[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + ((it * U + u) * NW + wv) * RPW + slot;
      ok[u] = r < r1;
      const int rr = min(r, r1 - 1);                           // r1 >= 1: the block exists
      const long long o = (long long)place_of<WIN>(rr, hidden, win) * ROWB;
      // lanes past the end re-read the block's last row (and ignore it): if that is the new row,
      // they too must take it from k_new/v_new, its place in the cache is not written yet
      const bool fresh = rr == new_row;
      kk[u] = *reinterpret_cast<const u32x4 *>(fresh ? k_new + new_byte : Kb + o);
      vv[u] = *reinterpret_cast<const u32x4 *>(fresh ? v_new + new_byte : Vb + o);
      if (r == new_row && grp == 0) {
        *reinterpret_cast<u32x4 *>(Kb + o) = kk[u];
        *reinterpret_cast<u32x4 *>(Vb + o) = vv[u];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float kf[EPL], sc[GW];
      Elem<T>::widen(kk[u], kf);
      bool grow = false;
#pragma unroll
      for (int gi = 0; gi < GW; ++gi) {
        float a = 0.0f;
#pragma unroll
        for (int e = 0; e < EPL; ++e) a = fmaf(qf[gi][e], kf[e], a);
        a = row_sum<LPR>(a);
        sc[gi] = ok[u] ? a : -INFINITY;
        grow |= sc[gi] > m[gi];
      }
      if (__any(grow)) {                       // a new running maximum somewhere in the wavefront
#pragma unroll
        for (int gi = 0; gi < GW; ++gi) {
          const float mn = fmaxf(m[gi], sc[gi]);
          const float corr = fast_exp2(m[gi] - mn);
          l[gi] *= corr;
#pragma unroll
          for (int e = 0; e < EPL; ++e) acc[gi][e] *= corr;
          m[gi] = mn;
        }
      }
      float vf[EPL];
      if (it == iters - 1 && !ok[u]) vv[u] = u32x4{0};         // (a weight of 0 times an infinite value would be a NaN)
      Elem<T>::widen(vv[u], vf);
#pragma unroll
      for (int gi = 0; gi < GW; ++gi) {
        const float p = fast_exp2(sc[gi] - m[gi]);
        l[gi] += p;
#pragma unroll
        for (int e = 0; e < EPL; ++e) acc[gi][e] = fmaf(p, vf[e], acc[gi][e]);
      }
    }
  }

  // ---- merge the RPW row slots of the wavefront, then the NW wavefronts of each head set --------
#pragma unroll
  for (int gi = 0; gi < GW; ++gi) {
    float M = m[gi];
#pragma unroll
    for (int o = LPR; o < 64; o <<= 1) M = fmaxf(M, __shfl_xor(M, o));
    const float f = fast_exp2(m[gi] - M);
    float ll = l[gi] * f;
#pragma unroll
    for (int o = LPR; o < 64; o <<= 1) ll += __shfl_xor(ll, o);
#pragma unroll
    for (int e = 0; e < EPL; ++e) {
      float a = acc[gi][e] * f;
#pragma unroll
      for (int o = LPR; o < 64; o <<= 1) a += __shfl_xor(a, o);
      acc[gi][e] = a;
    }
    if (slot == 0) {
      const int head = grp * GW + gi;
#pragma unroll
      for (int e = 0; e < EPL; ++e) sh_acc[wv][head][col * EPL + e] = acc[gi][e];
      if (col == 0) { sh_m[wv][head] = M; sh_l[wv][head] = ll; }
    }
  }
  __syncthreads();
  for (int t = tid; t < G * D; t += NT) {
    const int gi = t / D, e = t % D;
    float M = sh_m[0][gi];
#pragma unroll
    for (int w2 = 1; w2 < NW; ++w2) M = fmaxf(M, sh_m[w2][gi]);
    float a = 0.0f, ll = 0.0f;
#pragma unroll
    for (int w2 = 0; w2 < NW; ++w2) {
      const float f = fast_exp2(sh_m[w2][gi] - M);
      a = fmaf(sh_acc[w2][gi][e], f, a);
      ll = fmaf(sh_l[w2][gi], f, ll);
    }
    if constexpr (WHOLE) {
      const long long row = (long long)s * G + gi;
      res.out[row * D + e] = len > 0 ? a / ll : 0.0f;
      if (res.lse && e == 0) res.lse[row] = (M + log2f(ll)) * LN2;
    } else {
      res.part_acc[((long long)blockIdx.x * G + gi) * D + e] = a;
      if (e == 0) {
        res.part_ml[((long long)blockIdx.x * G + gi) * 2] = M;
        res.part_ml[((long long)blockIdx.x * G + gi) * 2 + 1] = ll;
      }
    }
  }
  // (nobody but this workgroup reads the segment's length, and all of it has: a barrier lies between)
  if (WHOLE && res.new_len && tid == 0) {
    if (new_row >= 0) res.new_len[s] = len + hidden;
    else if (res.overflow) *res.overflow = 1;  // the segment was full, its new row was dropped
  }
}

// ---------------------------------------------------------------------------------------------
// 16-bit caches: both products on the matrix cores (v_mfma_f32_16x16x32), one wavefront per tile of
// 32 rows, nothing staged through LDS and no data crossing lanes between the two products.
//
//   logits   D[row][head] = K Q^T: a lane loads 16-byte words of row l%16 (twice: 32 rows), and
//            ends up with head l%16 and the rows 4 (l/16) + i and 16 + 4 (l/16) + i, i < 4.  The
//            columns past the group repeat its heads.
//   values   D[head][column] += P V: what a lane holds is its part of the P operand if the rows are
//            numbered that way, so V is loaded in that numbering: a lane takes 8 rows x D/16
//            columns and turns its own 8 x (D/16) block with byte permutes.
//
// P stays in 32 bits: it is cut into three bf16 parts whose sum is P to 2^-24 (truncated to 8, 8 and 8
// bits), and the 16 rows of the P operand hold the parts side by side (the repeated heads).  For g = 8
// the third part goes through a product of its own.  Products of 16-bit values and their sums are exact
// in fp32 up to the accumulation, as they were on the vector units.  The parts are bf16 for fp16 caches
// too: fp16 parts run out of exponent 2^-39 below the maximum, so that a weight of 2^-28 kept 11 bits
// and an infinite value row behind a smaller one gave 0 * inf.  An fp16 value is exactly the sum of a
// bf16 value of its upper 8 bits and one of the lower 3, so its product takes two instructions, and P
// travels multiplied by 2^64, which leaves the parts of the smallest weight above the bf16 range's end.
//
// The vector form before this one (16 lanes per row, a dot product and two fused multiply-adds
// per element and head) issued 130 instructions per four rows at g = 4 and 240 at g = 8, which
// made it the bound from g = 8 on: a 134 MB cache at g = 8 took 77.2 us, now 29.8 (a plain
// read of as much: 25); 49 MB at g = 4 19.2, now 12.9 (kernel times, launch included).
template <bool F16> constexpr float P_SCALE = F16 ? 0x1p64f : 1.0f;    // (|V| < 2^16, 2^31 rows: below the fp32 range's end)

// (seg_len is also written, through res.new_len: after the barrier, by the one workgroup that read it)
template <bool F16, int D, int G, bool WHOLE, bool WIN>
__global__ __launch_bounds__(WHOLE ? 512 : 256) void decode_mfma_kernel(
    int nseg, int h, int per, int split, int headroom, float c_log2, const unsigned short *__restrict__ q,
    const char *__restrict__ k_new, const char *__restrict__ v_new, const int *__restrict__ cu,
    const int *seg_len, char *Kc, char *Vc, DecodeOut res, Window win) {
  constexpr int NW = WHOLE ? 8 : 4;            // wavefronts that share the rows of a split
  constexpr int ROWB = D * 2;
  constexpr int KS = D / 32;                   // k-steps of the logits
  constexpr int VC = D / 16;                   // columns of V per lane
  constexpr int TR = 32;                       // rows per tile
  constexpr int PARTS = G == 8 ? 2 : 3;        // parts of P held side by side
  constexpr bool THIRD = G == 8;               // the last part has accumulators of its own
  typedef unsigned int vword __attribute__((ext_vector_type(VC / 2)));

  __shared__ int sh_scan[24];                  // [0..15] the prefix sum's wavefront totals, [16..21] results
  __shared__ __align__(16) float sh_acc[NW][PARTS * G][D];
  __shared__ __align__(16) float sh_third[THIRD ? NW : 1][THIRD ? G : 1][THIRD ? D : 1];
  __shared__ float sh_m[NW][G], sh_l[NW][G];

  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, lg = lane >> 4;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);

  // ---- which (segment, split) is this workgroup?  (as in decode_attn_kernel) --------------------
  const int grow = k_new != nullptr ? 1 : 0;
  int s, len, cu_s, new_row, r0, r1, hidden = 0;
  if constexpr (WHOLE) {
    s = blockIdx.x;
    cu_s = cu[s];
    const int now = rows_held(cu, seg_len, s, headroom, grow);
    len = seen_rows<WIN>(now, win);
    hidden = now - len;
    new_row = now > rows_held(cu, seg_len, s, headroom, 0) ? len - 1 : -1;
    r0 = 0;
    r1 = len;
  } else {
    Work wk;
    if (!find_work<NW, WIN>(nseg, per, split, headroom, grow, cu, seg_len, sh_scan, res.seg_tab, wk, win)) return;
    s = wk.s;
    len = wk.rows;
    hidden = wk.hidden;
    cu_s = wk.first_row;
    new_row = wk.appended ? len - 1 : -1;
    // The segment's rows in equal parts, in whole rounds of the workgroup: the call lasts as long as its
    // longest workgroup, and with `split` rows for all but the last one 1024 rows were cut into 896 + 128
    // (40 sequences x 8 heads of as many rows, d = 128, g = 4: 42.9 us, now 34.7; the vector kernel's 832 + 192
    // at g = 1: 37.4, 40.4 with this one, then 33.0).  None is empty.  (Whole tiles instead of rounds: 40 uneven
    // segments of 900 rows 11.8 instead of 11.3 us, 320 of 400 rows 21.7 instead of 22.0.)
    const int rows = min(split, __builtin_amdgcn_readfirstlane(((len + wk.parts - 1) / wk.parts + NW * TR - 1) / (NW * TR) * (NW * TR)));
    r0 = wk.j * rows;
    r1 = min(len, r0 + rows);
  }
  const long long seg_byte = ((long long)cu_s + (long long)s * headroom) * ROWB;
  char *Kb = Kc + seg_byte;
  char *Vb = Vc + seg_byte;
  const char *kn = k_new + (long long)s * ROWB, *vn = v_new + (long long)s * ROWB;

  u32x4 qf[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks)
    qf[ks] = *reinterpret_cast<const u32x4 *>(q + ((long long)s * G + l16 % G) * D + (4 * ks + lg) * 8);

  float m = M_INIT, l = 0.0f;                  // of head l16 % G; m the same in all lanes of a head
  floatx4 acc[VC], acc3[THIRD ? VC : 1];
#pragma unroll
  for (int e = 0; e < VC; ++e) acc[e] = floatx4{0};
  if (THIRD) {
#pragma unroll
    for (int e = 0; e < VC; ++e) acc3[e] = floatx4{0};
  }
  const int part = l16 / G;                    // which part of P this lane's operand rows hold

  for (int t0 = r0 + wv * TR; t0 < r1; t0 += NW * TR) {
    u32x4 kk[2][KS];
    vword vv[8];
    // (a tile with the last sink and the window's first row in it is none of consecutive rows)
    const bool edge = t0 + TR > r1 || (new_row >= t0 && new_row < t0 + TR) || (WIN && t0 < win.sinks && win.sinks < t0 + TR);
    const long long t_at = place_of<WIN>(t0, hidden, win);
    const char *kt = Kb + t_at * ROWB, *vt = Vb + t_at * ROWB;
    const unsigned vcol = l16 * (VC * 2);
    if (!edge) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
          kk[t][ks] = *reinterpret_cast<const u32x4 *>(kt + (unsigned)((16 * t + l16) * ROWB + (4 * ks + lg) * 16));
#pragma unroll
      for (int j = 0; j < 8; ++j)
        vv[j] = *reinterpret_cast<const vword *>(vt + (unsigned)((16 * (j / 4) + 4 * lg + j % 4) * ROWB + vcol));
    } else {
      // rows past the end repeat the block's last one (and are masked below); the appended row comes from
      // k_new / v_new, its place in the cache is not written yet, and the lanes it falls to store it
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int r = t0 + 16 * t + l16, rr = min(r, r1 - 1);
        const long long o = (long long)place_of<WIN>(rr, hidden, win) * ROWB;
        const char *src = rr == new_row ? kn : Kb + o;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          kk[t][ks] = *reinterpret_cast<const u32x4 *>(src + (4 * ks + lg) * 16);
          if (r == new_row) *reinterpret_cast<u32x4 *>(Kb + o + (4 * ks + lg) * 16) = kk[t][ks];
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int r = t0 + 16 * (j / 4) + 4 * lg + j % 4, rr = min(r, r1 - 1);
        const long long o = (long long)place_of<WIN>(rr, hidden, win) * ROWB;
        const char *src = rr == new_row ? vn : Vb + o;
        vv[j] = *reinterpret_cast<const vword *>(src + vcol);
        if (r == new_row) *reinterpret_cast<vword *>(Vb + o + vcol) = vv[j];
      }
    }
    float sc[8];                               // row t0 + 16 (j/4) + 4 lg + j%4, not scaled yet
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      // a sum of its own per k-step, then a tree: the rounding of a logit is what the result's error
      // against 64 bits consists of (one chain of KS products: 1.3 times as much)
      floatx4 a[KS];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) a[ks] = mfma16<F16>(kk[t][ks], qf[ks], floatx4{0});
#pragma unroll
      for (int o = KS / 2; o > 0; o >>= 1)
#pragma unroll
        for (int ks = 0; ks < o; ++ks) a[ks] += a[ks + o];
#pragma unroll
      for (int i = 0; i < 4; ++i) sc[4 * t + i] = a[0][i];
    }
    if (edge) {
      // the values too: a weight of 0 times an infinite one would be a NaN (here and not between the
      // loads, where every one of them would be waited for: 64 segments of 1500 rows 15.7 -> 17.7 us)
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (t0 + 16 * (j / 4) + 4 * lg + j % 4 >= r1) { sc[j] = -INFINITY; vv[j] = vword{0}; }
    }
    float top = sc[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) top = fmaxf(top, sc[j]);
    top *= c_log2;
    if (__any(top > m)) {                      // a new running maximum somewhere in the wavefront
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float mn = fmaxf(m, top);
      const float corr = fast_exp2(m - mn);
      l *= corr;
      m = mn;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float ci = __shfl(corr, 4 * lg + i);   // accumulator row 4 lg + i: that lane's head
#pragma unroll
        for (int e = 0; e < VC; ++e) {
          acc[e][i] *= ci;
          if (THIRD) acc3[e][i] *= ci;
        }
      }
    }
    float p[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      p[j] = fast_exp2(fmaf(sc[j], c_log2, -m));
      l += p[j];
      p[j] *= P_SCALE<F16>;
    }
    u32x4 pa, pc;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float x0 = p[2 * k], x1 = p[2 * k + 1];
      x0 -= cut(x0, part >= 1);
      x1 -= cut(x1, part >= 1);
      if (!THIRD) {
        x0 -= cut(x0, part >= 2);
        x1 -= cut(x1, part >= 2);
      }
      pa[k] = pack(x0, x1);
      if (THIRD) {
        float y0 = p[2 * k], y1 = p[2 * k + 1];
        y0 -= cut(y0, true); y1 -= cut(y1, true);
        y0 -= cut(y0, true); y1 -= cut(y1, true);
        pc[k] = pack(y0, y1);
      }
    }
#pragma unroll
    for (int e = 0; e < VC; ++e) {
      u32x4 vb, vl;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const unsigned w0 = vv[2 * k][e / 2], w1 = vv[2 * k + 1][e / 2];
        if constexpr (F16) {
          const float x0 = half_of(w0, e & 1), x1 = half_of(w1, e & 1);
          vb[k] = pack(x0, x1);
          vl[k] = pack(low_part(x0), low_part(x1));
        } else {
          vb[k] = __builtin_amdgcn_perm(w1, w0, (e & 1) ? 0x07060302u : 0x05040100u);
        }
      }
      acc[e] = mfma16<false>(pa, vb, acc[e]);
      if (THIRD) acc3[e] = mfma16<false>(pc, vb, acc3[e]);
      if constexpr (F16) {
        acc[e] = mfma16<false>(pa, vl, acc[e]);
        if (THIRD) acc3[e] = mfma16<false>(pc, vl, acc3[e]);
      }
    }
  }

  // ---- the wavefronts' results meet in LDS -------------------------------------------------------
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (lane < G) { sh_m[wv][lane] = m; sh_l[wv][lane] = l; }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = 4 * lg + i;                // part * G + head
#pragma unroll
    for (int e = 0; e < VC; e += 4) {
      if (row < PARTS * G)
        *reinterpret_cast<float4 *>(&sh_acc[wv][row][l16 * VC + e]) =
            make_float4(acc[e][i], acc[e + 1][i], acc[e + 2][i], acc[e + 3][i]);
      if (THIRD && row < G)
        *reinterpret_cast<float4 *>(&sh_third[wv][row][l16 * VC + e]) =
            make_float4(acc3[e][i], acc3[e + 1][i], acc3[e + 2][i], acc3[e + 3][i]);
    }
  }
  __syncthreads();
  for (int t = tid; t < G * D; t += 64 * NW) {
    const int gi = t / D, e = t % D;
    float M = sh_m[0][gi];
#pragma unroll
    for (int w2 = 1; w2 < NW; ++w2) M = fmaxf(M, sh_m[w2][gi]);
    float a = 0.0f, ll = 0.0f;
#pragma unroll
    for (int w2 = 0; w2 < NW; ++w2) {
      const float f = fast_exp2(sh_m[w2][gi] - M);
      // an infinite value row makes the first part's sum infinite and 0 * inf = NaN of the others
      const float first = sh_acc[w2][gi][e];
      float rest = sh_acc[w2][G + gi][e];
      rest += THIRD ? sh_third[w2][gi][e] : sh_acc[w2][2 * G + gi][e];
      const float x = first + (__builtin_fabsf(first) < INFINITY ? rest : 0.0f);
      a = fmaf(x * (1.0f / P_SCALE<F16>), f, a);
      ll = fmaf(sh_l[w2][gi], f, ll);
    }
    if constexpr (WHOLE) {
      const long long row = (long long)s * G + gi;
      res.out[row * D + e] = len > 0 ? a / ll : 0.0f;
      if (res.lse && e == 0) res.lse[row] = (M + log2f(ll)) * LN2;
    } else {
      res.part_acc[((long long)blockIdx.x * G + gi) * D + e] = a;
      if (e == 0) {
        res.part_ml[((long long)blockIdx.x * G + gi) * 2] = M;
        res.part_ml[((long long)blockIdx.x * G + gi) * 2 + 1] = ll;
      }
    }
  }
  // (nobody but this workgroup reads the segment's length)
  if (WHOLE && res.new_len && tid == 0) {
    if (new_row >= 0) res.new_len[s] = len + hidden;
    else if (res.overflow) *res.overflow = 1;  // the segment was full, its new row was dropped
  }
}

#if ADAKV_DECODE_PART == 1
// One workgroup per (segment, query head of its group) merges that segment's splits and
// normalises.  A long segment has hundreds of splits, so they are merged NSLOT side by side
// (each by D/4 lanes holding a float4 of the value sum), four loads deep, then across slots.
template <int D, int G>
__global__ __launch_bounds__(1024) void decode_combine_kernel(
    const int4 *__restrict__ seg_tab, int *__restrict__ seg_len, int *__restrict__ overflow,
    const float *__restrict__ part_acc, const float *__restrict__ part_ml,
    float *__restrict__ out, float *__restrict__ lse) {
  constexpr int LPE = D / 4;
  constexpr int NSLOT = 1024 / LPE;
  constexpr int UC = 4;
  __shared__ float sh_a[NSLOT][D];
  __shared__ float sh_m[NSLOT], sh_l[NSLOT];
  const int tid = threadIdx.x;
  const int s = blockIdx.x, gi = blockIdx.y;
  const int4 ent = seg_tab[s];                 // first partial, partials, rows now, 1 if a row was appended
  const int p0 = ent.x, cnt = ent.y;
  if (seg_len && gi == 0 && tid == 0) {        // the call appended: the new lengths become visible
    if (ent.w) seg_len[s] = ent.z;
    else if (overflow) *overflow = 1;          // the segment was full, its new row was dropped
  }
  const int e4 = tid % LPE, slot = tid / LPE;

  float m = M_INIT, l = 0.0f;
  float4 a = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  for (int p = slot; p < cnt; p += NSLOT * UC) {
    float2 ml[UC];
    float4 pa[UC];
#pragma unroll
    for (int u = 0; u < UC; ++u) {
      const int pp = p + u * NSLOT;
      const long long pg = (long long)(p0 + (pp < cnt ? pp : p)) * G + gi;
      ml[u] = *reinterpret_cast<const float2 *>(part_ml + pg * 2);
      pa[u] = *reinterpret_cast<const float4 *>(part_acc + pg * D + e4 * 4);
      if (pp >= cnt) { ml[u] = make_float2(M_INIT, 0.0f); pa[u] = make_float4(0.0f, 0.0f, 0.0f, 0.0f); }
    }
#pragma unroll
    for (int u = 0; u < UC; ++u) {
      const float mn = fmaxf(m, ml[u].x);
      const float fo = fast_exp2(m - mn), fn = fast_exp2(ml[u].x - mn);
      l = l * fo + ml[u].y * fn;
      a.x = a.x * fo + pa[u].x * fn; a.y = a.y * fo + pa[u].y * fn;
      a.z = a.z * fo + pa[u].z * fn; a.w = a.w * fo + pa[u].w * fn;
      m = mn;
    }
  }
  // (only the slots that had partials: with all of them the end of the kernel took 0.7 us of 32 slots and 1.3 of 64; a step over 8 segments of
  // 512 rows, with the above, 9.1 -> 8.0 us, over 64 of 1500 16.5 -> 16.0)
  // (From half of them on all: the loops below are then of a fixed length, with every load ahead.  One segment's 64
  // slots, d = 64, 8 x 4160 rows: 10.4 us a step with a loop of variable length, 9.65 with this.)
  const int live = cnt > NSLOT / 2 ? NSLOT : cnt;
  if (slot < live) {
    *reinterpret_cast<float4 *>(&sh_a[slot][e4 * 4]) = a;
    if (e4 == 0) { sh_m[slot] = m; sh_l[slot] = l; }
  }
  __syncthreads();
  if (tid < D) {
    float M = M_INIT, acc = 0.0f, ll = 0.0f;
    auto add = [&](int k) {
      const float f = fast_exp2(sh_m[k] - M);
      acc = fmaf(sh_a[k][tid], f, acc);
      ll = fmaf(sh_l[k], f, ll);
    };
    if (live == NSLOT) {
#pragma unroll
      for (int k = 0; k < NSLOT; ++k) M = fmaxf(M, sh_m[k]);
#pragma unroll 8
      for (int k = 0; k < NSLOT; ++k) add(k);
    } else {
#pragma unroll 4
      for (int k = 0; k < live; ++k) M = fmaxf(M, sh_m[k]);
#pragma unroll 4
      for (int k = 0; k < live; ++k) add(k);
    }
    const long long row = (long long)s * G + gi;       // = (b*h + c)*G + gi
    out[row * D + tid] = cnt > 0 ? acc / ll : 0.0f;
    if (lse && tid == 0) lse[row] = (M + log2f(ll)) * LN2;
  }
}

// Eq. (1) for every segment: LPR lanes move the new K row and the new V row of one segment.
template <int LPR>
__global__ __launch_bounds__(256) void append_kernel(
    int nseg, int headroom, const char *__restrict__ k_new, const char *__restrict__ v_new,
    const int *__restrict__ cu, char *__restrict__ Kc, char *__restrict__ Vc,
    int *__restrict__ seg_len, int *__restrict__ overflow) {
  const int s = (blockIdx.x * 256 + threadIdx.x) / LPR;
  const int col = threadIdx.x % LPR;
  if (s >= nseg) return;
  const int cap = cu[s + 1] - cu[s] + headroom;
  const int len = seg_len[s];                  // read by all LPR lanes before lane 0 stores
  if (len < 0 || len >= cap) {
    if (col == 0 && overflow) *overflow = 1;
    return;
  }
  const uint4 kv = *reinterpret_cast<const uint4 *>(k_new + ((long long)s * LPR + col) * 16);
  const uint4 vv = *reinterpret_cast<const uint4 *>(v_new + ((long long)s * LPR + col) * 16);
  const long long o = (((long long)cu[s] + (long long)s * headroom + len) * LPR + col) * 16;
  *reinterpret_cast<uint4 *>(Kc + o) = kv;
  *reinterpret_cast<uint4 *>(Vc + o) = vv;
  if (col == 0) seg_len[s] = len + 1;
}
#endif

template <typename T, int D, int G>
void run_decode(const SeqTab &st, const Dims &dm, int headroom, const DecodePlan &pl,
                const void *q, const void *k_new, const void *v_new, const int *cu, void *Kc,
                void *Vc, int *seg_len, int *overflow, float *out, float *lse, char *ws,
                Window win, hipStream_t s) {
  const int nseg = st.batch * dm.h_kv;
  const int per = (nseg + 255) / 256;
  float *part_acc = (float *)(ws + pl.part_acc);
  float *part_ml = (float *)(ws + pl.part_ml);
  int4 *seg_tab = (int4 *)(ws + pl.seg_tab);
  constexpr bool F16 = std::is_same<T, f16_t>::value;
  // The matrix kernel multiplies 16 operand rows whatever the group, so with one head per KV head, and for
  // fp16 (two products per value) with two of 128 columns, the vector kernel is the faster one.  us per
  // step, vector | matrix, d = 128: 64 uneven segments of 4096 rows on average, 64 of 1500, 320 of 1024:
  //   bf16, g = 1   26.8 | 27.2   14.0 | 15.2   31.6 | 33.1      g = 2   30.6 | 29.9   15.0 | 15.0   33.6 | 33.2
  //   fp16, g = 1   26.4 | 29.2   13.7 | 14.9   31.2 | 35.5      g = 2   28.7 | 29.6   15.2 | 15.0   33.5 | 35.9
  // fp16, g = 2, d = 64: 20.1 | 19.5   11.7 | 11.3   22.5 | 22.2.
  // bf16, g = 1, d = 64 (kernels alone): 64 segments of 1500 rows 11.6 | 12.1, 256 of 6000 81.4 | 87.9, but 256
  // of 1500 26.0 | 23.8, the one shape measured that the matrix kernel does faster.
  constexpr bool VECTOR = sizeof(T) == 4 || G == 1 || (F16 && G == 2 && D == 128);
  const DecodeOut res = {part_acc, part_ml, seg_tab, out, lse, k_new ? seg_len : nullptr, overflow};
  if constexpr (sizeof(T) == 2) {
    if (pl.whole) {
      ADAKV_LAUNCH("decode_attn", (decode_mfma_kernel<F16, D, G, true, WIN_PART>), dim3(nseg), dim3(512), s, nseg, dm.h_kv,
                   per, pl.split, headroom, dm.scale * LOG2E, (const unsigned short *)q, (const char *)k_new,
                   (const char *)v_new, cu, (const int *)seg_len, (char *)Kc, (char *)Vc, res, win);
      return;
    }
    if constexpr (!VECTOR)
      ADAKV_LAUNCH("decode_attn", (decode_mfma_kernel<F16, D, G, false, WIN_PART>), dim3(pl.nblk), dim3(256), s, nseg,
                   dm.h_kv, per, pl.split, headroom, dm.scale * LOG2E, (const unsigned short *)q, (const char *)k_new,
                   (const char *)v_new, cu, (const int *)seg_len, (char *)Kc, (char *)Vc, res, win);
  } else if constexpr (WIN_PART) {
    if (pl.whole) {
      ADAKV_LAUNCH("decode_attn", (decode_attn_kernel<T, D, G, true, true>), dim3(nseg), dim3(1024), s, nseg, dm.h_kv, per,
                   pl.split, headroom, dm.scale * LOG2E, (const T *)q, (const char *)k_new, (const char *)v_new, cu,
                   (const int *)seg_len, (char *)Kc, (char *)Vc, res, win);
      return;
    }
  }
  if constexpr (VECTOR)
    ADAKV_LAUNCH("decode_attn", (decode_attn_kernel<T, D, G, false, WIN_PART>), dim3(pl.nblk), dim3(256 * HeadSplit<T, G>::NGRP), s,
                 nseg, dm.h_kv, per, pl.split, headroom, dm.scale * LOG2E, (const T *)q, (const char *)k_new,
                 (const char *)v_new, cu, (const int *)seg_len, (char *)Kc, (char *)Vc, res, win);
  // only a call that appends hands the lengths to the merge kernel for updating
  launch_decode_combine(nseg, D, G, pl, ws, k_new ? seg_len : nullptr, overflow, out, lse, s);
}

struct DecodeArgs {
  const void *q, *k_new, *v_new;
  const int *cu;
  void *Kc, *Vc;
  int *seg_len, *overflow;
  float *out, *lse;
  char *ws;
  Window win;
};

template <typename T, int D>
bool run_decode_g(const SeqTab &st, const Dims &dm, int headroom, const DecodePlan &pl,
                  const DecodeArgs &a, hipStream_t s) {
#define ADAKV_DECODE_G(G)                                                                       \
  run_decode<T, D, G>(st, dm, headroom, pl, a.q, a.k_new, a.v_new, a.cu, a.Kc, a.Vc, a.seg_len,   \
                      a.overflow, a.out, a.lse, a.ws, a.win, s)
  switch (dm.g) {
    case 1: ADAKV_DECODE_G(1); return true;
    case 2: ADAKV_DECODE_G(2); return true;
    case 4: ADAKV_DECODE_G(4); return true;
    case 8: ADAKV_DECODE_G(8); return true;
    default: return false;
  }
#undef ADAKV_DECODE_G
}

bool run_decode_t(const SeqTab &st, const Dims &dm, int dtype, int headroom, const DecodePlan &pl, const DecodeArgs &a,
                  hipStream_t s) {
  if (dtype == ADAKV_BF16)
    return dm.d == 64 ? run_decode_g<unsigned short, 64>(st, dm, headroom, pl, a, s)
                      : run_decode_g<unsigned short, 128>(st, dm, headroom, pl, a, s);
  if (dtype == ADAKV_FP16)
    return dm.d == 64 ? run_decode_g<f16_t, 64>(st, dm, headroom, pl, a, s)
                      : run_decode_g<f16_t, 128>(st, dm, headroom, pl, a, s);
  return dm.d == 64 ? run_decode_g<float, 64>(st, dm, headroom, pl, a, s)
                    : run_decode_g<float, 128>(st, dm, headroom, pl, a, s);
}

}  // namespace

#if ADAKV_DECODE_PART == 2

hipError_t launch_decode_window(const SeqTab &st, const Dims &dm, int dtype, int headroom, int limit, int sinks,
                                const void *q, const void *k_new, const void *v_new, const int *cu, void *Kc, void *Vc,
                                int *seg_len, int *overflow, float *out, float *lse, char *ws, hipStream_t s) {
  const DecodePlan pl = plan_decode(st, dm, dtype, headroom, limit);
  const DecodeArgs a = {q, k_new, v_new, cu, Kc, Vc, seg_len, overflow, out, lse, ws, {limit, sinks}};
  return run_decode_t(st, dm, dtype, headroom, pl, a, s) ? hipGetLastError() : hipErrorInvalidValue;
}

#else

void launch_decode_combine(int nseg, int d, int g, const DecodePlan &pl, char *ws, int *new_len, int *overflow,
                           float *out, float *lse, hipStream_t s) {
  const float *part_acc = (const float *)(ws + pl.part_acc), *part_ml = (const float *)(ws + pl.part_ml);
  const int4 *seg_tab = (const int4 *)(ws + pl.seg_tab);
#define ADAKV_COMBINE(D, G)                                                                       \
  if (d == D && g == G)                                                                           \
    ADAKV_LAUNCH("decode_combine", (decode_combine_kernel<D, G>), dim3(nseg, G), dim3(1024), s,   \
                 seg_tab, new_len, overflow, part_acc, part_ml, out, lse)
#define ADAKV_COMBINE_D(D) ADAKV_COMBINE(D, 1); ADAKV_COMBINE(D, 2); ADAKV_COMBINE(D, 4); ADAKV_COMBINE(D, 8)
  ADAKV_COMBINE_D(64);
  ADAKV_COMBINE_D(128);
#undef ADAKV_COMBINE_D
#undef ADAKV_COMBINE
}

bool decode_supported(const Dims &dm) {
  return (dm.g == 1 || dm.g == 2 || dm.g == 4 || dm.g == 8) && (dm.d == 64 || dm.d == 128);
}

DecodePlan plan_decode(const SeqTab &st, const Dims &dm, int dtype, int headroom, int limit) {
  DecodePlan pl;
  const long long nseg = (long long)st.batch * dm.h_kv;
  long long cap = (long long)st.out_off[st.batch] + nseg * headroom;
  if (cap > nseg * limit) cap = nseg * limit;               // (what a call with a window looks at)
  // Rows per workgroup: what fills one resident round, so that all workgroups start together and
  // none is left for a thin second round.  Three workgroups fit on a compute unit (768 on the
  // chip), two of the 16-bit kernel for g = 8 at d = 128, whose third part of P takes 32 more
  // registers (134 MB cache: 35.2 us with 500 workgroups, 41.0 with 752, 39.7 with 1500; at g = 4,
  // 49 MB: 17.6, 16.2, 18.2).  The split is a multiple of one round of the workgroup's loads: 128
  // rows in the 16-bit kernels, four wavefronts of 32 (16.2 us against 17.2 with multiples of 64), but of
  // half a round beyond two (segments of 4096 rows on average, uneven, 448 against 512: d = 128, g = 4
  // 28.3 | 30.2, d = 64 18.9 | 20.0; all of them 4096: 27.7 | 27.7, 18.6 | 17.4); 64 rows in the fp32
  // kernel and for caches so small that there are workgroups to spare.
  const bool mfma = dtype != ADAKV_FP32;
  const long long round_wgs = mfma && dm.g == 8 && dm.d == 128 ? 500 : 752;
  const long long room = round_wgs - nseg;                   // the segments' last, partial splits
  long long want = room > 64 ? (cap + room - 1) / room : cap / 512;
  if (want < 64) want = 64;
  const int unit = mfma && want > 64 && want <= 256 ? 128 : 64;
  const int split = (int)((want + unit - 1) / unit * unit);
  // One workgroup of eight wavefronts per segment, and no merge kernel, where no segment can be long: a
  // compute unit walks it alone, and what that takes follows its bytes.  us per step, split / whole, by rows of the
  // longest segment (the others a sixth to a half of it), 8 segments, bf16, d = 128, g = 4: 256 8.2 / 7.0, 384 8.3 / 8.1,
  // 512 8.4 / 9.2, 768 8.6 / 11.2, 1024 9.0 / 13.2; 64 segments 8.6 / 7.2, 8.9 / 9.3, 9.1 / 10.3, 10.1 / 12.5, 11.1 / 14.8;
  // g = 8, 8 segments 9.0 / 7.9, 9.1 / 9.0, 9.3 / 10.0, 9.4 / 12.2, 9.7 / 14.3; d = 64, fp16, g = 4: 512 7.6 / 6.9, 768 7.8 /
  // 8.3, 1024 7.9 / 9.6.  Heads are budgeted unevenly (the longest of a layer holds three to four times the
  // average), so the line is on four times the average, head-room full: 768 rows of 256 bytes; the most that the
  // layer allows, one head with all of its sequence's prefix budget, 1024; and 384 rows of capacity on average.  (768
  // is where both took the same while the split form's workgroups found their rows 1.5 us later.  They meet near 400
  // rows now: a layer at the line, with half to all of its 768 rows in use, takes up to 2.6 us more than in parts.)
  long long &likely = pl.likely = 0, &longest = pl.longest = 0;
  for (int b = 0; b < st.batch; ++b) {
    const long long most = st.Bp[b] < st.n[b] ? st.Bp[b] : st.n[b];
    const long long four = 4ll * ((st.Bp[b] + dm.h_kv - 1) / dm.h_kv);
    longest = most > longest ? most : longest;
    likely = (four < most ? four : most) > likely ? (four < most ? four : most) : likely;
  }
  const long long fixed = dm.w + headroom;
  likely = likely + fixed < limit ? likely + fixed : limit;
  longest = longest + fixed < limit ? longest + fixed : limit;
  pl.whole = mfma && cap <= nseg * 384 && likely * dm.d <= 768 * 128 && longest * dm.d <= 1024 * 128;
  pl.split = split;
  pl.nblk = (int)(cap / split + nseg);          // >= sum over segments of ceil(len / split)
  pl.part_acc = 0;
  pl.part_ml = align_up((size_t)pl.nblk * dm.g * dm.d * sizeof(float), 256);
  pl.seg_tab = pl.part_ml + align_up((size_t)pl.nblk * dm.g * 2 * sizeof(float), 256);
  pl.total = pl.seg_tab + align_up((size_t)nseg * sizeof(int4), 256);
  if (limit < INT_MAX) {
    // With a window segments are about as long as each other, so that one workgroup per segment pays further: with as
    // many segments as half the compute units or all of them (if they hold the window on average), longer ones too.
    // us per call, parts | whole, by rows that it looks at, 16-bit, d = 128, g = 4:
    //   8 segments     64 10.6 | 8.1   256 10.6 | 8.1   512 10.5 | 8.6   768 10.3 | 11.2   1024 10.4 | 13.1
    //   128 segments   64 10.1 | 8.0   256 10.3 | 7.8   512 11.5 | 9.1   768 15.3 | 12.8   1024 17.4 | 15.1   2048 26.2 | 25.0
    //   256 segments   64 10.3 | 8.0   256 12.4 | 8.2   512 19.2 | 13.9  768 23.5 | 18.2   1024 28.0 | 22.6   2048 46.2 | 40.6
    // (d = 64, 8 segments: 1024 10.4 | 9.6).  The fp32 kernel is bound by its vector instructions, which follow the rows, d and g
    // (d = 128, g = 4: 8 segments 128 12.1 | 8.8, 256 11.7 | 11.3, 512 11.9 | 18.5, 256 segments 15.1 | 8.8, 19.7 |
    // 15.2, 28.7 | 24.7, 1024 47.1 | 44.1; g = 8: 8 segments 128 11.5 | 11.4, 256 segments 20.8 | 12.1, 1024 82.5 | 77.6).
    const long long even = st.out_off[st.batch] >= nseg * limit ? nseg : 0, seen = longest * dm.d;
    if (longest < limit) {                                  // (it hides nothing: as without a window)
    } else if (mfma) {
      pl.whole |= seen <= 128 * (even >= 256 ? 2048 : even >= 128 ? 1024 : 640);
    } else {
      pl.whole = even >= 256 ? seen <= 128 * 1024 : seen * dm.g <= 128 * 4 * 256 && seen <= 128 * 512;
    }
    // a workspace is as large as the call without a window needs it: fewer rows in shorter parts can be more parts
    const DecodePlan full = plan_decode(st, dm, dtype, headroom, INT_MAX);
    if (pl.nblk > full.nblk) {
      const DecodePlan window = pl;
      pl = full;                                            // (never fewer parts than the window's rows make)
      pl.whole = window.whole, pl.likely = window.likely, pl.longest = window.longest;
    }
  }
  return pl;
}

hipError_t launch_decode_attn(const SeqTab &st, const Dims &dm, int dtype, int headroom,
                              const void *q, const void *k_new, const void *v_new, const int *cu,
                              void *Kc, void *Vc, int *seg_len, int *overflow, float *out,
                              float *lse, char *ws, hipStream_t s) {
  const DecodePlan pl = plan_decode(st, dm, dtype, headroom);
  const DecodeArgs a = {q, k_new, v_new, cu, Kc, Vc, seg_len, overflow, out, lse, ws, {}};
  return run_decode_t(st, dm, dtype, headroom, pl, a, s) ? hipGetLastError() : hipErrorInvalidValue;
}

hipError_t launch_append(const SeqTab &st, const Dims &dm, int dtype, int headroom,
                         const void *k_new, const void *v_new, const int *cu, void *Kc, void *Vc,
                         int *seg_len, int *overflow, hipStream_t s) {
  const int lpr = dm.d * (dtype == ADAKV_FP32 ? 4 : 2) / 16;
  const int nseg = st.batch * dm.h_kv;
  dim3 grid((nseg * lpr + 255) / 256), block(256);
#define ADAKV_LAUNCH_APPEND(LPR)                                                               \
  ADAKV_LAUNCH("append", append_kernel<LPR>, grid, block, s, nseg, headroom,                   \
               (const char *)k_new, (const char *)v_new, cu, (char *)Kc, (char *)Vc, seg_len,  \
               overflow)
  switch (lpr) {
    case 8: ADAKV_LAUNCH_APPEND(8); break;
    case 16: ADAKV_LAUNCH_APPEND(16); break;
    case 32: ADAKV_LAUNCH_APPEND(32); break;
    default: return hipErrorInvalidValue;
  }
#undef ADAKV_LAUNCH_APPEND
  return hipGetLastError();
}

#endif  // ADAKV_DECODE_PART

}  // namespace adakv
