// The flattened per-head cache in 8 bits (q8_parts.h says what a value is): the gather that quantises, the cache update of
// Eq. (1) and one decoding step of Eq. (2).  Layout and division of work as in decode.hip, with rows of d bytes and a
// scale per 32 rows of a segment, counted from the segment's first row, so that a tile of the attention kernel has one
// scale for its keys and one for its values.
//
// Attention is HBM-bound: 2 d bytes a row and 8 bytes a block for 4 g d flops a row, half of what a 16-bit cache reads.
// Codes are turned into 16-bit operands in registers (exact: 4 significant bits), two per instruction; fp16 queries
// meet fp16 keys, all others bf16.  fp32 queries are three bf16 parts, the products of which are added in 32 bits.
// 64 segments of 8192 rows on average, 64 query heads, d = 128, bf16: 27 us (4.8 TB/s) and 4.4 for the merge kernel (half as many rows in
// 16 bits: 30 and 4.2).
#include <float.h>
#include <math.h>

#include <type_traits>

#include "decode_parts.h"
#include "q8_parts.h"

namespace adakv {
namespace {

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
typedef __attribute__((__vector_size__(2 * sizeof(_Float16)))) _Float16 f16x2;

struct BF16 { static constexpr int EPL = 8; };
struct FP16 { static constexpr int EPL = 8; };
struct FP32 { static constexpr int EPL = 4; };
template <typename T> struct Same { static constexpr bool f16 = false, f32 = false; };
template <> struct Same<FP16> { static constexpr bool f16 = true, f32 = false; };
template <> struct Same<FP32> { static constexpr bool f16 = false, f32 = true; };

// The values of 16 bytes of a row.
template <typename T> __device__ __forceinline__ void widen16(u32x4 v, float (&f)[T::EPL]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const unsigned w = v[i];
    if constexpr (Same<T>::f32) {
      f[i] = __builtin_bit_cast(float, w);
    } else if constexpr (Same<T>::f16) {
      f[2 * i] = (float)__builtin_bit_cast(_Float16, (unsigned short)(w & 0xffffu));
      f[2 * i + 1] = (float)__builtin_bit_cast(_Float16, (unsigned short)(w >> 16));
    } else {
      f[2 * i] = __builtin_bit_cast(float, w << 16);
      f[2 * i + 1] = __builtin_bit_cast(float, w & 0xffff0000u);
    }
  }
}

// ---- the gather ---------------------------------------------------------------------------------------------------
// A wavefront takes a block's K rows or its V rows, all of them in registers (2 to 16 KB), so the rows are read once: the largest
// magnitude first, then the codes.  HBM-bound: 2 d (sizeof(T) + 1) bytes a row.
template <typename T, int D>
__global__ __launch_bounds__(256) void cache_build_q8_kernel(
    SeqTab st, int h, int nseg, int nblk, long long k_tok, long long k_head, long long v_tok, long long v_head,
    const char *__restrict__ K, const char *__restrict__ V, const int *__restrict__ indices, const int *__restrict__ cu,
    char *__restrict__ Kq, char *__restrict__ Vq, float *__restrict__ k_scale, float *__restrict__ v_scale, int rows_total, int w,
    int headroom, int *__restrict__ seg_len) {
  constexpr int EPL = T::EPL, LPR = D / EPL, RPI = 64 / LPR, NL = Q8_BLOCK / RPI;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i = blockIdx.x * 2 + wv / 2;
  const bool values = wv % 2;
  if (i >= nblk) return;
  // segment s whose blocks are counted from cu[s] / 32 + s: the numbers grow by one at least from segment to segment
  int lo = 0, hi = nseg;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cu[mid] / Q8_BLOCK + mid <= i) lo = mid; else hi = mid;
  }
  const int s = lo, from = min(max(cu[s], 0), rows_total), len = min(cu[s + 1], rows_total) - from;
  const int blk = i - (from / Q8_BLOCK + s), t0 = blk * Q8_BLOCK;
  if (blk == 0 && !values && lane == 0 && seg_len) seg_len[s] = max(len, 0);
  if (t0 < 0 || t0 >= len) return;             // (below 0: offsets that do not begin with 0)
  const int b = s / h, c = s % h, col = lane % LPR, slot = lane / LPR;
  const char *src = (values ? V + c * v_head : K + c * k_head) + col * 16;
  const long long stride = values ? v_tok : k_tok;
  int at[NL];
#pragma unroll
  for (int u = 0; u < NL; ++u) at[u] = indices[from + min(t0 + u * RPI + slot, len - 1)];
  u32x4 x[NL];
#pragma unroll
  for (int u = 0; u < NL; ++u) {
    // (clamped into the sequence's own rows, as in compact_kernel)
    const long long row = st.tok_off[b] + min(max(at[u], 0), st.n[b] + w - 1);
    x[u] = *reinterpret_cast<const u32x4 *>(src + row * stride);
  }
  float m = 0.0f;                              // (the rows past the end repeat the last one)
#pragma unroll
  for (int u = 0; u < NL; ++u) {
    float f[EPL];
    widen16<T>(x[u], f);
#pragma unroll
    for (int e = 0; e < EPL; ++e) m = fmaxf(m, magnitude(f[e]));
  }
  const int k = exponent_for(wave_max(m));
  const float inv = pow2(-k);
  const long long row0 = (long long)from + (long long)s * headroom;
  char *dst = (values ? Vq : Kq) + (row0 + t0) * D + col * EPL;
#pragma unroll
  for (int u = 0; u < NL; ++u) {
    const int r = u * RPI + slot;
    float f[EPL];
    widen16<T>(x[u], f);
#pragma unroll
    for (int e = 0; e < EPL; ++e) f[e] = to_range(f[e], inv);
    if (t0 + r < len) {
      // (past the caches: 96 000 rows of 128 bf16 values 16.8 us, 16.2 with this, 14.1 at the rate of a copy)
      const unsigned w0 = to_codes(f[0], f[1], f[2], f[3]);
      if constexpr (EPL == 8)
        __builtin_nontemporal_store(u32x2{w0, to_codes(f[4], f[5], f[6], f[7])}, reinterpret_cast<u32x2 *>(dst + r * D));
      else
        __builtin_nontemporal_store(w0, reinterpret_cast<unsigned *>(dst + r * D));
    }
  }
  if (lane == 0) (values ? v_scale : k_scale)[first_scale(row0, s) + blk] = pow2(k);
}

// ---- the cache update -----------------------------------------------------------------------------------------------
// One row of d values at row t of a segment, by one wavefront.  `block`: the first row of its block, `scale`: the block's.
// A block that the row does not begin keeps its exponent if that will do, else its earlier rows get the new one.
// Returns the block's scale.
template <typename T, int D>
__device__ __forceinline__ float append_row(int lane, const char *src, char *block, int t, float *scale) {
  constexpr int E = D / 64;                    // values per lane
  float x[E];
  if constexpr (Same<T>::f32) {
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = reinterpret_cast<const float *>(src)[lane * E + e];
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const unsigned short u = reinterpret_cast<const unsigned short *>(src)[lane * E + e];
      if constexpr (Same<T>::f16) x[e] = (float)__builtin_bit_cast(_Float16, u);
      else x[e] = __builtin_bit_cast(float, (unsigned)u << 16);
    }
  }
  float m = magnitude(x[0]);
  if constexpr (E == 2) m = fmaxf(m, magnitude(x[1]));
  int k = exponent_for(wave_max(m));
  if (t > 0) {
    const int was = exponent_of(*scale);
    if (k > was) {
      const float by = pow2(max(was - k, -100));       // (of 448 * 2^-100 nothing is left)
      for (int i = lane; i < t * (D / 4); i += 64) {
        const unsigned w = reinterpret_cast<const unsigned *>(block)[i];
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
        reinterpret_cast<unsigned *>(block)[i] = to_codes(lo[0] * by, lo[1] * by, hi[0] * by, hi[1] * by);
      }
    } else {
      k = was;
    }
  }
  const float inv = pow2(-k);
  if constexpr (E == 2) {
    const unsigned w = to_codes(to_range(x[0], inv), to_range(x[1], inv), 0.0f, 0.0f);
    reinterpret_cast<unsigned short *>(block + t * D)[lane] = (unsigned short)w;
  } else {
    block[t * D + lane] = (char)to_codes(to_range(x[0], inv), 0.0f, 0.0f, 0.0f);
  }
  if (lane == 0) *scale = pow2(k);
  return pow2(k);
}

// A wavefront per segment and tensor.
template <typename T, int D>
__global__ __launch_bounds__(128) void append_q8_kernel(
    int headroom, const char *__restrict__ k_new, const char *__restrict__ v_new, const int *__restrict__ cu, char *Kq, char *Vq,
    float *k_scale, float *v_scale, int *seg_len, int *__restrict__ overflow) {
  const int s = blockIdx.x, lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int cap = cu[s + 1] - cu[s] + headroom, len = seg_len[s];
  __syncthreads();                             // both have read the length before it changes
  if (len < 0 || len >= cap) {
    if (threadIdx.x == 0 && overflow) *overflow = 1;
    return;
  }
  const long long row0 = (long long)cu[s] + (long long)s * headroom;
  const int t0 = len / Q8_BLOCK * Q8_BLOCK;
  append_row<T, D>(lane, (wv ? v_new : k_new) + (long long)s * D * (16 / T::EPL), (wv ? Vq : Kq) + (row0 + t0) * D, len - t0,
                   (wv ? v_scale : k_scale) + first_scale(row0, s) + t0 / Q8_BLOCK);
  if (threadIdx.x == 0) seg_len[s] = len + 1;
}

// ---- one decoding step ----------------------------------------------------------------------------------------------
template <bool F16> __device__ __forceinline__ unsigned two(unsigned w, bool upper, float scale) {
  // (the selector is a constant of the instruction)
  if constexpr (F16) {
    const f16x2 r = upper ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, false);
    return __builtin_bit_cast(unsigned, r);
  } else {
    const bf16x2 r = upper ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false);
    return __builtin_bit_cast(unsigned, r);
  }
}

// Wavefronts of a workgroup that takes a whole segment: as many as its registers (100 to 120 at d = 64, 140 to 160 at
// d = 128, 213 with eight fp32 queries) and LDS (a wavefront's results, 6 or 12 KB with eight queries) allow.
template <int D, int G> constexpr int WHOLE_WAVES = D == 64 ? 16 : G == 8 ? 8 : 12;

// As decode_mfma_kernel, tile by tile of 32 rows, one block each:
//   logits   a lane loads 16 codes of a row at a time, which are two operands of 8; the queries' operands are loaded
//            in that order of the columns.
//   values   a lane takes 8 rows x D/16 columns, turns them 4 x 4 with byte permutes so that two rows of a column stand
//            side by side, and converts them with the block's scale on the way.
// The row that the call appends is stored by the wavefront whose tile it belongs to, before it loads that tile.
template <typename T, int D, int G, bool WHOLE>
__global__ __launch_bounds__((WHOLE ? 64 * WHOLE_WAVES<D, G> : 256)) void decode_q8_kernel(
    int nseg, int h, int per, int split, int headroom, float c_log2, const char *__restrict__ q, const char *__restrict__ k_new,
    const char *__restrict__ v_new, const int *__restrict__ cu, const int *seg_len, char *Kc, char *Vc, float *k_scale,
    float *v_scale, DecodeOut res) {
  constexpr bool F16 = Same<T>::f16, F32 = Same<T>::f32;
  constexpr int NW = WHOLE ? WHOLE_WAVES<D, G> : 4;
  constexpr int KC = D / 64;                   // 16-byte words of a K row per lane
  constexpr int KS = D / 32;                   // k-steps of the logits
  constexpr int QP = F32 ? 3 : 1;              // parts of a query
  constexpr int VC = D / 16, VW = VC / 4;      // columns of V per lane, in words
  constexpr int TR = Q8_BLOCK;
  constexpr int PARTS = G == 8 ? 2 : 3;
  constexpr bool THIRD = G == 8;
  constexpr int ESZ = 16 / T::EPL;
  typedef unsigned int vword __attribute__((ext_vector_type(VW)));

  __shared__ int sh_scan[24];
  __shared__ __align__(16) float sh_acc[NW][PARTS * G][D];
  __shared__ __align__(16) float sh_third[THIRD ? NW : 1][THIRD ? G : 1][THIRD ? D : 1];
  __shared__ float sh_m[NW][G], sh_l[NW][G];

  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, lg = lane >> 4;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int grow = k_new != nullptr ? 1 : 0;
  int s, len, cu_s, new_row, r0, r1;
  if constexpr (WHOLE) {
    s = blockIdx.x;
    cu_s = cu[s];
    len = rows_held(cu, seg_len, s, headroom, grow);
    new_row = len > rows_held(cu, seg_len, s, headroom, 0) ? len - 1 : -1;
    r0 = 0;
    r1 = len;
  } else {
    Work wk;
    if (!find_work<NW>(nseg, per, split, headroom, grow, cu, seg_len, sh_scan, res.seg_tab, wk)) return;
    s = wk.s;
    len = wk.rows;
    cu_s = wk.first_row;
    new_row = wk.appended ? len - 1 : -1;
    // equal parts, in whole rounds of the workgroup (none is empty, as in decode_mfma_kernel)
    const int rows = min(split, __builtin_amdgcn_readfirstlane(((len + wk.parts - 1) / wk.parts + NW * TR - 1) / (NW * TR) * (NW * TR)));
    r0 = wk.j * rows;
    r1 = min(len, r0 + rows);
  }
  const long long row0 = (long long)cu_s + (long long)s * headroom;
  char *Kb = Kc + row0 * D, *Vb = Vc + row0 * D;
  float *ksc = k_scale + first_scale(row0, s), *vsc = v_scale + first_scale(row0, s);

  // 8 query values of columns (lg + 4 (ks / 2)) * 16 + (ks % 2) * 8 on: those of a lane's ks-th half of a word of codes
  u32x4 qf[QP][KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    const char *src = q + (((long long)s * G + l16 % G) * D + (lg + 4 * (ks / 2)) * 16 + (ks % 2) * 8) * ESZ;
    if constexpr (!F32) {
      qf[0][ks] = *reinterpret_cast<const u32x4 *>(src);
    } else {
      const float4 a = *reinterpret_cast<const float4 *>(src), b = *reinterpret_cast<const float4 *>(src + 16);
      float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
      for (int p = 0; p < QP; ++p)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          qf[p][ks][i] = pack(x[2 * i], x[2 * i + 1]);
          x[2 * i] -= cut(x[2 * i], true);
          x[2 * i + 1] -= cut(x[2 * i + 1], true);
        }
    }
  }

  float m = M_INIT, l = 0.0f;
  floatx4 acc[VC], acc3[THIRD ? VC : 1];
#pragma unroll
  for (int e = 0; e < VC; ++e) acc[e] = floatx4{0};
  if (THIRD) {
#pragma unroll
    for (int e = 0; e < VC; ++e) acc3[e] = floatx4{0};
  }
  const int part = l16 / G;

  for (int t0 = r0 + wv * TR; t0 < r1; t0 += NW * TR) {
    char *kt = Kb + (long long)t0 * D, *vt = Vb + (long long)t0 * D;
    const int blk = t0 / Q8_BLOCK;
    float ks_now, vs_now;
    const bool mine = new_row >= t0 && new_row < t0 + TR;
    if (mine) {
      ks_now = append_row<T, D>(lane, k_new + (long long)s * D * ESZ, kt, new_row - t0, ksc + blk);
      vs_now = append_row<T, D>(lane, v_new + (long long)s * D * ESZ, vt, new_row - t0, vsc + blk);
      // the stores are seen by the loads below: one wavefront's, in order, through one compute unit's cache
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
    } else {
      ks_now = ksc[blk];
      vs_now = vsc[blk];
    }
    u32x4 kk[2][KC];
    vword vv[8];
    const bool edge = t0 + TR > r1;
    const int last = r1 - 1 - t0;              // rows past the end repeat the last one and are masked below
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int r = edge ? min(16 * t + l16, last) : 16 * t + l16;
#pragma unroll
      for (int c = 0; c < KC; ++c) kk[t][c] = *reinterpret_cast<const u32x4 *>(kt + (unsigned)(r * D + (lg + 4 * c) * 16));
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int r = 16 * (j / 4) + 4 * lg + j % 4;
      vv[j] = *reinterpret_cast<const vword *>(vt + (unsigned)((edge ? min(r, last) : r) * D + l16 * VC));
    }
    float sc[8];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      floatx4 a[KS];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        u32x4 op;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const unsigned w = kk[t][ks / 2][2 * (ks % 2) + i];
          op[2 * i] = two<F16>(w, false, 1.0f);
          op[2 * i + 1] = two<F16>(w, true, 1.0f);
        }
        a[ks] = floatx4{0};
#pragma unroll
        for (int p = QP - 1; p >= 0; --p) a[ks] = mfma16<F16>(op, qf[p][ks], a[ks]);
      }
#pragma unroll
      for (int o = KS / 2; o > 0; o >>= 1)
#pragma unroll
        for (int ks = 0; ks < o; ++ks) a[ks] += a[ks + o];
#pragma unroll
      for (int i = 0; i < 4; ++i) sc[4 * t + i] = a[0][i];
    }
    if (edge) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (16 * (j / 4) + 4 * lg + j % 4 > last) { sc[j] = -INFINITY; vv[j] = vword{0}; }
    }
    const float cs = fmaxf(c_log2 * ks_now, FLT_MIN);          // (0 times the -inf of a row past the end would be a NaN)
    float top = sc[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) top = fmaxf(top, sc[j]);
    top *= cs;
    if (__any(top > m)) {
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float mn = fmaxf(m, top);
      const float corr = fast_exp2(m - mn);
      l *= corr;
      m = mn;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float ci = __shfl(corr, 4 * lg + i);
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
      p[j] = fast_exp2(fmaf(sc[j], cs, -m));
      l += p[j];
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
    for (int v = 0; v < VW; ++v) {
      unsigned pair[2][4];                     // [columns 4v, 4v+1 | 4v+2, 4v+3][rows 0,1 | 2,3 | 4,5 | 6,7]: two columns of two rows
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const unsigned w0 = vv[2 * k][v], w1 = vv[2 * k + 1][v];
        pair[0][k] = __builtin_amdgcn_perm(w1, w0, 0x05010400u);
        pair[1][k] = __builtin_amdgcn_perm(w1, w0, 0x07030602u);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        u32x4 vb;
#pragma unroll
        for (int k = 0; k < 4; ++k) vb[k] = two<false>(pair[e / 2][k], e % 2, vs_now);
        acc[4 * v + e] = mfma16<false>(pa, vb, acc[4 * v + e]);
        if (THIRD) acc3[4 * v + e] = mfma16<false>(pc, vb, acc3[4 * v + e]);
      }
    }
  }

  // ---- the wavefronts' results meet in LDS, as in decode_mfma_kernel (no value is infinite here) -----------------
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (lane < G) { sh_m[wv][lane] = m; sh_l[wv][lane] = l; }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = 4 * lg + i;
#pragma unroll
    for (int e = 0; e < VC; e += 4) {
      if (row < PARTS * G)
        *reinterpret_cast<float4 *>(&sh_acc[wv][row][l16 * VC + e]) = make_float4(acc[e][i], acc[e + 1][i], acc[e + 2][i], acc[e + 3][i]);
      if (THIRD && row < G)
        *reinterpret_cast<float4 *>(&sh_third[wv][row][l16 * VC + e]) = make_float4(acc3[e][i], acc3[e + 1][i], acc3[e + 2][i], acc3[e + 3][i]);
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
      float rest = sh_acc[w2][G + gi][e];
      rest += THIRD ? sh_third[w2][gi][e] : sh_acc[w2][2 * G + gi][e];
      a = fmaf(sh_acc[w2][gi][e] + rest, f, a);
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
  if (WHOLE && res.new_len && tid == 0) {
    if (new_row >= 0) res.new_len[s] = len;
    else if (res.overflow) *res.overflow = 1;
  }
}

template <typename T, int D, int G>
void run_decode_q8(const SeqTab &st, const Dims &dm, int headroom, const DecodePlan &pl, const void *q, const void *k_new,
                   const void *v_new, const int *cu, const Q8Cache &c, int *seg_len, int *overflow, float *out, float *lse, char *ws,
                   hipStream_t s) {
  const int nseg = st.batch * dm.h_kv, per = (nseg + 255) / 256;
  const DecodeOut res = {(float *)(ws + pl.part_acc), (float *)(ws + pl.part_ml), (int4 *)(ws + pl.seg_tab), out, lse,
                         k_new ? seg_len : nullptr, overflow};
#define ADAKV_DECODE_Q8(WHOLE, grid, block)                                                                              \
  ADAKV_LAUNCH("decode_q8", (decode_q8_kernel<T, D, G, WHOLE>), dim3(grid), dim3(block), s, nseg, dm.h_kv, per, pl.split,  \
               headroom, dm.scale *LOG2E, (const char *)q, (const char *)k_new, (const char *)v_new, cu, (const int *)seg_len, \
               c.K, c.V, c.k_scale, c.v_scale, res)
  if (pl.whole) {
    ADAKV_DECODE_Q8(true, nseg, (64 * WHOLE_WAVES<D, G>));
    return;
  }
  ADAKV_DECODE_Q8(false, pl.nblk, 256);
#undef ADAKV_DECODE_Q8
  launch_decode_combine(nseg, D, G, pl, ws, k_new ? seg_len : nullptr, overflow, out, lse, s);
}

// A template's call by the layer's type, d (and g): `false` where there is none.
template <typename F> bool by_type(int dtype, int d, F &&f) {
  if (d != 64 && d != 128) return false;
  auto at = [&](auto t) {
    if (d == 64) f(t, std::integral_constant<int, 64>());
    else f(t, std::integral_constant<int, 128>());
  };
  if (dtype == ADAKV_BF16) at(BF16());
  else if (dtype == ADAKV_FP16) at(FP16());
  else at(FP32());
  return true;
}

}  // namespace

long long q8_scales(const SeqTab &st, const Dims &dm, int headroom) {
  const long long nseg = (long long)st.batch * dm.h_kv;
  return ((long long)st.out_off[st.batch] + nseg * headroom) / ADAKV_Q8_BLOCK + nseg;
}

hipError_t launch_cache_build_q8(const SeqTab &st, const Dims &dm, int dtype, const void *K, const void *V, const int *indices,
                                 const int *cu, int headroom, const Q8Cache &c, int *seg_len, hipStream_t s) {
  const int nseg = st.batch * dm.h_kv, rows = st.out_off[st.batch];
  const int nblk = rows / Q8_BLOCK + nseg, esz = dtype == ADAKV_FP32 ? 4 : 2;
  const bool ok = by_type(dtype, dm.d, [&](auto t, auto d) {
    ADAKV_LAUNCH("cache_build_q8", (cache_build_q8_kernel<decltype(t), decltype(d)::value>), dim3((nblk + 1) / 2), dim3(256), s, st,
                 dm.h_kv, nseg, nblk, dm.k_stride_tok * esz, dm.k_stride_head * esz, dm.v_stride_tok * esz, dm.v_stride_head * esz,
                 (const char *)K, (const char *)V, indices, cu, c.K, c.V, c.k_scale, c.v_scale, rows, dm.w, headroom, seg_len);
  });
  return ok ? hipGetLastError() : hipErrorInvalidValue;
}

hipError_t launch_append_q8(const SeqTab &st, const Dims &dm, int dtype, int headroom, const void *k_new, const void *v_new,
                            const int *cu, const Q8Cache &c, int *seg_len, int *overflow, hipStream_t s) {
  const bool ok = by_type(dtype, dm.d, [&](auto t, auto d) {
    ADAKV_LAUNCH("append_q8", (append_q8_kernel<decltype(t), decltype(d)::value>), dim3(st.batch * dm.h_kv), dim3(128), s, headroom,
                 (const char *)k_new, (const char *)v_new, cu, c.K, c.V, c.k_scale, c.v_scale, seg_len, overflow);
  });
  return ok ? hipGetLastError() : hipErrorInvalidValue;
}

DecodePlan plan_decode_q8(const SeqTab &st, const Dims &dm, int dtype, int headroom) {
  // the 16-bit kernels' division (the same tiles and registers); the workspace is as large as the layer's own type has it
  DecodePlan pl = plan_decode(st, dm, ADAKV_BF16, headroom);
  const DecodePlan full = plan_decode(st, dm, dtype, headroom);
  if (pl.nblk > full.nblk) pl = full;
  // One workgroup per segment and no merge kernel up to a longest segment of, in bytes of codes, 768 rows of 128 (512
  // with fp32 queries, which take three products for one).  us per step, parts | whole, by rows of the longest segment
  // (the others a third of it): 8 segments, d = 128, g = 4, bf16: 64 8.1 | 5.5, 256 8.5 | 7.0, 512 8.4 | 8.1, 768 8.7 |
  // 9.2, 1024 8.9 | 11.3; g = 8: 9.1 | 6.1, 9.3 | 7.2, 9.5 | 8.4, 9.5 | 9.8, 9.7 | 11.1; d = 64, fp16: 8.0 | 5.0, 8.1 |
  // 5.2, 8.2 | 5.8, 8.3 | 6.6, 8.4 | 6.8, 1536 8.5 | 8.3, 2048 8.7 | 9.5; fp32, d = 128: 256 9.3 | 8.2, 512 9.3 | 9.9,
  // 768 9.7 | 11.0.  From half as many segments as compute units on the parts fill the chip less evenly, and the merge
  // takes longer: segments of 512 and of 1024 rows, d = 128, g = 4, bf16: 64 segments 9.7 | 8.3 and 10.8 | 11.4, 256
  // 14.5 | 9.3 and 19.4 | 14.5, 512 24.3 | 18.4 and 33.2 | 27.3; fp32, 256: 15.6 | 10.6 and 20.2 | 15.9.
  const long long nseg = (long long)st.batch * dm.h_kv;
  const long long line = 128ll * (nseg >= 128 ? 1024 : dtype == ADAKV_FP32 ? 512 : 768);
  pl.whole = pl.likely * dm.d <= line && pl.longest * dm.d <= line + line / 3;
  return pl;
}

hipError_t launch_decode_q8(const SeqTab &st, const Dims &dm, int dtype, int headroom, const void *q, const void *k_new,
                            const void *v_new, const int *cu, const Q8Cache &c, int *seg_len, int *overflow, float *out, float *lse,
                            char *ws, hipStream_t s) {
  const DecodePlan pl = plan_decode_q8(st, dm, dtype, headroom);
  bool ok = false;
  by_type(dtype, dm.d, [&](auto t, auto d) {
#define ADAKV_G(G)                                                                                                          \
  if (dm.g == G)                                                                                                            \
    ok = true, run_decode_q8<decltype(t), decltype(d)::value, G>(st, dm, headroom, pl, q, k_new, v_new, cu, c, seg_len, overflow, out, \
                                                                 lse, ws, s)
    ADAKV_G(1);
    ADAKV_G(2);
    ADAKV_G(4);
    ADAKV_G(8);
#undef ADAKV_G
  });
  return ok ? hipGetLastError() : hipErrorInvalidValue;
}

}  // namespace adakv
