// Rotary positions of queries and keys, of a prompt or of a batch's new tokens, and the norm of every head in the same pass.
//
// Elements a and b of a pair i of a row at position p become a cos t - b sin t and b cos t + a sin t, t = p f_i, times the
// magnitude; a norm divides a head by the root of its mean square first, and multiplies it by a weight per element.  All of it in 32
// bits with one rounding at the end, but for the angle: p f_i reaches 10^5 and more radians, of which 32 bits would leave a
// hundredth, so the product and its remainder by quarter turns are made in 64.
//
// Bound by memory: 2 d e bytes a head for some 6 d operations.  A wavefront takes a row of all heads.  Each of its lanes makes
// the cosine and the sine of one pair (64 pairs at d = 128), through LDS they reach the lanes that have the pair's elements: a lane has
// the same pairs of every head it sees, 16 bytes of elements a and 16 of elements b, and 16 (d = 64) or 8 heads go by at a time.  16384 rows of 40 heads, bf16, d = 128, behind
// a norm: 58.6 us, 5.7 TB/s read and written, where a copy of as many bytes reaches 5.4.
#include <math.h>

#include "common.h"
#include "row_parts.h"

namespace adakv {
namespace {

typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// E elements of a row, 16 bytes, as they are in memory.
template <typename T, int E> struct Chunk;
template <typename T> struct Chunk<T, 4> : Elem<T> {
  typedef u32x4 Word;
  static __device__ __forceinline__ Word narrow(const float (&f)[4]) {
    return {__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
  }
};
template <typename T> __device__ __forceinline__ unsigned round2(float x0, float x1);
template <> __device__ __forceinline__ unsigned round2<unsigned short>(float x0, float x1) {
  return __builtin_bit_cast(unsigned, __builtin_convertvector(floatx2{x0, x1}, bf16x2));
}
template <> __device__ __forceinline__ unsigned round2<f16_t>(float x0, float x1) {
  return __builtin_bit_cast(unsigned, __builtin_convertvector(floatx2{x0, x1}, f16x2));
}
template <typename T> struct Chunk<T, 8> : Elem<T> {
  typedef u32x4 Word;
  static __device__ __forceinline__ Word narrow(const float (&f)[8]) {
    return {round2<T>(f[0], f[1]), round2<T>(f[2], f[3]), round2<T>(f[4], f[5]), round2<T>(f[6], f[7])};
  }
};
// The rows of a call, each in `shares` pieces of `share` heads; without positions the rows of `batch` sequences, which begin at `off` among
// them and at `tok` in the tensors.
struct Rows {
  int total, batch, items, shares, share;
  const int *positions;
  int off[ADAKV_MAX_BATCH];
  long long tok[ADAKV_MAX_BATCH];
};
struct Heads {                                 // of queries or of keys; strides in bytes
  const char *x;
  char *out;
  long long tok, head, out_tok, out_head;
  int count;
};

// cos and sin of p * f, f in quarter turns.  Taylor series on an eighth of a turn either way: what is left out is below 2 x 10^-9.
__device__ __forceinline__ float2 cos_sin(double p, double f) {
  const double t = p * f, k = __builtin_rint(t);
  const float x = (float)(t - k) * 1.57079632679489662f, y = x * x;
  float s = fmaf(y, 1.0f / 362880.0f, -1.0f / 5040.0f), c = fmaf(y, -1.0f / 3628800.0f, 1.0f / 40320.0f);
  s = fmaf(y, s, 1.0f / 120.0f);
  c = fmaf(y, c, -1.0f / 720.0f);
  s = fmaf(y, s, -1.0f / 6.0f);
  c = fmaf(y, c, 1.0f / 24.0f);
  s = fmaf(x * y, s, x);
  c = fmaf(y, c, -0.5f);
  c = fmaf(y, c, 1.0f);
  const int quarter = (int)(k - 4.0 * __builtin_floor(0.25 * k));
  const float a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
  return make_float2((quarter + 1) & 2 ? -a : a, quarter & 2 ? -b : b);
}

// Rows are read once and written for another kernel: neither is to push anything out of the caches.  (But half a line is not to be dropped
// before its other half is read.)  us, plain | stores | both: 16384 rows of 40 heads, bf16, d = 128 63.8 | 60.6 | 59.0; fp16, d = 64 34.0 |
// 32.4 | 34.1; 8192 rows, fp32, d = 64 35.6 | 33.5 | 32.4.
template <bool ONCE, typename Word> __device__ __forceinline__ Word load_word(const Word *p) {
  if constexpr (ONCE) return __builtin_nontemporal_load(p);
  else return *p;
}

// How a lane comes by its pairs.  HALVES: it has elements a of a half and elements b of the other.  NEIGHBOURS: its elements are whole pairs.  SHIFTED: halves
// that are not 16 bytes apart by some number; an element's other one is another lane's, and they meet in LDS.  (One element a lane at a time
// instead: 63.9 us, now 34.3, 8192 rows of 40 heads in bf16, d = 128, 100 of it turned.)
enum Way { HALVES, NEIGHBOURS, SHIFTED };

template <typename T, int D, Way WAY, bool NORM>
__global__ __launch_bounds__(256) void rotary_kernel(Rows rows, Heads q, Heads k, int dims, float magnitude, const double *__restrict__ freq,
                                                     const void *__restrict__ q_weight, const void *__restrict__ k_weight, float eps) {
  constexpr int E = 16 / (int)sizeof(T);
  typedef Chunk<T, E> C;
  typedef typename C::Word Word;
  constexpr int S = (int)sizeof(T), LPH = D / 2 / E;           // lanes a head
  constexpr int HPW = 64 / LPH;                                // heads a wavefront sees at a time
  constexpr bool ONCE = D * S / 2 >= 128;                      // (a load is of whole lines of 128 bytes)
  constexpr int U = 4;                                         // ... times those whose loads are in flight together
  constexpr int MINE = WAY == SHIFTED ? 2 * E : E;             // angles of a lane: its pairs', or its elements'
  __shared__ float2 sh_cs[4][D / 2];
  // the heads of a wavefront, elements of a lane an odd number of words from the next lane's
  __shared__ float sh_x[WAY == SHIFTED ? 4 : 1][WAY == SHIFTED ? HPW * (D + D / E) : 1];
  const int lane = threadIdx.x & 63, unit = lane % LPH, slot = lane / LPH;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = dims / 2;
  // the lane's elements: a and b of the same pairs, and behind the turned ones some of the others, as they come; or a piece of either half of the
  // head, so that neighbouring lanes read on (NEIGHBOURS with 16 of every 32 bytes at a time: 68.7 us, now 58.4, 16384 rows of 40 heads in bf16)
  const int ea = WAY != HALVES || E * unit < half ? E * unit : dims + 2 * (E * unit - half);
  const int eb = WAY != HALVES ? ea + D / 2 : E * unit >= half ? ea + E : ea + half;
  const auto pair = [&](int e) {
    if constexpr (WAY == HALVES) return E * unit + e;
    if constexpr (WAY == NEIGHBOURS) return E / 2 * unit + (e < E / 2 ? e : e - E / 2 + D / 4);
    const int at = e < E ? ea + e : eb + e - E;                // (SHIFTED: of the lane's element e)
    return at < half ? at : at < dims ? at - half : half;
  };
  Word wa[2], wb[2];
  if constexpr (NORM) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const char *w = (const char *)(i ? k_weight : q_weight);
      if (w) {
        wa[i] = *(const Word *)(w + ea * S);
        wb[i] = *(const Word *)(w + eb * S);
      }
    }
  }
  const double f = lane < half ? freq[lane] * 0.63661977236758134308 : 0.0;    // 2 / pi

  const int heads = q.count + k.count;
  for (int item = blockIdx.x * 4 + wv; item < rows.items; item += gridDim.x * 4) {
    // a row, or some of its heads where there are few rows
    const int r = rows.shares > 1 ? item / rows.shares : item;
    const int from = (item - r * rows.shares) * rows.share, end = min(heads, from + rows.share);
    long long row = r;
    int pos;
    if (rows.positions) {
      pos = rows.positions[r];
      if (pos < 0) continue;
    } else {
      const int b = __popcll(__ballot(lane > 0 && lane < rows.batch && r >= rows.off[lane]));
      pos = r - rows.off[b];
      row = rows.tok[b] + pos;
    }
    float cs[MINE], sn[MINE];
    if (half) {
      if (lane < D / 2) {
        const float2 v = cos_sin(pos, f);
        sh_cs[wv][lane] = make_float2(v.x * magnitude, v.y * magnitude);
      }
      lanes_meet();
#pragma unroll
      for (int e = 0; e < MINE; ++e) {
        const float2 v = sh_cs[wv][WAY == SHIFTED ? min(pair(e), D / 2 - 1) : pair(e)];
        cs[e] = v.x;
        sn[e] = v.y;
      }
      lanes_meet();
    }
    for (int h0 = from; h0 < end; h0 += HPW * U) {
      Word xa[U], xb[U];
      char *out[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = h0 + u * HPW + slot;
        out[u] = nullptr;
        if (h < end) {
          const bool is_k = h >= q.count;
          const int hh = is_k ? h - q.count : h;
          const char *x = (is_k ? k.x : q.x) + row * (is_k ? k.tok : q.tok) + hh * (is_k ? k.head : q.head);
          out[u] = (is_k ? k.out : q.out) + row * (is_k ? k.out_tok : q.out_tok) + hh * (is_k ? k.out_head : q.out_head);
          xa[u] = load_word<ONCE>((const Word *)(x + ea * S));
          xb[u] = load_word<ONCE>((const Word *)(x + eb * S));
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (h0 + u * HPW >= end) break;        // (of all lanes)
        float a[E], b[E];
        C::widen(xa[u], a);
        C::widen(xb[u], b);
        if constexpr (NORM) {
          float sum = 0.0f;
#pragma unroll
          for (int e = 0; e < E; ++e) sum = fmaf(a[e], a[e], fmaf(b[e], b[e], sum));
          sum = row_sum<LPH>(sum);
          const float by = rsqrtf(fmaf(sum, 1.0f / D, eps));
          const bool is_k = h0 + u * HPW + slot >= q.count;
          float w0[E], w1[E];
          C::widen(is_k ? wa[1] : wa[0], w0);
          C::widen(is_k ? wb[1] : wb[0], w1);
#pragma unroll
          for (int e = 0; e < E; ++e) {
            a[e] = a[e] * by * w0[e];
            b[e] = b[e] * by * w1[e];
          }
        }
        if (half) {
          float x[2 * E];                      // as they lie in memory
#pragma unroll
          for (int e = 0; e < E; ++e) {
            x[e] = a[e];
            x[E + e] = b[e];
          }
          if constexpr (WAY == SHIFTED) {
            float *mine = sh_x[wv] + slot * (D + D / E);
            const auto place = [](int at) { return at + at / E; };
#pragma unroll
            for (int e = 0; e < 2 * E; ++e) mine[place(e < E ? ea + e : eb + e - E)] = x[e];
            lanes_meet();
#pragma unroll
            for (int e = 0; e < 2 * E; ++e) {
              const int at = e < E ? ea + e : eb + e - E;
              const float other = mine[place(at < half ? at + half : at < dims ? at - half : at)];
              const float y = fmaf(x[e], cs[e], at < half ? -other * sn[e] : other * sn[e]);
              x[e] = at < dims ? y : x[e];
            }
            lanes_meet();
          } else {
#pragma unroll
            for (int e = 0; e < E; ++e) {
              const int i = WAY == NEIGHBOURS ? 2 * e : e, j = WAY == NEIGHBOURS ? i + 1 : E + e;
              const bool turned = pair(e) < half;
              const float y0 = fmaf(x[i], cs[e], -x[j] * sn[e]), y1 = fmaf(x[j], cs[e], x[i] * sn[e]);
              x[i] = turned ? y0 : x[i];
              x[j] = turned ? y1 : x[j];
            }
          }
#pragma unroll
          for (int e = 0; e < E; ++e) {
            a[e] = x[e];
            b[e] = x[E + e];
          }
        }
        if (out[u]) {
          __builtin_nontemporal_store(C::narrow(a), (Word *)(out[u] + ea * S));
          __builtin_nontemporal_store(C::narrow(b), (Word *)(out[u] + eb * S));
        }
      }
    }
  }
}

template <typename T, int D, bool NORM>
void run_rotary(bool neighbours, int dims, Rows rows, const Heads &q, const Heads &k, float magnitude, const double *freq, const void *qw,
                const void *kw, float eps, hipStream_t s) {
  constexpr int E = 16 / (int)sizeof(T);
  // A wavefront takes a row, and where there are fewer rows than the chip holds wavefronts (a batch's new tokens), some of its heads.  64 rows of 72
  // heads, bf16, d = 128, behind a norm: 7.6 us a call with a row each, 5.1 with 8 heads each; 1021 rows of 10 fp32 heads, halves that are not aligned, where there is
  // little to share: 5.7 and 5.9 with four each.
  const int at_a_time = 64 / (D / 2 / E), heads = q.count + k.count;
  const int pieces = (heads + at_a_time - 1) / at_a_time, most = 8192 / rows.total;
  rows.share = most <= 1 ? heads : (pieces + most - 1) / most * at_a_time;
  rows.shares = (heads + rows.share - 1) / rows.share;
  rows.items = rows.total * rows.shares;
  const dim3 grid((unsigned)((rows.items + 3) / 4 < 4096 ? (rows.items + 3) / 4 : 4096));
  const char *name = NORM ? "norm_rotary" : "rotary";
#define ADAKV_ROTARY(WAY) \
  ADAKV_LAUNCH(name, (rotary_kernel<T, D, WAY, NORM>), grid, dim3(256), s, rows, q, k, dims, magnitude, freq, qw, kw, eps)
  if (neighbours) ADAKV_ROTARY(NEIGHBOURS);
  else if (dims % (2 * E) == 0) ADAKV_ROTARY(HALVES);
  else ADAKV_ROTARY(SHIFTED);
#undef ADAKV_ROTARY
}

}  // namespace

hipError_t launch_rotary(const SeqTab &st, const Dims &dm, int dtype, const adakv_rotation &R, int rows, const int *positions,
                         const adakv_heads *q, const adakv_heads *k, const adakv_heads *q_out, const adakv_heads *k_out, bool norm,
                         const void *q_weight, const void *k_weight, float eps, hipStream_t s) {
  const long long e = dtype == ADAKV_FP32 ? 4 : 2;
  const auto heads = [&](const adakv_heads *x, const adakv_heads *o, int count) {
    if (!x) return Heads{nullptr, nullptr, 0, 0, 0, 0, 0};
    return Heads{(const char *)x->x, (char *)o->x, x->stride_tok * e, x->stride_head * e, o->stride_tok * e, o->stride_head * e, count};
  };
  Rows r = {};
  r.positions = positions;
  r.batch = st.batch;
  long long total = 0;
  for (int b = 0; b < st.batch; ++b) {
    r.off[b] = (int)total;
    r.tok[b] = st.tok_off[b];
    total += st.n[b] + dm.w;
  }
  r.total = positions ? rows : (int)total;
  if (r.total == 0) return hipSuccess;
  const Heads hq = heads(q, q_out, dm.h_q), hk = heads(k, k_out, dm.h_kv);
  const float by = R.magnitude > 0.0f ? R.magnitude : 1.0f;
  const bool nb = R.layout == ADAKV_ROTARY_INTERLEAVED;
#define ADAKV_ROTARY_N(T, D, N) run_rotary<T, D, N>(nb, R.dims, r, hq, hk, by, R.freq, q_weight, k_weight, eps, s)
#define ADAKV_ROTARY_D(T, D) (norm ? ADAKV_ROTARY_N(T, D, true) : ADAKV_ROTARY_N(T, D, false))
#define ADAKV_ROTARY_T(T) (dm.d == 64 ? ADAKV_ROTARY_D(T, 64) : ADAKV_ROTARY_D(T, 128))
  if (dtype == ADAKV_BF16) ADAKV_ROTARY_T(unsigned short);
  else if (dtype == ADAKV_FP16) ADAKV_ROTARY_T(f16_t);
  else ADAKV_ROTARY_T(float);
#undef ADAKV_ROTARY_T
#undef ADAKV_ROTARY_D
#undef ADAKV_ROTARY_N
  return hipGetLastError();
}

}  // namespace adakv
