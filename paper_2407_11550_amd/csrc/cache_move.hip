// Sequences of a flattened cache into another one: the destination's sequence i takes the rows that sequence from[i] of
// the source holds, behind a head-room of its own.  Named twice a sequence is forked, not named it is dropped.
//
// Pure byte movement, bound by HBM: distinct held rows are read and all destination rows written.  A sequence's segments lie
// one behind the other in the source (head-room between them), so a workgroup takes consecutive rows of the
// sequence's place there, as 16-byte words by LPR lanes a row, and skips what no segment holds.  Capacities are
// copied, so where a destination segment begins follows from the source's offsets without a prefix sum.
#include "common.h"

namespace adakv {
namespace {

struct MoveTab {
  int count;
  int from[ADAKV_MAX_BATCH];
  int src_row[ADAKV_MAX_BATCH];            // sum of B of the source's sequences before it
  int rows[ADAKV_MAX_BATCH];               // its B
  int dst_row[ADAKV_MAX_BATCH + 1];        // sum of B of the destination's sequences before it
  int blk[ADAKV_MAX_BATCH + 1];            // first workgroup
};

template <int LPR, int RPT, bool Q8>
__global__ __launch_bounds__(256) void cache_move_kernel(
    MoveTab mt, int h, int headroom, int headroom_out, const int *__restrict__ cu, const int *__restrict__ seg_len,
    const char *__restrict__ K, const char *__restrict__ V, const float *__restrict__ k_scale, const float *__restrict__ v_scale,
    int *__restrict__ cu_out, int *__restrict__ len_out, char *__restrict__ K_out, char *__restrict__ V_out,
    float *__restrict__ ks_out, float *__restrict__ vs_out, int *__restrict__ overflow) {
  constexpr int RPB = 256 / LPR;
  int i = 0;
  while (i + 1 < mt.count && (int)blockIdx.x >= mt.blk[i + 1]) ++i;
  const int b = mt.from[i], src_row = mt.src_row[i], rows = mt.rows[i];
  const int u0 = ((int)blockIdx.x - mt.blk[i]) * (RPB * RPT);
  const int *cu_b = cu + b * h, *len_b = seg_len + b * h;
  // (offsets are clamped into the sequence, so that corrupt ones cannot leave the buffers)
  auto begin = [&](int c) { return min(max(cu_b[c] - src_row, 0), rows); };

  if (u0 == 0 && (int)threadIdx.x < h) {
    const int c = threadIdx.x, size = max(begin(c + 1) - begin(c), 0), held = min(max(len_b[c], 0), size + headroom);
    cu_out[i * h + c] = mt.dst_row[i] + begin(c);
    len_out[i * h + c] = min(held, size + headroom_out);
    if (held > size + headroom_out && overflow) *overflow = 1;
    if (i == mt.count - 1 && c == 0) cu_out[mt.count * h] = mt.dst_row[mt.count];
  }

  const int lane = threadIdx.x % LPR, slot = threadIdx.x / LPR;
  // segment c whose place in the source has row u0 of the sequence's
  int lo = 0, hi = h;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (begin(mid) + (long long)mid * headroom <= u0) lo = mid; else hi = mid;
  }
  uint4 kv[RPT], vv[RPT];
  long long to[RPT];
  int c = lo;
#pragma unroll
  for (int r = 0; r < RPT; ++r) {
    const long long u = u0 + r * RPB + slot;
    while (c + 1 < h && begin(c + 1) + (long long)(c + 1) * headroom <= u) ++c;
    const int at = begin(c), size = max(begin(c + 1) - at, 0);
    const int held = min(min(max(len_b[c], 0), size + headroom), size + headroom_out);
    const long long t = u - (at + (long long)c * headroom);
    const bool on = t < held;
    const long long first = src_row + (long long)at + (long long)(b * h + c) * headroom, row = first + t;
    const long long first_out = mt.dst_row[i] + (long long)at + (long long)(i * h + c) * headroom_out;
    to[r] = on ? first_out + t : -1;
    if (on) {
      kv[r] = *reinterpret_cast<const uint4 *>(K + (row * LPR + lane) * 16);
      vv[r] = *reinterpret_cast<const uint4 *>(V + (row * LPR + lane) * 16);
      if (Q8 && lane == 0 && t % ADAKV_Q8_BLOCK == 0) {        // blocks are counted from a segment's first row: they move whole
        const long long src = first / ADAKV_Q8_BLOCK + b * h + c + t / ADAKV_Q8_BLOCK;
        const long long dst = first_out / ADAKV_Q8_BLOCK + i * h + c + t / ADAKV_Q8_BLOCK;
        ks_out[dst] = k_scale[src];
        vs_out[dst] = v_scale[src];
      }
    }
  }
#pragma unroll
  for (int r = 0; r < RPT; ++r)
    if (to[r] >= 0) {
      *reinterpret_cast<uint4 *>(K_out + (to[r] * LPR + lane) * 16) = kv[r];
      *reinterpret_cast<uint4 *>(V_out + (to[r] * LPR + lane) * 16) = vv[r];
    }
}

}  // namespace

hipError_t launch_cache_move(const SeqTab &st, const Dims &dm, int row_bytes, int count, const int *from, const int *cu, int headroom,
                             const void *K, const void *V, const float *k_scale, const float *v_scale, const int *seg_len,
                             int headroom_out, int *cu_out, void *K_out, void *V_out, float *ks_out, float *vs_out, int *len_out,
                             int *overflow, hipStream_t s) {
  const int lpr = row_bytes / 16;
  constexpr int RPT = 2;
  MoveTab mt;
  mt.count = count;
  long long row = 0, blk = 0;
  for (int i = 0; i < count; ++i) {
    const int b = from[i], rows = st.out_off[b + 1] - st.out_off[b], per = 256 / lpr * RPT;
    mt.from[i] = b;
    mt.src_row[i] = st.out_off[b];
    mt.rows[i] = rows;
    mt.dst_row[i] = (int)row;
    mt.blk[i] = (int)blk;
    row += rows;
    blk += (rows + (long long)dm.h_kv * headroom + per - 1) / per;
  }
  for (int i = count; i <= ADAKV_MAX_BATCH; ++i) {
    mt.dst_row[i] = (int)row;
    mt.blk[i] = (int)blk;
  }
#define ADAKV_MOVE(LPR, Q8)                                                                                                    \
  ADAKV_LAUNCH("cache_move", (cache_move_kernel<LPR, RPT, Q8>), dim3((unsigned)blk), dim3(256), s, mt, dm.h_kv, headroom, headroom_out, \
               cu, seg_len, (const char *)K, (const char *)V, k_scale, v_scale, cu_out, len_out, (char *)K_out, (char *)V_out, ks_out,  \
               vs_out, overflow)
  const bool q8 = k_scale != nullptr;
  if (q8 && lpr == 4) ADAKV_MOVE(4, true);
  else if (q8 && lpr == 8) ADAKV_MOVE(8, true);
  else if (!q8 && lpr == 8) ADAKV_MOVE(8, false);
  else if (!q8 && lpr == 16) ADAKV_MOVE(16, false);
  else if (!q8 && lpr == 32) ADAKV_MOVE(32, false);
  else return hipErrorInvalidValue;
#undef ADAKV_MOVE
  return hipGetLastError();
}

}  // namespace adakv
