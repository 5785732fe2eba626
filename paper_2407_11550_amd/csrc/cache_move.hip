// Sequences of a flattened cache into another one: the destination's sequence i takes the rows that sequence from[i] of
// the source holds, behind a head-room of its own.  Named twice a sequence is forked, not named it is dropped.
//
// Pure byte movement, bound by HBM: a workgroup reads a piece of a segment once and writes it to every destination that
// names its sequence.  A segment is one contiguous byte range in both caches, so a piece is too.  Capacities are copied, so
// where a destination segment begins follows from the source's offsets without a prefix sum, and so that a
// workgroup finds its piece with one look at the sequence's offsets, pieces are numbered by their place in the
// source, with one more number for each segment: place / PIECE + segment on, which no two segments share.
#include "common.h"

namespace adakv {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

struct MoveTab {
  int sources;                             // distinct ones
  int blk[ADAKV_MAX_BATCH + 1];            // first workgroup of each
  int b[ADAKV_MAX_BATCH], src_row[ADAKV_MAX_BATCH], rows[ADAKV_MAX_BATCH];   // sequence, sum of B before it, its B
  int first[ADAKV_MAX_BATCH + 1];          // its destinations: to[first[i]] .. to[first[i + 1] - 1]
  int to[ADAKV_MAX_BATCH], dst_row[ADAKV_MAX_BATCH];                         // sequence there, sum of B before it
  int count, rows_out;
};

// ROWB: bytes of a row.  grid.y: K, V.  U 16-byte words per thread and piece.
template <int ROWB, int U, bool Q8>
__global__ __launch_bounds__(256) void cache_move_kernel(
    MoveTab mt, int h, int headroom, int headroom_out, const int *__restrict__ cu, const int *__restrict__ seg_len,
    const char *__restrict__ K, const char *__restrict__ V, const float *__restrict__ k_scale, const float *__restrict__ v_scale,
    int *__restrict__ cu_out, int *__restrict__ len_out, char *__restrict__ K_out, char *__restrict__ V_out,
    float *__restrict__ ks_out, float *__restrict__ vs_out, int *__restrict__ overflow) {
  constexpr int PIECE = 256 * 16 * U / ROWB;               // rows
  const int tid = threadIdx.x, lane = tid & 63, blk = blockIdx.x;
  const bool values = blockIdx.y != 0;
  int i = 0;
  while (i + 1 < mt.sources && blk >= mt.blk[i + 1]) ++i;
  const int b = mt.b[i], src_row = mt.src_row[i], rows = mt.rows[i], k = blk - mt.blk[i];
  const int d0 = mt.first[i], d1 = mt.first[i + 1];

  // a segment a lane; offsets are clamped into the sequence, so that corrupt ones cannot leave the buffers
  const int c_l = min(lane, h - 1);
  const int at_l = min(max(cu[b * h + c_l] - src_row, 0), rows), end_l = min(max(cu[b * h + c_l + 1] - src_row, at_l), rows);
  const int held_l = max(seg_len[b * h + c_l], 0);         // (a corrupt length: no more rows than the source has)
  const int fit_l = min(held_l, end_l - at_l + min(headroom, headroom_out));
  if (k == 0 && !values && tid < h) {
    for (int d = d0; d < d1; ++d) {
      cu_out[mt.to[d] * h + tid] = mt.dst_row[d] + at_l;
      len_out[mt.to[d] * h + tid] = fit_l;
      if (mt.to[d] == mt.count - 1 && tid == 0) cu_out[mt.count * h] = mt.rows_out;
    }
    if (fit_l < held_l && overflow) *overflow = 1;
  }
  const int first_l = (int)((at_l + (long long)lane * headroom) / PIECE) + lane;
  const int c = __builtin_amdgcn_readfirstlane(max(__popcll(__ballot(lane < h && first_l <= k)) - 1, 0));
  const int at = __builtin_amdgcn_readlane(at_l, c), fit = __builtin_amdgcn_readlane(fit_l, c);
  const int t0 = (k - __builtin_amdgcn_readlane(first_l, c)) * PIECE;
  if (t0 < 0 || t0 >= fit) return;         // (below 0: offsets that do not ascend)

  const long long from = src_row + (long long)at + (long long)(b * h + c) * headroom;
  const int words = min(fit - t0, PIECE) * (ROWB / 16);
  const u32x4 *src = reinterpret_cast<const u32x4 *>((values ? V : K) + (from + t0) * ROWB);
  u32x4 x[U];
#pragma unroll
  for (int u = 0; u < U; ++u) x[u] = src[min(tid + 256 * u, words - 1)];
  const int s_in = b * h + c, blocks = Q8 ? (words / (ROWB / 16) + ADAKV_Q8_BLOCK - 1) / ADAKV_Q8_BLOCK : 0;
  float scale = 0.0f;                      // (blocks are counted from a segment's first row: they move whole)
  if (Q8 && tid < blocks) scale = (values ? v_scale : k_scale)[from / ADAKV_Q8_BLOCK + s_in + t0 / ADAKV_Q8_BLOCK + tid];
  for (int d = d0; d < d1; ++d) {
    const int s = mt.to[d] * h + c;
    const long long to = mt.dst_row[d] + (long long)at + (long long)s * headroom_out;
    u32x4 *dst = reinterpret_cast<u32x4 *>((values ? V_out : K_out) + (to + t0) * ROWB);
    // (past the caches, which would hold none of it by the time it is read: 33 MB forked into 137 MB 42.0 us, 28.3 with this)
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (tid + 256 * u < words) __builtin_nontemporal_store(x[u], dst + tid + 256 * u);
    if (Q8 && tid < blocks) (values ? vs_out : ks_out)[to / ADAKV_Q8_BLOCK + s + t0 / ADAKV_Q8_BLOCK + tid] = scale;
  }
}

}  // namespace

hipError_t launch_cache_move(const SeqTab &st, const Dims &dm, int row_bytes, int count, const int *from, const int *cu, int headroom,
                             const void *K, const void *V, const float *k_scale, const float *v_scale, const int *seg_len,
                             int headroom_out, int *cu_out, void *K_out, void *V_out, float *ks_out, float *vs_out, int *len_out,
                             int *overflow, hipStream_t s) {
  constexpr int U = 4;
  const int piece = 256 * 16 * U / row_bytes;
  MoveTab mt = {};
  int dst_row[ADAKV_MAX_BATCH], row = 0;
  for (int i = 0; i < count; ++i) {
    dst_row[i] = row;
    row += st.out_off[from[i] + 1] - st.out_off[from[i]];
  }
  mt.count = count;
  mt.rows_out = row;
  long long blk = 0;
  int n = 0, d = 0;
  for (int b = 0; b < st.batch; ++b) {
    const int begin = d;
    for (int i = 0; i < count; ++i)
      if (from[i] == b) { mt.to[d] = i; mt.dst_row[d] = dst_row[i]; ++d; }
    if (d == begin) continue;
    mt.b[n] = b;
    mt.src_row[n] = st.out_off[b];
    mt.rows[n] = st.out_off[b + 1] - st.out_off[b];
    mt.first[n] = begin;
    mt.blk[n] = (int)blk;
    blk += (mt.rows[n] + (long long)dm.h_kv * headroom) / piece + dm.h_kv;
    ++n;
  }
  mt.sources = n;
  mt.first[n] = d;
  mt.blk[n] = (int)blk;
#define ADAKV_MOVE(ROWB, Q8)                                                                                                     \
  ADAKV_LAUNCH("cache_move", (cache_move_kernel<ROWB, U, Q8>), dim3((unsigned)blk, 2), dim3(256), s, mt, dm.h_kv, headroom,      \
               headroom_out, cu, seg_len, (const char *)K, (const char *)V, k_scale, v_scale, cu_out, len_out, (char *)K_out,     \
               (char *)V_out, ks_out, vs_out, overflow)
  const bool q8 = k_scale != nullptr;
  if (q8 && row_bytes == 64) ADAKV_MOVE(64, true);
  else if (q8 && row_bytes == 128) ADAKV_MOVE(128, true);
  else if (!q8 && row_bytes == 128) ADAKV_MOVE(128, false);
  else if (!q8 && row_bytes == 256) ADAKV_MOVE(256, false);
  else if (!q8 && row_bytes == 512) ADAKV_MOVE(512, false);
  else return hipErrorInvalidValue;
#undef ADAKV_MOVE
  return hipGetLastError();
}

}  // namespace adakv
