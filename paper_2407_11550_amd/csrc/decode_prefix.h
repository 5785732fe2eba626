// A decoding step over shared caches: what its kernels and the entry points share (decode_prefix.hip, api.hip).
#pragma once

#include "common.h"

namespace adakv {

// Which sequences share which cache, passed to kernels by value.
struct Sharing {
  int groups, h, log_g;                        // shared caches; KV heads; query heads to one of them, a power of two
  unsigned char order[ADAKV_MAX_BATCH];        // sequences, those of a shared cache one after the other
  unsigned char first[ADAKV_MAX_BATCH + 1];    // of a shared cache among them
  int whose[ADAKV_MAX_BATCH];                  // a sequence's shared cache, and 256 times which of that cache's sequences it is; or -1
};
// A flattened cache with head-room.
struct Segments {
  const char *K, *V;
  const int *cu, *seg_len;
  int headroom;
};
// How segments are split.  Shared ones, which come first: query rows of a workgroup; parts beyond one for each segment and block of rows;
// workgroups, an upper bound; what a part's sums cost (tiles_a_part).  Own ones: rows of a part; segments, and how many of them a thread counts.
struct PrefixSplit {
  int rb, spare, shared_blocks;
  float sums_cost;
  int own_split, own_segments, own_per;
};
// Partial results: sums, maxima and sums of weights, and which are whose.
struct PrefixSums {
  float *shared_acc, *own_acc;
  float2 *shared_ml, *own_ml;
  int4 *shared_tab, *own_tab;
};
struct PrefixPlan {
  PrefixSplit split;
  int own_blocks;                              // workgroups of the own segments, an upper bound as shared_blocks is
  size_t shared_acc, own_acc, shared_ml, own_ml, shared_tab, own_tab, total;   // byte offsets
};
Sharing share(const SeqTab &st, const Dims &dm, int groups, const int *of);
PrefixPlan plan_prefix(const SeqTab &st, const Dims &dm, int dtype, int headroom, const Sharing &sh);
// k_new == nullptr: attention only
hipError_t launch_decode_prefix(const Dims &dm, int dtype, const PrefixPlan &pl, const Sharing &sh, const Segments &shared, const Segments &own,
                                const void *q, const void *k_new, const void *v_new, int *seg_len, int *overflow, float *out, float *lse,
                                char *ws, hipStream_t s);

}  // namespace adakv
