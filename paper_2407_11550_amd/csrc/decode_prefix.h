// A decoding step over shared caches: what its kernels and the entry points share (decode_prefix.hip, api.hip).
#pragma once

#include "common.h"

namespace adakv {

// Which sequences share which cache, passed to kernels by value.
struct Sharing {
  static constexpr unsigned char NONE = 255;
  int groups, h, g;
  unsigned char order[ADAKV_MAX_BATCH];        // sequences, those of a shared cache one after the other
  unsigned char first[ADAKV_MAX_BATCH + 1];    // of a shared cache among them
  unsigned char group[ADAKV_MAX_BATCH];        // a sequence's shared cache, or NONE
  unsigned char place[ADAKV_MAX_BATCH];        // and which of that cache's sequences it is
};
struct SharedCache {
  const void *K, *V;
  const int *cu, *seg_len;
  int headroom;
};
struct PrefixPlan {
  DecodePlan own;                              // of the sequences' own segments
  int rb, split, nblk;                         // query rows of a workgroup; rows of a shared segment per part; workgroups at most
  size_t part_acc, part_ml, tab, total;        // byte offsets: the shared segments' partial results; their first workgroups
};
Sharing share(const SeqTab &st, const Dims &dm, int groups, const int *of);
PrefixPlan plan_prefix(const SeqTab &st, const Dims &dm, int dtype, int headroom, const Sharing &sh, const SeqTab &shared, int shared_headroom);
hipError_t launch_decode_prefix(const SeqTab &st, const Dims &dm, int dtype, int headroom, const PrefixPlan &pl, const Sharing &sh,
                                const SharedCache &sc, const void *q, const void *k_new, const void *v_new, const int *cu, void *Kc,
                                void *Vc, int *seg_len, int *overflow, float *out, float *lse, char *ws, hipStream_t s);

}  // namespace adakv
