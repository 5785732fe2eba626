// C ABI entry points: argument checks, workspace planning, kernel launches.
// Each call only enqueues work on the caller's stream.
#include <math.h>
#include <stdio.h>

#include <mutex>

#include "common.h"
#include "decode_prefix.h"
#include "places.h"

namespace adakv {

static int build_tables(const adakv_layer *L, SeqTab &st, Dims &dm) {
  if (!L || !L->n || !L->B) return ADAKV_EINVAL;
  if (L->h_q < 1 || L->h_kv < 1 || L->h_q % L->h_kv != 0) return ADAKV_EINVAL;
  if (L->w < 1 || L->pool_k < 1 || L->pool_k % 2 == 0) return ADAKV_EINVAL;
  if (!(L->alpha >= 0.0f && L->alpha <= 1.0f)) return ADAKV_EINVAL;
  if (!(L->scale >= 0.0f) || isinf(L->scale)) return ADAKV_EINVAL;
  if (L->batch < 1 || L->batch > ADAKV_MAX_BATCH) return ADAKV_EINVAL;
  if (L->batch > 1 && !L->tok_off) return ADAKV_EINVAL;
  if (L->d < 1) return ADAKV_EINVAL;
  long long sc = 0, out = 0;
  st.batch = L->batch;
  for (int b = 0; b < L->batch; ++b) {
    long long n = L->n[b], B = L->B[b];
    long long wh = (long long)L->w * L->h_kv;
    if (n < 1 || B < wh || B - wh > (long long)L->h_kv * n) return ADAKV_EINVAL;
    long long t0 = L->tok_off ? L->tok_off[b] : 0;
    if (t0 < 0) return ADAKV_EINVAL;
    if (L->tok_off && L->tok_off[b + 1] - t0 < n + L->w) return ADAKV_EINVAL;
    st.n[b] = (int)n;
    st.Bp[b] = (int)(B - wh);
    st.tok_off[b] = t0;
    st.score_off[b] = (int)sc;
    st.out_off[b] = (int)out;
    sc += (long long)L->h_kv * n;
    out += B;
    if (sc >= (1ll << 31) || out >= (1ll << 31)) return ADAKV_EUNSUPPORTED;
  }
  for (int b = L->batch; b < ADAKV_MAX_BATCH; ++b) {
    st.n[b] = 0; st.Bp[b] = 0; st.tok_off[b] = 0;
  }
  for (int b = L->batch; b <= ADAKV_MAX_BATCH; ++b) {
    st.score_off[b] = (int)sc;
    st.out_off[b] = (int)out;
  }
  if (L->dtype != ADAKV_BF16 && L->dtype != ADAKV_FP32 && L->dtype != ADAKV_FP16) return ADAKV_EUNSUPPORTED;
  if (L->d != 64 && L->d != 128) return ADAKV_EUNSUPPORTED;
  if (L->h_kv > 64 || (long long)L->h_q * L->w > (1 << 20)) return ADAKV_EUNSUPPORTED;
  const long long esz = L->dtype == ADAKV_FP32 ? 4 : 2;
  const long long strides[4] = {L->k_stride_tok, L->k_stride_head, L->v_stride_tok,
                                L->v_stride_head};
  for (long long sd : strides) {
    if (sd < L->d) return ADAKV_EINVAL;
    if ((sd * esz) % 16 != 0) return ADAKV_EUNSUPPORTED;   // rows are moved as 16-byte words
  }
  dm.h_q = L->h_q; dm.h_kv = L->h_kv; dm.g = L->h_q / L->h_kv; dm.d = L->d; dm.w = L->w;
  dm.pool_k = L->pool_k;
  dm.scale = L->scale > 0.0f ? L->scale : 1.0f / sqrtf((float)L->d);
  dm.alpha_fix = (int)floor((double)L->alpha * 65536.0 + 0.5);
  dm.k_stride_tok = L->k_stride_tok; dm.k_stride_head = L->k_stride_head;
  dm.v_stride_tok = L->v_stride_tok; dm.v_stride_head = L->v_stride_head;
  return ADAKV_OK;
}

// Workspace: the scoring part first, the Top-k part behind it (they must not overlap: in
// pipeline mode the scoring call already writes into the Top-k part).
static bool pool_first(const adakv_layer *L) { return (L->flags & ADAKV_FLAG_POOL_THEN_MEAN) != 0; }
// Which kernel family scores the layer: the matrix cores (16-bit inputs, at most 512 window rows
// per KV head; with ADAKV_FLAG_POOL_THEN_MEAN a pool radius of at most 7), else the fp32 kernels.
static bool on_mfma(const Dims &dm, const adakv_layer *L) {
  return pool_first(L) ? mfma_pool_rows_supported(dm, L->dtype) : mfma_path_supported(dm, L->dtype);
}
// (planning looks at every sequence a few times: once per call)
struct Plan {
  ScorePlan score;
  size_t topk, bytes;       // start of the Top-k part; workspace size
};
static Plan make_plan(const SeqTab &st, const Dims &dm, const adakv_layer *L) {
  Plan p;
  p.score = plan_score(st, dm, L->dtype, on_mfma(dm, L));
  p.topk = align_up(p.score.total, 256);
  p.bytes = p.topk + plan_topk_bytes(st, dm) + 256;
  return p;
}
static bool pipeline_mode(const adakv_layer *L, const Dims &dm) {
  return (L->flags & ADAKV_FLAG_PIPELINE) != 0 && carry_supported(dm, L->dtype) && on_mfma(dm, L);
}

static bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }

static thread_local struct {
  void *const *events = nullptr;
  int capacity = 0, used = 0;
  const char *names[ADAKV_TRACE_MAX];
} g_trace;

bool trace_pair(const char *name, hipEvent_t *start, hipEvent_t *stop) {
  if (!g_trace.events || g_trace.used + 2 > g_trace.capacity) return false;
  g_trace.names[g_trace.used] = name;
  g_trace.names[g_trace.used + 1] = name;
  *start = (hipEvent_t)g_trace.events[g_trace.used];
  *stop = (hipEvent_t)g_trace.events[g_trace.used + 1];
  g_trace.used += 2;
  return true;
}

}  // namespace adakv

// Scratch for adakv_compress_static.  In host code this name is only a handle for
// hipGetSymbolAddress; the device address differs per GPU and is looked up once per device.
static __device__ __align__(256) unsigned char scratch[ADAKV_STATIC_SCRATCH_BYTES];

namespace {
constexpr int MAX_DEVICES = 64;
std::mutex g_scratch_mutex;
void *g_scratch_ptr[MAX_DEVICES] = {};

// Device address of `scratch` on the current device (nullptr if HIP refuses).
void *static_scratch() {
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= MAX_DEVICES) return nullptr;
  std::lock_guard<std::mutex> lock(g_scratch_mutex);
  if (!g_scratch_ptr[dev]) {
    void *p = nullptr;
    if (hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)) != hipSuccess) return nullptr;
    g_scratch_ptr[dev] = p;
  }
  return g_scratch_ptr[dev];
}
}  // namespace

using namespace adakv;

extern "C" {

size_t adakv_workspace_bytes(const adakv_layer *L) {
  SeqTab st; Dims dm;
  if (build_tables(L, st, dm) != ADAKV_OK) return 0;
  return make_plan(st, dm, L).bytes;
}

int adakv_pyramid_budgets(int32_t n_layers, int64_t avg_budget, double ratio, int64_t *out) {
  if (n_layers < 1 || avg_budget < 0 || !(ratio >= 1.0) || isinf(ratio) || !out) return ADAKV_EINVAL;
  if (avg_budget > (1ll << 40) || n_layers > (1 << 24) || ratio > 1048576.0) return ADAKV_EUNSUPPORTED;
  if (n_layers == 1) { out[0] = avg_budget; return ADAKV_OK; }
  // Exact integer arithmetic (a product of doubles can land one unit in the last place off an
  // integer and the floor below would then be wrong by one).  A finite double is p / q with q a
  // power of two, so with L = n_layers
  //   real_l = b_max - (b_max - b_min) l / (L-1),  b_min = 2 avg / (1 + r),  b_max = r b_min
  //          = 2 avg (p (L-1) - (p - q) l) / ((p + q) (L-1)).
  // p < 2^53, q <= 2^52, avg <= 2^40, L <= 2^24: the numerator stays below 2^119.
  int e = 0;
  const double mant = frexp(ratio, &e);                        // ratio = mant * 2^e, 0.5 <= mant < 1
  unsigned __int128 p = (unsigned __int128)(uint64_t)ldexp(mant, 53), q = 1;   // ratio = p * 2^(e-53)
  if (e >= 53) p <<= (e - 53); else q <<= (53 - e);
  while (!(p & 1) && !(q & 1)) { p >>= 1; q >>= 1; }
  const unsigned __int128 Lm1 = (unsigned __int128)(n_layers - 1);
  const unsigned __int128 den = (p + q) * Lm1;
  int64_t given = 0;
  for (int32_t l = 0; l < n_layers; ++l) {
    const unsigned __int128 num = (unsigned __int128)(2 * avg_budget) * (p * Lm1 - (p - q) * (unsigned __int128)l);
    out[l] = (int64_t)(num / den);                             // floor: everything is non-negative
    given += out[l];
  }
  // the real values sum to exactly L * avg, and every floor lost less than one unit
  int64_t left = (int64_t)n_layers * avg_budget - given;
  for (int32_t l = 0; l < n_layers && left > 0; ++l, --left) out[l] += 1;
  return left == 0 ? ADAKV_OK : ADAKV_EINVAL;
}

int adakv_trace_arm(void *const *events, int n_events) {
  if (!events || n_events < 2 || n_events > ADAKV_TRACE_MAX) return ADAKV_EINVAL;
  g_trace.events = events;
  g_trace.capacity = n_events;
  g_trace.used = 0;
  return ADAKV_OK;
}

int adakv_trace_disarm(void) {
  const int used = g_trace.used;
  g_trace.events = nullptr;
  g_trace.capacity = 0;
  return used;
}

const char *adakv_trace_name(int i) {
  return (i >= 0 && i < g_trace.used) ? g_trace.names[i] : "";
}

const char *adakv_strerror(int status) {
  switch (status) {
    case ADAKV_OK: return "ok";
    case ADAKV_EINVAL: return "invalid argument (NULL pointer or parameter outside its domain)";
    case ADAKV_EUNSUPPORTED: return "shape, dtype or alignment not supported by this build";
    case ADAKV_EWORKSPACE: return "workspace missing or smaller than adakv_workspace_bytes";
    case ADAKV_EHIP: return "a HIP runtime call failed";
    case ADAKV_ESCRATCH: return "the layer needs more scratch memory than the built-in array of adakv_compress_static holds";
    default: return "unknown status";
  }
}

int adakv_score(const adakv_layer *L, const void *q_window, const void *K, const float *row_lse,
                float *scores, void *ws, size_t ws_bytes, void *hip_stream) {
  SeqTab st; Dims dm;
  int rc = build_tables(L, st, dm);
  if (rc != ADAKV_OK) return rc;
  if (!q_window || !K || !scores) return ADAKV_EINVAL;
  if (!aligned16(q_window) || !aligned16(K) || !aligned16(scores)) return ADAKV_EUNSUPPORTED;
  const Plan plan = make_plan(st, dm, L);
  if (!ws || ws_bytes < plan.bytes) return ADAKV_EWORKSPACE;
  char *wsp = (char *)(((uintptr_t)ws + 255) & ~(uintptr_t)255);
  hipStream_t s = (hipStream_t)hip_stream;
  if (pool_first(L) && dm.pool_k / 2 > 100) return ADAKV_EUNSUPPORTED;
  TopkCarry tc = {nullptr, 0u, nullptr, nullptr};
  if (pipeline_mode(L, dm)) tc = plan_carry(st, dm, wsp + plan.topk);
  hipError_t e = on_mfma(dm, L)
                     ? launch_score_mfma(st, dm, L->dtype, q_window, K, row_lse, scores, wsp, plan.score, tc,
                                         pool_first(L), s)
                     : launch_score_generic(st, dm, L->dtype, q_window, K, row_lse, scores, wsp,
                                            plan.score, pool_first(L), s);
  return e == hipSuccess ? ADAKV_OK : ADAKV_EHIP;
}

int adakv_allocate(const adakv_layer *L, const float *scores, int32_t *budgets,
                   int32_t *cu_seqlens, void *ws, size_t ws_bytes, void *hip_stream) {
  SeqTab st; Dims dm;
  int rc = build_tables(L, st, dm);
  if (rc != ADAKV_OK) return rc;
  if (!scores || !budgets || !cu_seqlens) return ADAKV_EINVAL;
  if (!aligned16(scores)) return ADAKV_EUNSUPPORTED;
  const Plan plan = make_plan(st, dm, L);
  if (!ws || ws_bytes < plan.bytes) return ADAKV_EWORKSPACE;
  char *wsp = (char *)(((uintptr_t)ws + 255) & ~(uintptr_t)255);
  hipError_t e = launch_allocate(st, dm, scores, budgets, cu_seqlens,
                                 wsp + plan.topk, pipeline_mode(L, dm),
                                 (hipStream_t)hip_stream);
  return e == hipSuccess ? ADAKV_OK : ADAKV_EHIP;
}

int adakv_select(const adakv_layer *L, const float *scores, const int32_t *budgets,
                 const int32_t *cu_seqlens, int32_t *indices, void *ws, size_t ws_bytes,
                 void *hip_stream) {
  SeqTab st; Dims dm;
  int rc = build_tables(L, st, dm);
  if (rc != ADAKV_OK) return rc;
  if (!scores || !budgets || !cu_seqlens || !indices) return ADAKV_EINVAL;
  if (!aligned16(scores)) return ADAKV_EUNSUPPORTED;
  const Plan plan = make_plan(st, dm, L);
  if (!ws || ws_bytes < plan.bytes) return ADAKV_EWORKSPACE;
  char *wsp = (char *)(((uintptr_t)ws + 255) & ~(uintptr_t)255);
  hipError_t e = launch_select(st, dm, scores, budgets, cu_seqlens, indices,
                               wsp + plan.topk, pipeline_mode(L, dm),
                               (hipStream_t)hip_stream);
  return e == hipSuccess ? ADAKV_OK : ADAKV_EHIP;
}

int adakv_compact(const adakv_layer *L, const void *K, const void *V, const int32_t *indices,
                  const int32_t *cu_seqlens, void *K_out, void *V_out, void *hip_stream) {
  SeqTab st; Dims dm;
  int rc = build_tables(L, st, dm);
  if (rc != ADAKV_OK) return rc;
  if (!K || !V || !indices || !cu_seqlens || !K_out || !V_out) return ADAKV_EINVAL;
  if (!aligned16(K) || !aligned16(V) || !aligned16(K_out) || !aligned16(V_out))
    return ADAKV_EUNSUPPORTED;
  hipError_t e = launch_compact(st, dm, L->dtype, K, V, indices, cu_seqlens, K_out, V_out, 0,
                                nullptr, (hipStream_t)hip_stream);
  return e == hipSuccess ? ADAKV_OK : ADAKV_EHIP;
}

int adakv_compress(const adakv_layer *L, const void *q_window, const void *K, const void *V,
                   const float *row_lse, float *scores, int32_t *budgets, int32_t *cu_seqlens,
                   int32_t *indices, void *K_out, void *V_out, void *ws, size_t ws_bytes,
                   void *hip_stream) {
  // every argument is checked before the first kernel is enqueued
  SeqTab st; Dims dm;
  int rc = build_tables(L, st, dm);
  if (rc != ADAKV_OK) return rc;
  if (!q_window || !K || !V || !scores || !budgets || !cu_seqlens || !indices || !K_out || !V_out)
    return ADAKV_EINVAL;
  if (!aligned16(q_window) || !aligned16(K) || !aligned16(V) || !aligned16(scores) ||
      !aligned16(K_out) || !aligned16(V_out))
    return ADAKV_EUNSUPPORTED;
  if (pool_first(L) && dm.pool_k / 2 > 100) return ADAKV_EUNSUPPORTED;
  const Plan plan = make_plan(st, dm, L);
  if (!ws || ws_bytes < plan.bytes) return ADAKV_EWORKSPACE;
  adakv_layer P = *L;
  P.flags |= ADAKV_FLAG_PIPELINE;
  if ((rc = adakv_score(&P, q_window, K, row_lse, scores, ws, ws_bytes, hip_stream)) != ADAKV_OK) return rc;
  char *wsp = (char *)(((uintptr_t)ws + 255) & ~(uintptr_t)255);
  if (launch_topk(st, dm, scores, budgets, cu_seqlens, indices, wsp + plan.topk,
                  pipeline_mode(&P, dm), wsp, plan.topk, (hipStream_t)hip_stream) != hipSuccess)
    return ADAKV_EHIP;
  return adakv_compact(&P, K, V, indices, cu_seqlens, K_out, V_out, hip_stream);
}

// ---- the whole step without a workspace argument ------------------------------------------------
int adakv_compress_static(const adakv_layer *L, const void *q_window, const void *K, const void *V,
                          const float *row_lse, float *scores, int32_t *budgets,
                          int32_t *cu_seqlens, int32_t *indices, void *K_out, void *V_out,
                          void *hip_stream) {
  SeqTab st; Dims dm;
  int rc = build_tables(L, st, dm);
  if (rc != ADAKV_OK) return rc;
  if (make_plan(st, dm, L).bytes > (size_t)ADAKV_STATIC_SCRATCH_BYTES) return ADAKV_ESCRATCH;
  void *ws = static_scratch();
  if (!ws) return ADAKV_EHIP;
  return adakv_compress(L, q_window, K, V, row_lse, scores, budgets, cu_seqlens, indices, K_out,
                        V_out, ws, ADAKV_STATIC_SCRATCH_BYTES, hip_stream);
}

struct Range { const void *at; size_t bytes; };
static bool overlap(const Range &a, const Range &b) {
  const uintptr_t x = (uintptr_t)a.at, y = (uintptr_t)b.at;
  return a.at && b.at && x < y + b.bytes && y < x + a.bytes;
}

// ---- decode side ------------------------------------------------------------------------------
static int check_headroom(const SeqTab &st, const Dims &dm, int32_t headroom) {
  if (headroom < 0) return ADAKV_EINVAL;
  const long long rows = (long long)st.out_off[st.batch] + (long long)st.batch * dm.h_kv * headroom;
  return rows < (1ll << 31) ? ADAKV_OK : ADAKV_EUNSUPPORTED;
}

int adakv_cache_build(const adakv_layer *L, const void *K, const void *V, const int32_t *indices,
                      const int32_t *cu_seqlens, int32_t headroom, void *K_cache, void *V_cache,
                      int32_t *seg_len, void *hip_stream) {
  SeqTab st; Dims dm;
  int rc = build_tables(L, st, dm);
  if (rc != ADAKV_OK) return rc;
  if ((rc = check_headroom(st, dm, headroom)) != ADAKV_OK) return rc;
  if (!K || !V || !indices || !cu_seqlens || !K_cache || !V_cache || !seg_len) return ADAKV_EINVAL;
  if (!aligned16(K) || !aligned16(V) || !aligned16(K_cache) || !aligned16(V_cache))
    return ADAKV_EUNSUPPORTED;
  hipError_t e = launch_compact(st, dm, L->dtype, K, V, indices, cu_seqlens, K_cache, V_cache,
                                headroom, seg_len, (hipStream_t)hip_stream);
  return e == hipSuccess ? ADAKV_OK : ADAKV_EHIP;
}

int adakv_append(const adakv_layer *L, const void *k_new, const void *v_new,
                 const int32_t *cu_seqlens, int32_t headroom, void *K_cache, void *V_cache,
                 int32_t *seg_len, int32_t *overflow, void *hip_stream) {
  SeqTab st; Dims dm;
  int rc = build_tables(L, st, dm);
  if (rc != ADAKV_OK) return rc;
  if ((rc = check_headroom(st, dm, headroom)) != ADAKV_OK) return rc;
  if (!k_new || !v_new || !cu_seqlens || !K_cache || !V_cache || !seg_len) return ADAKV_EINVAL;
  if (!aligned16(k_new) || !aligned16(v_new) || !aligned16(K_cache) || !aligned16(V_cache))
    return ADAKV_EUNSUPPORTED;
  hipError_t e = launch_append(st, dm, L->dtype, headroom, k_new, v_new, cu_seqlens, K_cache,
                               V_cache, seg_len, overflow, (hipStream_t)hip_stream);
  return e == hipSuccess ? ADAKV_OK : ADAKV_EHIP;
}

size_t adakv_decode_workspace_bytes(const adakv_layer *L, int32_t headroom) {
  SeqTab st; Dims dm;
  if (build_tables(L, st, dm) != ADAKV_OK || check_headroom(st, dm, headroom) != ADAKV_OK) return 0;
  if (!decode_supported(dm)) return 0;
  return plan_decode(st, dm, L->dtype, headroom).total + 256;
}

int adakv_decode_attn(const adakv_layer *L, const void *q_new, const int32_t *cu_seqlens,
                      int32_t headroom, const void *K_cache, const void *V_cache,
                      const int32_t *seg_len, float *out, float *lse, void *ws, size_t ws_bytes,
                      void *hip_stream) {
  SeqTab st; Dims dm;
  int rc = build_tables(L, st, dm);
  if (rc != ADAKV_OK) return rc;
  if ((rc = check_headroom(st, dm, headroom)) != ADAKV_OK) return rc;
  if (!q_new || !cu_seqlens || !K_cache || !V_cache || !seg_len || !out) return ADAKV_EINVAL;
  if (!decode_supported(dm)) return ADAKV_EUNSUPPORTED;
  if (!aligned16(q_new) || !aligned16(K_cache) || !aligned16(V_cache)) return ADAKV_EUNSUPPORTED;
  if (!ws || ws_bytes < plan_decode(st, dm, L->dtype, headroom).total + 256) return ADAKV_EWORKSPACE;
  char *wsp = (char *)(((uintptr_t)ws + 255) & ~(uintptr_t)255);
  hipError_t e = launch_decode_attn(st, dm, L->dtype, headroom, q_new, nullptr, nullptr,
                                    cu_seqlens, (void *)K_cache, (void *)V_cache,
                                    (int *)seg_len, nullptr, out, lse, wsp,
                                    (hipStream_t)hip_stream);
  return e == hipSuccess ? ADAKV_OK : ADAKV_EHIP;
}

int adakv_decode_step(const adakv_layer *L, const void *q_new, const void *k_new,
                      const void *v_new, const int32_t *cu_seqlens, int32_t headroom,
                      void *K_cache, void *V_cache, int32_t *seg_len, int32_t *overflow,
                      float *out, float *lse, void *ws, size_t ws_bytes, void *hip_stream) {
  SeqTab st; Dims dm;
  int rc = build_tables(L, st, dm);
  if (rc != ADAKV_OK) return rc;
  if ((rc = check_headroom(st, dm, headroom)) != ADAKV_OK) return rc;
  if (!q_new || !k_new || !v_new || !cu_seqlens || !K_cache || !V_cache || !seg_len || !out)
    return ADAKV_EINVAL;
  if (!decode_supported(dm)) return ADAKV_EUNSUPPORTED;
  if (!aligned16(q_new) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(K_cache) ||
      !aligned16(V_cache))
    return ADAKV_EUNSUPPORTED;
  if (!ws || ws_bytes < plan_decode(st, dm, L->dtype, headroom).total + 256) return ADAKV_EWORKSPACE;
  char *wsp = (char *)(((uintptr_t)ws + 255) & ~(uintptr_t)255);
  hipError_t e = launch_decode_attn(st, dm, L->dtype, headroom, q_new, k_new, v_new, cu_seqlens,
                                    K_cache, V_cache, seg_len, overflow, out, lse, wsp,
                                    (hipStream_t)hip_stream);
  return e == hipSuccess ? ADAKV_OK : ADAKV_EHIP;
}

// ---- attention limited to a window and sinks ------------------------------------------------------
int adakv_window_attn(const adakv_layer *L, const void *q, int64_t q_stride_tok, int64_t q_stride_head,
                      const void *K, const void *V, int32_t window, int32_t sinks, void *out,
                      float *row_lse, void *hip_stream) {
  SeqTab st; Dims dm;
  int rc = build_tables(L, st, dm);
  if (rc != ADAKV_OK) return rc;
  if (window < 1 || sinks < 0 || q_stride_tok < L->d || q_stride_head < L->d) return ADAKV_EINVAL;
  // a launch holds fewer than 2^32 threads: workgroups of 256, one for 128 rows of a head (sharing is for few)
  long long blocks = 0;
  for (int b = 0; b < st.batch; ++b) {
    const long long rows = (long long)st.n[b] + dm.w;
    if (rows > (1 << 28)) return ADAKV_EUNSUPPORTED;
    blocks += (rows + 127) / 128;
  }
  if (blocks * dm.h_q >= (1 << 24)) return ADAKV_EUNSUPPORTED;
  if (!q || !K || !V || !out) return ADAKV_EINVAL;
  const int esz = L->dtype == ADAKV_FP32 ? 4 : 2;
  if (q_stride_tok * esz % 16 != 0 || q_stride_head * esz % 16 != 0) return ADAKV_EUNSUPPORTED;
  if (!aligned16(q) || !aligned16(K) || !aligned16(V) || !aligned16(out)) return ADAKV_EUNSUPPORTED;
  // (a tile has up to 128 rows, whose offsets are below 2^31)
  if (L->k_stride_tok >= (1 << 24) / esz || L->v_stride_tok >= (1 << 24) / esz) return ADAKV_EUNSUPPORTED;
  hipError_t e = launch_window_attn(st, dm, L->dtype, q, q_stride_tok, q_stride_head, K, V, window, sinks, out, row_lse,
                                    (hipStream_t)hip_stream);
  return e == hipSuccess ? ADAKV_OK : ADAKV_EHIP;
}

// (both forms; k_new == NULL: attention only)
static int decode_window(const adakv_layer *L, const void *q_new, const void *k_new, const void *v_new, const int32_t *cu_seqlens,
                         int32_t headroom, void *K_cache, void *V_cache, int32_t *seg_len, int32_t *overflow, int32_t window,
                         int32_t sinks, float *out, float *lse, void *ws, size_t ws_bytes, void *hip_stream) {
  SeqTab st; Dims dm;
  int rc = build_tables(L, st, dm);
  if (rc != ADAKV_OK) return rc;
  if ((rc = check_headroom(st, dm, headroom)) != ADAKV_OK) return rc;
  if (window < 1 || sinks < 0) return ADAKV_EINVAL;
  if (!q_new || !cu_seqlens || !K_cache || !V_cache || !seg_len || !out) return ADAKV_EINVAL;
  if (!decode_supported(dm)) return ADAKV_EUNSUPPORTED;
  if (!aligned16(q_new) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(K_cache) || !aligned16(V_cache))
    return ADAKV_EUNSUPPORTED;
  if (!ws || ws_bytes < plan_decode(st, dm, L->dtype, headroom).total + 256) return ADAKV_EWORKSPACE;
  char *wsp = (char *)(((uintptr_t)ws + 255) & ~(uintptr_t)255);
  const long long limit = (long long)window + sinks;
  hipError_t e = launch_decode_window(st, dm, L->dtype, headroom, limit < INT_MAX ? (int)limit : INT_MAX, sinks, q_new, k_new, v_new,
                                      cu_seqlens, K_cache, V_cache, seg_len, overflow, out, lse, wsp, (hipStream_t)hip_stream);
  return e == hipSuccess ? ADAKV_OK : ADAKV_EHIP;
}

int adakv_decode_window_attn(const adakv_layer *L, const void *q_new, const int32_t *cu_seqlens,
                             int32_t headroom, const void *K_cache, const void *V_cache,
                             const int32_t *seg_len, int32_t window, int32_t sinks, float *out,
                             float *lse, void *ws, size_t ws_bytes, void *hip_stream) {
  return decode_window(L, q_new, nullptr, nullptr, cu_seqlens, headroom, (void *)K_cache, (void *)V_cache, (int32_t *)seg_len,
                       nullptr, window, sinks, out, lse, ws, ws_bytes, hip_stream);
}

int adakv_decode_window_step(const adakv_layer *L, const void *q_new, const void *k_new,
                             const void *v_new, const int32_t *cu_seqlens, int32_t headroom,
                             void *K_cache, void *V_cache, int32_t *seg_len, int32_t *overflow,
                             int32_t window, int32_t sinks, float *out, float *lse, void *ws,
                             size_t ws_bytes, void *hip_stream) {
  if (!k_new || !v_new) return ADAKV_EINVAL;
  return decode_window(L, q_new, k_new, v_new, cu_seqlens, headroom, K_cache, V_cache, seg_len, overflow, window, sinks, out, lse,
                       ws, ws_bytes, hip_stream);
}

// ---- a decoding step over shared caches ---------------------------------------------------------------
// The layer's and the shared caches' tables, and what follows from both.
struct PrefixTables {
  SeqTab st, shared;
  Dims dm, shared_dm;
  Sharing sh;
  PrefixPlan plan;
};
static int prefix_tables(const adakv_layer *L, int32_t headroom, const adakv_prefix *P, PrefixTables &t) {
  int rc = build_tables(L, t.st, t.dm);
  if (rc != ADAKV_OK) return rc;
  if ((rc = check_headroom(t.st, t.dm, headroom)) != ADAKV_OK) return rc;
  if (!P || !P->L || !P->of) return ADAKV_EINVAL;
  if ((rc = build_tables(P->L, t.shared, t.shared_dm)) != ADAKV_OK) return rc;
  if ((rc = check_headroom(t.shared, t.shared_dm, P->headroom)) != ADAKV_OK) return rc;
  if (P->L->dtype != L->dtype || P->L->h_q != L->h_q || P->L->h_kv != L->h_kv || P->L->d != L->d) return ADAKV_EINVAL;
  for (int b = 0; b < t.st.batch; ++b)
    if (P->of[b] < -1 || P->of[b] >= t.shared.batch) return ADAKV_EINVAL;
  if (!decode_supported(t.dm)) return ADAKV_EUNSUPPORTED;
  t.sh = share(t.st, t.dm, t.shared.batch, P->of);
  t.plan = plan_prefix(t.st, t.dm, L->dtype, headroom, t.sh);
  return ADAKV_OK;
}

size_t adakv_prefix_workspace_bytes(const adakv_layer *L, int32_t headroom, const adakv_prefix *P) {
  PrefixTables t;
  return prefix_tables(L, headroom, P, t) == ADAKV_OK ? t.plan.total + 256 : 0;
}

// (both forms; k_new == NULL: attention only)
static int decode_prefix(const adakv_layer *L, const void *q_new, const void *k_new, const void *v_new, const int32_t *cu_seqlens,
                         int32_t headroom, void *K_cache, void *V_cache, int32_t *seg_len, int32_t *overflow, const adakv_prefix *P,
                         float *out, float *lse, void *ws, size_t ws_bytes, void *hip_stream) {
  PrefixTables t;
  const int rc = prefix_tables(L, headroom, P, t);
  if (rc == ADAKV_EINVAL) return rc;
  if (!q_new || !cu_seqlens || !K_cache || !V_cache || !seg_len || !out) return ADAKV_EINVAL;
  if (!P->cu_seqlens || !P->K_cache || !P->V_cache || !P->seg_len) return ADAKV_EINVAL;
  if (rc != ADAKV_OK) return rc;
  if (!aligned16(q_new) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(K_cache) || !aligned16(V_cache) ||
      !aligned16(P->K_cache) || !aligned16(P->V_cache))
    return ADAKV_EUNSUPPORTED;
  if (k_new) {
    const size_t row = (size_t)t.dm.d * (L->dtype == ADAKV_FP32 ? 4 : 2), heads = (size_t)t.dm.h_kv;
    const size_t own = (t.st.out_off[t.st.batch] + t.st.batch * heads * headroom) * row;
    const size_t theirs = (t.shared.out_off[t.shared.batch] + t.shared.batch * heads * P->headroom) * row;
    for (const void *x : {(const void *)K_cache, (const void *)V_cache})
      for (const void *y : {P->K_cache, P->V_cache})
        if (overlap({x, own}, {y, theirs})) return ADAKV_EINVAL;
    if (overlap({seg_len, t.st.batch * heads * sizeof(int32_t)}, {P->seg_len, t.shared.batch * heads * sizeof(int32_t)})) return ADAKV_EINVAL;
  }
  if (!ws || ws_bytes < t.plan.total + 256) return ADAKV_EWORKSPACE;
  char *wsp = (char *)(((uintptr_t)ws + 255) & ~(uintptr_t)255);
  const Segments shared = {(const char *)P->K_cache, (const char *)P->V_cache, P->cu_seqlens, P->seg_len, P->headroom};
  const Segments own = {(const char *)K_cache, (const char *)V_cache, cu_seqlens, seg_len, headroom};
  hipError_t e = launch_decode_prefix(t.dm, L->dtype, t.plan, t.sh, shared, own, q_new, k_new, v_new, seg_len, overflow, out, lse, wsp,
                                      (hipStream_t)hip_stream);
  return e == hipSuccess ? ADAKV_OK : ADAKV_EHIP;
}

int adakv_decode_prefix_attn(const adakv_layer *L, const void *q_new, const int32_t *cu_seqlens, int32_t headroom, const void *K_cache,
                             const void *V_cache, const int32_t *seg_len, const adakv_prefix *P, float *out, float *lse, void *ws,
                             size_t ws_bytes, void *hip_stream) {
  return decode_prefix(L, q_new, nullptr, nullptr, cu_seqlens, headroom, (void *)K_cache, (void *)V_cache, (int32_t *)seg_len, nullptr, P,
                       out, lse, ws, ws_bytes, hip_stream);
}

int adakv_decode_prefix_step(const adakv_layer *L, const void *q_new, const void *k_new, const void *v_new, const int32_t *cu_seqlens,
                             int32_t headroom, void *K_cache, void *V_cache, int32_t *seg_len, int32_t *overflow, const adakv_prefix *P,
                             float *out, float *lse, void *ws, size_t ws_bytes, void *hip_stream) {
  if (!k_new || !v_new) return ADAKV_EINVAL;
  return decode_prefix(L, q_new, k_new, v_new, cu_seqlens, headroom, K_cache, V_cache, seg_len, overflow, P, out, lse, ws, ws_bytes,
                       hip_stream);
}

// ---- rotary positions and head norms ----------------------------------------------------------------
int adakv_rotary_frequencies(int32_t dims, double base, int32_t scaling, double factor, int32_t original_len, double low, double high,
                             double *freq) {
  if (!freq || dims < 2 || dims % 2 != 0 || !(base > 0.0) || isinf(base)) return ADAKV_EINVAL;
  if (scaling < ADAKV_ROTARY_PLAIN || scaling > ADAKV_ROTARY_PARTS) return ADAKV_EINVAL;
  if (scaling != ADAKV_ROTARY_PLAIN && (!(factor >= 1.0) || isinf(factor))) return ADAKV_EINVAL;
  if (scaling == ADAKV_ROTARY_PARTS && (original_len < 1 || !(low >= 0.0) || !(high > low) || isinf(high))) return ADAKV_EINVAL;
  if (dims > 128) return ADAKV_EUNSUPPORTED;
  if (scaling == ADAKV_ROTARY_BASE && dims > 2) base *= pow(factor, dims / (dims - 2.0));
  if (isinf(base) || isinf(pow(base, 2.0 / dims - 1.0))) return ADAKV_EINVAL;        // (of a base below 1 the last frequency is the largest)
  for (int i = 0; i < dims / 2; ++i) {
    const double f = pow(base, -2.0 * i / dims);
    double by = 1.0;
    if (scaling == ADAKV_ROTARY_LINEAR) by = 1.0 / factor;
    if (scaling == ADAKV_ROTARY_PARTS) {
      const double u = (original_len * f / 6.283185307179586477 - low) / (high - low), share = u < 0.0 ? 0.0 : u > 1.0 ? 1.0 : u;
      by = share + (1.0 - share) / factor;
    }
    freq[i] = f * by;
  }
  return ADAKV_OK;
}

// An input and its output, of `rows` rows of `count` heads.
static int check_heads(const adakv_heads *x, const adakv_heads *o, long long rows, int count, int d, int esz) {
  if (!x->x || !o->x) return ADAKV_EINVAL;
  const int64_t strides[4] = {x->stride_tok, x->stride_head, o->stride_tok, o->stride_head};
  for (int64_t sd : strides)
    if (sd < d || sd > (1ll << 40)) return ADAKV_EINVAL;
  const __int128 tok = o->stride_tok, head = o->stride_head;
  if (tok < (count - 1) * head + d && head < (rows - 1) * tok + d) return ADAKV_EINVAL;
  if (x->x == o->x && (x->stride_tok != o->stride_tok || x->stride_head != o->stride_head)) return ADAKV_EINVAL;
  if (!aligned16(x->x) || !aligned16(o->x)) return ADAKV_EUNSUPPORTED;
  for (int64_t sd : strides)
    if (sd * esz % 16 != 0) return ADAKV_EUNSUPPORTED;
  return ADAKV_OK;
}

// From its first byte to its last (as far as there are addresses).
static Range reach_of(const adakv_heads *x, long long rows, int count, int d, int esz) {
  if (!x || rows < 1) return {nullptr, 0};
  const wide bytes = ((wide)(rows - 1) * x->stride_tok + (wide)(count - 1) * x->stride_head + d) * esz, most = UINTPTR_MAX - (uintptr_t)x->x;
  return {x->x, (size_t)(bytes < most ? bytes : most)};
}

// Whether an output has memory of another tensor of the call, which is rows of `x_count` heads or, with x_count == 0, `piece` bytes at x->x.
// `rows` rows; without positions only st's sequences' count.
static int check_apart(const SeqTab &st, const Dims &dm, long long rows, bool positions, int esz, const adakv_heads *o, int o_count,
                       const adakv_heads *x, int x_count, long long piece = 0) {
  const auto places = [&](const adakv_heads *t, int count, long long from, long long n) {
    if (count == 0) return Places((uintptr_t)t->x, piece);
    const long long tok = t->stride_tok * esz, head = t->stride_head * esz;
    return Places((uintptr_t)t->x + (uintptr_t)from * (uintptr_t)tok, (long long)dm.d * esz, {n, tok}, {count, head});
  };
  if (x_count && o->stride_tok == x->stride_tok) {             // parts of one tensor's rows: their places within a row tell
    const bool o_first = (uintptr_t)o->x <= (uintptr_t)x->x;
    const uintptr_t tok = (uintptr_t)(o->stride_tok * esz), apart = o_first ? (uintptr_t)x->x - (uintptr_t)o->x : (uintptr_t)o->x - (uintptr_t)x->x;
    const wide o_row = ((wide)(o_count - 1) * o->stride_head + dm.d) * esz, x_row = ((wide)(x_count - 1) * x->stride_head + dm.d) * esz;
    if ((o_first ? o_row : x_row) <= apart % tok && apart % tok + (o_first ? x_row : o_row) <= tok) return ADAKV_OK;
  }
  const auto said = [](Meet m) { return m == Meet::NO ? ADAKV_OK : m == Meet::YES ? ADAKV_EINVAL : ADAKV_EUNSUPPORTED; };
  const Meet all = meet_places(places(o, o_count, 0, rows), places(x, x_count, 0, rows));
  if (all == Meet::NO || positions) return said(all);
  // what meets may be rows of no sequence: once more by the runs of sequences one behind the other
  long long from[ADAKV_MAX_BATCH], n[ADAKV_MAX_BATCH];
  int runs = 0;
  for (int b = 0; b < st.batch; ++b) {
    const long long mine = (long long)st.n[b] + dm.w;
    if (runs && from[runs - 1] + n[runs - 1] == st.tok_off[b]) n[runs - 1] += mine;
    else from[runs] = st.tok_off[b], n[runs++] = mine;
  }
  for (int i = 0; i < runs; ++i)
    for (int j = 0; j < (x_count ? runs : 1); ++j) {
      const Meet m = meet_places(places(o, o_count, from[i], n[i]), places(x, x_count, from[j], n[j]));
      if (m != Meet::NO) return said(m);
    }
  return ADAKV_OK;
}

// (both forms)
static int rotary(const adakv_layer *L, const adakv_rotation *R, int64_t rows, const int32_t *positions, const adakv_heads *q,
                  const adakv_heads *k, const adakv_heads *q_out, const adakv_heads *k_out, bool norm, const void *q_weight,
                  const void *k_weight, float eps, void *hip_stream) {
  SeqTab st; Dims dm;
  int rc = build_tables(L, st, dm);
  if (rc != ADAKV_OK) return rc;
  if (!R || (R->layout != ADAKV_ROTARY_HALF && R->layout != ADAKV_ROTARY_INTERLEAVED)) return ADAKV_EINVAL;
  if (R->dims < 0 || R->dims % 2 != 0 || R->dims > L->d || (R->dims > 0 && !R->freq)) return ADAKV_EINVAL;
  if (!(R->magnitude >= 0.0f) || isinf(R->magnitude)) return ADAKV_EINVAL;
  if ((!q && !k) || !q != !q_out || !k != !k_out) return ADAKV_EINVAL;
  if (norm && ((q && !q_weight) || (k && !k_weight) || !(eps >= 0.0f) || isinf(eps))) return ADAKV_EINVAL;
  long long all = 0, reach = rows;             // rows; one past the last one
  if (positions) {
    if (rows < 0) return ADAKV_EINVAL;
    all = rows;
  } else {
    reach = 0;
    for (int b = 0; b < st.batch; ++b) {
      const long long mine = (long long)st.n[b] + dm.w, end = st.tok_off[b] + mine;
      all += mine;
      reach = end > reach ? end : reach;
    }
  }
  if (all > (1 << 30) || reach > (1ll << 40)) return ADAKV_EUNSUPPORTED;
  const int esz = L->dtype == ADAKV_FP32 ? 4 : 2;
  if (q && (rc = check_heads(q, q_out, reach, dm.h_q, dm.d, esz)) != ADAKV_OK) return rc;
  if (k && (rc = check_heads(k, k_out, reach, dm.h_kv, dm.d, esz)) != ADAKV_OK) return rc;
  // outputs against all else: by where they begin and end, and only if these meet, place by place
  const Range ends[4] = {reach_of(q, reach, dm.h_q, dm.d, esz), reach_of(k, reach, dm.h_kv, dm.d, esz), reach_of(q_out, reach, dm.h_q, dm.d, esz),
                         reach_of(k_out, reach, dm.h_kv, dm.d, esz)};
  const adakv_heads *const all_heads[4] = {q, k, q_out, k_out};
  for (int o = 2; o < 4 && rc == ADAKV_OK; ++o) {
    const int o_count = o == 2 ? dm.h_q : dm.h_kv;
    for (int x = 0; x < o && rc == ADAKV_OK; ++x)
      if (overlap(ends[o], ends[x]) && !(x == o - 2 && ends[x].at == ends[o].at))      // (an output at its input's address has its places)
        rc = check_apart(st, dm, reach, positions != nullptr, esz, all_heads[o], o_count, all_heads[x], x % 2 == 0 ? dm.h_q : dm.h_kv);
    const Range pieces[4] = {{positions, positions ? (size_t)rows * sizeof(int32_t) : 0}, {R->freq, (size_t)(R->dims / 2) * sizeof(double)},
                             {q_weight, norm && q ? (size_t)dm.d * esz : 0}, {k_weight, norm && k ? (size_t)dm.d * esz : 0}};
    for (const Range &x : pieces)
      if (rc == ADAKV_OK && x.bytes && overlap(ends[o], x)) {
        const adakv_heads at = {const_cast<void *>(x.at), 0, 0};
        rc = check_apart(st, dm, reach, positions != nullptr, esz, all_heads[o], o_count, &at, 0, (long long)x.bytes);
      }
  }
  if (rc != ADAKV_OK) return rc;
  if (norm && (!aligned16(q_weight) || !aligned16(k_weight))) return ADAKV_EUNSUPPORTED;
  if (((uintptr_t)R->freq & 7u) != 0 || ((uintptr_t)positions & 3u) != 0) return ADAKV_EUNSUPPORTED;
  hipError_t e = launch_rotary(st, dm, L->dtype, *R, (int)all, positions, q, k, q_out, k_out, norm, q_weight, k_weight, eps,
                               (hipStream_t)hip_stream);
  return e == hipSuccess ? ADAKV_OK : ADAKV_EHIP;
}

int adakv_rotary(const adakv_layer *L, const adakv_rotation *R, int64_t rows, const int32_t *positions, const adakv_heads *q,
                 const adakv_heads *k, const adakv_heads *q_out, const adakv_heads *k_out, void *hip_stream) {
  return rotary(L, R, rows, positions, q, k, q_out, k_out, false, nullptr, nullptr, 0.0f, hip_stream);
}

int adakv_norm_rotary(const adakv_layer *L, const adakv_rotation *R, int64_t rows, const int32_t *positions, const adakv_heads *q,
                      const adakv_heads *k, const void *q_weight, const void *k_weight, float eps, const adakv_heads *q_out,
                      const adakv_heads *k_out, void *hip_stream) {
  return rotary(L, R, rows, positions, q, k, q_out, k_out, true, q_weight, k_weight, eps, hip_stream);
}

// ---- the cache in 8 bits --------------------------------------------------------------------------
size_t adakv_q8_scales(const adakv_layer *L, int32_t headroom) {
  SeqTab st; Dims dm;
  if (build_tables(L, st, dm) != ADAKV_OK || check_headroom(st, dm, headroom) != ADAKV_OK) return 0;
  return (size_t)q8_scales(st, dm, headroom);
}

int adakv_cache_build_q8(const adakv_layer *L, const void *K, const void *V,
                         const int32_t *indices, const int32_t *cu_seqlens, int32_t headroom,
                         void *K_q8, void *V_q8, float *k_scale, float *v_scale, int32_t *seg_len,
                         void *hip_stream) {
  SeqTab st; Dims dm;
  int rc = build_tables(L, st, dm);
  if (rc != ADAKV_OK) return rc;
  if ((rc = check_headroom(st, dm, headroom)) != ADAKV_OK) return rc;
  // a launch holds fewer than 2^32 threads: workgroups of 256 for two blocks
  if (st.out_off[st.batch] > 1000000000) return ADAKV_EUNSUPPORTED;
  if (!K || !V || !indices || !cu_seqlens || !K_q8 || !V_q8 || !k_scale || !v_scale || !seg_len) return ADAKV_EINVAL;
  if (!aligned16(K) || !aligned16(V) || !aligned16(K_q8) || !aligned16(V_q8)) return ADAKV_EUNSUPPORTED;
  hipError_t e = launch_cache_build_q8(st, dm, L->dtype, K, V, indices, cu_seqlens, headroom,
                                       {(char *)K_q8, (char *)V_q8, k_scale, v_scale}, seg_len, (hipStream_t)hip_stream);
  return e == hipSuccess ? ADAKV_OK : ADAKV_EHIP;
}

int adakv_append_q8(const adakv_layer *L, const void *k_new, const void *v_new,
                    const int32_t *cu_seqlens, int32_t headroom, void *K_q8, void *V_q8,
                    float *k_scale, float *v_scale, int32_t *seg_len, int32_t *overflow,
                    void *hip_stream) {
  SeqTab st; Dims dm;
  int rc = build_tables(L, st, dm);
  if (rc != ADAKV_OK) return rc;
  if ((rc = check_headroom(st, dm, headroom)) != ADAKV_OK) return rc;
  if (!k_new || !v_new || !cu_seqlens || !K_q8 || !V_q8 || !k_scale || !v_scale || !seg_len) return ADAKV_EINVAL;
  if (!aligned16(k_new) || !aligned16(v_new) || !aligned16(K_q8) || !aligned16(V_q8)) return ADAKV_EUNSUPPORTED;
  hipError_t e = launch_append_q8(st, dm, L->dtype, headroom, k_new, v_new, cu_seqlens,
                                  {(char *)K_q8, (char *)V_q8, k_scale, v_scale}, seg_len, overflow, (hipStream_t)hip_stream);
  return e == hipSuccess ? ADAKV_OK : ADAKV_EHIP;
}

// (both forms; k_new == NULL: attention only)
static int decode_q8(const adakv_layer *L, const void *q_new, const void *k_new, const void *v_new, const int32_t *cu_seqlens,
                     int32_t headroom, const Q8Cache &c, int32_t *seg_len, int32_t *overflow, float *out, float *lse, void *ws,
                     size_t ws_bytes, void *hip_stream) {
  SeqTab st; Dims dm;
  int rc = build_tables(L, st, dm);
  if (rc != ADAKV_OK) return rc;
  if ((rc = check_headroom(st, dm, headroom)) != ADAKV_OK) return rc;
  if (!q_new || !cu_seqlens || !c.K || !c.V || !c.k_scale || !c.v_scale || !seg_len || !out) return ADAKV_EINVAL;
  if (!decode_supported(dm)) return ADAKV_EUNSUPPORTED;
  if (!aligned16(q_new) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(c.K) || !aligned16(c.V)) return ADAKV_EUNSUPPORTED;
  if (!ws || ws_bytes < plan_decode(st, dm, L->dtype, headroom).total + 256) return ADAKV_EWORKSPACE;
  char *wsp = (char *)(((uintptr_t)ws + 255) & ~(uintptr_t)255);
  hipError_t e = launch_decode_q8(st, dm, L->dtype, headroom, q_new, k_new, v_new, cu_seqlens, c, seg_len, overflow, out, lse, wsp,
                                  (hipStream_t)hip_stream);
  return e == hipSuccess ? ADAKV_OK : ADAKV_EHIP;
}

int adakv_decode_attn_q8(const adakv_layer *L, const void *q_new, const int32_t *cu_seqlens,
                         int32_t headroom, const void *K_q8, const void *V_q8,
                         const float *k_scale, const float *v_scale, const int32_t *seg_len,
                         float *out, float *lse, void *ws, size_t ws_bytes, void *hip_stream) {
  return decode_q8(L, q_new, nullptr, nullptr, cu_seqlens, headroom, {(char *)K_q8, (char *)V_q8, (float *)k_scale, (float *)v_scale},
                   (int32_t *)seg_len, nullptr, out, lse, ws, ws_bytes, hip_stream);
}

int adakv_decode_step_q8(const adakv_layer *L, const void *q_new, const void *k_new,
                         const void *v_new, const int32_t *cu_seqlens, int32_t headroom,
                         void *K_q8, void *V_q8, float *k_scale, float *v_scale, int32_t *seg_len,
                         int32_t *overflow, float *out, float *lse, void *ws, size_t ws_bytes,
                         void *hip_stream) {
  if (!k_new || !v_new) return ADAKV_EINVAL;
  return decode_q8(L, q_new, k_new, v_new, cu_seqlens, headroom, {(char *)K_q8, (char *)V_q8, k_scale, v_scale}, seg_len, overflow,
                   out, lse, ws, ws_bytes, hip_stream);
}

// ---- sequences of a cache, moved --------------------------------------------------------------------
// (both forms; a cache in 8 bits has scales)
static int cache_move(const adakv_layer *L, int32_t count, const int32_t *from, const int32_t *cu_seqlens, int32_t headroom,
                      const Q8Cache &c, const int32_t *seg_len, int32_t headroom_out, int32_t *cu_out, const Q8Cache &o,
                      int32_t *len_out, int32_t *overflow, void *hip_stream) {
  SeqTab st; Dims dm;
  int rc = build_tables(L, st, dm);
  if (rc != ADAKV_OK) return rc;
  if ((rc = check_headroom(st, dm, headroom)) != ADAKV_OK) return rc;
  if (!from || count < 1 || count > ADAKV_MAX_BATCH || headroom_out < 0) return ADAKV_EINVAL;
  const bool q8 = c.k_scale != nullptr;
  if (!cu_seqlens || !c.K || !c.V || !seg_len || !cu_out || !o.K || !o.V || !len_out) return ADAKV_EINVAL;
  const long long nseg = (long long)st.batch * dm.h_kv, nseg_out = (long long)count * dm.h_kv;
  const long long rows = st.out_off[st.batch] + nseg * headroom;
  long long rows_out = nseg_out * headroom_out;
  for (int i = 0; i < count; ++i) {
    if (from[i] < 0 || from[i] >= st.batch) return ADAKV_EINVAL;
    rows_out += st.out_off[from[i] + 1] - st.out_off[from[i]];
  }
  if (rows_out >= (1ll << 31)) return ADAKV_EUNSUPPORTED;
  if (!aligned16(c.K) || !aligned16(c.V) || !aligned16(o.K) || !aligned16(o.V)) return ADAKV_EUNSUPPORTED;
  const size_t row = (size_t)dm.d * (q8 ? 1 : L->dtype == ADAKV_FP32 ? 4 : 2);
  const size_t sc = (size_t)(rows / ADAKV_Q8_BLOCK + nseg) * 4, sc_out = (size_t)(rows_out / ADAKV_Q8_BLOCK + nseg_out) * 4;
  const Range in[6] = {{c.K, rows * row}, {c.V, rows * row}, {cu_seqlens, (size_t)(nseg + 1) * 4}, {seg_len, (size_t)nseg * 4},
                       {c.k_scale, sc}, {c.v_scale, sc}};
  const Range res[7] = {{o.K, rows_out * row}, {o.V, rows_out * row}, {cu_out, (size_t)(nseg_out + 1) * 4},
                        {len_out, (size_t)nseg_out * 4}, {o.k_scale, sc_out}, {o.v_scale, sc_out}, {overflow, 4}};
  for (int i = 0; i < 7; ++i) {
    for (const Range &r : in)
      if (overlap(res[i], r)) return ADAKV_EINVAL;
    for (int j = 0; j < i; ++j)
      if (overlap(res[i], res[j])) return ADAKV_EINVAL;
  }
  hipError_t e = launch_cache_move(st, dm, (int)row, count, from, cu_seqlens, headroom, c.K, c.V, c.k_scale, c.v_scale, seg_len,
                                   headroom_out, cu_out, o.K, o.V, o.k_scale, o.v_scale, len_out, overflow, (hipStream_t)hip_stream);
  return e == hipSuccess ? ADAKV_OK : ADAKV_EHIP;
}

int adakv_cache_move(const adakv_layer *L, int32_t count, const int32_t *from,
                     const int32_t *cu_seqlens, int32_t headroom, const void *K_cache,
                     const void *V_cache, const int32_t *seg_len, int32_t headroom_out,
                     int32_t *cu_out, void *K_out, void *V_out, int32_t *len_out,
                     int32_t *overflow, void *hip_stream) {
  return cache_move(L, count, from, cu_seqlens, headroom, {(char *)K_cache, (char *)V_cache, nullptr, nullptr}, seg_len, headroom_out,
                    cu_out, {(char *)K_out, (char *)V_out, nullptr, nullptr}, len_out, overflow, hip_stream);
}

int adakv_cache_move_q8(const adakv_layer *L, int32_t count, const int32_t *from,
                        const int32_t *cu_seqlens, int32_t headroom, const void *K_q8,
                        const void *V_q8, const float *k_scale, const float *v_scale,
                        const int32_t *seg_len, int32_t headroom_out, int32_t *cu_out,
                        void *K_out, void *V_out, float *k_scale_out, float *v_scale_out,
                        int32_t *len_out, int32_t *overflow, void *hip_stream) {
  if (!k_scale || !v_scale || !k_scale_out || !v_scale_out) return ADAKV_EINVAL;
  return cache_move(L, count, from, cu_seqlens, headroom, {(char *)K_q8, (char *)V_q8, (float *)k_scale, (float *)v_scale}, seg_len,
                    headroom_out, cu_out, {(char *)K_out, (char *)V_out, k_scale_out, v_scale_out}, len_out, overflow, hip_stream);
}

int adakv_describe(const adakv_layer *L, int have_row_lse, char *out, size_t out_bytes) {
  SeqTab st; Dims dm;
  int rc = build_tables(L, st, dm);
  if (rc != ADAKV_OK) return rc;
  if (!out || out_bytes == 0) return ADAKV_EINVAL;
  if (pool_first(L) && dm.pool_k / 2 > 100) return ADAKV_EUNSUPPORTED;
  const char *dt = L->dtype == ADAKV_FP32 ? "fp32" : L->dtype == ADAKV_FP16 ? "fp16" : "bf16";
  const char *topk = pipeline_mode(L, dm) ? "carried" : "separate";
  const char *stats = have_row_lse ? "caller" : "sweep";
  int len;
  if (on_mfma(dm, L)) {
    const MfmaVariant v = choose_mfma_variant(st, dm);
    len = snprintf(out, out_bytes,
                   "score=%s dtype=%s d=%d rows=%d mb=%d rs=%d kg=%d chunk=%d keys=%d stat_keys=%d stats=%s lse=%s pool=%s topk=%s",
                   pool_first(L) ? "mfma-pool-first" : "mfma", dt, dm.d, dm.g * dm.w, v.mb, v.rs, v.kg,
                   v.chunk, v.len, v.part_len, stats, have_row_lse ? "caller" : v.fuse_lse ? "fused" : "kernel",
                   pool_first(L) ? "rows" : v.fuse_pool ? "fused" : "kernel", topk);
  } else {
    const int stat_keys = plan_score(st, dm, L->dtype, false).part_chunk;
    len = snprintf(out, out_bytes, "score=%s dtype=%s d=%d rows=%d products=%s stat_keys=%d stats=%s lse=%s pool=%s topk=%s",
                   pool_first(L) ? "fma-pool-first" : "fma", dt, dm.d, dm.g * dm.w,
                   f32_cut(dm, L->dtype) ? "parts" : "fp32", stat_keys, stats,
                   have_row_lse ? "caller"
                   : !pool_first(L) && f32_lse_fused(st, stat_keys) ? "fused" : "kernel",
                   !pool_first(L) && f32_pool_fused(st, dm, L->dtype) ? "fused" : "kernel", topk);
  }
  return (len < 0 || (size_t)len >= out_bytes) ? ADAKV_EINVAL : ADAKV_OK;
}

int adakv_probe_read(const void *src, size_t bytes, void *sink, void *hip_stream) {
  if ((!src && bytes > 0) || !sink || bytes % 16 != 0) return ADAKV_EINVAL;
  if (!aligned16(src) || !aligned16(sink)) return ADAKV_EUNSUPPORTED;
  static_assert(ADAKV_PROBE_SINK_BYTES == ADAKV_PROBE_BLOCKS * 4 * 16, "one word per wave");
  if (probe_waves_per_block() != 4) return ADAKV_EHIP;
  hipError_t e = launch_probe_read(src, (long long)(bytes / 16), sink, ADAKV_PROBE_BLOCKS,
                                   (hipStream_t)hip_stream);
  return e == hipSuccess ? ADAKV_OK : ADAKV_EHIP;
}

}  // extern "C"
