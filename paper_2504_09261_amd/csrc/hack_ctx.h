// The context behind the C ABI and what its entry points share: the error path, the checks of common arguments and the
// report of conditions that kernels found.  Host code only; hack_api.cpp has the steps and their stages, ops_api.cpp the operators around them.
#pragma once

#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <string>

#include "../../include/hack.h"
#include "hack_internal.h"
#include "table_cache.h"

namespace hack {

// Launch-table storage in device memory with a pinned host mirror.
struct HipTableBackend {
  bool alloc(size_t bytes, uint8_t** dev, uint8_t** host) {
    if (hipMalloc((void**)dev, bytes) != hipSuccess) return false;
    if (hipHostMalloc((void**)host, bytes, hipHostMallocDefault) != hipSuccess) {
      (void)hipFree(*dev);
      return false;
    }
    return true;
  }
  void release(uint8_t* dev, uint8_t* host) {
    (void)hipFree(dev);
    (void)hipHostFree(host);
  }
  bool upload(uint8_t* dev, const uint8_t* host, size_t bytes, void* stream) {
    return hipMemcpyAsync(dev, host, bytes, hipMemcpyHostToDevice, static_cast<hipStream_t>(stream)) == hipSuccess;
  }
  bool may_alloc(void* stream) {
    hipStreamCaptureStatus cs = hipStreamCaptureStatusNone;
    (void)hipStreamIsCapturing(static_cast<hipStream_t>(stream), &cs);
    return cs == hipStreamCaptureStatusNone;
  }
};

}  // namespace hack

struct hack_ctx {
  hack_config cfg;
  int elem_bytes = 2;
  // workspace
  float* importance = nullptr;   // [max_units, ws_stride]
  int32_t* kept = nullptr;       // [max_units, ws_stride]
  int32_t* seam = nullptr;       // [max_units] kept rows of the step's selection that come from the cache
  int32_t* iota = nullptr;       // [kIotaRows] 0, 1, 2, ...
  double* f32_logits = nullptr;  // fp32 path: [score_select_f32_max_groups, kF32GroupLogits] logits of short units
  double* stats = nullptr;       // fp32 path: [score_f32_max_groups, 32, 2] softmax partials
  unsigned long long* rowstat = nullptr;  // bf16 path: [max_units, score_groups, 32] row-sum exchange slots, all-ones between launches
  unsigned long long* rowstat_side = nullptr;  // the same for the side branch of hack_step (two-pass form: its slots are not re-armed)
  int score_groups = 0;          // work-groups a unit of max_cache_len keys is scored by
  int spin_limit = 0;            // polls after which a score work-group gives up its wait for the unit's other work-groups
  unsigned* abort_flag = nullptr; // bf16 path: device word behind the counters; set by a fused score launch that gave up
  size_t n_slots = 0;            // 64-bit words in rowstat
  int score_mode = HACK_SCORE_FUSED;   // hack_score_mode: fused single launch / two launches without in-kernel waits
  int skip_publish = -1;         // test hook: work-group of a fused score launch that withholds its sums
  unsigned* counters = nullptr;  // [max_units, 2], zero between launches; bf16 path: reader counters, fp32 path: tickets of short units
  float* hv_stats = nullptr;     // head variance: [max_units, max_queries, 2] softmax statistics of every query
  int32_t* merge_nn = nullptr;   // final-step merge (bf16): [max_units, ws_stride] nearest kept row of every cache row
  float* merge_w = nullptr;      //   ... its weight
  float* merge_inv = nullptr;    //   ... inverse key norms of the kept rows
  int* fault = nullptr;          // pinned, device-visible int[2]: [0] a score wave's bounded wait gave up (fatal),
                                 // [1] a logit exceeded the range the bf16 score kernel supports
  int cus = 1;                   // compute units of the device
  int score_capacity[hack::kScoreSizes] = {};   // bf16 path: score items one fused launch may hold (resident waves), by item size (kScoreItemKeys)
  int split_max_items = -1;      // launches with at most this many 32-query attention items use the key-split kernel (HACK_ATTN_SPLIT_ITEMS); -1 (default): see use_split_attention
  int attn_kernel = -1;          // bf16 kernel of the 128-query items (kAttnPlain ...); -1 (default): the deeper pipeline, keys in halves where use_key_halves says so
  int packed_queries = 0;        // attention over packed caches: queries of a work-group (HACK_ATTN_PACKED_QUERIES: 16, 32 or 128); 0 (default): see queries_per_group
  // streamed form of that kernel: the launch is cut into equal runs of key blocks, one per resident work-group
  int attn_stream = -1;          // HACK_ATTN_STREAM; -1 (default): cut single work items where the pair model gains, 0: never, 1: equal runs
                                 // for every launch of the 128-query kernel, 2: A/B aid, 4: every cut the model likes (see use_stream_attention)
  int attn_slots = 0;            // work-groups of the streamed kernel the device holds at once
  float* part_o = nullptr;       // [2 * attn_slots, 128, head_dim] unnormalised partial outputs (fp32 contexts: [part_rows, head_dim])
  float* part_ml = nullptr;      // [2 * attn_slots, 2, 128] their references and normalisers ([part_rows, 2])
  int64_t part_rows = 0;         // rows of part_o
  unsigned* part_count = nullptr; // [attn_slots] ticket counters, zero between launches
  // hack_step overlap: the compression chain of one group of units runs beside the attention of the other group
  int lds_bytes = 0;             // of a work-group, as the device has it
  bool step_overlap = false;     // off by default (measured slower on MI355X, see step_impl); HACK_STEP_OVERLAP=1 switches it on
  hipStream_t aux_stream = nullptr;
  hipEvent_t ev_fork = nullptr, ev_join = nullptr;
  int64_t ws_stride = 0;
  // launch-table cache: tables keep their device address for the life of the context
  hack::TableCache<hack::HipTableBackend>* tables = nullptr;
  std::string err;
};

namespace hack {

inline hack_status fail(hack_ctx* ctx, hack_status s, const char* fmt, ...) {
  if (ctx) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    try {
      ctx->err = buf;
    } catch (...) {   // no memory for the message: the status says enough
      ctx->err.clear();
    }
  }
  return s;
}

// Ends the body of an entry point that allocates host memory (`try { ... } HACK_NO_THROW(ctx)`): exceptions stop here.
#define HACK_NO_THROW(ctx) \
  catch (...) { return fail(ctx, HACK_EHIP, "out of host memory"); }

#define HIP_TRY(ctx, call)                                                              \
  do {                                                                                  \
    hipError_t e_ = (call);                                                             \
    if (e_ != hipSuccess)                                                               \
      return fail(ctx, HACK_EHIP, "%s failed: %s", #call, hipGetErrorString(e_));      \
  } while (0)

inline int64_t round_up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Brings the exchange workspace of the fused score kernel back to its idle state
// (every slot empty, counters and abort word zero).  Synchronises the device.
inline hipError_t rearm_score_workspace(hack_ctx* ctx) {
  hipError_t e = hipDeviceSynchronize();
  if (e == hipSuccess && ctx->rowstat) e = hipMemset(ctx->rowstat, 0xFF, ctx->n_slots * sizeof(unsigned long long));
  if (e == hipSuccess && ctx->counters) e = hipMemset(ctx->counters, 0, ((size_t)ctx->cfg.max_units * 2 + 64) * sizeof(unsigned));
  if (e == hipSuccess) e = hipDeviceSynchronize();
  return e;
}

// Conditions that kernels of earlier calls found on the device.
inline hack_status device_report(hack_ctx* ctx) {
  volatile int* f = ctx->fault;
  if (f && f[0]) {
    // A fused score launch gave up its wait (the device did not keep the launch resident as a
    // whole, e.g. because other work held compute units).  Later fused launches have refused to
    // run since.  Recover: drain, re-arm the workspace, and from now on score in two launches
    // that do not wait for each other inside a kernel.
    if (rearm_score_workspace(ctx) != hipSuccess)
      return fail(ctx, HACK_EHIP, "a score launch gave up its wait and the workspace could not be re-armed");
    f[0] = 0;
    ctx->score_mode = HACK_SCORE_TWO_PASS;
    return fail(ctx, HACK_EHIP, "a score launch gave up waiting for a unit's other work-groups: importance (and whatever "
                                "was derived from it) of the calls since the last successful check is incomplete and those "
                                "calls must be issued again; the context has been re-armed and now scores in two passes "
                                "without in-kernel waits");
  }
  if (f && f[1]) {
    f[1] = 0;
    return fail(ctx, HACK_EUNSUPPORTED, "an earlier bf16 score launch met a logit beyond +-354 (scale * q.k); such logits "
                                        "are clamped, so its importance may differ from the definition");
  }
  return HACK_OK;
}

inline hack_status check_common(hack_ctx* ctx, int32_t B, int32_t N_k, bool need_nk) {
  if (!ctx) return HACK_EINVAL;
  const hack_status dev = device_report(ctx);
  if (dev != HACK_OK) return dev;
  if (B < 1) return fail(ctx, HACK_EINVAL, "B must be >= 1 (got %d)", B);
  if ((int64_t)B * ctx->cfg.heads > ctx->cfg.max_units)
    return fail(ctx, HACK_ECAPACITY, "B*H = %lld exceeds max_units %d", (long long)B * ctx->cfg.heads, ctx->cfg.max_units);
  if (need_nk) {
    if (N_k < 1) return fail(ctx, HACK_EINVAL, "N_k must be >= 1 (got %d)", N_k);
    if (N_k > ctx->cfg.max_queries) return fail(ctx, HACK_ECAPACITY, "N_k = %d exceeds max_queries %d", N_k, ctx->cfg.max_queries);
  }
  return HACK_OK;
}

inline hack_status check_cache(hack_ctx* ctx, const hack_cache* c, int n_units, const char* name, bool need_v) {
  if (!c) return fail(ctx, HACK_EINVAL, "%s is NULL", name);
  if (!c->k || (need_v && !c->v) || !c->off || !c->len) return fail(ctx, HACK_EINVAL, "%s has a NULL member", name);
  if (!aligned16(c->k) || (c->v && !aligned16(c->v))) return fail(ctx, HACK_EINVAL, "%s k/v must be 16-byte aligned", name);
  if (c->rows < 0) return fail(ctx, HACK_EINVAL, "%s rows < 0", name);
  for (int u = 0; u < n_units; ++u) {
    if (c->len[u] < 0 || c->off[u] < 0 || (c->off[u] & 7) || c->off[u] + c->len[u] > c->rows)
      return fail(ctx, HACK_EINVAL, "%s unit %d: off %lld len %d outside [0, %lld) or off not a multiple of 8", name, u,
                  (long long)c->off[u], c->len[u], (long long)c->rows);
  }
  return HACK_OK;
}

inline bool scale_ok(float s) { return std::isfinite(s) && s > 0.f; }

}  // namespace hack
