// Host-side helpers that the operators around the cache share: checks of devices, of memory that operands share and of the operands of a rotation, and the
// shape of its launch.  ops_api.cpp has the operators over rows and packed caches, pages_api.cpp those over caches in pages.
#pragma once

#include <algorithm>
#include <climits>
#include <initializer_list>

#include "hack_ctx.h"
#include "ops_internal.h"

namespace hack {

constexpr int kMostGroups = (1 << 24) - 1;   // of 256 threads, which a launch counts in 32 bits

// Kernels run on the device that is current when they are launched; the context's memory lies on its own.
inline hack_status check_device(hack_ctx* ctx) {
  int dev = -1;
  HIP_TRY(ctx, hipGetDevice(&dev));
  if (dev != ctx->cfg.device) return fail(ctx, HACK_EINVAL, "the current device is %d, the context's is %d", dev, ctx->cfg.device);
  return HACK_OK;
}

// ---- rotary positions, norms ------------------------------------------------

struct Range {   // bytes
  uintptr_t lo, hi;
  bool meets(const Range& o) const { return lo < o.hi && o.lo < hi; }
};

inline Range range_of(const void* p, int64_t n, int64_t bytes) {   // n elements; none for NULL
  const uintptr_t lo = (uintptr_t)p;
  return p ? Range{lo, lo + (uintptr_t)(std::min<int64_t>(n, (int64_t)1 << 44) * bytes)} : Range{0, 0};
}
// A stride whose product with a count fits 64 bits.
inline int64_t apart(int64_t stride) { return std::min<int64_t>(stride, (int64_t)1 << 32); }
// Whether an output shares memory with an input or with another output.
inline bool share(std::initializer_list<Range> out, std::initializer_list<Range> in) {
  for (const Range* o = out.begin(); o != out.end(); ++o) {
    for (const Range& i : in)
      if (o->meets(i)) return true;
    for (const Range* p = o + 1; p != out.end(); ++p)
      if (o->meets(*p)) return true;
  }
  return false;
}

// Checks one operand and fills in its part of the launch; pages: its rows go to pages, not to an output of its own.
inline hack_status take_rows(hack_ctx* ctx, int32_t B, int32_t N, const hack_rows* r, const char* name, RotateTensor* t, Range* in, Range* out,
                             bool pages = false) {
  if (!r) return fail(ctx, HACK_EINVAL, "%s is NULL", name);
  if (pages && r->out) return fail(ctx, HACK_EINVAL, "%s goes to pages, its out must be NULL", name);
  if (!r->x || (!pages && !r->out)) return fail(ctx, HACK_EINVAL, "%s has a NULL member", name);
  if (r->heads < 1) return fail(ctx, HACK_EINVAL, "%s heads must be >= 1 (got %d)", name, r->heads);
  const int d = ctx->cfg.head_dim, e = ctx->elem_bytes, piece = 16 / e;
  if (!aligned16(r->x) || !aligned16(r->out)) return fail(ctx, HACK_EINVAL, "%s x/out must be 16-byte aligned", name);
  const int64_t strides[3] = {r->stride_b, r->stride_h, r->stride_n}, counts[3] = {B, r->heads, N};
  int64_t span = d;   // elements from the first to behind the last
  for (int i = 0; i < 3; ++i) {
    if (strides[i] < 0 || strides[i] % piece != 0)
      return fail(ctx, HACK_EINVAL, "%s strides must be non-negative multiples of 16 bytes (got %lld elements)", name, (long long)strides[i]);
    if (strides[i] > (INT64_MAX >> 4) / counts[i]) return fail(ctx, HACK_EINVAL, "%s strides are too large", name);
    span += strides[i] * (counts[i] - 1);
  }
  if (r->weight && ((uintptr_t)r->weight & 15)) return fail(ctx, HACK_EINVAL, "%s weight must be 16-byte aligned", name);
  if (r->weight && r->weight_stride_h != 0 && (r->weight_stride_h < d || r->weight_stride_h % 4 != 0 || r->weight_stride_h > INT32_MAX))
    return fail(ctx, HACK_EINVAL, "%s weight_stride_h must be 0 or a multiple of 4 from head_dim on (got %lld)", name, (long long)r->weight_stride_h);
  t->x = r->x;
  t->out = r->out;
  t->w = r->weight;
  t->w_stride = (int32_t)r->weight_stride_h;
  t->sb = r->stride_b;
  t->sh = r->stride_h;
  t->sn = r->stride_n;
  t->heads = r->heads;
  const int64_t rows = (int64_t)B * r->heads * N;
  if (rows > (int64_t)1 << 34 || r->heads > 1 << 30) return fail(ctx, HACK_ECAPACITY, "%s has %lld rows, more than a launch takes", name, (long long)rows);
  *in = Range{(uintptr_t)r->x, (uintptr_t)r->x + (uintptr_t)span * e};
  *out = pages ? Range{0, 0} : Range{(uintptr_t)r->out, (uintptr_t)r->out + (uintptr_t)(rows * d) * e};
  return HACK_OK;
}

// Whether a thread that reads an element of x is the one that writes that place of out.
inline bool in_place(const hack_ctx* ctx, int32_t B, int32_t N, const hack_rows* r) {
  const int64_t d = ctx->cfg.head_dim;
  return r->x == r->out && (N == 1 || r->stride_n == d) && (r->heads == 1 || r->stride_h == d * N) && (B == 1 || r->stride_b == d * N * r->heads);
}

inline hack_status take_rope(hack_ctx* ctx, const hack_rope* rope, int32_t N, const int32_t* pos, int64_t pos_stride_b, int32_t pos0, RotateArgs* a) {
  const int d = ctx->cfg.head_dim;
  if (rope->layout != HACK_ROPE_HALF && rope->layout != HACK_ROPE_INTERLEAVED) return fail(ctx, HACK_EINVAL, "bad rope layout %d", rope->layout);
  if (rope->axes != 1 && rope->axes != 2) return fail(ctx, HACK_EINVAL, "rope axes must be 1 or 2 (got %d)", rope->axes);
  if (rope->rot_dim < 1 || rope->rot_dim > d) return fail(ctx, HACK_EINVAL, "rot_dim %d outside [1, head_dim]", rope->rot_dim);
  if (rope->rot_dim % (16 * rope->axes) != 0) return fail(ctx, HACK_EUNSUPPORTED, "rot_dim %d is no multiple of 16 for each axis", rope->rot_dim);
  if (!rope->freq) return fail(ctx, HACK_EINVAL, "rope freq is NULL");
  if (!std::isfinite(rope->gain)) return fail(ctx, HACK_EINVAL, "rope gain must be finite");
  if (!pos && rope->axes != 1) return fail(ctx, HACK_EINVAL, "two axes need positions");
  if ((uintptr_t)pos & 3) return fail(ctx, HACK_EINVAL, "pos must be 4-byte aligned");
  if (pos && pos_stride_b != 0 && pos_stride_b < (int64_t)rope->axes * N)
    return fail(ctx, HACK_EINVAL, "pos_stride_b must be 0 or at least axes * N (got %lld)", (long long)pos_stride_b);
  if (!pos && (int64_t)pos0 + N - 1 > INT32_MAX) return fail(ctx, HACK_EINVAL, "positions from %d on leave 32 bits", pos0);
  for (int i = 0; i < rope->rot_dim / 2; ++i) {
    if (!(std::fabs(rope->freq[i]) <= 1e6)) return fail(ctx, HACK_EINVAL, "freq[%d] is not a number of at most 1e6", i);
    // freq / 2 pi as the sum of two doubles, without its whole turns, which do not matter; then in units of 2^-64.  From the magnitude, whose fraction is
    // exact (that of a small number below zero is one less something, cut at 2^-54: 7.5e-7 at the farthest position), and turned round at the end.
    constexpr double kInv = 0.15915494309189535, kInvLow = -9.839338337591243e-18;
    const double f = std::fabs(rope->freq[i]), t = f * kInv, low = std::fma(f, kInv, -t) + f * kInvLow;
    const uint64_t turns = (uint64_t)((t - std::floor(t)) * 18446744073709551616.0) + (uint64_t)(int64_t)(low * 18446744073709551616.0);
    a->turns[i] = rope->freq[i] < 0.0 ? 0 - turns : turns;
  }
  a->pos = pos;
  a->pos_b = pos_stride_b;
  a->pos0 = pos0;
  a->rot_dim = rope->rot_dim;
  a->section = rope->rot_dim / rope->axes;
  a->gain = rope->gain;
  return HACK_OK;
}

// The launch shape of a rotation, and its number of work-groups.
inline int64_t shape_rotation(int head_dim, int batch, int n_tensors, RotateArgs* a) {
  constexpr int kMaxSteps = 8;
  constexpr int kWantGroups = 2048;   // work-groups that fill the chip: eight a compute unit
  const int slots = kRotateThreads / (head_dim / 16);
  for (int i = 0; i < n_tensors; ++i) {
    RotateTensor& t = a->t[i];
    // Rows of one head side by side: few, so that the rest of the work-group takes the heads beside it, which lie behind each other in a projection
    // (4, 8, 32 rows: 16384 rows of 32 + 8 heads 64.8, 66.7, 65.4 us, 32 x 256 of 30 + 30 heads 26.0, 29.0, 28.5, 2 x 4096 of 16 heads 15.4, 14.0, 14.6),
    // but as many as leave no more than a quarter of the lanes without a head (2 x 11844 rows of 10 + 2 heads of 64: 22.7 us with as few as fit the heads of
    // the larger tensor, 15.8 so; 8 x 10948 of 2 + 1 heads 21.1, 18.6).
    const auto idle = [&](int log2) {
      const int64_t across = slots >> log2, taken = (t.heads + across - 1) / across * across;
      return 4 * (taken - t.heads) > taken;
    };
    int log2 = 0;
    while ((1 << log2) < slots && (1 << log2) < a->n && (log2 < 2 || idle(log2))) ++log2;
    t.tokens_log2 = log2;
    t.tiles = (int32_t)(((int64_t)a->n + (1 << log2) - 1) >> log2);
  }
  // A thread walks over as many heads as leave enough work-groups: it forms its angles once for all of them.
  for (a->steps = kMaxSteps;; a->steps /= 2) {
    int64_t groups = 0;
    for (int i = 0; i < n_tensors; ++i) {
      const RotateTensor& t = a->t[i];
      const int64_t each = (slots >> t.tokens_log2) * a->steps;
      groups += (t.heads + each - 1) / each * t.tiles;
      a->groups[i] = (uint32_t)groups;
    }
    a->groups[1] = (uint32_t)groups;
    groups *= batch;
    if (a->steps == 1 || groups >= kWantGroups) return groups;
  }
}

}  // namespace hack
