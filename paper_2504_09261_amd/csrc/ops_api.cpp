// Host side of the operators around the cache that include/hack.h declares: rotary positions and norms of queries and keys, rows
// packed into 4 bits and read back, attention over them.  Arguments are checked here, launches take everything by value.
#include <algorithm>
#include <climits>
#include <utility>
#include <vector>

#include "ops_host.h"

using namespace hack;

namespace {

hack_status rotate(hack_ctx* ctx, int32_t B, int32_t N, const hack_rows* q, const hack_rows* k, int norm, float eps, const hack_rope* rope,
                   const int32_t* pos, int64_t pos_stride_b, int32_t pos0, hack_stream stream) {
  hack_status st = check_common(ctx, B, N, true);
  if (st != HACK_OK) return st;
  RotateArgs a{};
  const int n = k ? 2 : 1;
  const hack_rows* r[2] = {q, k};
  Range in[2], out[2];
  for (int i = 0; i < n; ++i)
    if ((st = take_rows(ctx, B, N, r[i], i ? "k" : norm == kNormNone ? "x" : "q", &a.t[i], &in[i], &out[i])) != HACK_OK) return st;
  for (int i = 0; i < n; ++i)
    for (int j = 0; j < n; ++j)
      if (out[i].meets(in[j]) && !(i == j && in_place(ctx, B, N, r[i])))
        return fail(ctx, HACK_EINVAL, "outputs overlap rows that are read (in place: x in the layout of out, from the same address)");
  if (n == 2 && out[0].meets(out[1])) return fail(ctx, HACK_EINVAL, "the outputs overlap each other");
  a.n = N;
  a.eps = eps;
  a.norm = norm;
  if (rope && (st = take_rope(ctx, rope, N, pos, pos_stride_b, pos0, &a)) != HACK_OK) return st;
  for (int i = 0; i < n; ++i) {   // work-groups that store would change what others still have to read
    if (rope && out[i].meets(range_of(pos, apart(pos_stride_b) * (B - 1) + (int64_t)rope->axes * N, 4))) return fail(ctx, HACK_EINVAL, "an output overlaps the positions");
    for (int j = 0; j < n; ++j)
      if (out[i].meets(range_of(r[j]->weight, r[j]->weight_stride_h * (r[j]->heads - 1) + ctx->cfg.head_dim, 4)))
        return fail(ctx, HACK_EINVAL, "an output overlaps the weights");
  }
  if ((st = check_device(ctx)) != HACK_OK) return st;
  const int64_t groups = shape_rotation(ctx->cfg.head_dim, B, n, &a);
  if (groups > kMostGroups) return fail(ctx, HACK_ECAPACITY, "%lld work-groups are more than a launch takes", (long long)groups);
  launch_rotate(static_cast<hipStream_t>(stream), ctx->elem_bytes, ctx->cfg.head_dim, !rope || rope->layout == HACK_ROPE_HALF, B, n, a);
  HIP_TRY(ctx, hipGetLastError());
  return HACK_OK;
}

// ---- packed cache -----------------------------------------------------------

hack_status check_packed(hack_ctx* ctx, const hack_packed_cache* c, int n_units, const char* name) {
  if (!c) return fail(ctx, HACK_EINVAL, "%s is NULL", name);
  if (!c->k || !c->v || !c->off || !c->len) return fail(ctx, HACK_EINVAL, "%s has a NULL member", name);
  if (!aligned16(c->k) || !aligned16(c->v) || ((uintptr_t)c->pos & 3)) return fail(ctx, HACK_EINVAL, "%s k/v must be 16-byte, pos 4-byte aligned", name);
  if (c->rows < 0 || c->rows % kPackRows != 0) return fail(ctx, HACK_EINVAL, "%s rows must be a non-negative multiple of %d", name, kPackRows);
  if (c->rows / kPackRows > INT32_MAX) return fail(ctx, HACK_ECAPACITY, "%s has more than 2^31 blocks of %d rows", name, kPackRows);
  for (int u = 0; u < n_units; ++u)
    if (c->len[u] < 0 || c->off[u] < 0 || c->off[u] % kPackRows != 0 || c->off[u] > c->rows || c->len[u] > c->rows - c->off[u])
      return fail(ctx, HACK_EINVAL, "%s unit %d: off %lld len %d outside [0, %lld) or off not a multiple of %d", name, u, (long long)c->off[u],
                  c->len[u], (long long)c->rows, kPackRows);
  return HACK_OK;
}

// Whether two units' rows [off + first, off + len), rounded out to `step`, share any.
template <typename Lo, typename Hi>
bool units_overlap(int n_units, Lo lo, Hi hi) {
  bool sorted = true;
  int64_t end = INT64_MIN;
  for (int u = 0; u < n_units && sorted; ++u) {
    if (hi(u) <= lo(u)) continue;
    sorted = lo(u) >= end;
    end = hi(u);
  }
  if (sorted) return false;
  std::vector<std::pair<int64_t, int64_t>> r;
  for (int u = 0; u < n_units; ++u)
    if (hi(u) > lo(u)) r.emplace_back(lo(u), hi(u));
  std::sort(r.begin(), r.end());
  for (size_t i = 1; i < r.size(); ++i)
    if (r[i].first < r[i - 1].second) return true;
  return false;
}

int blocks_of(int len) { return (int)(((int64_t)len + kPackRows - 1) / kPackRows); }

int tiles_of(int N_k, int queries) { return (int)(((int64_t)N_k + queries - 1) / queries); }

// Partial results of work-groups of so many queries that the workspace holds.
int64_t partial_slots(const hack_ctx* ctx, int queries) { return ctx->part_rows / queries; }

void measure(const int32_t* len, int n, int64_t* blocks, int64_t* longest) {
  *blocks = *longest = 0;
  for (int i = 0; i < n; ++i) {
    const int64_t b = blocks_of(len[i]);
    *blocks += b;
    *longest = std::max(*longest, b);
  }
}

// How units are cut, if at all.  Work-groups of less to do fill the chip and end together, but each leaves a part, and merging the parts is a launch of its
// own: neither the most nor the fewest work-groups are best.  Tried by an estimate of the time are: no cut; chunks that give each compute unit one work-group,
// and two (by the mean, by the mean and half a chunk left over in every unit, by the longest); chunks that balance their own time with that of their parts.
// Fitted to 250 bf16 launches of 4 to 600 units, even and ragged, 500 to 32000 keys, 1 to 1500 queries, each cut into 1 to 32 chunks (float32 contexts are cut by the
// rates of the 16-query bf16 form as they are; no fit was made for them): what it picks takes
// 1.03 times the best of them on average, 1.38 at most (always two work-groups to a compute unit: 1.06, 2.1).  Us a launch, always two / so: 14 units
// of 21747 to 27815 keys, 472 queries 132 / 103, 12 of 1009 to 1591, 5 queries 9.1 / 6.9.
double plan_chunks(const hack_ctx* ctx, int queries, const int32_t* len, int64_t blocks, int64_t longest, AttnPackedHead* a) {
  struct Rates { double block, merge, part; };   // us of 64 keys to a work-group alone, of the merge, of a work-group's part
  static constexpr Rates kRates[2][3] = {{{.16, 2.7, .003}, {.28, 2.5, .005}, {.80, 5.5, .011}}, {{.23, 3.0, .006}, {.45, 4.0, .022}, {1.45, 4.8, .036}}};
  constexpr int kXcds = 8, kLeast = 4;   // blocks of a chunk: one for each wave of the smaller forms
  const Rates& r = kRates[ctx->cfg.head_dim == 128][queries == 16 ? 0 : queries == 32 ? 1 : 2];
  const int64_t n = a->n_units, tiles = a->q_tiles, cus = std::max(ctx->cus / kXcds, 1);
  const int64_t most = std::min<int64_t>(kMostChunks, std::max<int64_t>(1, partial_slots(ctx, queries) / (n * tiles)));   // ... whose partial results the workspace holds
  constexpr int kRows = 256;
  int32_t ends[kRows + 1];   // units of so many chunks
  const auto us = [&](int64_t chunk) {
    const int64_t rows = (longest + chunk - 1) / chunk;
    const bool exact = tiles > 1 && rows > 1 && rows <= kRows;
    if (exact) std::fill(ends, ends + rows + 1, 0);
    int64_t parts = 0;
    const float inv = 1.f / chunk;
    const auto chunks_of = [&](int i) { return (int)(((len[i] - 1) / kPackRows + 0.5f) * inv) + 1; };
    if (rows == 1) {
      parts = n;
    } else if (exact) {
      for (int i = 0; i < n; ++i) {
        const int chunks = std::min<int>(chunks_of(i), rows);
        parts += chunks;
        ++ends[chunks];
      }
    } else {
      for (int i = 0; i < n; ++i) parts += chunks_of(i);
    }
    // Chunks on one XCD: chunk c of the i-th unit, by length, is on (c n + i) mod 8.  Its query tiles share it, so that one chunk more may be many work-groups.
    int64_t on = (parts + kXcds - 1) / kXcds;
    if (exact) {
      int64_t left = n, even = 0, more[kXcds] = {};
      for (int64_t c = 0; c < rows; ++c) {
        left -= ends[c];
        even += left / kXcds;
        for (int64_t i = 0; i < left % kXcds; ++i) ++more[(c * n + i) % kXcds];
      }
      on = even + *std::max_element(more, more + kXcds);
    }
    const double fill = (double)(on * tiles) / cus;   // work-groups of a compute unit
    const double slower = queries == 16 ? std::max(1.0 + 0.6 * fill, 1.1 * fill) : std::max(1.0, 0.76 * std::ceil(fill));
    const double t = r.block * std::max((double)chunk, (double)blocks / parts * slower);
    return parts == n ? t : t + r.merge + r.part * parts * tiles + 3e-4 * (rows * n * tiles);   // the last: empty work-groups
  };
  int64_t best = longest;
  double best_us = us(longest);
  if (most > 1 && longest > kLeast) {
    // no cut can be faster than the merge and the blocks spread evenly: most launches of short units end here
    const double least = r.merge + r.part * n * tiles + r.block * std::max((double)kLeast, 0.76 * blocks * tiles / (kXcds * cus));
    const auto consider = [&](int64_t chunk) {
      chunk = std::max<int64_t>({chunk, kLeast, (longest + most - 1) / most});
      if (chunk >= longest) return;
      const double t = us(chunk);
      if (t < best_us) best = chunk, best_us = t;
    };
    for (int each = 1; each <= 2 && best_us > least; ++each) {
      const int64_t groups = kXcds * (each * cus / tiles);   // a query tile's
      if (groups < 1) continue;
      consider((blocks + groups - 1) / groups);
      if (2 * groups > n) consider((2 * blocks + 2 * groups - n - 1) / (2 * groups - n));
      if (groups > n) consider((longest + groups / n - 1) / (groups / n));
    }
    if (best_us > least) consider((int64_t)std::ceil(std::sqrt(r.part * tiles * blocks / r.block)));
  }
  a->chunk = (int32_t)best;
  a->n_chunks = (int32_t)((longest + best - 1) / best);
  return best_us;
}

// Queries of a work-group.  Sixteen and 32 have every wave convert the keys it takes, 128 (kTileQueries) share every converted block, which is what a large
// launch wants, but give an eighth of the work-groups.  Which is fastest goes by the plan's estimate, scaled and with the start of the work-groups added as
// fitted to 257 drawn launches of 1 to 500 units, even and ragged, 100 to 60000 keys, 17 to 2000 queries: what it picks takes 1.014 times the best on
// average, 1.30 at most (114 others: 1.02, 1.32; always 16: 1.16, 2.4; always 32: 1.08, 1.6; always 128: 1.33, 2.6).  Us a launch, 16 / 32 / 128 queries,
// head_dim 128: 9 units of 1440 keys, 207 queries 10.6 / 13.2 / 15.6, 46 of 12401, 187 88.8 / 70.7 / 85.3, 14 of 20679, 378 108 / 77 / 64.
int queries_per_group(const hack_ctx* ctx, const int32_t* len, int n_units, int N_k) {
  if (ctx->cfg.dtype == HACK_F32) return 16;
  if (ctx->packed_queries != 0) return ctx->packed_queries;
  if (N_k <= 16) return 16;
  struct Form { int queries; double scale, start, groups; };   // us of a launch's start, of 256 work-groups'
  static constexpr Form kForms[2][3] = {{{16, .81, 4.0, .36}, {32, .85, 4.1, .75}, {kTileQueries, 1.10, 4.6, 2.2}},
                                        {{16, 1.00, 4.2, 1.1}, {32, .83, 4.5, 2.0}, {kTileQueries, .86, 4.3, 3.35}}};
  int64_t blocks, longest;
  measure(len, n_units, &blocks, &longest);
  int queries = 0;
  double best = 0.0;
  for (const Form& f : kForms[ctx->cfg.head_dim == 128]) {
    AttnPackedHead a{};
    a.n_units = n_units;
    a.q_tiles = tiles_of(N_k, f.queries);
    const double us = f.scale * plan_chunks(ctx, f.queries, len, blocks, longest, &a) + f.start + f.groups * n_units * a.q_tiles / 256.0;
    if (queries == 0 || us < best) queries = f.queries, best = us;
  }
  return queries;
}

// In what order units start: the longest first, except that where all work-groups start at once, two to a compute unit (one on each first, then a second
// one in the same order), the long ones get the short ones beside them.
void order_units(const hack_ctx* ctx, const int32_t* len, const AttnPackedHead& a, std::vector<int32_t>* order, std::vector<int32_t>* count) {
  const int n = a.n_units;
  int lo = INT_MAX, hi = 0;
  for (int i = 0; i < n; ++i) {
    lo = std::min(lo, blocks_of(len[i]));
    hi = std::max(hi, blocks_of(len[i]));
  }
  std::vector<int32_t>& o = *order;
  if (lo == hi || n == 1) {
    for (int i = 0; i < n; ++i) o[i] = i;
    return;
  }
  // by length in steps of a 255th of the range, equal ones in the order of the units
  constexpr int kSteps = 256;
  const auto step = [&](int i) { return (int)((int64_t)(hi - blocks_of(len[i])) * (kSteps - 1) / (hi - lo)); };
  count->assign(kSteps + 1, 0);
  for (int i = 0; i < n; ++i) ++(*count)[step(i) + 1];
  for (int i = 0; i < kSteps; ++i) (*count)[i + 1] += (*count)[i];
  for (int i = 0; i < n; ++i) o[(*count)[step(i)]++] = i;
  if (a.q_tiles == 1 && a.n_chunks == 1 && n > ctx->cus && n <= 2 * ctx->cus) std::reverse(o.begin() + ctx->cus, o.begin() + n);
}

}  // namespace

extern "C" hack_status hack_rope_freqs(int32_t rot_dim, int32_t axes, int32_t scaling, double base, double factor, double trained_len, double* freq,
                                       float* gain) {
  if (!freq || (axes != 1 && axes != 2) || rot_dim < 2 || rot_dim > 2 * kMaxPairs || rot_dim % (2 * axes) != 0) return HACK_EINVAL;
  if (!std::isfinite(base) || base <= 1.0 || !std::isfinite(factor) || factor < 1.0) return HACK_EINVAL;
  if (scaling < HACK_ROPE_PLAIN || scaling > HACK_ROPE_PARTS) return HACK_EINVAL;
  if (scaling == HACK_ROPE_PARTS && (!std::isfinite(trained_len) || trained_len < 1.0)) return HACK_EINVAL;
  const int size = rot_dim / axes, n = size / 2;
  double g = 1.0;
  if (scaling == HACK_ROPE_BASE && size > 2) base *= std::pow(factor, (double)size / (size - 2));
  double low = 0.0, high = 0.0;
  if (scaling == HACK_ROPE_PARTS) {
    // pair that makes `turns` turns over the length trained on
    const auto at = [&](double turns) { return size * std::log(trained_len / (turns * 6.283185307179586)) / (2.0 * std::log(base)); };
    low = std::max(std::floor(at(32.0)), 0.0);
    high = std::min(std::ceil(at(1.0)), size - 1.0);
    g = 0.1 * std::log(factor) + 1.0;
  }
  for (int i = 0; i < n; ++i) {
    double f = std::pow(base, -2.0 * i / size);
    if (scaling == HACK_ROPE_LINEAR) f /= factor;
    if (scaling == HACK_ROPE_PARTS) {
      // no pair between where the fastest turns less than once (all are slow) or the slowest more than 32 times (all are fast)
      const double ramp = high > low ? std::min(std::max((i - low) / (high - low), 0.0), 1.0) : i >= low ? 1.0 : 0.0;
      f = f * (1.0 - ramp) + f / factor * ramp;
    }
    for (int a = 0; a < axes; ++a) freq[a * n + i] = f;
  }
  if (gain) *gain = (float)g;
  return HACK_OK;
}

extern "C" hack_status hack_rotate(hack_ctx* ctx, int32_t B, int32_t N, const hack_rows* x, const hack_rope* rope, const int32_t* pos,
                                   int64_t pos_stride_b, int32_t pos0, hack_stream stream) {
  if (!ctx) return HACK_EINVAL;
  if (!rope) return fail(ctx, HACK_EINVAL, "rope is NULL");
  if (x && x->weight) return fail(ctx, HACK_EINVAL, "a rotation without a norm takes no weight");
  return rotate(ctx, B, N, x, nullptr, kNormNone, 0.f, rope, pos, pos_stride_b, pos0, stream);
}

extern "C" hack_status hack_norm_rotate(hack_ctx* ctx, int32_t B, int32_t N, const hack_rows* q, const hack_rows* k, int32_t norm, float eps,
                                        const hack_rope* rope, const int32_t* pos, int64_t pos_stride_b, int32_t pos0, hack_stream stream) {
  if (!ctx) return HACK_EINVAL;
  if (norm != HACK_NORM_RMS && norm != HACK_NORM_UNIT) return fail(ctx, HACK_EINVAL, "bad norm %d", norm);
  if (!std::isfinite(eps) || eps <= 0.f) return fail(ctx, HACK_EINVAL, "eps must be finite and > 0");
  return rotate(ctx, B, N, q, k, norm == HACK_NORM_RMS ? kNormRms : kNormL2, eps, rope, pos, pos_stride_b, pos0, stream);
}

extern "C" hack_status hack_packed_bytes(int32_t head_dim, int64_t rows, int64_t* bytes) {
  if (!bytes || (head_dim != 64 && head_dim != 128) || rows < 0 || rows > ((int64_t)INT32_MAX) * kPackRows) return HACK_EINVAL;
  *bytes = (rows + kPackRows - 1) / kPackRows * packed_block_bytes(head_dim);
  return HACK_OK;
}

extern "C" hack_status hack_pack(hack_ctx* ctx, int32_t B, int32_t N_k, const hack_cache* in, const void* k_new, const void* v_new, int32_t pos_new,
                                 const int32_t* kept_idx, int64_t idx_stride, const int32_t* first, const hack_packed_cache* out,
                                 hack_stream stream) try {
  const bool has_new = k_new != nullptr;
  hack_status st = check_common(ctx, B, N_k, has_new);
  if (st != HACK_OK) return st;
  const int U = B * ctx->cfg.heads;
  if (has_new != (v_new != nullptr)) return fail(ctx, HACK_EINVAL, "k_new and v_new must both be given or both be NULL");
  if (!has_new && !in) return fail(ctx, HACK_EINVAL, "neither cached nor new rows are given");
  if (has_new && (!aligned16(k_new) || !aligned16(v_new))) return fail(ctx, HACK_EINVAL, "k_new/v_new must be 16-byte aligned");
  if ((uintptr_t)kept_idx & 3) return fail(ctx, HACK_EINVAL, "kept_idx must be 4-byte aligned");
  if (in && (st = check_cache(ctx, in, U, "in", true)) != HACK_OK) return st;
  if ((st = check_packed(ctx, out, U, "out")) != HACK_OK) return st;
  const int n_new = has_new ? N_k : 0;
  std::vector<PackUnit> units(U);
  bool any = false;
  for (int u = 0; u < U; ++u) {
    const int at = first ? first[u] : 0, there = in ? in->len[u] : 0;
    if (at < 0 || at > out->len[u]) return fail(ctx, HACK_EINVAL, "first[%d] = %d outside [0, out->len = %d]", u, at, out->len[u]);
    const int n = out->len[u] - at;
    if (n > (int64_t)there + n_new) return fail(ctx, HACK_EINVAL, "unit %d takes %d rows of %lld", u, n, (long long)there + n_new);
    if (kept_idx && n > idx_stride) return fail(ctx, HACK_ECAPACITY, "idx_stride %lld < the %d rows of unit %d", (long long)idx_stride, n, u);
    if ((int64_t)there + n_new > INT32_MAX) return fail(ctx, HACK_ECAPACITY, "unit %d has more than 2^31 rows", u);
    units[u] = PackUnit{in ? in->off[u] : 0, there, (int32_t)(out->off[u] / kPackRows), at, n};
    any |= n > 0;
  }
  if (!any) return HACK_OK;
  if (units_overlap(U, [&](int u) { return out->off[u] + units[u].first; }, [&](int u) { return out->off[u] + out->len[u]; }))
    return fail(ctx, HACK_EINVAL, "units of out overlap");
  const int64_t row = (int64_t)ctx->cfg.head_dim * ctx->elem_bytes, block = packed_block_bytes(ctx->cfg.head_dim), blocks = out->rows / kPackRows;
  const int64_t rows = in ? in->rows : 0, fresh = (int64_t)U * n_new;
  if (share({range_of(out->k, blocks, block), range_of(out->v, blocks, block), range_of(out->pos, out->rows, 4)},
            {range_of(in ? in->k : nullptr, rows, row), range_of(in ? in->v : nullptr, rows, row), range_of(in ? in->pos : nullptr, rows, 4),
             range_of(k_new, fresh, row), range_of(v_new, fresh, row), range_of(kept_idx, U * apart(idx_stride), 4)}))
    return fail(ctx, HACK_EINVAL, "out shares memory with what is read, or K with V");
  if ((st = check_device(ctx)) != HACK_OK) return st;
  PackHead a{};
  if (in) a.plain = CachePtrs{in->k, in->v, in->pos};
  a.packed = CachePtrs{out->k, out->v, out->pos};
  a.k_new = k_new;
  a.v_new = v_new;
  a.kept = kept_idx;
  a.kept_stride = idx_stride;
  a.n_new = n_new;
  a.pos_new = pos_new;
  launch_pack(static_cast<hipStream_t>(stream), ctx->elem_bytes, ctx->cfg.head_dim, a, units.data(), U);
  HIP_TRY(ctx, hipGetLastError());
  return HACK_OK;
} HACK_NO_THROW(ctx)

extern "C" hack_status hack_unpack(hack_ctx* ctx, int32_t B, const hack_packed_cache* in, const int32_t* first, const hack_cache* out,
                                   hack_stream stream) try {
  hack_status st = check_common(ctx, B, 0, false);
  if (st != HACK_OK) return st;
  const int U = B * ctx->cfg.heads;
  if ((st = check_packed(ctx, in, U, "in")) != HACK_OK) return st;
  if ((st = check_cache(ctx, out, U, "out", true)) != HACK_OK) return st;
  std::vector<PackUnit> units(U);
  bool any = false;
  for (int u = 0; u < U; ++u) {
    const int at = first ? first[u] : 0;
    if (at < 0 || at > in->len[u] || out->len[u] > in->len[u] - at)
      return fail(ctx, HACK_EINVAL, "unit %d: rows %d to %lld of %d", u, at, (long long)at + out->len[u], in->len[u]);
    units[u] = PackUnit{out->off[u], 0, (int32_t)(in->off[u] / kPackRows), at, out->len[u]};
    any |= out->len[u] > 0;
  }
  if (!any) return HACK_OK;
  if (units_overlap(U, [&](int u) { return out->off[u]; }, [&](int u) { return out->off[u] + out->len[u]; }))
    return fail(ctx, HACK_EINVAL, "units of out overlap");
  const int64_t row = (int64_t)ctx->cfg.head_dim * ctx->elem_bytes, block = packed_block_bytes(ctx->cfg.head_dim), blocks = in->rows / kPackRows;
  if (share({range_of(out->k, out->rows, row), range_of(out->v, out->rows, row), range_of(out->pos, out->rows, 4)},
            {range_of(in->k, blocks, block), range_of(in->v, blocks, block), range_of(in->pos, in->rows, 4)}))
    return fail(ctx, HACK_EINVAL, "out shares memory with what is read, or K with V");
  if ((st = check_device(ctx)) != HACK_OK) return st;
  PackHead a{};
  a.plain = CachePtrs{out->k, out->v, out->pos};
  a.packed = CachePtrs{in->k, in->v, in->pos};
  launch_unpack(static_cast<hipStream_t>(stream), ctx->elem_bytes, ctx->cfg.head_dim, a, units.data(), U);
  HIP_TRY(ctx, hipGetLastError());
  return HACK_OK;
} HACK_NO_THROW(ctx)

extern "C" hack_status hack_attn_packed(hack_ctx* ctx, int32_t B, int32_t N_k, const void* q, const hack_packed_cache* kv, float scale, void* out,
                                        hack_stream stream) try {
  hack_status st = check_common(ctx, B, N_k, true);
  if (st != HACK_OK) return st;
  const int U = B * ctx->cfg.heads, d = ctx->cfg.head_dim;
  if (!q || !out) return fail(ctx, HACK_EINVAL, "q and out must not be NULL");
  if (!aligned16(q) || !aligned16(out)) return fail(ctx, HACK_EINVAL, "q/out must be 16-byte aligned");
  if (!scale_ok(scale)) return fail(ctx, HACK_EINVAL, "scale must be finite and > 0");
  if ((st = check_packed(ctx, kv, U, "kv")) != HACK_OK) return st;
  for (int u = 0; u < U; ++u)
    if (kv->len[u] < 1) return fail(ctx, HACK_EINVAL, "unit %d has an empty cache", u);
  const int64_t rows = (int64_t)U * N_k, row = (int64_t)d * ctx->elem_bytes;
  if (range_of(q, rows, row).meets(range_of(out, rows, row))) return fail(ctx, HACK_EINVAL, "q and out overlap");
  if ((st = check_device(ctx)) != HACK_OK) return st;
  AttnPackedHead a{};
  AttnPackedUnit units[kAttnPackedUnits];
  a.k = static_cast<const uint8_t*>(kv->k);
  a.v = static_cast<const uint8_t*>(kv->v);
  a.part_o = ctx->part_o;
  a.part_ml = ctx->part_ml;
  a.q = q;
  a.out = out;
  a.N_k = N_k;
  a.scale = scale;
  const int queries = queries_per_group(ctx, kv->len, U, N_k);
  a.q_tiles = tiles_of(N_k, queries);
  // Units of a launch: its work-groups are a multiple of eight times the tiles.  (Units that are cut have few.)
  const int most = std::min(kAttnPackedUnits, kMostGroups / a.q_tiles / 8 * 8);
  if (most < 1) return fail(ctx, HACK_ECAPACITY, "%d queries are more than a launch takes", N_k);
  std::vector<int32_t> order(std::min(U, most)), count;
  for (int u0 = 0; u0 < U; u0 += most) {
    a.n_units = std::min(most, U - u0);
    const int32_t* len = kv->len + u0;
    int64_t blocks, longest;
    measure(len, a.n_units, &blocks, &longest);
    plan_chunks(ctx, queries, len, blocks, longest, &a);
    order_units(ctx, len, a, &order, &count);
    for (int i = 0; i < a.n_units; ++i) units[i] = AttnPackedUnit{(int32_t)(kv->off[u0 + order[i]] / kPackRows), len[order[i]], u0 + order[i]};
    launch_attn_packed(static_cast<hipStream_t>(stream), ctx->elem_bytes, d, queries, a, units);
  }
  HIP_TRY(ctx, hipGetLastError());
  return HACK_OK;
} HACK_NO_THROW(ctx)
