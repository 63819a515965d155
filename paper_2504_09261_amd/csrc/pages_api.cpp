// Host side of the caches in pages that include/hack.h declares: appending to them and attention over them.  Arguments are checked here and launches laid
// out for the longest caches they may meet; tables and lengths are device memory that only the kernels read.
#include "ops_host.h"
#include "pages_internal.h"

using namespace hack;

namespace {

struct Dim { int64_t stride, count; };

// Whether rows of `width` bytes at the multiples of nested dimensions (the widest first), and the same ones delta bytes on, keep clear of each other.
bool clear_of(int64_t delta, const Dim* dim, int n, int64_t width) {
  if (n == 0) return delta >= width || -delta >= width;
  const int64_t s = dim->stride, below = delta / s - (delta % s < 0);   // numbers differ by this, or one more
  for (int64_t k = below; k <= below + 1; ++k)
    if (k > -dim->count && k < dim->count && !clear_of(delta - k * s, dim + 1, n - 1, width)) return false;
  return true;
}

struct PageMemory {
  Range k, v, table, len, fresh;
};

// Checks a cache and fills in what kernels take of it.
hack_status take_pages(hack_ctx* ctx, int32_t B, int32_t N, const hack_pages* c, const int32_t* fresh, Pages* p, PageMemory* mem) {
  if (!c) return fail(ctx, HACK_EINVAL, "cache is NULL");
  if (!c->k || !c->v || !c->table || !c->len) return fail(ctx, HACK_EINVAL, "cache has a NULL member");
  if (!aligned16(c->k) || !aligned16(c->v)) return fail(ctx, HACK_EINVAL, "cache k/v must be 16-byte aligned");
  if (((uintptr_t)c->table & 3) || ((uintptr_t)c->len & 3) || ((uintptr_t)fresh & 3)) return fail(ctx, HACK_EINVAL, "table, len and fresh must be 4-byte aligned");
  if (c->pages < 1 || c->pages > INT32_MAX) return fail(ctx, HACK_EINVAL, "cache pages %lld outside [1, 2^31)", (long long)c->pages);
  if (c->page_rows < 16 || c->page_rows > 65536 || (c->page_rows & (c->page_rows - 1)))
    return fail(ctx, HACK_EINVAL, "page_rows %d is no power of two in [16, 65536]", c->page_rows);
  if (c->table_pages < 1 || c->table_stride < c->table_pages) return fail(ctx, HACK_EINVAL, "a table has at least an entry and table_stride covers its entries");
  const int64_t H = ctx->cfg.heads, d = ctx->cfg.head_dim, e = ctx->elem_bytes, piece = 16 / e;
  const int64_t strides[3] = {c->stride_page, c->stride_row, c->stride_head};
  for (int64_t s : strides)
    if (s < 0 || s % piece != 0) return fail(ctx, HACK_EINVAL, "cache strides must be non-negative multiples of 16 bytes (got %lld elements)", (long long)s);
  if (c->stride_row * e > 1 << 26) return fail(ctx, HACK_EINVAL, "cache stride_row is beyond 64 MiB");
  const bool one = c->stride_head == 0;   // a page holds the rows of one head
  if (one && H > 1 && !c->by_head) return fail(ctx, HACK_EINVAL, "stride_head 0 needs tables by head");
  Dim dims[3] = {{c->stride_page, c->pages}, {c->stride_row, c->page_rows}, {one ? 0 : c->stride_head, one ? 1 : H}};
  std::sort(dims, dims + 3, [](const Dim& a, const Dim& b) { return a.stride > b.stride; });
  int64_t span = d;   // elements from a row's first to behind the last of the dimensions so far
  for (int i = 2; i >= 0; --i) {
    if (dims[i].count == 1) continue;
    if (dims[i].stride < span) return fail(ctx, HACK_EINVAL, "rows of the cache overlap");
    if (dims[i].stride > (INT64_MAX >> 4) / dims[i].count) return fail(ctx, HACK_EINVAL, "cache strides are too large");
    span += dims[i].stride * (dims[i].count - 1);
  }
  mem->k = range_of(c->k, span, e);
  mem->v = range_of(c->v, span, e);
  if (mem->k.meets(mem->v)) {
    int n = 0;
    for (const Dim& x : dims)
      if (x.count > 1) dims[n++] = Dim{x.stride * e, x.count};
    if (!clear_of((int64_t)((uintptr_t)c->v - (uintptr_t)c->k), dims, n, d * e)) return fail(ctx, HACK_EINVAL, "rows of K and V overlap");
  }
  const int64_t rows = c->by_head ? B * H : B, most = std::min<int64_t>((int64_t)c->table_pages * c->page_rows, INT32_MAX - 2 * kKeys);
  if (c->table_stride > (INT64_MAX >> 4) / rows) return fail(ctx, HACK_EINVAL, "table_stride is too large");
  if (c->max_len < 0 || c->max_len > most) return fail(ctx, HACK_EINVAL, "max_len %d outside [0, %lld]", c->max_len, (long long)most);
  mem->table = range_of(c->table, apart(c->table_stride) * (rows - 1) + c->table_pages, 4);
  mem->len = range_of(c->len, rows, 4);
  mem->fresh = range_of(fresh, B, 4);
  *p = Pages{static_cast<uint8_t*>(c->k), static_cast<uint8_t*>(c->v), c->stride_page * e, c->stride_row * e, one ? 0 : c->stride_head * e, c->table, c->table_stride,
             c->len, fresh, ctx->fault + 2, (int32_t)c->pages, __builtin_ctz((unsigned)c->page_rows), c->max_len ? c->max_len : (int32_t)most, (int32_t)H,
             c->by_head != 0, N};
  return HACK_OK;
}

constexpr int kFewUncut = 24, kTilesUncut = 48;   // blocks of the longest entry up to which nothing is cut: joining the parts takes a launch of 4 us

// Queries of a tile for so many queries of each of `units` caches.  Tiles of 128 share every block through LDS, in the smaller ones every wave reads blocks of its
// own.  Us a call, tiles of 16 / 32 / 128, head_dim 128, 64 elements of 8 caches of 900 to 4000 rows, 20 queries 157 / 140 / 147; of 300 to 1500 rows, 32 queries
// 73 / 64 / 61, 48 87 / 80 / 64, 80 114 / 97 / 70.  Where short caches leave compute units without a tile of 32, more tiles of 16 end earlier: 64 units of
// 61 to 424 rows at head_dim 64, 17 queries 8.8 / 11.2 / 12.0, float32, 169 queries 18.0 / 22.7.
// Tiles of 64 instead of 128 as long as the device holds all of them at once, four a compute unit at head_dim 64 and two at 128: twice the work-groups, whose stages
// are half the work, but read all of K and V again.  64 / 128: head_dim 128, 32 units of 680 rows, 256 queries 17.1 / 23.0, a causal prompt of 300 11.1 / 15.2, 64 units,
// 676 queries (704 work-groups of 64) 36.4 / 34.6; head_dim 64, 16 units of 3900 rows, as many queries (976) 91 / 99, 480 units, 256 queries (1920) 57 / 50.
int tile_queries(const hack_ctx* ctx, int64_t queries, int64_t units, int32_t max_len) {
  if (queries <= 16) return 16;
  if (ctx->cfg.dtype != HACK_F32 && queries > 32)
    return queries <= kHalfTileQueries || (queries + kHalfTileQueries - 1) / kHalfTileQueries * units <= (ctx->cfg.head_dim == 64 ? 4 : 2) * (int64_t)ctx->cus ? kHalfTileQueries : kPageTileQueries;
  return max_len < kFewUncut * kKeys && (queries + 31) / 32 * units < 3 * (int64_t)ctx->cus ? 16 : 32;
}

// How the parts of a call are laid out: tiles of queries, at most how many (entry, head, chunk) there may be, and where their partial results go.  Lengths are
// not known here, so all bounds hold for any up to max_len.  false: more work-groups than a launch takes.
bool plan_parts(const hack_ctx* ctx, AttnPagesArgs* a) {
  const int64_t H = a->c.heads, GN = (int64_t)a->G * a->c.n, units = (int64_t)a->batch * H;
  AttnPart* const part = a->part;
  const auto rows_of = [](const AttnPart& p, int64_t entries) { return entries * p.tiles * p.queries; };   // of partial results, without a cut
  const auto lay_out = [&](int i, int64_t queries, int tile) {
    const bool large = tile >= kHalfTileQueries;
    part[i] = AttnPart{tile, (int32_t)((queries + tile - 1) / tile), 0, large ? kTilesUncut : kFewUncut, large ? 16 : 4, 0.f, 0.f, 0};
  };
  int64_t most = 0, saved = 0, members = 0;   // queries of a group; bytes that sharing spares; batch elements in groups
  int32_t fewest = a->c.max_len, longest = 0; // shared rows of a group
  for (int i = 0; i < a->n_shared; ++i) {
    const Shared& s = a->shared[i];
    most = std::max(most, s.count * GN);
    members += s.count;
    fewest = std::min(fewest, s.rows);
    longest = std::max(longest, s.rows);
    saved += (int64_t)(s.count - 1) * s.rows * H * 2 * ctx->cfg.head_dim * ctx->elem_bytes;
  }
  if (saved < ctx->share_bytes) a->n_shared = 0;
  int own_tile, shared_tile;
  const auto choose_tiles = [&]() {
    own_tile = shared_tile = tile_queries(ctx, GN, units, a->c.max_len);
    if (a->n_shared > 0) {   // tiles of 16 and of 32 are not mixed, nor those of 64 and of 128
      if (tile_queries(ctx, most, a->n_shared * H, a->c.max_len) >= kHalfTileQueries) shared_tile = kPageTileQueries;
      if (own_tile >= kHalfTileQueries) own_tile = kPageTileQueries;
    }
    lay_out(1, GN, own_tile);
    lay_out(0, most, shared_tile);
  };
  choose_tiles();
  if (rows_of(part[0], a->n_shared * H) + rows_of(part[1], units) > ctx->part_rows && a->n_shared > 0) {
    a->n_shared = 0;   // no room to join the parts: every element reads all of its rows
    choose_tiles();
  }
  const int64_t shared_rows = rows_of(part[0], a->n_shared * H);
  // Work-groups that blocks are cut for: of few queries four a compute unit (two, three, four, six: 643 MB 121, 120, 119, 118 us, one long cache 105, 107, 103, 106),
  // of 128 two, which is what it holds.  Shorter chunks than kChunk are worth it only up to one a compute unit: 8 units of 20000 rows in 296 chunks 26.3 us, in 256 22.3.
  int64_t spare = ctx->part_rows - shared_rows - rows_of(part[1], units);   // rows that chunks may take beyond, three quarters for those of shared rows
  const bool large = std::max(own_tile, shared_tile) >= kHalfTileQueries;
  // Float32 tiles of 32, whose products bound them: one, less half of what entries' last chunks may add (8 units of 20000 rows, 100 queries, four / two / one 144 / 121 /
  // 125 us, 16 at head_dim 64, 32 queries 60 / 60 / 51, 32 of 2000 to 9000 rows 70 / 70 / 70, less the half 51).
  const int64_t uncut = units * part[1].tiles;
  const int64_t want = ctx->cfg.dtype == HACK_F32 && own_tile == 32 ? ctx->cus - std::min<int64_t>(uncut / 2, ctx->cus / 4) : (large ? 2 : 4) * (int64_t)ctx->cus;
  int64_t rows = 0, groups = 0;
  for (int i = 0; i < 2; ++i) {
    AttnPart& p = part[i];
    const int64_t pairs = i ? units : a->n_shared * H;
    const int64_t rows_most = i == 0 ? longest : a->n_shared && members == a->batch ? a->c.max_len - fewest : a->c.max_len;   // of an entry
    const int64_t blocks = (rows_most + kKeys - 1) / kKeys + 1, cuts = blocks <= p.uncut ? 1 : (blocks + p.least - 1) / p.least;   // chunks of an entry at most
    const int64_t more = pairs ? std::min(want, (i ? spare : spare * 3 / 4) / p.queries) : 0;
    spare -= std::max<int64_t>(more, 0) * p.queries;
    // A chunk has a `more`-th of all blocks at least, so no entry is cut whose heads and tiles are as many: the longest one alone brings so many times its blocks.
    const bool never = (i && a->c.by_head ? 1 : H) * p.tiles >= more;
    p.share = !never && cuts > 1 && pairs > 0 ? (float)more : 0.f;
    p.fill = (float)std::min<int64_t>(more, ctx->cus);
    p.pairs = (int32_t)std::min(pairs * cuts, p.share > 0.f ? (more + pairs * p.tiles) / p.tiles : pairs);
    p.row0 = rows;
    rows += (int64_t)p.pairs * p.tiles * p.queries;
    groups += pairs_grid(p.pairs, p.tiles);
  }
  return groups <= kMostGroups;
}

}  // namespace

extern "C" hack_status hack_append_pages(hack_ctx* ctx, int32_t B, int32_t N, const hack_rows* q, const hack_rows* k, const hack_rows* v, int32_t norm,
                                         float eps, const hack_rope* rope, const int32_t* pos, int64_t pos_stride_b, const int32_t* fresh,
                                         const hack_pages* cache, hack_stream stream) {
  hack_status st = check_common(ctx, B, N, true);
  if (st != HACK_OK) return st;
  if (norm != HACK_NORM_NONE && norm != HACK_NORM_RMS && norm != HACK_NORM_UNIT) return fail(ctx, HACK_EINVAL, "bad norm %d", norm);
  if (norm != HACK_NORM_NONE && (!std::isfinite(eps) || eps <= 0.f)) return fail(ctx, HACK_EINVAL, "eps must be finite and > 0");
  AppendArgs a{};
  Range in[3] = {}, out[3] = {};
  if (q && (st = take_rows(ctx, B, N, q, "q", &a.t[0], &in[0], &out[0])) != HACK_OK) return st;
  if ((st = take_rows(ctx, B, N, k, "k", &a.t[1], &in[1], &out[1], true)) != HACK_OK) return st;
  if ((st = take_rows(ctx, B, N, v, "v", &a.v, &in[2], &out[2], true)) != HACK_OK) return st;
  if (k->heads != ctx->cfg.heads || v->heads != ctx->cfg.heads) return fail(ctx, HACK_EINVAL, "k and v have the context's %d heads", ctx->cfg.heads);
  if (v->weight || (norm == HACK_NORM_NONE && (k->weight || (q && q->weight)))) return fail(ctx, HACK_EINVAL, "rows without a norm take no weight");
  PageMemory mem;
  if ((st = take_pages(ctx, B, N, cache, fresh, &a.c, &mem)) != HACK_OK) return st;
  a.n = N;
  a.eps = eps;
  a.norm = norm == HACK_NORM_NONE ? kNormNone : norm == HACK_NORM_RMS ? kNormRms : kNormL2;
  if (rope) {
    if (!pos && cache->by_head) return fail(ctx, HACK_EINVAL, "lengths by head need positions");
    if ((st = take_rope(ctx, rope, N, pos, pos_stride_b, 0, &a)) != HACK_OK) return st;
    a.own_rows = !pos;
  }
  // what is read, and what is written: the pages and the queries
  Range read[12];
  int n_read = 0;
  for (const Range& r : in) read[n_read++] = r;
  read[n_read++] = mem.table;
  read[n_read++] = mem.len;
  read[n_read++] = mem.fresh;
  if (rope) read[n_read++] = range_of(pos, apart(pos_stride_b) * (B - 1) + (int64_t)rope->axes * N, 4);
  for (const hack_rows* r : {q, k})
    if (r) read[n_read++] = range_of(r->weight, r->weight_stride_h * (r->heads - 1) + ctx->cfg.head_dim, 4);
  for (int i = 0; i < n_read; ++i) {
    if (mem.k.meets(read[i]) || mem.v.meets(read[i])) return fail(ctx, HACK_EINVAL, "the cache shares memory with what is read");
    if (q && out[0].meets(read[i]) && !(i == 0 && in_place(ctx, B, N, q)))
      return fail(ctx, HACK_EINVAL, "the queries' output shares memory with what is read (in place: x in the layout of out, from the same address)");
  }
  if (q && (out[0].meets(mem.k) || out[0].meets(mem.v))) return fail(ctx, HACK_EINVAL, "the queries' output shares memory with the cache");
  if ((st = check_device(ctx)) != HACK_OK) return st;
  // v takes the launch shape of k
  if (!q) std::swap(a.t[0], a.t[1]);
  shape_rotation(ctx->cfg.head_dim, B, q ? 2 : 1, &a);
  uint32_t k_groups = a.groups[1] - (q ? a.groups[0] : 0);
  if (!q) {
    std::swap(a.t[0], a.t[1]);
    a.groups[0] = 0;
  }
  a.v.tokens_log2 = a.t[1].tokens_log2;
  a.v.tiles = a.t[1].tiles;
  const int64_t all = (int64_t)a.groups[1] + k_groups;
  if (all * B > kMostGroups) return fail(ctx, HACK_ECAPACITY, "%lld work-groups are more than a launch takes", (long long)all * B);
  a.all_groups = (uint32_t)all;
  launch_append(static_cast<hipStream_t>(stream), ctx->elem_bytes, ctx->cfg.head_dim, !rope || rope->layout == HACK_ROPE_HALF, B, a);
  HIP_TRY(ctx, hipGetLastError());
  return HACK_OK;
}

extern "C" hack_status hack_attn_pages(hack_ctx* ctx, int32_t B, int32_t N, int32_t heads, const void* q, const hack_pages* cache, const int32_t* fresh,
                                       int32_t causal, const hack_shared* shared, int32_t n_shared, float scale, void* out, hack_stream stream) {
  hack_status st = check_common(ctx, B, N, true);
  if (st != HACK_OK) return st;
  const int H = ctx->cfg.heads, d = ctx->cfg.head_dim;
  if (heads < 1 || heads % H != 0) return fail(ctx, HACK_EINVAL, "heads %d are no multiple of the context's %d", heads, H);
  if (!q || !out) return fail(ctx, HACK_EINVAL, "q and out must not be NULL");
  if (!aligned16(q) || !aligned16(out)) return fail(ctx, HACK_EINVAL, "q/out must be 16-byte aligned");
  if (!scale_ok(scale)) return fail(ctx, HACK_EINVAL, "scale must be finite and > 0");
  if (n_shared < 0 || (n_shared > 0 && !shared)) return fail(ctx, HACK_EINVAL, "shared is NULL or n_shared negative");
  if (n_shared > kMostShared) return fail(ctx, HACK_ECAPACITY, "%d groups are more than %d", n_shared, kMostShared);
  AttnPagesArgs a;
  PageMemory mem;
  if ((st = take_pages(ctx, B, N, cache, fresh, &a.c, &mem)) != HACK_OK) return st;
  const int64_t GN = (int64_t)(heads / H) * N, rows = (int64_t)B * H * GN;
  if (rows > ((int64_t)1 << 31) - 2 * kPageTileQueries) return fail(ctx, HACK_ECAPACITY, "%lld queries are more than a launch takes", (long long)rows);
  const Range from = range_of(q, rows, (int64_t)d * ctx->elem_bytes), to = range_of(out, rows, (int64_t)d * ctx->elem_bytes);
  for (const Range& r : {from, mem.k, mem.v, mem.table, mem.len, mem.fresh})
    if (to.meets(r)) return fail(ctx, HACK_EINVAL, "out shares memory with what is read");
  a.n_shared = 0;
  for (int i = 0, end = 0; i < n_shared; ++i) {
    const hack_shared& s = shared[i];
    if (s.first < end || s.count < 1 || s.count > B - s.first || s.rows < 0 || s.rows > a.c.max_len)
      return fail(ctx, HACK_EINVAL, "group %d: batch elements %d + %d outside [%d, %d) or %d rows outside [0, %d]", i, s.first, s.count, end, B, s.rows, a.c.max_len);
    end = s.first + s.count;
    if (s.count > 1 && s.rows > 0) a.shared[a.n_shared++] = Shared{s.first, s.count, s.rows};
  }
  if ((st = check_device(ctx)) != HACK_OK) return st;
  a.q = q;
  a.out = out;
  a.part_o = ctx->part_o;
  a.part_ml = ctx->part_ml;
  a.plan = ctx->page_plan;
  a.batch = B;
  a.G = heads / H;
  a.causal = causal != 0;
  a.scale = scale;
  if (!plan_parts(ctx, &a)) return fail(ctx, HACK_ECAPACITY, "%lld queries are more than a launch takes", (long long)rows);
  launch_attn_pages(static_cast<hipStream_t>(stream), ctx->elem_bytes, d, a.part[1].share > 0.f || a.n_shared > 0, a);
  HIP_TRY(ctx, hipGetLastError());
  return HACK_OK;
}
