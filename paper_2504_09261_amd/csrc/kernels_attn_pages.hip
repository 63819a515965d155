// Attention over caches in pages for few queries of a cache (single tokens, small scales) and in float32 contexts for all, and the merge of partial results
// (the arithmetic: attn_pages_few.h; many queries: kernels_attn_pages_tiles.hip).
//
// Measured, bf16, head_dim 128: one token of 64 elements with 32 heads over 8 caches of 900 to 4000 rows, 643 MB, 112 us (5.7 TB/s; a plain kernel that only
// reads reaches 5.9), 64 heads over 8 caches of 131071 rows, 537 MB, 95; float32, head_dim 64: 64 units of 61 to 424 rows, 169 queries 18 us, of which the
// products are 5: the start of a work-group, 5 us, and uneven units.
#include "attn_pages_few.h"

namespace hack {

namespace {

using namespace dev;

// At head_dim 128 two work-groups a compute unit with all the registers they ask for (three: some spill, 643 MB 120 -> 123 us, float32 122 -> 132).
template <typename T, int D, int NQ, bool NT>
__global__ __launch_bounds__(kThreads, D == 128 ? 2 : NQ == 1 ? 4 : 3) void attn_pages(const AttnPagesArgs a) {
  __shared__ __attribute__((aligned(1024))) unsigned char lds[kFewLds<D, NQ>];
  const int grid0 = a.parts & 1 ? (a.part[0].pairs + 7) / 8 * 8 * a.part[0].tiles : 0, part = (int)blockIdx.x >= grid0 ? 1 : 0;
  attn_pages_few<T, D, NQ, NT>(a, part, blockIdx.x - (part ? grid0 : 0), lds);
}

// Joins the partial results of rows: ROWS of them a work-group, each by 256 / ROWS threads, D / 4 lanes a slot, which walk over its slots.  With references m_i, sums l_i
// and outputs o_i of a row's slots, o = sum 2^(m_i - M) o_i / sum 2^(m_i - M) l_i.  Bound by reading the slots (6144 rows of 11 or 12: 38 MB, 8 us); where rows are few, the way of one
// through them counts, and a work-group takes one.
template <typename T, int D, int ROWS>
__global__ __launch_bounds__(256) void attn_pages_merge(const AttnPagesArgs a) {
  constexpr int LPR = D / 4, SIDE = 256 / LPR / ROWS;   // slots of a row at a time
  const Pages& c = a.c;
  const int tid = threadIdx.x, lane = tid % LPR, side = tid / LPR % SIDE;
  const int64_t row = (int64_t)blockIdx.x * ROWS + tid / (LPR * SIDE);
  const int GN = a.G * c.n;
  __shared__ float4 o_sh[ROWS][SIDE][LPR];
  __shared__ float2 ml_sh[ROWS][SIDE];
  bool mine = row < (int64_t)a.batch * c.heads * GN;
  const int u = mine ? (int)(row / GN) : 0, r = (int)(row - (int64_t)u * GN), b = u / c.heads, h = u - b * c.heads, n = r % c.n, x0 = n * a.G + r / c.n;
  const int entry = c.by_head ? u : b, group = mine ? group_of(a, b) : -1;
  const int2 own = a.plan[a.n_shared + entry];
  int2 common = make_int2(0, 0);
  if (group >= 0) common = a.plan[group];
  const int fresh = fresh_of(c, b);
  mine = mine && n < fresh && (group >= 0 || own.y > 1);
  const int slots = mine ? common.y + own.y : 0;
  // A part's slots are tiles of whole rows, one tile behind the other: query x of an entry is row x of its pair, and pairs of a head are its chunks.  The order of an
  // entry's queries: by element, number, head.
  const int64_t j = group >= 0 ? (int64_t)(b - a.shared[group].first) * GN + x0 : 0;
  const int64_t rows0 = (int64_t)a.part[0].tiles * a.part[0].queries, rows1 = (int64_t)a.part[1].tiles * a.part[1].queries;
  const int64_t at0 = a.part[0].row0 + ((int64_t)common.x + (int64_t)h * common.y) * rows0 + j;
  const int64_t at1 = a.part[1].row0 + ((int64_t)own.x + (c.by_head ? 0 : (int64_t)h * own.y)) * rows1 + x0;
  const float2* const ml = reinterpret_cast<const float2*>(a.part_ml);
  const float4* const po = reinterpret_cast<const float4*>(a.part_o) + lane;
  float M = -FLT_MAX, L = 0.f;
  floatx4 o = {0.f, 0.f, 0.f, 0.f};
  constexpr int kAhead = 4;   // slots whose loads are under way together
  for (int s0 = side; s0 < slots; s0 += kAhead * SIDE) {
    float2 x[kAhead];
    float4 p[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int s = min(s0 + i * SIDE, slots - 1);
      const int64_t at = s < common.y ? at0 + s * rows0 : at1 + (s - common.y) * rows1;
      x[i] = ml[at];
      p[i] = po[at * LPR];
    }
    float m = M;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) m = maximum(m, x[i].x);
    const float old = __builtin_amdgcn_exp2f(M - m);
    M = m;
    L *= old;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] *= old;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (s0 + i * SIDE >= slots) continue;
      const float f = __builtin_amdgcn_exp2f(x[i].x - M);
      L = fmaf(f, x[i].y, L);
      o[0] = fmaf(f, p[i].x, o[0]);
      o[1] = fmaf(f, p[i].y, o[1]);
      o[2] = fmaf(f, p[i].z, o[2]);
      o[3] = fmaf(f, p[i].w, o[3]);
    }
  }
  if constexpr (SIDE > 1) {
    const int k = tid / (LPR * SIDE);
    o_sh[k][side][lane] = make_float4(o[0], o[1], o[2], o[3]);
    if (lane == 0) ml_sh[k][side] = make_float2(M, L);
    __syncthreads();
    if (side != 0) return;
    float2 x[SIDE];
    M = -FLT_MAX;
#pragma unroll
    for (int i = 0; i < SIDE; ++i) {
      x[i] = ml_sh[k][i];
      M = maximum(M, x[i].x);
    }
    L = 0.f;
    o = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < SIDE; ++i) {
      const float f = __builtin_amdgcn_exp2f(x[i].x - M);
      const float4 p = o_sh[k][i][lane];
      L = fmaf(f, x[i].y, L);
      o[0] = fmaf(f, p.x, o[0]);
      o[1] = fmaf(f, p.y, o[1]);
      o[2] = fmaf(f, p.z, o[2]);
      o[3] = fmaf(f, p.w, o[3]);
    }
  }
  if (!mine) return;
  const int len = rows_of(c, entry);
  const float inv = (a.causal ? len - fresh + n + 1 : len) > 0 ? 1.f / L : 0.f;
  float y[4] = {o[0], o[1], o[2], o[3]};
  store_some(static_cast<T*>(a.out) + row * D + 4 * lane, y, 4, inv);
}

template <typename T, int D>
void launch_some(hipStream_t s, bool merge, AttnPagesArgs& a) {
  const bool both = a.n_shared > 0;
  a.parts = both ? 3 : 2;
  if (a.part[1].queries >= kHalfTileQueries || (both && a.part[0].queries >= kHalfTileQueries)) {
    launch_attn_pages_tiles(s, D, a);
  } else {
    const dim3 grid((unsigned)(part_grid(a, 0) + part_grid(a, 1)));
    const bool once = reads_once(a);
#define HACK_ATTN_PAGES(NQ, NT) hipLaunchKernelGGL((attn_pages<T, D, NQ, NT>), grid, dim3(kThreads), 0, s, a)
    if (a.part[1].queries == 16) {
      if (once) HACK_ATTN_PAGES(1, true);
      else HACK_ATTN_PAGES(1, false);
    } else {
      if (once) HACK_ATTN_PAGES(2, true);
      else HACK_ATTN_PAGES(2, false);
    }
#undef HACK_ATTN_PAGES
  }
  if (!merge) return;
  const int64_t rows = (int64_t)a.batch * a.c.heads * a.G * a.c.n;
  constexpr int kRows = 1024 / D;
  if (rows >= 4096) hipLaunchKernelGGL((attn_pages_merge<T, D, kRows>), dim3((unsigned)((rows + kRows - 1) / kRows)), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((attn_pages_merge<T, D, 1>), dim3((unsigned)rows), dim3(256), 0, s, a);
}

}  // namespace

void launch_attn_pages(hipStream_t s, int elem_bytes, int head_dim, bool merge, AttnPagesArgs a) {
  if (elem_bytes == 4) {
    if (head_dim == 64) launch_some<float, 64>(s, merge, a);
    else launch_some<float, 128>(s, merge, a);
  } else {
    if (head_dim == 64) launch_some<__bf16, 64>(s, merge, a);
    else launch_some<__bf16, 128>(s, merge, a);
  }
}

}  // namespace hack
