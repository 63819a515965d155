// New rows into the pages of their sequences: keys normed and rotated on the way, values as they are, and the queries of the same tokens normed and rotated
// in the same launch.
//
// The arithmetic and the lanes' share of a row are those of the rotation (rotate_device.h); a token's place is its sequence's table entry.  Memory-bound: every
// row is read and written once.  Measured, bf16: 16384 tokens of 32 + 8 + 8 heads of 128 out of one projection 79 us (403 MB, 5.1 TB/s of the 6.2 of a plain elementwise kernel),
// 32 x 256 of 30 + 30 + 30 heads of 64, normed and turned in two axes, into pages of 16 rows 42 us (189 MB, 4.5 TB/s; a plain kernel of this size 5.4), one
// token of each of 64 sequences 4.5 us.  More or fewer tokens or heads a work-group, the next head's loads ahead of this one's arithmetic: within 3 %.
#include "pages_device.h"
#include "rotate_device.h"

namespace hack {

namespace {

using namespace dev;

// A length or a number of new rows that is out of range stores nothing, no queries either: the rows and positions that it would name are others'.
__device__ __forceinline__ int stored_rows(const Pages& c, int entry) {
  const int len = c.len[entry];
  if (__builtin_expect((unsigned)len <= (unsigned)c.max_len, 1)) return len;
  report(c);
  return -1;   // no row lies in front of the sequence's first
}
__device__ __forceinline__ int stored_fresh(const Pages& c, int b) {
  if (!c.fresh) return c.n;
  const int fresh = c.fresh[b];
  if (__builtin_expect((unsigned)fresh <= (unsigned)c.n, 1)) return fresh;
  report(c);
  return 0;
}
// Where row r of a table's sequence lies; NULL where it lies nowhere.
__device__ __forceinline__ uint8_t* find_row(const Pages& c, uint8_t* mem, int entry, int r) {
  if (r < 0) return nullptr;
  const int page = c.table[entry * c.table_stride + (r >> c.log2_rows)];
  if ((unsigned)page >= (unsigned)c.pages) {
    report(c);
    return nullptr;
  }
  return mem + page * c.stride_page + (r & ((1 << c.log2_rows) - 1)) * c.stride_row;
}
template <typename T> struct ToPages {
  static constexpr bool kDrops = true;
  bool taken;
  Pages c;
  uint8_t* mem;
  uint8_t* row;       // of all heads; by_head: each has its own
  int unit0, back;    // by_head: the first head's unit; rows between the sequence's end and this one
  __device__ __forceinline__ T* operator()(int h) const {
    uint8_t* p = row;
    if (c.by_head) p = find_row(c, mem, unit0 + h, stored_rows(c, unit0 + h) - back);
    return p ? reinterpret_cast<T*>(p + h * c.stride_head) : nullptr;
  }
};

template <typename T, int D, bool HALF, bool NORM, bool STREAM>
__global__ __launch_bounds__(kRotateThreads) void append_rows(const AppendArgs a) {
  const int b = blockIdx.x / a.all_groups;
  unsigned x = blockIdx.x - (unsigned)b * a.all_groups;
  const int which = x < a.groups[0] ? 0 : x < a.groups[1] ? 1 : 2;   // q, k, v
  const int len = a.c.by_head ? 0 : stored_rows(a.c, b), fresh = len < 0 ? 0 : stored_fresh(a.c, b);
  const int first = a.c.by_head ? 0 : len - fresh;   // row of the first new one
  const int pos0 = a.own_rows ? first : 0;
  if (which == 0) {
    turn_rows<T, D, HALF, NORM, STREAM>(a, a.t[0], b, x, a.rot_dim, pos0, [&](int64_t n) {
      return ToArray<T>{n < fresh, static_cast<T*>(a.t[0].out) + ((int64_t)b * a.t[0].heads * a.n + n) * D, (int64_t)a.n * D};
    });
    return;
  }
  uint8_t* const mem = which == 1 ? a.c.k : a.c.v;
  const auto place = [&](int64_t n) {
    ToPages<T> to{n < fresh, a.c, mem, nullptr, b * a.c.heads, fresh - (int)n};
    if (to.taken && !a.c.by_head) to.taken = (to.row = find_row(a.c, mem, b, first + (int)n)) != nullptr;
    return to;
  };
  if (which == 1) turn_rows<T, D, HALF, NORM, STREAM>(a, a.t[1], b, x - a.groups[0], a.rot_dim, pos0, place);
  else turn_rows<T, D, HALF, false, STREAM>(a, a.v, b, x - a.groups[1], 0, 0, place);
}

template <typename T, int D, bool HALF>
void launch_form(hipStream_t s, bool stream, unsigned groups, const AppendArgs& a) {
#define HACK_APPEND(NORM, STREAM) hipLaunchKernelGGL((append_rows<T, D, HALF, NORM, STREAM>), dim3(groups), dim3(kRotateThreads), 0, s, a)
  if (a.norm == kNormNone) {
    if (stream) HACK_APPEND(false, true);
    else HACK_APPEND(false, false);
  } else {
    if (stream) HACK_APPEND(true, true);
    else HACK_APPEND(true, false);
  }
#undef HACK_APPEND
}

template <typename T, int D>
void launch_typed(hipStream_t s, bool half_layout, bool stream, unsigned groups, const AppendArgs& a) {
  if (half_layout) launch_form<T, D, true>(s, stream, groups, a);
  else launch_form<T, D, false>(s, stream, groups, a);
}

}  // namespace

void launch_append(hipStream_t s, int elem_bytes, int head_dim, bool half_layout, int batch, AppendArgs a) {
  const int64_t rows = (int64_t)batch * a.n * ((a.groups[0] ? a.t[0].heads : 0) + 2 * (int64_t)a.c.heads);
  a.low = a.eps < 0x1p-50f ? 0x1p-100f : 0.f;   // as in the rotation
  const bool stream = streams(a, half_layout, head_dim, rows * head_dim * elem_bytes);
  const unsigned groups = a.all_groups * (unsigned)batch;
  if (elem_bytes == 4) {
    if (head_dim == 64) launch_typed<float, 64>(s, half_layout, stream, groups, a);
    else launch_typed<float, 128>(s, half_layout, stream, groups, a);
  } else {
    if (head_dim == 64) launch_typed<__bf16, 64>(s, half_layout, stream, groups, a);
    else launch_typed<__bf16, 128>(s, half_layout, stream, groups, a);
  }
}

}  // namespace hack
