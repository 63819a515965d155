// Rotary positions of queries and keys, alone or behind the norm of each head's row.
//
// A pair (a, b) of a head's row at position p turns by p f: (a c - b s, a s + b c) with c, s = gain cos(p f), gain sin(p f).  Pairs are (i, i + S/2)
// or (2i, 2i + 1) of a section of S elements; with two axes a head has two sections, each turned by a position of its own.  In front of it, RMS norm
// x / sqrt(mean x^2 + eps) w or unit norm x / max(|x|, eps) w over the whole row.
//
// Memory-bound: a row is read and written once, whatever the strides it is read with.  A lane holds 16 elements of a row, pieces of 16 bytes chosen so
// that its pairs are its own and the lanes of an access lie side by side: no exchange but the sum of squares over the 8 (head_dim 128) or 4 lanes of a row.  Angles are formed
// once for a token and used for all heads that the thread walks over.  They are exact where it matters: the frequency is held in units of 2^-64
// turns, so the product with a position wraps to its fraction of a turn in integers, however far the position (cut at 2^-32 turns, 1.5e-9 rad).
// Measured: 16384 rows of 32 + 8 heads of 128 out of a projection, normed and turned, 66 us (5.1 TB/s of the 6.2 that a plain elementwise
// kernel reaches), 2 x 4096 rows of 16 heads in two axes 13 us (5.1).
#include "rotate_device.h"

namespace hack {

namespace {

using namespace dev;

constexpr int kThreads = kRotateThreads;

template <typename T, int D, bool HALF, bool NORM, bool STREAM>
__global__ __launch_bounds__(kThreads) void rotate_rows(const RotateArgs a) {
  const int64_t b = blockIdx.x / a.groups[1];
  unsigned x = blockIdx.x - (unsigned)b * a.groups[1];
  const bool second = x >= a.groups[0];
  const RotateTensor& t = a.t[second ? 1 : 0];
  if (second) x -= a.groups[0];
  turn_rows<T, D, HALF, NORM, STREAM>(a, t, b, x, a.rot_dim, a.pos0, [&](int64_t n) {
    return ToArray<T>{true, static_cast<T*>(t.out) + (b * t.heads * a.n + n) * D, (int64_t)a.n * D};
  });
}

template <typename T, int D, bool HALF>
void launch_form(hipStream_t s, bool stream, unsigned groups, const RotateArgs& a) {
#define HACK_ROTATE(NORM, STREAM) hipLaunchKernelGGL((rotate_rows<T, D, HALF, NORM, STREAM>), dim3(groups), dim3(kThreads), 0, s, a)
  if (a.norm == kNormNone) {
    if (stream) HACK_ROTATE(false, true);
    else HACK_ROTATE(false, false);
  } else {
    if (stream) HACK_ROTATE(true, true);
    else HACK_ROTATE(true, false);
  }
#undef HACK_ROTATE
}

template <typename T, int D>
void launch_typed(hipStream_t s, bool half_layout, bool stream, unsigned groups, const RotateArgs& a) {
  if (half_layout) launch_form<T, D, true>(s, stream, groups, a);
  else launch_form<T, D, false>(s, stream, groups, a);
}

}  // namespace

void launch_rotate(hipStream_t s, int elem_bytes, int head_dim, bool half_layout, int batch, int n_tensors, RotateArgs a) {
  int64_t rows = 0;
  for (int i = 0; i < n_tensors; ++i) rows += (int64_t)batch * a.n * a.t[i].heads;
  // With an eps from 2^-50 on, what a sum of squares below 2^-100 is off by does not reach the result.
  a.low = a.eps < 0x1p-50f ? 0x1p-100f : 0.f;
  const bool stream = streams(a, half_layout, head_dim, rows * head_dim * elem_bytes);
  const unsigned groups = a.groups[1] * (unsigned)batch;
  if (elem_bytes == 4) {
    if (head_dim == 64) launch_typed<float, 64>(s, half_layout, stream, groups, a);
    else launch_typed<float, 128>(s, half_layout, stream, groups, a);
  } else {
    if (head_dim == 64) launch_typed<__bf16, 64>(s, half_layout, stream, groups, a);
    else launch_typed<__bf16, 128>(s, half_layout, stream, groups, a);
  }
}

}  // namespace hack
