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
#include <algorithm>
#include <cfloat>

#include "device_util.h"
#include "ops_internal.h"

namespace hack {

namespace {

using namespace dev;

constexpr int kThreads = kRotateThreads;
constexpr int64_t kL2Bytes = 32 << 20;   // of eight XCDs

// 2^32 u turns -> cosine and sine.  The nearest quarter turn, then the Taylor series of the rest (at most pi / 4: the first terms
// left out are 1.8e-9 of the sine, 1.2e-10 of the cosine).  The rest is a float32 number of radians: rounded twice, up to 7.5e-8 off.
__device__ __forceinline__ void cos_sin(unsigned u, float& c, float& s) {
  const unsigned q = (u + 0x20000000u) >> 30;
  const float x = (float)(int)(u - (q << 30)) * 1.4629180792671596e-9f;   // 2 pi 2^-32
  const float y = x * x;
  const float sx = fmaf(x * y, fmaf(y, fmaf(y, fmaf(y, 2.7557319e-6f, -1.9841270e-4f), 8.3333333e-3f), -1.6666667e-1f), x);
  const float cx = fmaf(y, fmaf(y, fmaf(y, fmaf(y, fmaf(y, -2.7557319e-7f, 2.4801587e-5f), -1.3888889e-3f), 4.1666667e-2f), -0.5f), 1.f);
  const float a = (q & 1) ? sx : cx, b = (q & 1) ? cx : sx;
  c = ((q + 1) & 2) ? -a : a;
  s = (q & 2) ? -b : b;
}

template <bool STREAM, typename V> __device__ __forceinline__ void put(V* p, const V& x) {
  if constexpr (STREAM) __builtin_nontemporal_store(x, p);
  else *p = x;
}
template <typename T> struct Piece;   // 16 bytes
template <> struct Piece<float> {
  static constexpr int kElements = 4;
  static __device__ __forceinline__ void load(const float* p, float* v) {
    const floatx4 a = *reinterpret_cast<const floatx4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a[i];
  }
  template <bool STREAM> static __device__ __forceinline__ void store(float* p, const float* v) {
    put<STREAM>(reinterpret_cast<floatx4*>(p), floatx4{v[0], v[1], v[2], v[3]});
  }
};
template <> struct Piece<__bf16> {
  static constexpr int kElements = 8;
  static __device__ __forceinline__ void load(const __bf16* p, float* v) {
    const bf16x8 x = *reinterpret_cast<const bf16x8*>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)x[i];
  }
  template <bool STREAM> static __device__ __forceinline__ void store(__bf16* p, const float* v) {
    bf16x8 x;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (__bf16)v[i];
    put<STREAM>(reinterpret_cast<bf16x8*>(p), x);
  }
};

template <int CTRL> __device__ __forceinline__ float dpp_add(float v) {
  return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}

// Of the lanes of a row, in all of them.
template <int LPR> __device__ __forceinline__ float row_sum(float v) {
  v = dpp_add<0xB1>(v);    // lane ^ 1
  v = dpp_add<0x4E>(v);    // lane ^ 2
  return LPR == 8 ? dpp_add<0x141>(v) : v;   // mirrored within eight lanes
}
template <int CTRL> __device__ __forceinline__ unsigned dpp_max(unsigned v) {
  return max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true));
}
template <int LPR> __device__ __forceinline__ unsigned row_max(unsigned v) {
  v = dpp_max<0xB1>(v);
  v = dpp_max<0x4E>(v);
  return LPR == 8 ? dpp_max<0x141>(v) : v;
}
__device__ __forceinline__ float sum_of_squares(const float* v) {
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) ss = fmaf(v[i], v[i], ss);
  return ss;
}

template <int E> __device__ __forceinline__ void load_weights(const float* p, float* v) {
#pragma unroll
  for (int i = 0; i < E; i += 4) Piece<float>::load(p + i, v + i);
}

template <typename T, int D, bool HALF, bool NORM, bool STREAM>
__global__ __launch_bounds__(kThreads) void rotate_rows(const RotateArgs a) {
  constexpr int LPR = D / 16;             // lanes of a row
  constexpr int SLOTS = kThreads / LPR;   // rows of a work-group at a time
  const int j = threadIdx.x % LPR, slot = threadIdx.x / LPR;
  const int64_t b = blockIdx.x / a.groups[1];
  unsigned x = blockIdx.x - (unsigned)b * a.groups[1];
  const bool second = x >= a.groups[0];
  const RotateTensor& t = a.t[second ? 1 : 0];
  if (second) x -= a.groups[0];
  const int chunk = x / (unsigned)t.tiles, tile = x - (unsigned)chunk * t.tiles;
  const int64_t n = (int64_t)(tile << t.tokens_log2) + (slot & ((1 << t.tokens_log2) - 1));
  if (n >= a.n) return;   // all lanes of a row

  // This lane's 16 elements: a piece of every part of its region of a row.  Pairs side by side lie in one piece, so that the region is the whole row and
  // pieces turn or not; pairs (i, i + S/2) need a region each for an axis' section and for what does not rotate, and lanes turn or not.  (Regions for the
  // former too: 3 x 1369 float32 rows of 20 heads of 64, of which 16 elements rotate, 11.8 us, so 9.6; 50 x 900 of 8 + 1 heads 70, 37.)
  constexpr int E = Piece<T>::kElements, PIECES = 16 / E;
  const bool lane_turns = 16 * j < a.rot_dim;
  int base = 0, size = D;
  if (HALF) {
    base = lane_turns ? (16 * j >= a.section ? a.section : 0) : a.rot_dim;
    size = lane_turns ? a.section : D - a.rot_dim;
  }
  const int part = size / PIECES, in_part = (16 * j - base) / PIECES, at = base + in_part;   // elements of a part, and this lane's first one
  const auto turns = [&](int piece) { return HALF ? lane_turns : at + piece * part < a.rot_dim; };
  constexpr int STEP = HALF ? 8 : E / 2;   // pairs that turn or not together
  const int* const pos = a.pos ? a.pos + b * a.pos_b + n : nullptr;
  const bool two = HALF ? lane_turns && base > 0 : a.section < a.rot_dim;   // the second axis' position is needed
  int p0 = a.pos0 + (int)n, p1 = p0;   // on the two axes
  if (pos) {
    p0 = pos[0];
    if (two) p1 = pos[a.n];
  }
  uint64_t f[8];   // loaded in front of the branches; numbers of pairs that do not turn are below D / 2 too
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = a.turns[HALF ? base / 2 + i / E * part + in_part + i % E : (at + 2 * i / E * part + 2 * i % E) / 2];
  float c[8], s[8];
#pragma unroll
  for (int i0 = 0; i0 < 8; i0 += STEP) {   // pair i: elements i and 8 + i, or 2 i and 2 i + 1
    const int piece = 2 * i0 / E;
    if (!turns(piece)) continue;
    const int p = (HALF ? base > 0 : at + piece * part >= a.section) ? p1 : p0;
#pragma unroll
    for (int i = i0; i < i0 + STEP; ++i) {
      // upper half of the low 64 bits of p f; the low half of f makes up for p < 0 standing for p + 2^32
      const unsigned u = __umulhi((unsigned)p, (unsigned)f[i]) + (unsigned)p * (unsigned)(f[i] >> 32) - (p < 0 ? (unsigned)f[i] : 0u);
      cos_sin(u, c[i], s[i]);
      c[i] *= a.gain;
      s[i] *= a.gain;
    }
  }
  const T* src = static_cast<const T*>(t.x) + b * t.sb + n * t.sn;
  T* dst = static_cast<T*>(t.out) + (b * t.heads * a.n + n) * D;
  const int across = SLOTS >> t.tokens_log2;   // heads at a time
  const int h0 = chunk * across * a.steps + (slot >> t.tokens_log2);
  const int h1 = min(t.heads, (chunk + 1) * across * a.steps);
  float w[16];
  if (NORM && t.w != nullptr && t.w_stride == 0) {
#pragma unroll
    for (int k = 0; k < PIECES; ++k) load_weights<E>(t.w + at + k * part, w + k * E);
  }
  for (int h = h0; h < h1; h += across) {
    float v[16];
#pragma unroll
    for (int k = 0; k < PIECES; ++k) Piece<T>::load(src + h * t.sh + at + k * part, v + k * E);
    if (NORM) {
      if (t.w != nullptr && t.w_stride != 0) {
#pragma unroll
        for (int k = 0; k < PIECES; ++k) load_weights<E>(t.w + (int64_t)h * t.w_stride + at + k * part, w + k * E);
      }
      float ss = row_sum<LPR>(sum_of_squares(v)), eps = a.eps, eps2 = a.eps;
      // Squares that float32 does not hold, and do matter: the row is scaled by a power of two (eps with it, for the mean of squares twice) that brings its largest
      // element to about one.  The RMS norm leaves a tiny row where eps, 2^-149 at least, still fits scaled by 2^120, and decides.
      if (__builtin_expect(!(ss >= a.low && ss <= FLT_MAX), 0)) {
        unsigned top = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) top = max(top, __builtin_bit_cast(unsigned, v[i]) & 0x7FFFFFFFu);
        top = row_max<LPR>(top);
        if (top == 0) {
          eps = eps2 = 1.f;   // a row of zeros stays one, whatever 1 / eps is
        } else if (top < 0x7F800000u) {
          const int e = 253 - (int)(top >> 23);
          const float scale = __builtin_bit_cast(float, (unsigned)min(max(e, 1), a.norm == kNormRms ? 187 : 253) << 23);
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] *= scale;
          ss = row_sum<LPR>(sum_of_squares(v));
          eps *= scale;
          eps2 = eps * scale;
        }
      }
      const float r = 1.f / (a.norm == kNormRms ? sqrtf(ss * (1.f / D) + eps2) : fmaxf(sqrtf(ss), eps));
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        v[i] *= r;
        if (t.w != nullptr) v[i] *= w[i];
      }
    }
#pragma unroll
    for (int i0 = 0; i0 < 8; i0 += STEP) {
      if (!turns(2 * i0 / E)) continue;
#pragma unroll
      for (int i = i0; i < i0 + STEP; ++i) {
        const int ia = HALF ? i : 2 * i, ib = HALF ? 8 + i : 2 * i + 1;
        const float p = v[ia], q = v[ib];
        v[ia] = fmaf(p, c[i], -(q * s[i]));
        v[ib] = fmaf(p, s[i], q * c[i]);
      }
    }
    T* o = dst + (int64_t)h * a.n * D;
#pragma unroll
    for (int k = 0; k < PIECES; ++k) Piece<T>::template store<STREAM>(o + at + k * part, v + k * E);
  }
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
  // Outputs that the L2 caches cannot hold pass them by (16384 rows of 32 + 8 heads 71.7 -> 65.3 us, 32 x 256 of 30 + 30 heads 30.2 -> 26.6); smaller ones
  // are for the next launch to find there, and where a row's pieces of an access make up less than 32 bytes (as many as its region has elements) they
  // need the caches to become lines (8 x 8192 float32 rows of 16 heads of 64, of which 16 elements rotate: 129 us, past the caches 326; 32 elements of bf16 rows 61, 51).
  const auto wide = [&](int region) { return !half_layout || region == 0 || region >= 32; };
  const bool stream = rows * head_dim * elem_bytes > kL2Bytes && wide(a.section) && wide(head_dim - a.rot_dim);
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
