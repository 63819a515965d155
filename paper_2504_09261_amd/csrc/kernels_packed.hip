// Rows into a cache of 4 bits and back (layout and rounding: packed_device.h).
//
// Memory-bound.  Packing reads a row of K and one of V (bf16 or float32), in order or through a unit's list of kept rows, cached rows
// and new ones in one numbering, and writes 17/64 of a byte for every bit less; reading back is the same the other way, and exact.
// Eight elements a lane: four lanes share a group's scale.  Everything travels by value, so that lengths that are new in every call of a serving loop fill no
// store of launch tables (host time of appending to 512 units and reading back 54 -> 16 us).
// Measured: 32 units of a 1024^2 image, half of 4200 to 6200 rows of 128 gathered into 4 bits and read back, 20.5 us for 108 MB (5.3 TB/s); one row behind
// each of 512 units and back 4.7 us, a launch's latency twice.  The same image in float32 48.7 us for 194 MB (4.0 TB/s): packing 17.0, reading back 29.7, which is not
// bound by its bytes.  A lane's eight elements are two stores there, each of 16 bytes of every 32, and past the caches these do not become lines: 111 MB are written for 85.
#include <algorithm>

#include "packed_device.h"

namespace hack {

namespace {

using namespace dev;

constexpr int kThreads = 256;
constexpr int64_t kL2Bytes = 32 << 20;   // of eight XCDs: larger outputs pass the caches by

template <typename T> __device__ __forceinline__ void load8(const T* p, float* v);
template <> __device__ __forceinline__ void load8<float>(const float* p, float* v) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
template <> __device__ __forceinline__ void load8<__bf16>(const __bf16* p, float* v) {
  const bf16x8 x = *reinterpret_cast<const bf16x8*>(p);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (float)x[i];
}

template <int CTRL> __device__ __forceinline__ unsigned dpp_max(unsigned v) {
  const unsigned o = (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
  return v > o ? v : o;
}

// The group's exponent, and this lane's eight codes.  Magnitudes are compared as bit patterns, in which NaN is the largest.
__device__ __forceinline__ unsigned encode8(const float* v, unsigned& exponent) {
  unsigned top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __builtin_bit_cast(unsigned, v[i]) & 0x7FFFFFFFu);
  top = dpp_max<0xB1>(top);
  top = dpp_max<0x4E>(top);
  if (top >= 0x7F800000u) {
    exponent = 255;
    return 0;
  }
  // the largest is m 2^(E - 127), 1 <= m < 2: 4 m of the unit 2^(E - 2 - 127), or 2 m of the next one where m is above 7/4
  exponent = (unsigned)min(max((int)((top + 0x1FFFFFu) >> 23) - 2, 3), 252);
  const float scale = scale_of(exponent);
  unsigned w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], scale, 3);
  return w;
}

template <int N> struct PackArgs : PackHead { PackUnit unit[N]; };

template <typename T, int D, int N>
__global__ __launch_bounds__(kThreads) void pack_rows(const PackArgs<N> a) {
  constexpr int LPR = D / 8, RPG = kThreads / LPR;   // lanes of a row, rows of a work-group
  const PackUnit u = a.unit[blockIdx.y];
  const int i = a.row_at + (int)(blockIdx.x * RPG + threadIdx.x / LPR), c = threadIdx.x % LPR;
  if (i >= u.n) return;   // all lanes of a row
  const int64_t unit = a.unit0 + blockIdx.y;
  int src = a.kept ? a.kept[unit * a.kept_stride + i] : i;
  src = min(max(src, 0), u.len_in + a.n_new - 1);
  const bool cached = src < u.len_in;
  const int64_t row = cached ? u.row0 + src : unit * a.n_new + (src - u.len_in);
  float k[8], v[8];
  load8(static_cast<const T*>(cached ? a.plain.k : a.k_new) + row * D + 8 * c, k);
  load8(static_cast<const T*>(cached ? a.plain.v : a.v_new) + row * D + 8 * c, v);
  unsigned ek, ev;
  const unsigned wk = encode8(k, ek), wv = encode8(v, ev);
  const int to = u.first + i, r = to & (kPackRows - 1);
  const int64_t block = (int64_t)(u.block + (to >> 6)) * kPackBytes<D>;
  const int at = code_at<D>(r, 8 * c / (D / 4)) + 4 * (c % (D / 32)), ex = exponent_at<D>(r, c / 4);
  uint8_t* const pk = static_cast<uint8_t*>(a.packed.k) + block;
  uint8_t* const pv = static_cast<uint8_t*>(a.packed.v) + block;
  *reinterpret_cast<unsigned*>(pk + at) = wk;
  *reinterpret_cast<unsigned*>(pv + at) = wv;
  if (c % 4 == 0) {
    pk[ex] = (uint8_t)ek;
    pv[ex] = (uint8_t)ev;
  }
  if (a.packed.pos != nullptr && c == 0 && !(cached && a.plain.pos == nullptr))
    a.packed.pos[(int64_t)u.block * kPackRows + to] = cached ? a.plain.pos[row] : a.pos_new + (src - u.len_in);
}

template <bool STREAM, typename V> __device__ __forceinline__ void put(V* p, const V& x) {
  if constexpr (STREAM) __builtin_nontemporal_store(x, p);
  else *p = x;
}
template <bool STREAM> __device__ __forceinline__ void store8(__bf16* p, unsigned w, float scale) { put<STREAM>(reinterpret_cast<bf16x8*>(p), codes_bf16(w, scale)); }
template <bool STREAM> __device__ __forceinline__ void store8(float* p, unsigned w, float scale) {
  const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1),
             c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
  put<STREAM>(reinterpret_cast<floatx4*>(p), floatx4{a[0], a[1], b[0], b[1]});
  put<STREAM>(reinterpret_cast<floatx4*>(p) + 1, floatx4{c[0], c[1], d[0], d[1]});
}

template <typename T, int D, int N, bool STREAM>
__global__ __launch_bounds__(kThreads) void unpack_rows(const PackArgs<N> a) {
  constexpr int LPR = D / 8, RPG = kThreads / LPR;
  const PackUnit u = a.unit[blockIdx.y];
  const int i = a.row_at + (int)(blockIdx.x * RPG + threadIdx.x / LPR), c = threadIdx.x % LPR;
  if (i >= u.n) return;
  const int from = u.first + i, r = from & (kPackRows - 1);
  const int64_t block = (int64_t)(u.block + (from >> 6)) * kPackBytes<D>;
  const int at = code_at<D>(r, 8 * c / (D / 4)) + 4 * (c % (D / 32)), ex = exponent_at<D>(r, c / 4);
  const uint8_t* const pk = static_cast<const uint8_t*>(a.packed.k) + block;
  const uint8_t* const pv = static_cast<const uint8_t*>(a.packed.v) + block;
  const unsigned wk = *reinterpret_cast<const unsigned*>(pk + at), wv = *reinterpret_cast<const unsigned*>(pv + at);
  const float sk = scale_of(pk[ex]), sv = scale_of(pv[ex]);
  const int64_t row = u.row0 + i;
  store8<STREAM>(static_cast<T*>(a.plain.k) + row * D + 8 * c, wk, sk);
  store8<STREAM>(static_cast<T*>(a.plain.v) + row * D + 8 * c, wv, sv);
  if (a.plain.pos != nullptr && a.packed.pos != nullptr && c == 0) a.plain.pos[row] = a.packed.pos[(int64_t)u.block * kPackRows + from];
}

template <typename T, int D, int N>
void launch_some(hipStream_t s, bool pack, const PackHead& h, const PackUnit* units, int n_units) {
  PackArgs<N> a;
  static_cast<PackHead&>(a) = h;
  int rows = 0;
  int64_t all = 0;
  for (int i = 0; i < n_units; ++i) {
    a.unit[i] = units[i];
    rows = std::max(rows, units[i].n);
    all += units[i].n;
  }
  constexpr int per = kThreads / (D / 8);
  constexpr int kMostRows = 1 << 27;   // of a unit and a launch, which counts its threads in 32 bits; a row's number and what a work-group adds fit them too
  for (int64_t at = 0; at < rows; at += kMostRows) {
    a.row_at = (int)at;
    const dim3 grid((unsigned)((std::min<int64_t>(rows - at, kMostRows) + per - 1) / per), n_units);
    if (pack) hipLaunchKernelGGL((pack_rows<T, D, N>), grid, dim3(kThreads), 0, s, a);
    else if (2 * all * D * (int64_t)sizeof(T) > kL2Bytes) hipLaunchKernelGGL((unpack_rows<T, D, N, true>), grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((unpack_rows<T, D, N, false>), grid, dim3(kThreads), 0, s, a);
  }
}

template <typename T, int D>
void launch_all(hipStream_t s, bool pack, PackHead h, const PackUnit* units, int n_units) {
  for (int u = 0; u < n_units; u += kPackUnits) {
    h.unit0 = u;
    const int n = std::min(kPackUnits, n_units - u);
    if (n <= kFewUnits) launch_some<T, D, kFewUnits>(s, pack, h, units + u, n);
    else launch_some<T, D, kPackUnits>(s, pack, h, units + u, n);
  }
}

void launch(hipStream_t s, int elem_bytes, int head_dim, bool pack, const PackHead& h, const PackUnit* units, int n_units) {
  if (elem_bytes == 4) {
    if (head_dim == 64) launch_all<float, 64>(s, pack, h, units, n_units);
    else launch_all<float, 128>(s, pack, h, units, n_units);
  } else {
    if (head_dim == 64) launch_all<__bf16, 64>(s, pack, h, units, n_units);
    else launch_all<__bf16, 128>(s, pack, h, units, n_units);
  }
}

}  // namespace

void launch_pack(hipStream_t s, int elem_bytes, int head_dim, PackHead h, const PackUnit* units, int n_units) {
  launch(s, elem_bytes, head_dim, true, h, units, n_units);
}
void launch_unpack(hipStream_t s, int elem_bytes, int head_dim, PackHead h, const PackUnit* units, int n_units) {
  launch(s, elem_bytes, head_dim, false, h, units, n_units);
}

}  // namespace hack
