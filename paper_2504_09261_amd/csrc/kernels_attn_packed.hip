// Attention over a cache held in 4 bits: O = Softmax(scale Q K^T) V for every unit over its own rows, no mask (layout and rounding of
// the rows: packed_device.h).
//
// A code times its power of two is a bf16 number, so K and V enter the 16x16x32 bf16 matrix instructions exactly; what is rounded is what
// attention over bf16 rows rounds, the probabilities and the output.  In a float32 context queries and probabilities enter as three bf16 pieces each, which add up
// to them exactly, so products and sums are those of float32.
//
// A work-group takes 16 NQ queries of a unit and a chunk of its keys, its four waves every fourth block of 64 keys, each by itself.  K comes from
// memory in the order of the A operand of S^T = K Q^T: conversion is all that stands between the load and the product.  V^T needs
// keys side by side where memory has head-dim: a wave writes the converted rows to LDS and reads them with the transposing LDS read, in the order of keys in
// which the accumulators hold the probabilities.  One softmax update a block.  The next block's codes are loaded into the registers of this one's as soon as those have
// been converted.  The partial results of the waves are merged through LDS, those of several chunks of a unit in memory, by a launch of their own.
//
// One token reads its cache once and is bound by that: 768 units of 4096 rows at head_dim 128 (428 MB) take 86 us, 5.0 TB/s, 512 units (285 MB, part of which the
// last-level cache keeps from launch to launch) 46, and 58 and 44 where all units share one cache, so arithmetic is not far behind.  A block takes a wave 2.9 us with another work-group on the
// compute unit and 1.6 alone.  Tried: four work-groups a compute unit (128 registers spill) 41 -> 56 us for 512 units of 900 to 4000 rows; V in two halves of
// 32 rows, three work-groups a compute unit, equal within 3 %; the last work-group of a unit to end merges its chunks (tickets), 8.9 -> 9.6 us for 8 units of 4000 rows,
// 13.6 -> 15.8 for 32.  In float32 contexts there are three matrix instructions for every bf16 one: 512 units of 900 to 4000 rows, 4 queries 45 us (bf16 37), 32 units of
// 3000 rows, 1000 queries 136 us (362 TFLOP/s; bf16 in its form of 128 queries 66).  K by the scaled matrix instruction, codes as they are and queries in two 8-bit or three 6-bit pieces: the sums keep 16 bits of the largest
// product, or the pieces 14 of the largest query element, where bf16 operands lose nothing.
#include <cfloat>
#include <type_traits>

#include "packed_device.h"

namespace hack {

namespace {

using namespace dev;

constexpr int kWaves = 4;

template <int D> struct PackedRows {   // a lane's share of a block of 64 rows
  uintx4 code[D / 32];
  unsigned exponents;
  __device__ __forceinline__ void load(const uint8_t* block, int lane) {
    const uintx4* c = reinterpret_cast<const uintx4*>(block) + lane;
#pragma unroll
    for (int p = 0; p < D / 32; ++p) code[p] = c[64 * p];
    exponents = reinterpret_cast<const unsigned*>(block + 32 * D)[D == 128 ? lane : (lane >> 5) * 16 + (lane & 15)];
  }
  // of tile t (16 rows) the eight elements of slice s of the lane's quarter
  __device__ __forceinline__ unsigned slice(int t, int s) const { return D == 128 ? code[t][s] : code[t >> 1][(t & 1) * 2 + s]; }
  __device__ __forceinline__ float scale(int t) const { return scale_of((exponents >> (8 * t)) & 255u); }
};

// A number as a sum of bf16 pieces: itself, or three pieces of eight bits each, exactly.  (Cut, not rounded: a piece never passes the number.)
template <typename T> struct Pieces;
template <> struct Pieces<__bf16> {
  static constexpr int kCount = 1;
  static __device__ __forceinline__ void load(const __bf16* p, bf16x8 (&f)[1]) { f[0] = *reinterpret_cast<const bf16x8*>(p); }
  static __device__ __forceinline__ void split(float x, int j, bf16x8 (&f)[1]) { f[0][j] = (__bf16)x; }
};
template <> struct Pieces<float> {
  static constexpr int kCount = 3;
  static __device__ __forceinline__ void split(float x, int j, bf16x8 (&f)[3]) {
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      const unsigned top = __builtin_bit_cast(unsigned, x) & 0xFFFF0000u;
      f[i][j] = __builtin_bit_cast(__bf16, (unsigned short)(top >> 16));
      x -= __builtin_bit_cast(float, top);
    }
  }
  static __device__ __forceinline__ void load(const float* p, bf16x8 (&f)[3]) {
    const floatx4 a = reinterpret_cast<const floatx4*>(p)[0], b = reinterpret_cast<const floatx4*>(p)[1];
#pragma unroll
    for (int j = 0; j < 8; ++j) split(j < 4 ? a[j] : b[j - 4], j, f);
  }
};
__device__ __forceinline__ void store4(__bf16* p, const floatx4& x, float f) {
  *reinterpret_cast<bf16x4*>(p) = bf16x4{(__bf16)(x[0] * f), (__bf16)(x[1] * f), (__bf16)(x[2] * f), (__bf16)(x[3] * f)};
}
__device__ __forceinline__ void store4(float* p, const floatx4& x, float f) { *reinterpret_cast<floatx4*>(p) = floatx4{x[0] * f, x[1] * f, x[2] * f, x[3] * f}; }

template <typename T, int D, int NQ, int N>
__global__ __launch_bounds__(64 * kWaves, NQ == 2 || sizeof(T) == 4 ? 2 : D == 64 ? 4 : 2) void attn_packed(const AttnPackedArgs<N> a) {
  constexpr int KC = D / 32, MT = D / 16, QROWS = 16 * NQ, NP = Pieces<T>::kCount;
  constexpr int SLOT = 64 * D;   // elements: a block of V, then the wave's partial results
  // The query tiles of a unit and a chunk follow each other on an XCD (work-group id mod 8).
  const int local = blockIdx.x >> 3, pair = (local / a.q_tiles) * 8 + (blockIdx.x & 7), q_tile = local % a.q_tiles;
  if (pair >= a.n_units * a.n_chunks) return;
  const int ui = pair % a.n_units, chunk = pair / a.n_units;
  const AttnPackedUnit u = a.unit[ui];
  const int len = u.len, n_blocks = packed_blocks(len);
  const int chunks = chunks_of(n_blocks, a.chunk);
  if (chunk >= chunks) return;
  const int first = chunk_at(n_blocks, chunks, chunk), last = chunk_at(n_blocks, chunks, chunk + 1);
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, g = lane >> 4;
  const int q0 = q_tile * QROWS;
  const int64_t row0 = (int64_t)u.unit * a.N_k;

  __shared__ __attribute__((aligned(1024))) __bf16 ring[kWaves][SLOT];
  __shared__ float m_sh[kWaves][QROWS], l_sh[kWaves][QROWS];

  // This wave's blocks: first + w, first + w + kWaves, ...  A block's K is needed until its scores are formed, its V until it lies in LDS: the
  // next ones are loaded into the same registers then and have the rest of the iteration to arrive.
  int b = first + w;
  const uint8_t* kb = a.k + ((int64_t)u.block + b) * kPackBytes<D>;
  const uint8_t* vb = a.v + ((int64_t)u.block + b) * kPackBytes<D>;
  PackedRows<D> kr, vr;
  if (b < last) {
    kr.load(kb, lane);
    vr.load(vb, lane);
  }
  // Queries as the B operand, in the order in which the lane's quarter of a key comes: element 8 s + j of quarter g
  bf16x8 qf[NQ][KC][NP];
#pragma unroll
  for (int qt = 0; qt < NQ; ++qt) {
    const T* row = static_cast<const T*>(a.q) + (row0 + min(q0 + 16 * qt + col, a.N_k - 1)) * D + g * (D / 4);
#pragma unroll
    for (int s = 0; s < KC; ++s) Pieces<T>::load(row + 8 * s, qf[qt][s]);
  }
  floatx4 o[MT][NQ];   // O^T: head-dim 16 mt + 4 g + r, query 16 qt + col
  floatx4 ls[NQ];      // row sums of P: all four rows hold the same
  float mc[NQ];        // probabilities are 2^(c2 s - mc); finite from the start, so that keys whose score is -inf get 0
  const float c2 = a.scale * kLog2eF;
  bf16x8 ones;
#pragma unroll
  for (int j = 0; j < 8; ++j) ones[j] = (__bf16)1.0f;
#pragma unroll
  for (int qt = 0; qt < NQ; ++qt) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) o[mt][qt] = floatx4{0.f, 0.f, 0.f, 0.f};
    ls[qt] = floatx4{0.f, 0.f, 0.f, 0.f};
    mc[qt] = -FLT_MAX;
  }
  // V^T operand: rows 4 g + e and 16 + 4 g + e, head-dim 16 mt + 4 qd; even and odd mt
  const int qd = col & 3, v_even = v_chunk<D>(4 * g + (col >> 2), qd >> 1) + 4 * (qd & 1), v_odd = v_even ^ 16;
  __bf16* const slot = &ring[w][0];

  // RAGGED: rows of this block lie behind the unit's last one.  They may hold anything: their scores are masked, and as their probabilities are
  // zero, V is zero there too, since the product must not meet a NaN.
  auto block = [&](auto ragged_tag) {
    constexpr bool RAGGED = decltype(ragged_tag)::value;
    const bool more = b + kWaves < last;
    floatx4 sc[4][NQ];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const float scale = kr.scale(t);
#pragma unroll
      for (int qt = 0; qt < NQ; ++qt) sc[t][qt] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < KC; ++s) {
        const bf16x8 kf = codes_bf16(kr.slice(t, s), scale);
#pragma unroll
        for (int qt = 0; qt < NQ; ++qt)
#pragma unroll
          for (int i = NP - 1; i >= 0; --i) sc[t][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[qt][s][i], sc[t][qt], 0, 0, 0);
      }
    }
    const int left = len - b * kPackRows;   // rows of this block and behind it
    wave_lds_order();   // the last reads of the slot
#pragma unroll
    for (int t = 0; t < 4; ++t) {   // V as bf16
      const int r = 16 * t + col;
      const bool there = !RAGGED || r < left;
      const float scale = there ? vr.scale(t) : 1.f;
#pragma unroll
      for (int s = 0; s < KC; ++s)
        *reinterpret_cast<bf16x8*>(&slot[v_chunk<D>(r, KC * g + s)]) = codes_bf16(there ? vr.slice(t, s) : 0u, scale);
    }
    wave_lds_order();
    kb += kWaves * kPackBytes<D>;
    vb += kWaves * kPackBytes<D>;
    if (more) {
      kr.load(kb, lane);
      vr.load(vb, lane);
    }
    if constexpr (RAGGED) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (16 * t + 4 * g + r >= left) {
#pragma unroll
            for (int qt = 0; qt < NQ; ++qt) sc[t][qt][r] = -INFINITY;
          }
    }
    // The reference is the largest score so far: the largest probabilities lie just below one, where bf16 rounds them finest.
    float m_new[NQ];
    bool moved = false;
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) {
      float mx = sc[0][qt][0];
#pragma unroll
      for (int j = 1; j < 16; ++j) mx = maximum(mx, sc[j >> 2][qt][j & 3]);
      m_new[qt] = maximum(mc[qt], quad_maximum(mx) * c2);
      moved |= m_new[qt] != mc[qt];
    }
    if (__any(moved)) {
#pragma unroll
      for (int qt = 0; qt < NQ; ++qt) {
        const float f = __builtin_amdgcn_exp2f(mc[qt] - m_new[qt]);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          ls[qt][r] *= f;
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) o[mt][qt][r] *= f;
        }
        mc[qt] = m_new[qt];
      }
    }
    bf16x8 pf[2][NQ][NP];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int qt = 0; qt < NQ; ++qt) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          Pieces<T>::split(__builtin_amdgcn_exp2f(fmaf(sc[2 * h + (j >> 2)][qt][j & 3], c2, -mc[qt])), j, pf[h][qt]);
#pragma unroll
        for (int i = NP - 1; i >= 0; --i)   // sums over the numbers that the PV product uses
          ls[qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[h][qt][i], ls[qt], 0, 0, 0);
      }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        const __bf16* const at = slot + 32 * h * D + 128 * (mt >> 1) + (mt & 1 ? v_odd : v_even);
        const bf16x4 v0 = lds_read_tr(at), v1 = lds_read_tr(at + 16 * D);
        const bf16x8 vf = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
#pragma unroll
        for (int qt = 0; qt < NQ; ++qt)
#pragma unroll
          for (int i = NP - 1; i >= 0; --i) o[mt][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[h][qt][i], o[mt][qt], 0, 0, 0);
      }
  };
  const int full = min(last, len / kPackRows);
  for (; b < full; b += kWaves) block(std::false_type{});
  if (b < last) block(std::true_type{});

  // ---- merge the waves' partial results ----
  constexpr int kPart = SLOT * 2 / 16;   // float4 per wave
  static_assert(NQ * MT * 64 <= kPart && kWaves % NQ == 0, "partial results fit the slots");
  wave_lds_order();
  float4* mine = reinterpret_cast<float4*>(slot) + lane;
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) mine[(mt * NQ + qt) * 64] = make_float4(o[mt][qt][0], o[mt][qt][1], o[mt][qt][2], o[mt][qt][3]);
  if (g == 0) {
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) {
      m_sh[w][16 * qt + col] = mc[qt];
      l_sh[w][16 * qt + col] = ls[qt][0];
    }
  }
  __syncthreads();
  // wave w finishes query tile w % NQ, head-dim tiles w / NQ, w / NQ + kWaves / NQ, ...
  const int qt = w % NQ;
  float M = -FLT_MAX;
#pragma unroll
  for (int x = 0; x < kWaves; ++x) M = fmaxf(M, m_sh[x][16 * qt + col]);
  float f[kWaves], L = 0.f;
#pragma unroll
  for (int x = 0; x < kWaves; ++x) {
    f[x] = __builtin_amdgcn_exp2f(m_sh[x][16 * qt + col] - M);   // a wave without blocks has summed nothing
    L = fmaf(f[x], l_sh[x][16 * qt + col], L);
  }
  const bool whole = chunks == 1;
  const float inv = whole ? 1.f / L : 1.f;
  const int qi = q0 + 16 * qt + col;
  const int64_t part = (((int64_t)ui * a.q_tiles + q_tile) * a.n_chunks + chunk) * QROWS + 16 * qt + col;
  const float4* const parts = reinterpret_cast<const float4*>(&ring[0][0]) + lane;
#pragma unroll
  for (int m = 0; m < MT; m += kWaves / NQ) {
    const int mt = m + w / NQ;
    if (mt >= MT) break;
    floatx4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < kWaves; ++x) {
      const float4 p = parts[x * kPart + (mt * NQ + qt) * 64];
      acc[0] = fmaf(f[x], p.x, acc[0]);
      acc[1] = fmaf(f[x], p.y, acc[1]);
      acc[2] = fmaf(f[x], p.z, acc[2]);
      acc[3] = fmaf(f[x], p.w, acc[3]);
    }
    if (qi >= a.N_k) continue;
    if (whole) store4(static_cast<T*>(a.out) + (row0 + qi) * D + 16 * mt + 4 * g, acc, inv);
    else *reinterpret_cast<floatx4*>(a.part_o + part * D + 16 * mt + 4 * g) = acc;
  }
  if (!whole && w < NQ && g == 0 && qi < a.N_k) {
    a.part_ml[2 * part] = M;
    a.part_ml[2 * part + 1] = L;
  }
}

// Rows of units that were cut, where these are few and the chunks many: a work-group takes one query, D / 4 lanes a chunk.
template <typename T, int D, int N>
__global__ __launch_bounds__(256) void attn_packed_merge(const AttnPackedArgs<N> a, int q_rows) {
  constexpr int LPR = D / 4, SIDE = 256 / LPR;   // chunks at a time
  const int ui = blockIdx.y, n = chunks_of(packed_blocks(a.unit[ui].len), a.chunk);
  if (n == 1) return;
  const int tid = threadIdx.x, qi = blockIdx.x, c0 = tid / LPR, lane = tid % LPR;
  const int64_t part0 = ((int64_t)ui * a.q_tiles + qi / q_rows) * a.n_chunks * q_rows + qi % q_rows;
  const float2* const ml = reinterpret_cast<const float2*>(a.part_ml) + part0;
  const float4* const po = reinterpret_cast<const float4*>(a.part_o + part0 * D) + lane;
  __shared__ float4 o_sh[SIDE][LPR];
  __shared__ float f_sh[kMostChunks], m_sh[4], l_sh[4];
  // The first results are on their way while the factors are formed.
  constexpr int kEarly = 8;
  float4 early[kEarly];
#pragma unroll
  for (int i = 0; i < kEarly; ++i)
    if (c0 + i * SIDE < n) early[i] = po[(int64_t)(c0 + i * SIDE) * q_rows * LPR];
  float M = -FLT_MAX, L = 0.f;
  for (int c = tid; c < n; c += 256) M = fmaxf(M, ml[(int64_t)c * q_rows].x);
#pragma unroll
  for (int x = 1; x < 64; x *= 2) M = fmaxf(M, __shfl_xor(M, x, 64));
  if ((tid & 63) == 0) m_sh[tid >> 6] = M;
  __syncthreads();
  M = fmaxf(fmaxf(m_sh[0], m_sh[1]), fmaxf(m_sh[2], m_sh[3]));
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](float f, const float4& x) {
    o.x = fmaf(f, x.x, o.x);
    o.y = fmaf(f, x.y, o.y);
    o.z = fmaf(f, x.z, o.z);
    o.w = fmaf(f, x.w, o.w);
  };
  for (int c = tid; c < n; c += 256) {
    const float2 x = ml[(int64_t)c * q_rows];
    const float f = __builtin_amdgcn_exp2f(x.x - M);
    f_sh[c] = f;
    L = fmaf(f, x.y, L);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kEarly; ++i)
    if (c0 + i * SIDE < n) add(f_sh[c0 + i * SIDE], early[i]);
#pragma unroll 4
  for (int c = c0 + kEarly * SIDE; c < n; c += SIDE) add(f_sh[c], po[(int64_t)c * q_rows * LPR]);
#pragma unroll
  for (int x = 1; x < 64; x *= 2) L += __shfl_xor(L, x, 64);
  if ((tid & 63) == 0) l_sh[tid >> 6] = L;
  o_sh[c0][lane] = o;
  __syncthreads();
  if (c0 != 0) return;
#pragma unroll
  for (int x = 1; x < SIDE; ++x) {
    const float4 p = o_sh[x][lane];
    o.x += p.x;
    o.y += p.y;
    o.z += p.z;
    o.w += p.w;
  }
  const float inv = 1.f / (l_sh[0] + l_sh[1] + l_sh[2] + l_sh[3]);
  store4(static_cast<T*>(a.out) + ((int64_t)a.unit[ui].unit * a.N_k + qi) * D + 4 * lane, floatx4{o.x, o.y, o.z, o.w}, inv);
}

// The same for many rows or few chunks: a query to D / 4 lanes, which walk over its chunks.
template <typename T, int D, int N>
__global__ __launch_bounds__(256) void attn_packed_merge_rows(const AttnPackedArgs<N> a, int q_rows) {
  constexpr int LPR = D / 4, ROWS = 256 / LPR;
  const int ui = blockIdx.y, n = chunks_of(packed_blocks(a.unit[ui].len), a.chunk);
  const int tid = threadIdx.x, qi = blockIdx.x * ROWS + tid / LPR, lane = tid % LPR;
  if (n == 1 || qi >= a.N_k) return;
  const int64_t part0 = ((int64_t)ui * a.q_tiles + qi / q_rows) * a.n_chunks * q_rows + qi % q_rows;
  const float2* const ml = reinterpret_cast<const float2*>(a.part_ml) + part0;
  const float4* const po = reinterpret_cast<const float4*>(a.part_o + part0 * D) + lane;
  float M = -FLT_MAX, L = 0.f;
  floatx4 o = {0.f, 0.f, 0.f, 0.f};
  constexpr int kAhead = 8;   // chunks whose loads are under way together
  for (int c0 = 0; c0 < n; c0 += kAhead) {
    float2 x[kAhead];
    float4 p[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int64_t at = (int64_t)min(c0 + i, n - 1) * q_rows;
      x[i] = ml[at];
      p[i] = po[at * LPR];
    }
    float m = M;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) m = fmaxf(m, x[i].x);
    const float old = __builtin_amdgcn_exp2f(M - m);
    M = m;
    L *= old;
#pragma unroll
    for (int r = 0; r < 4; ++r) o[r] *= old;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const float f = c0 + i < n ? __builtin_amdgcn_exp2f(x[i].x - M) : 0.f;
      L = fmaf(f, x[i].y, L);
      o[0] = fmaf(f, p[i].x, o[0]);
      o[1] = fmaf(f, p[i].y, o[1]);
      o[2] = fmaf(f, p[i].z, o[2]);
      o[3] = fmaf(f, p[i].w, o[3]);
    }
  }
  store4(static_cast<T*>(a.out) + ((int64_t)a.unit[ui].unit * a.N_k + qi) * D + 4 * lane, o, 1.f / L);
}

template <typename T, int D, int N>
void launch_some(hipStream_t s, int queries, const AttnPackedHead& h, const AttnPackedUnit* units) {
  AttnPackedArgs<N> a;
  static_cast<AttnPackedHead&>(a) = h;
  for (int i = 0; i < h.n_units; ++i) a.unit[i] = units[i];
  const int pairs = h.n_units * h.n_chunks;
  const dim3 grid((pairs + 7) / 8 * 8 * h.q_tiles), block(64 * kWaves);
  if constexpr (sizeof(T) == 4) {
    hipLaunchKernelGGL((attn_packed<T, D, 1, N>), grid, block, 0, s, a);
  } else {
    if (queries == kTileQueries) launch_attn_packed_tiles(s, D, h, units);
    else if (queries == 16) hipLaunchKernelGGL((attn_packed<T, D, 1, N>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((attn_packed<T, D, 2, N>), grid, block, 0, s, a);
  }
  if (h.n_chunks == 1) return;
  // One query to a work-group reads many chunks at a time; where a query has few or the queries fill the chip, D / 4 lanes each are as fast and more of them
  // run (launch and merge, us, a work-group / D / 4 lanes a query, head_dim 128: 4 chunks, 64 units, 1 query 9.6 / 8.5, 472 queries 111 / 73; 16 chunks, 64
  // units, 1 query 12.3 / 12.0, 4 units 7.8 / 8.1, 64 units, 100 queries 59 / 54).
  constexpr int kRows = 1024 / D;
  if (h.n_chunks <= 8 || (int64_t)h.N_k * h.n_units >= 2048)
    hipLaunchKernelGGL((attn_packed_merge_rows<T, D, N>), dim3((h.N_k + kRows - 1) / kRows, h.n_units), dim3(256), 0, s, a, queries);
  else
    hipLaunchKernelGGL((attn_packed_merge<T, D, N>), dim3(h.N_k, h.n_units), dim3(256), 0, s, a, queries);
}

template <typename T>
void launch_typed(hipStream_t s, int head_dim, int queries, const AttnPackedHead& h, const AttnPackedUnit* units) {
  const bool few = h.n_units <= kFewUnits;
  if (head_dim == 64 && few) launch_some<T, 64, kFewUnits>(s, queries, h, units);
  else if (head_dim == 64) launch_some<T, 64, kAttnPackedUnits>(s, queries, h, units);
  else if (few) launch_some<T, 128, kFewUnits>(s, queries, h, units);
  else launch_some<T, 128, kAttnPackedUnits>(s, queries, h, units);
}

}  // namespace

void launch_attn_packed(hipStream_t s, int elem_bytes, int head_dim, int queries, const AttnPackedHead& h, const AttnPackedUnit* units) {
  if (elem_bytes == 4) launch_typed<float>(s, head_dim, queries, h, units);
  else launch_typed<__bf16>(s, head_dim, queries, h, units);
}

}  // namespace hack
