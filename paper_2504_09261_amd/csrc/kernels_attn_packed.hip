// Attention over a cache held in 4 bits: O = Softmax(scale Q K^T) V for every unit over its own rows, no mask (layout and rounding of
// the rows: packed_device.h).
//
// A code times its power of two is a bf16 number, so K and V enter the 16x16x32 bf16 matrix instructions exactly; what is rounded is what
// attention over bf16 rows rounds, the probabilities and the output.
//
// A work-group takes 16 NQ queries of a unit and a chunk of its keys, its four waves every fourth block of 64 keys.  K comes from
// memory in the order of the A operand of S^T = K Q^T: conversion is all that stands between the load and the product.  V^T needs
// keys side by side where memory has head-dim: each wave writes 32 converted rows to LDS and reads them with the transposing LDS read.  Scores,
// probabilities and the PV product of 32 keys are those of SplitStage.  The partial results of the waves are merged through LDS, those of several chunks
// of a unit in memory, by a launch of their own.
#include <cfloat>

#include "packed_device.h"
#include "split_stage.h"

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

template <int D, int NQ>
__global__ __launch_bounds__(64 * kWaves, 2) void attn_packed(const AttnPackedArgs a) {
  constexpr int KC = D / 32, MT = D / 16, CPR = D / 8, QROWS = 16 * NQ;
  constexpr int SLOT = (NQ == 2 ? 64 : 32) * D;   // elements: 32 rows of V, then the wave's partial results
  // The query tiles of a unit and a chunk follow each other on an XCD (work-group id mod 8).
  const int local = blockIdx.x >> 3, pair = (local / a.q_tiles) * 8 + (blockIdx.x & 7), q_tile = local % a.q_tiles;
  if (pair >= a.n_units * a.n_chunks) return;
  const int ui = pair % a.n_units, chunk = pair / a.n_units;
  const AttnPackedUnit u = a.unit[ui];
  const int len = u.len, n_blocks = (len + kPackRows - 1) / kPackRows;
  const int first = chunk * a.chunk;
  if (first >= n_blocks) return;
  const int last = min(first + a.chunk, n_blocks);
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, g = lane >> 4;
  const int q0 = q_tile * QROWS;
  const int64_t row0 = (int64_t)(a.unit0 + ui) * a.N_k;

  __shared__ __attribute__((aligned(1024))) __bf16 ring[kWaves][SLOT];
  __shared__ float m_sh[kWaves][QROWS], l_sh[kWaves][QROWS];

  const uint8_t* const kb = a.k + (int64_t)u.block * kPackBytes<D>;
  const uint8_t* const vb = a.v + (int64_t)u.block * kPackBytes<D>;
  PackedRows<D> kr, vr;
  int b = first + w;
  if (b < last) {
    kr.load(kb + (int64_t)b * kPackBytes<D>, lane);
    vr.load(vb + (int64_t)b * kPackBytes<D>, lane);
  }
  // Queries as the B operand, in the order in which the lane's quarter of a key comes: element 8 s + j of quarter g
  bf16x8 qf[NQ][KC];
#pragma unroll
  for (int qt = 0; qt < NQ; ++qt) {
    const __bf16* row = static_cast<const __bf16*>(a.q) + (row0 + min(q0 + 16 * qt + col, a.N_k - 1)) * D + g * (D / 4);
#pragma unroll
    for (int s = 0; s < KC; ++s) qf[qt][s] = *reinterpret_cast<const bf16x8*>(row + 8 * s);
  }
  SplitStage<D, NQ> att;
  att.init(a.scale, lane);
  __bf16* const slot = &ring[w][0];

  for (; b < last; b += kWaves) {
    const PackedRows<D> kc = kr, vc = vr;
    if (b + kWaves < last) {
      kr.load(kb + (int64_t)(b + kWaves) * kPackBytes<D>, lane);
      vr.load(vb + (int64_t)(b + kWaves) * kPackBytes<D>, lane);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {   // 32 keys
      if (b * kPackRows + 32 * h >= len) break;
      floatx4 sc[2][NQ];
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        const float scale = kc.scale(2 * h + kt);
#pragma unroll
        for (int qt = 0; qt < NQ; ++qt) sc[kt][qt] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < KC; ++s) {
          const bf16x8 kf = codes_bf16(kc.slice(2 * h + kt, s), scale);
#pragma unroll
          for (int qt = 0; qt < NQ; ++qt) sc[kt][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[qt][s], sc[kt][qt], 0, 0, 0);
        }
      }
      att.mask(sc, 2 * b + h, len);
      wave_lds_order();   // the last reads of the slot
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        const int r = 16 * kt + col;
        // What lies behind the last row may be anything, and its probability is zero: the product must not meet a NaN there.
        const bool there = b * kPackRows + 32 * h + r < len;
        const float scale = there ? vc.scale(2 * h + kt) : 1.f;
#pragma unroll
        for (int s = 0; s < KC; ++s)
          *reinterpret_cast<bf16x8*>(&slot[r * D + (((KC * g + s) ^ swz_v16<D>(r)) & (CPR - 1)) * 8]) =
              codes_bf16(there ? vc.slice(2 * h + kt, s) : 0u, scale);
      }
      bf16x8 pf[NQ];
      att.follow(sc, b == first + w && h == 0);
      att.probs(sc, pf);
      wave_lds_order();
      att.row_sums(pf);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) att.pv(slot, pf, mt);
    }
  }

  // ---- merge the waves' partial results ----
  constexpr int kPart = SLOT * 2 / 16;   // float4 per wave
  static_assert(NQ * MT * 64 <= kPart && kWaves % NQ == 0, "partial results fit the slots");
  wave_lds_order();
  float4* mine = reinterpret_cast<float4*>(slot) + lane;
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) mine[(mt * NQ + qt) * 64] = make_float4(att.o[mt][qt][0], att.o[mt][qt][1], att.o[mt][qt][2], att.o[mt][qt][3]);
  if (g == 0) {
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) {
      m_sh[w][16 * qt + col] = att.mc[qt];
      l_sh[w][16 * qt + col] = att.ls[qt][0];
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
  const bool whole = n_blocks <= a.chunk;
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
    if (whole) att.store(static_cast<__bf16*>(a.out) + (row0 + qi) * D, mt, acc, inv);
    else *reinterpret_cast<floatx4*>(a.part_o + part * D + 16 * mt + 4 * g) = acc;
  }
  if (!whole && w < NQ && g == 0 && qi < a.N_k) {
    a.part_ml[2 * part] = M;
    a.part_ml[2 * part + 1] = L;
  }
}

// Rows of units that were cut: a work-group takes one query, D / 4 lanes a chunk.
template <int D>
__global__ __launch_bounds__(256) void attn_packed_merge(const AttnPackedArgs a, int q_rows) {
  constexpr int LPR = D / 4, SIDE = 256 / LPR;   // chunks at a time
  const int ui = blockIdx.y, n_blocks = (a.unit[ui].len + kPackRows - 1) / kPackRows;
  if (n_blocks <= a.chunk) return;
  const int n = (n_blocks + a.chunk - 1) / a.chunk;
  const int qi = blockIdx.x, c0 = threadIdx.x / LPR, lane = threadIdx.x % LPR;
  const int64_t part0 = ((int64_t)ui * a.q_tiles + qi / q_rows) * a.n_chunks * q_rows + qi % q_rows;
  __shared__ float4 o_sh[SIDE][LPR];
  __shared__ float l_sh[SIDE];
  float M = -FLT_MAX;
  for (int c = 0; c < n; ++c) M = fmaxf(M, a.part_ml[2 * (part0 + (int64_t)c * q_rows)]);
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  float L = 0.f;
  for (int c = c0; c < n; c += SIDE) {
    const int64_t p = part0 + (int64_t)c * q_rows;
    const float f = __builtin_amdgcn_exp2f(a.part_ml[2 * p] - M);
    const float4 x = reinterpret_cast<const float4*>(a.part_o + p * D)[lane];
    L = fmaf(f, a.part_ml[2 * p + 1], L);
    o.x = fmaf(f, x.x, o.x);
    o.y = fmaf(f, x.y, o.y);
    o.z = fmaf(f, x.z, o.z);
    o.w = fmaf(f, x.w, o.w);
  }
  o_sh[c0][lane] = o;
  if (lane == 0) l_sh[c0] = L;
  __syncthreads();
  if (c0 != 0) return;
#pragma unroll
  for (int x = 1; x < SIDE; ++x) {
    const float4 p = o_sh[x][lane];
    o.x += p.x;
    o.y += p.y;
    o.z += p.z;
    o.w += p.w;
    L += l_sh[x];
  }
  const float inv = 1.f / L;
  __bf16* row = static_cast<__bf16*>(a.out) + ((int64_t)(a.unit0 + ui) * a.N_k + qi) * D;
  *reinterpret_cast<bf16x4*>(row + 4 * lane) = bf16x4{(__bf16)(o.x * inv), (__bf16)(o.y * inv), (__bf16)(o.z * inv), (__bf16)(o.w * inv)};
}

template <int D>
void launch_dim(hipStream_t s, int queries, const AttnPackedArgs& a) {
  const int pairs = a.n_units * a.n_chunks;
  const dim3 grid((pairs + 7) / 8 * 8 * a.q_tiles), block(64 * kWaves);
  if (queries == 16) hipLaunchKernelGGL((attn_packed<D, 1>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((attn_packed<D, 2>), grid, block, 0, s, a);
  if (a.n_chunks > 1) hipLaunchKernelGGL((attn_packed_merge<D>), dim3(a.N_k, a.n_units), dim3(256), 0, s, a, queries);
}

}  // namespace

void launch_attn_packed(hipStream_t s, int head_dim, int queries, const AttnPackedArgs& a) {
  if (head_dim == 64) launch_dim<64>(s, queries, a);
  else launch_dim<128>(s, queries, a);
}

}  // namespace hack
