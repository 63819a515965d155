// Attention over a cache held in 4 bits for many queries: work items of 128 queries, four waves of 32, which share every converted block of 32 keys through
// LDS (layout and rounding of the rows: packed_device.h; few queries: kernels_attn_packed.hip).
//
// The arithmetic and its three strands are those of the 128-query kernel over bf16 rows: a stage forms the scores of block j + 1, the probabilities of
// block j and the PV product of block j - 1, in slots of one matrix instruction, an LDS read and a share of the vector work.  Where that kernel copies
// rows to LDS, here every thread loads 16 codes of K and 16 of V (8 at head_dim 64) stages ahead, and in the first half of a stage
// turns them into bf16 and writes them: K(j + 2) and V(j), which the barrier in the middle of the stage publishes and the next stage reads.
//
// Bound by the matrix cores and the vector work beside them.  Measured, head_dim 128: 32 units of 1943 and 3885 keys, 4096 queries 179 to 186 us (1.05 to 1.09
// PFLOP/s; a large library product reaches 1.2), over 10521 keys 605 to 617 us (1.14 to 1.17), where the kernel over bf16 rows, which converts nothing,
// takes 568.  Conversions earlier in the stage 1 % slower, explicit waits equal.
#include <cfloat>
#include <type_traits>

#include "packed_device.h"

namespace hack {

namespace {

using namespace dev;

constexpr int kKB = 32;           // keys per stage
constexpr int kNW = 4;            // waves of a work-group
constexpr int kNS = 4;            // LDS slots per tensor
constexpr int kAhead = 4;         // stages between the load of codes and their conversion
constexpr float kHeadroom = 15.f; // the reference lies 2^15 above the running maximum: the exponent's top bit says that a probability reached 2

template <int I, int N, typename F>
__device__ __forceinline__ void for_each(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    for_each<I + 1, N>(f);
  }
}

// Vector work of a stage, in the order of issue.  Softmax: 16 scores a lane become probabilities: multiply-add, exponential, and
// a conversion for two of them, dependent ones two elements apart.
struct Step {
  int kind, index;   // 0 multiply-add, 1 exponential, 2 conversion of elements index and index + 1
};
constexpr int kSteps = 40;
constexpr Step softmax_step(int t) {
  int n = 0;
  for (int j = -2; j < 18; ++j) {   // element j's exponential, with element j + 2's multiply-add behind it and the conversion of j - 2 and j - 1
    if (j >= 0 && j < 16 && n++ == t) return Step{1, j};
    if (j + 2 < 16 && n++ == t) return Step{0, j + 2};
    if (j >= 2 && j % 2 == 0 && n++ == t) return Step{2, j - 2};
  }
  return Step{-1, 0};
}
constexpr int step_cycles(int t) { return softmax_step(t).kind == 1 ? 8 : 4; }
constexpr int kSoftmaxCycles = 16 * 4 + 16 * 8 + 8 * 4;
// Steps in front of slot s: `first` of the cycles are spread over the slots up to the middle, where the conversions of codes are, the rest over those up to `end`.
constexpr int steps_before(int s, int middle, int end, int first) {
  if (s >= end) return kSteps;
  const int budget = s <= middle ? first * s / middle : first + (kSoftmaxCycles - first) * (s - middle) / (end - middle);
  int c = 0, t = 0;
  while (t < kSteps && c + step_cycles(t) <= budget) c += step_cycles(t++);
  return t;
}

template <int D, int N>
__global__ __launch_bounds__(64 * kNW, 2) void attn_packed_tiles(const AttnPackedArgs<N> a) {
  constexpr int KC = D / 32;        // MFMA steps over head_dim for S^T
  constexpr int MT = D / 16;        // 16-row tiles of O^T
  constexpr int BLK = kKB * D;      // elements per block and tensor
  constexpr int CW = D / 64;        // dwords of codes a thread converts of a block, per tensor
  // The query tiles of a unit and a chunk follow each other on an XCD (work-group id mod 8).
  const int local = blockIdx.x >> 3, pair = (local / a.q_tiles) * 8 + (blockIdx.x & 7), q_tile = local % a.q_tiles;
  if (pair >= a.n_units * a.n_chunks) return;
  const int ui = pair % a.n_units, chunk = pair / a.n_units;
  const AttnPackedUnit u = a.unit[ui];
  const int all = packed_blocks(u.len), chunks = chunks_of(all, a.chunk);
  if (chunk >= chunks) return;
  const int first = chunk_at(all, chunks, chunk), last = chunk_at(all, chunks, chunk + 1);
  const int len = rows_in(u.len, first, last), n_blocks = stages_of(len, kKB);   // keys of this work-group
  const int tid = threadIdx.x;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63, col = lane & 15, g = lane >> 4;

  __shared__ __attribute__((aligned(1024))) __bf16 Ks[kNS][BLK];
  __shared__ __attribute__((aligned(1024))) __bf16 Vs[kNS][BLK];

  // ---- codes: thread's share of block b, and where it goes in LDS ----
  const uint8_t* const kg = a.k + ((int64_t)u.block + first) * kPackBytes<D>;
  const uint8_t* const vg = a.v + ((int64_t)u.block + first) * kPackBytes<D>;
  const unsigned code_off = lane * 16 + (D == 128 ? (w >> 1) * 1024 + (w & 1) * 8 : (w >> 1) * 8 + (w & 1) * 4);
  const unsigned exp_off = 32 * D + (D == 128 ? lane : (lane >> 5) * 16 + col) * 4 + (w >> 1);
  struct Codes {
    unsigned w[CW];
    unsigned char exponent;
  };
  auto load_codes = [&](Codes& c, const uint8_t* base, int b) {
    const uint8_t* p = base + (int64_t)(b >> 1) * kPackBytes<D>;
    const uint8_t* q = p + (b & 1) * (16 * D);
    if constexpr (CW == 2) {
      const uint2 x = *reinterpret_cast<const uint2*>(q + code_off);
      c.w[0] = x.x;
      c.w[1] = x.y;
    } else {
      c.w[0] = *reinterpret_cast<const unsigned*>(q + code_off);
    }
    c.exponent = p[exp_off + (b & 1) * 2];
  };
  // Rows in groups of four, a group's 64-byte pieces row after row, 16-byte chunks permuted by two bits of the row (packed_device.h).  Written 8 rows at one
  // chunk at a time, K read 16 rows at one chunk, V^T 8 rows x 32 bytes.
  const int row = 16 * (w >> 1) + col, chunk0 = D == 128 ? 4 * g + 2 * (w & 1) : 2 * g + (w & 1);
  int to[CW];   // the same place for K and V
#pragma unroll
  for (int i = 0; i < CW; ++i) to[i] = v_chunk<D>(row, chunk0 + i);

  // Block 0 is the last one, ragged or not, blocks 1 .. n_blocks - 1 are the full ones in front of it: what is particular about a ragged block stays in front
  // of the main loop.  Past the last block the one before is loaded and converted again, into slots that nobody reads any more.
  const int last_full = max(n_blocks - 2, 0);
  Codes kc[kAhead], vc[kAhead];   // of stage j in [j % kAhead]
  {
    Codes k0, k1, k2, v0;
    load_codes(k0, kg, n_blocks - 1);
    load_codes(v0, vg, n_blocks - 1);
    load_codes(k1, kg, 0);
    load_codes(k2, kg, min(1, last_full));
#pragma unroll
    for (int j = 1; j <= kAhead; ++j) {
      load_codes(kc[j % kAhead], kg, min(j + 1, last_full));
      load_codes(vc[j % kAhead], vg, min(j - 1, last_full));
    }
    // What lies behind the last row may be anything: its scores are masked, and the PV product must not meet a NaN there.
    const bool there = (n_blocks - 1) * kKB + row < len;
#pragma unroll
    for (int i = 0; i < CW; ++i) {
      *reinterpret_cast<bf16x8*>(&Ks[0][to[i]]) = codes_bf16(k0.w[i], scale_of(k0.exponent));
      *reinterpret_cast<bf16x8*>(&Vs[0][to[i]]) = codes_bf16(there ? v0.w[i] : 0u, there ? scale_of(v0.exponent) : 1.f);
      *reinterpret_cast<bf16x8*>(&Ks[1][to[i]]) = codes_bf16(k1.w[i], scale_of(k1.exponent));
      *reinterpret_cast<bf16x8*>(&Ks[2][to[i]]) = codes_bf16(k2.w[i], scale_of(k2.exponent));
    }
  }
  int k_at = min(kAhead + 2, last_full), v_at = min(kAhead, last_full);   // the next blocks to load

  // Q fragments (B operand of S^T = K Q^T): query 16 qt + col, head-dim slice [32 kc + 8 g, +8)
  const int q0 = q_tile * (kNW * 32) + w * 32;
  const int64_t row0 = (int64_t)u.unit * a.N_k;
  bf16x8 qf[2][KC];
#pragma unroll
  for (int qt = 0; qt < 2; ++qt) {
    const __bf16* qrow = static_cast<const __bf16*>(a.q) + (row0 + min(q0 + 16 * qt + col, a.N_k - 1)) * D;
#pragma unroll
    for (int c = 0; c < KC; ++c) qf[qt][c] = *reinterpret_cast<const bf16x8*>(qrow + 32 * c + 8 * g);
  }

  floatx4 o[MT][2];        // O^T: head-dim 16 mt + 4 g + r, query 16 qt + col
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) o[mt][0] = o[mt][1] = floatx4{0.f, 0.f, 0.f, 0.f};
  floatx4 ls[2] = {floatx4{0.f, 0.f, 0.f, 0.f}, floatx4{0.f, 0.f, 0.f, 0.f}};   // row sums of P (equal in all four rows)
  const float c2 = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, a.scale * kLog2eF)));
  float mc[2] = {-FLT_MAX, -FLT_MAX};   // probabilities are 2^(c2 s - mc); finite from the start, so that keys whose score is -inf get 0

  const int e = col >> 2, qd = col & 3;
  const int k_off = e * 4 * D + (col & 3) * 32 + (g ^ v_flip(col)) * 8;                          // K operand: row 16 kt + col, chunk 4 c + g
  const int v_even = v_chunk<D>(4 * g + e, qd >> 1) + 4 * (qd & 1), v_odd = v_even ^ 16;   // V^T operand: rows 4 g + e and 16 + 4 g + e
  bf16x8 ones;
#pragma unroll
  for (int j = 0; j < 8; ++j) ones[j] = (__bf16)1.0f;
  asm volatile("" : "+v"(ones));   // stays in registers

  struct Scores { floatx4 t[2][2]; };   // keys 16 kt + 4 g + r, query 16 qt + col
  auto probs = [&](const Scores& sc, int qt, bf16x8& pf) {
#pragma unroll
    for (int j = 0; j < 8; ++j) pf[j] = (__bf16)__builtin_amdgcn_exp2f(fmaf(sc.t[j >> 2][qt][j & 3], c2, -mc[qt]));
  };
  auto too_large = [&](const bf16x8 (&pf)[2]) -> bool {
    const uintx4 x = __builtin_bit_cast(uintx4, pf[0]), y = __builtin_bit_cast(uintx4, pf[1]);
    return (((x[0] | x[1] | x[2]) | x[3] | y[0]) | y[1] | y[2] | y[3]) & 0x40004000u;
  };
  auto rescale = [&](const Scores& sc, bf16x8 (&pf)[2]) {
#pragma unroll
    for (int qt = 0; qt < 2; ++qt) {
      float mx = sc.t[0][qt][0];
#pragma unroll
      for (int j = 1; j < 8; ++j) mx = fmaxf(mx, sc.t[j >> 2][qt][j & 3]);
      const float m_new = fmaxf(mc[qt], fmaf(quad_max(mx), c2, kHeadroom));
      const float f = __builtin_amdgcn_exp2f(mc[qt] - m_new);
      mc[qt] = m_new;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        ls[qt][r] *= f;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) o[mt][qt][r] *= f;
      }
      probs(sc, qt, pf[qt]);
    }
  };
  // Operands of step i of a stage: head-dim slice i of S^T and two head-dim tiles of O^T.
  struct Frags {
    bf16x8 k[2];
    bf16x4 v[2][2];
  };
  auto load_frag = [&](Frags& f, const __bf16* Kt, const __bf16* Vt, int i, int part) {   // one LDS read, parts 0 .. 5
    if (part < 2) f.k[part] = *reinterpret_cast<const bf16x8*>(&Kt[16 * part * D + 128 * i + k_off]);
    else f.v[(part >> 1) - 1][part & 1] = lds_read_tr(&Vt[16 * (part & 1) * D + 128 * i + ((part >> 1) - 1 ? v_odd : v_even)]);
  };
  auto joined = [](const bf16x4 (&v)[2]) { return bf16x8{v[0][0], v[0][1], v[0][2], v[0][3], v[1][0], v[1][1], v[1][2], v[1][3]}; };
  auto qk = [&](Scores& sn, const Frags& f, int c, int n) {
    const int kt = n >> 1, qt = kt ^ (n & 1);
    sn.t[kt][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.k[kt], qf[qt][c], sn.t[kt][qt], 0, 0, 0);
  };
  auto pv = [&](const Frags& f, const bf16x8 (&p)[2], int i, int n) {
    const int m = n >> 1, qt = m ^ (n & 1);
    o[2 * i + m][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(joined(f.v[m]), p[qt], o[2 * i + m][qt], 0, 0, 0);
  };
  auto row_sums = [&](const bf16x8 (&p)[2], int qt) { ls[qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, p[qt], ls[qt], 0, 0, 0); };

  bf16x8 P[2][2];   // probabilities of block j in P[j & 1]: those of the previous block wait for their PV product
  Frags pre;        // operands of the next stage's first step

  // Stage j, slot S = j % 4 (compile time).  On entry sc = scores of block j, on exit those of block j + 1.  FIRST: j = 0 (no previous block, and K(2) and V(0) lie
  // in LDS already).
  auto stage = [&](auto slot_tag, auto first_tag, Scores& sc) {
    constexpr int S = decltype(slot_tag)::value;
    constexpr bool FIRST = decltype(first_tag)::value;
    const __bf16* const Kt = &Ks[(S + 1) % kNS][0];
    const __bf16* const Vt = &Vs[(S + 3) % kNS][0];
    Scores sn;
#pragma unroll
    for (int i = 0; i < 4; ++i) sn.t[i >> 1][i & 1] = floatx4{0.f, 0.f, 0.f, 0.f};
    bf16x8 (&pp)[2] = P[(S + 1) & 1], (&pf)[2] = P[S & 1];
    Codes &ck = kc[S % kAhead], &cv = vc[S % kAhead];
    Frags f = pre, nx;
    float x[16];
    bf16x8 conv;
    float k_scale = 0.f, v_scale = 0.f;
    auto vec_op = [&](auto t_tag) {
      constexpr Step op = softmax_step(decltype(t_tag)::value);
      constexpr int j = op.index, qt = (j >> 3) & 1, jj = j & 7;
      if constexpr (op.kind == 0) x[j] = fmaf(sc.t[jj >> 2][qt][jj & 3], c2, -mc[qt]);
      else if constexpr (op.kind == 1) x[j] = __builtin_amdgcn_exp2f(x[j]);
      else { pf[qt][jj] = (__bf16)x[j]; pf[qt][jj + 1] = (__bf16)x[j + 1]; }
    };
    // conversion i of 8 CW: codes 2 (i % 4) .. of dword (i / 4) % CW, K before V; the fourth of a dword writes it
    auto convert = [&](auto i_tag) {
      constexpr int i = decltype(i_tag)::value, d = (i / 4) % CW, p = i % 4;
      constexpr bool is_k = i < 4 * CW;
      if constexpr (i == 0) k_scale = scale_of(ck.exponent);
      if constexpr (i == 4 * CW) v_scale = scale_of(cv.exponent);
      const bf16x2 y = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(is_k ? ck.w[d] : cv.w[d], is_k ? k_scale : v_scale, p);
      conv[2 * p] = y[0];
      conv[2 * p + 1] = y[1];
      if constexpr (p == 3) *reinterpret_cast<bf16x8*>(is_k ? &Ks[(S + 2) % kNS][to[d]] : &Vs[S][to[d]]) = conv;
    };
    constexpr int SLOTS = 8 * KC + 2, END = SLOTS - 3 * KC / 4, MIDDLE = 4 * KC;
    constexpr int CONV_SLOTS = MIDDLE - KC / 2, FIRST_CYCLES = kSoftmaxCycles * 2 / 5;
    bool large = false;
    // one MFMA, one LDS read, a share of the vector work
    auto slot = [&](auto s_tag) {
      constexpr int T = decltype(s_tag)::value, I = T / 8 < KC ? T / 8 : KC - 1, M = T - 8 * I;   // the last step has two more
      if constexpr (M < 4) qk(sn, f, I, M);
      else if constexpr (M < 8) { if (!FIRST) pv(f, pp, I, M - 4); }
      else { if (!FIRST) row_sums(pp, M - 8); }
      if constexpr (!FIRST && T < CONV_SLOTS) for_each<8 * CW * T / CONV_SLOTS, 8 * CW * (T + 1) / CONV_SLOTS>(convert);
      for_each<steps_before(T, MIDDLE, END, FIRST_CYCLES), steps_before(T + 1, MIDDLE, END, FIRST_CYCLES)>(vec_op);
      if constexpr (T == END) large = __any(too_large(pf));
      if constexpr (M < 2 || (M >= 4 && M < 8)) {
        constexpr int part = M < 2 ? M : M - 2;
        if constexpr (I + 1 < KC) load_frag(nx, Kt, Vt, I + 1, part);
        else load_frag(nx, &Ks[(S + 2) % kNS][0], &Vs[S][0], 0, part);
      }
      if constexpr (M == 7 && I + 1 < KC) f = nx;
      __builtin_amdgcn_sched_barrier(0);
    };
    for_each<0, MIDDLE>(slot);
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");   // K(j + 2) and V(j) lie in LDS
    __builtin_amdgcn_sched_barrier(0);
    if (!FIRST) {
      load_codes(ck, kg, k_at);   // K(j + 2 + kAhead)
      load_codes(cv, vg, v_at);   // V(j + kAhead)
      k_at = min(k_at + 1, last_full);
      v_at = min(v_at + 1, last_full);
    }
    __builtin_amdgcn_sched_barrier(0);
    for_each<MIDDLE, SLOTS>(slot);
    pre = nx;
    if (__builtin_expect(large, 0)) rescale(sc, pf);
    sc = sn;
  };

  __syncthreads();
  Scores sc;
#pragma unroll
  for (int i = 0; i < 4; ++i) sc.t[i >> 1][i & 1] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int c = 0; c < KC; ++c) {
    Frags f;
    for (int n = 0; n < 2; ++n) load_frag(f, &Ks[0][0], nullptr, c, n);
    for (int n = 0; n < 4; ++n) qk(sc, f, c, n);
  }
  for (int n = 0; n < 2; ++n) load_frag(pre, &Ks[1][0], nullptr, 0, n);
  for (int n = 2; n < 6; ++n) load_frag(pre, nullptr, &Vs[0][0], 0, n);
#pragma unroll
  for (int kt = 0; kt < 2; ++kt)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if ((n_blocks - 1) * kKB + 16 * kt + 4 * g + r >= len) sc.t[kt][0][r] = sc.t[kt][1][r] = -INFINITY;

  using No = std::false_type;
  using Yes = std::true_type;
  if (n_blocks > 1) {
    stage(std::integral_constant<int, 0>{}, Yes{}, sc);
    for (int b = 1;; b += 4) {
      if (b >= n_blocks - 1) break;
      stage(std::integral_constant<int, 1>{}, No{}, sc);
      if (b + 1 >= n_blocks - 1) break;
      stage(std::integral_constant<int, 2>{}, No{}, sc);
      if (b + 2 >= n_blocks - 1) break;
      stage(std::integral_constant<int, 3>{}, No{}, sc);
      if (b + 3 >= n_blocks - 1) break;
      stage(std::integral_constant<int, 0>{}, No{}, sc);
    }
  }
  // the last block: its probabilities, its PV product and the one of the block before
  auto pv_block = [&](const __bf16* Vt, const bf16x8 (&p)[2]) {
#pragma unroll
    for (int i = 0; i < KC; ++i) {
      Frags f;
      for (int n = 2; n < 6; ++n) load_frag(f, nullptr, Vt, i, n);
      for (int n = 0; n < 4; ++n) pv(f, p, i, n);
    }
    row_sums(p, 0);
    row_sums(p, 1);
  };
  if (n_blocks > 1) {
    const bool odd = n_blocks & 1;   // the block before the last has an odd number
    Codes cv = vc[0];                // V of the last block, loaded for a stage that did not come
#pragma unroll
    for (int j = 1; j < kAhead; ++j)
      if ((n_blocks - 1) % kAhead == j) cv = vc[j];
#pragma unroll
    for (int i = 0; i < CW; ++i)
      *reinterpret_cast<bf16x8*>(&Vs[(n_blocks - 1) % kNS][to[i]]) = codes_bf16(cv.w[i], scale_of(cv.exponent));
    const bf16x8 pl[2] = {odd ? P[1][0] : P[0][0], odd ? P[1][1] : P[0][1]};
    pv_block(&Vs[(n_blocks - 2) % kNS][0], pl);
    __syncthreads();
  }
  probs(sc, 0, P[0][0]);
  probs(sc, 1, P[0][1]);
  if (__any(too_large(P[0]))) rescale(sc, P[0]);
  pv_block(&Vs[(n_blocks - 1) % kNS][0], P[0]);

  // ---- normalise and store: a lane holds head-dim 16 mt + 4 g .. +4 of queries 16 qt + col ----
  const bool whole = chunks == 1;
  const int64_t part = (((int64_t)ui * a.q_tiles + q_tile) * a.n_chunks + chunk) * (kNW * 32) + w * 32 + col;
#pragma unroll
  for (int qt = 0; qt < 2; ++qt) {
    const int qi = q0 + 16 * qt + col;
    if (qi >= a.N_k) continue;
    const float inv = 1.f / ls[qt][0];
    __bf16* orow = static_cast<__bf16*>(a.out) + (row0 + qi) * D;
    float* prow = a.part_o + (part + 16 * qt) * D;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      if (!whole) {
        *reinterpret_cast<floatx4*>(prow + 16 * mt + 4 * g) = o[mt][qt];
        continue;
      }
      bf16x4 pk;
#pragma unroll
      for (int r = 0; r < 4; ++r) pk[r] = (__bf16)(o[mt][qt][r] * inv);
      *reinterpret_cast<bf16x4*>(orow + 16 * mt + 4 * g) = pk;
    }
    if (!whole && g == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * (part + 16 * qt)) = make_float2(mc[qt], ls[qt][0]);
  }
}

template <int D, int N>
void launch_some(hipStream_t s, const AttnPackedHead& h, const AttnPackedUnit* units) {
  AttnPackedArgs<N> a;
  static_cast<AttnPackedHead&>(a) = h;
  for (int i = 0; i < h.n_units; ++i) a.unit[i] = units[i];
  const int pairs = h.n_units * h.n_chunks;
  hipLaunchKernelGGL((attn_packed_tiles<D, N>), dim3((pairs + 7) / 8 * 8 * h.q_tiles), dim3(64 * kNW), 0, s, a);
}

}  // namespace

void launch_attn_packed_tiles(hipStream_t s, int head_dim, const AttnPackedHead& h, const AttnPackedUnit* units) {
  const bool few = h.n_units <= kFewUnits;
  if (head_dim == 64 && few) launch_some<64, kFewUnits>(s, h, units);
  else if (head_dim == 64) launch_some<64, kAttnPackedUnits>(s, h, units);
  else if (few) launch_some<128, kFewUnits>(s, h, units);
  else launch_some<128, kAttnPackedUnits>(s, h, units);
}

}  // namespace hack
