// Attention over caches in pages, few queries (tiles of 16 and 32), as the kernels that have such tiles alone, beside larger ones and in
// place of results of larger ones share it: O = Softmax(scale Q K^T) V
// over the rows that a query sees.  HIP device code only.
//
// A work-group takes 16 NQ queries and a chunk of keys, its four waves every fourth block (32 keys, float32 16), each by itself.  S^T = K Q^T, one softmax update a block, O^T +=
// V^T P^T: the probabilities go from the accumulators into the B operand.  V^T wants keys side by side where memory has head-dim: a lane loads the
// same 8 elements of eight rows (at head_dim 64, of four, and trades halves with a neighbour) and turns the square around in registers.  Float32 enters the
// 16x16x4 matrix instruction as it is, whose operands need no turning.  The next block is loaded into the registers of this one as soon as they are free, the
// page numbers of the one behind it are under way by then.
// Bound by reading the cache: two work-groups keep 128 KB a compute unit under way.  Of the 137 us of one token over 643 MB, whole rows side by side in a load took 15 (K through
// LDS; 16 rows' 64 bytes each before), loads past the caches 5.
#pragma once

#include <type_traits>

#include "attn_pages_device.h"

namespace hack {
namespace dev {

// ---- rows of a block -----------------------------------------------------------
template <bool NT, typename V> __device__ __forceinline__ V load_piece(const uint8_t* p) {
  if constexpr (NT) return __builtin_nontemporal_load(reinterpret_cast<const V*>(p));
  else return *reinterpret_cast<const V*>(p);
}

// K: whole rows side by side in the lanes of a load, in chunks of 16 bytes, and through LDS into the order of the A operand.  Chunk c of row r lies at c ^ turn(r),
// so that neither the writes (whole rows) nor the reads (16 rows at one chunk) meet a bank twice.  (A load of 16 rows' 64 bytes each into the operand's
// registers needs no LDS, but reads half lines: 64 tokens over 643 MB 134 us, so 116.)
template <typename T, int D, bool NT> struct KeyRows {
  static constexpr int kRows = sizeof(T) == 2 ? 32 : 16, kChunks = D * (int)sizeof(T) / 16, kAtOnce = 64 / kChunks, kLoads = kRows / kAtOnce;
  uintx4 x[kLoads];
  static __device__ __forceinline__ int turn(int r) { return kChunks >= 16 ? r & 15 : (r >> 1) & 7; }
  static constexpr int tile(int i) { return i * kAtOnce >> 4; }
  // off: lane_offset.  (What is the same in all lanes goes into the base.)
  static __device__ __forceinline__ unsigned lane_offset(unsigned stride, int lane) { return lane / kChunks * stride + 16 * (lane % kChunks); }
  __device__ __forceinline__ void load(int i, const uint8_t* tile_base, unsigned stride, unsigned off) {
    x[i] = load_piece<NT, uintx4>(tile_base + (uint64_t)((i * kAtOnce & 15) * stride) + off);
  }
  __device__ __forceinline__ void put(uintx4* lds, int lane) const {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = i * kAtOnce + lane / kChunks;
      lds[r * kChunks + ((lane % kChunks) ^ turn(r))] = x[i];
    }
  }
  static __device__ __forceinline__ uintx4 get(const uintx4* lds, int t, int s, int col, int g) {   // chunk 4 s + g of row col of tile t
    const int r = 16 * t + col;
    return lds[r * kChunks + ((4 * s + g) ^ turn(r))];
  }
};

// V: a lane's head-dims of the rows that the accumulators of S^T hold in its group of 16 lanes.
template <typename T, int D, bool NT> struct ValueRows;
template <int D, bool NT> struct ValueRows<__bf16, D, NT> {   // 32 rows: 8 head-dims of eight rows (128), or, until turned, of every second one (64)
  static constexpr int kLoads = D / 16;
  uintx4 x[kLoads];
  static constexpr int tile(int i) { return i >= kLoads / 2; }
  static __device__ __forceinline__ int row(int i, int g, int col) {   // within its tile
    return D == 128 ? 4 * g + (i & 3) : 4 * g + 2 * (i & 1) + (col >> 3);
  }
  static __device__ __forceinline__ unsigned lane_offset(unsigned stride, int g, int col) { return row(0, g, col) * stride + 16 * (D == 128 ? col : col & 7); }
  __device__ __forceinline__ void load(int i, const uint8_t* tile_base, unsigned stride, unsigned off) {
    x[i] = load_piece<NT, uintx4>(tile_base + (uint64_t)(row(i, 0, 0) * stride) + off);
  }
  __device__ __forceinline__ void clear(int i) { x[i] = uintx4{0, 0, 0, 0}; }
  __device__ __forceinline__ bool strange(int i) const {   // an infinity or a NaN
    bool s = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) s |= (x[i][j] & 0x7F80u) == 0x7F80u || (x[i][j] & 0x7F800000u) == 0x7F800000u;
    return s;
  }
  __device__ __forceinline__ void clear_strange(int i) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if ((x[i][j] & 0x7F80u) == 0x7F80u) x[i][j] &= 0xFFFF0000u;
      if ((x[i][j] & 0x7F800000u) == 0x7F800000u) x[i][j] &= 0xFFFFu;
    }
  }
  // Operands of tiles 2 j and 2 j + 1 of O^T: elements 2 j and 2 j + 1 of the lane's head-dims in all eight rows.
  __device__ __forceinline__ void operands(int j, int col, bf16x8 (&v)[2]) const {
    uintx4 y[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      unsigned even_row, odd_row;
      if constexpr (D == 128) {
        even_row = x[2 * i][j];
        odd_row = x[2 * i + 1][j];
      } else {
        // Lanes col and col ^ 8 hold the even and the odd rows of the same eight head-dims: each takes four of these in all rows.
        const bool odd = col >> 3;
        const unsigned keep = odd ? x[i][2 + j] : x[i][j], give = odd ? x[i][j] : x[i][2 + j];
        const unsigned got = (unsigned)__builtin_amdgcn_update_dpp(0, (int)give, 0x128, 0xF, 0xF, true);   // row_ror 8
        even_row = odd ? got : keep;
        odd_row = odd ? keep : got;
      }
      y[0][i] = __builtin_amdgcn_perm(odd_row, even_row, 0x05040100u);
      y[1][i] = __builtin_amdgcn_perm(odd_row, even_row, 0x07060302u);
    }
    v[0] = __builtin_bit_cast(bf16x8, y[0]);
    v[1] = __builtin_bit_cast(bf16x8, y[1]);
  }
  // head-dim of row m of tile mt of O^T
  static __device__ __forceinline__ int dim(int mt, int m) { return D == 128 ? 8 * m + mt : 8 * (m & 7) + 4 * (m >> 3) + mt; }
};
template <int D, bool NT> struct ValueRows<float, D, NT> {   // 16 rows: four head-dims of each quarter (128) or all (64) of the head in four rows
  static constexpr int kLoads = 4;
  floatx4 x[kLoads][D / 64];
  static constexpr int tile(int) { return 0; }
  static __device__ __forceinline__ int row(int i, int g, int) { return 4 * g + i; }
  static __device__ __forceinline__ unsigned lane_offset(unsigned stride, int g, int col) { return 4 * g * stride + 16 * col; }
  __device__ __forceinline__ void load(int i, const uint8_t* tile_base, unsigned stride, unsigned off) {
#pragma unroll
    for (int p = 0; p < D / 64; ++p) x[i][p] = load_piece<NT, floatx4>(tile_base + (uint64_t)(i * stride) + 256 * p + off);
  }
  __device__ __forceinline__ void clear(int i) {
#pragma unroll
    for (int p = 0; p < D / 64; ++p) x[i][p] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  static __device__ __forceinline__ bool odd(float y) { return (__builtin_bit_cast(unsigned, y) & 0x7F800000u) == 0x7F800000u; }
  __device__ __forceinline__ bool strange(int i) const {
    bool s = false;
#pragma unroll
    for (int j = 0; j < D / 16; ++j) s |= odd(x[i][j >> 2][j & 3]);
    return s;
  }
  __device__ __forceinline__ void clear_strange(int i) {
#pragma unroll
    for (int j = 0; j < D / 16; ++j)
      if (odd(x[i][j >> 2][j & 3])) x[i][j >> 2][j & 3] = 0.f;
  }
  static __device__ __forceinline__ int dim(int mt, int m) { return 64 * (mt >> 2) + 4 * m + (mt & 3); }
};

// floats of the four (float32) or D / 16 (bf16) head-dims that lie side by side, from dim(mt, m) on
__device__ __forceinline__ void store_some(__bf16* p, const float* x, int n, float f) {
  if (n == 8) {
    bf16x8 y;
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = (__bf16)(x[i] * f);
    *reinterpret_cast<bf16x8*>(p) = y;
  } else {
    *reinterpret_cast<bf16x4*>(p) = bf16x4{(__bf16)(x[0] * f), (__bf16)(x[1] * f), (__bf16)(x[2] * f), (__bf16)(x[3] * f)};
  }
}
__device__ __forceinline__ void store_some(float* p, const float* x, int n, float f) {
#pragma unroll
  for (int i = 0; i < n; i += 4) *reinterpret_cast<floatx4*>(p + i) = floatx4{x[i] * f, x[i + 1] * f, x[i + 2] * f, x[i + 3] * f};
}

// Elements that are no numbers alone are replaced.
template <typename T> __device__ __forceinline__ void mend_some(T* p, const float* x, int n, float f) {
#pragma unroll
  for (int i = 0; i < n; ++i)
    if ((float)p[i] * 0.f != 0.f) p[i] = (T)(x[i] * f);
}

template <int D, int NQ> constexpr int kFewLds = kWaves * 16 * NQ * (D + 2) * (int)sizeof(float);   // bytes

// What a work-group takes: queries of an entry and head from number query0 on, and a chunk of the keys.
struct FewItem {
  int b0, h, entry0;     // the first (or only) batch element; row of the table
  int group, common;     // whose shared rows the element has, and how many these are
  int lo, n_rows;        // first row of this part, queries of the entry
  int query0;
  int chunks, chunk;
  int64_t row0;          // of the partial results of query0
  // MEND: the chunk is blocks first to end of kKeys keys; all: results of a tile are replaced, not only their elements that are no numbers
  int first, end;
  bool all;
};

// lds: kFewLds bytes, 1024-byte aligned.  NT: rows are read once, past the caches.  MEND: over results of a tile, which stand in `out` or among the partial results.
template <typename T, int D, int NQ, bool NT, bool MEND>
__device__ __forceinline__ void few_queries(const AttnPagesArgs& a, int part, const FewItem& item, unsigned char* lds) {
  using Keys = KeyRows<T, D, NT>;
  using Values = ValueRows<T, D, NT>;
  constexpr int ROWS = Keys::kRows, TILES = ROWS / 16, PIECES = Keys::kChunks / 4;
  static_assert(ROWS * D * (int)sizeof(T) <= 16 * NQ * D * (int)sizeof(float), "a wave's block of K fits where its results go");
  constexpr bool kBf16 = sizeof(T) == 2;
  // Sums that a float32 score is made of, each over a quarter of the products: one after the other 128 roundings add up where 32 do (one token of 2 caches in each of 4
  // elements, 1249 to 1787 rows: 1.5e-6 off, so 6e-7; products over as many elements in a tree 5e-7).  32 queries have no registers for them, and are as far off as large products are.
  constexpr int SUMS = !kBf16 && NQ == 1 ? 4 : 1;
  constexpr int MT = D / 16, QROWS = 16 * NQ, SIDE = kBf16 ? MT : 4;   // head-dims of a lane that lie side by side
  const Pages& c = a.c;
  const int b0 = item.b0, h = item.h, entry0 = item.entry0, group = item.group, common = item.common, lo = item.lo, n_rows = item.n_rows, GN = a.G * c.n;
  int tid = threadIdx.x;
  if constexpr (MEND) asm volatile("" : "+v"(tid));   // what follows from it does not stay in registers through the tile's stages
  const int lane = tid & 63, col = lane & 15, g = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);

  float (&ring)[kWaves][16 * NQ * D] = *reinterpret_cast<float (*)[kWaves][16 * NQ * D]>(lds);
  float (&m_sh)[kWaves][QROWS] = *reinterpret_cast<float (*)[kWaves][QROWS]>(lds + sizeof ring);
  float (&l_sh)[kWaves][QROWS] = *reinterpret_cast<float (*)[kWaves][QROWS]>(lds + sizeof ring + sizeof m_sh);

  // ---- queries and the rows that they see ----
  int sees[NQ];        // keys in front of it, of this part
  int64_t row[NQ];     // of q and out; < 0: not computed
  int most = 0, fewest = c.max_len;
#pragma unroll
  for (int qt = 0; qt < NQ; ++qt) {
    const int j = min(item.query0 + 16 * qt + col, n_rows - 1), m = j / GN, r = j - m * GN, n = r / a.G, b = b0 + m;
    const int fresh = fresh_of(c, b), len = rows_of(c, c.by_head ? b * c.heads + h : b);
    const bool there = item.query0 + 16 * qt + col < n_rows && n < fresh;
    sees[qt] = max(0, a.causal ? len - fresh + n + 1 : len);
    if (part == 0) sees[qt] = min(sees[qt], common);
    if (there) {
      most = max(most, sees[qt]);
      fewest = min(fewest, sees[qt]);
    } else {
      sees[qt] = 0;
    }
    row[qt] = ((int64_t)b * c.heads + h) * GN + (r - n * a.G) * c.n + n;
    if (!there) row[qt] = -1 - row[qt];
  }
  most = row_most(most);
  fewest = row_fewest(fewest);
  most = __builtin_amdgcn_readfirstlane(most);
  fewest = __builtin_amdgcn_readfirstlane(fewest);
  uintx4 qf[NQ][PIECES];
#pragma unroll
  for (int qt = 0; qt < NQ; ++qt) {
    const uint8_t* p = static_cast<const uint8_t*>(a.q) + (row[qt] < 0 ? -1 - row[qt] : row[qt]) * (D * (int)sizeof(T)) + 16 * g;
#pragma unroll
    for (int s = 0; s < PIECES; ++s) qf[qt][s] = *reinterpret_cast<const uintx4*>(p + 64 * s);
  }

  // ---- this wave's blocks of kRows keys: first + w, first + w + 4, ... ----
  constexpr int PER = kKeys / ROWS;
  const int n_blocks = blocks_between(lo, most), begin = lo / kKeys;
  const int first = (MEND ? item.first : begin + chunk_at(n_blocks, item.chunks, item.chunk)) * PER;
  const int last = (MEND ? min(item.end, begin + n_blocks) : begin + chunk_at(n_blocks, item.chunks, item.chunk + 1)) * PER;
  const ConstInts table = as_const(c.table) + entry0 * c.table_stride;
  const int in_page = (1 << c.log2_rows) - 1;
  // Tiles of 16 rows lie in one page.  Tiles behind the last row that is seen, or in front of the first one, are the nearest again (their scores are masked).
  const auto tile_row = [&](int blk, int t) { return max(min(blk * ROWS + 16 * t, (most - 1) & ~15), lo & ~15); };
  const auto pages_of = [&](int blk, int (&p)[TILES]) {
#pragma unroll
    for (int t = 0; t < TILES; ++t) p[t] = table[tile_row(blk, t) >> c.log2_rows];
  };
  Keys kr;
  Values vr;
  const unsigned stride = (unsigned)c.stride_row, k_off = Keys::lane_offset(stride, lane), v_off = Values::lane_offset(stride, g, col);
  uintx4* const k_lds = reinterpret_cast<uintx4*>(&ring[w][0]);
  int pg[TILES], bad = 0, next_bad = 0;   // pages of the next block; tiles of this and of the next one whose page is none
  int64_t at[TILES];                  // of the next block's tiles in k and v
  const auto place = [&](int blk) {
    next_bad = 0;
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      int p = pg[t];
      if (__builtin_expect((unsigned)p >= (unsigned)c.pages, 0)) {
        p = 0;
        next_bad |= 1 << t;
      }
      at[t] = p * c.stride_page + (tile_row(blk, t) & in_page) * c.stride_row + h * c.stride_head;
    }
    if (next_bad) report(c);
  };
  const auto load_k = [&]() {
#pragma unroll
    for (int i = 0; i < Keys::kLoads; ++i) kr.load(i, c.k + at[Keys::tile(i)], stride, k_off);
  };
  const auto load_v = [&]() {
#pragma unroll
    for (int i = 0; i < Values::kLoads; ++i) vr.load(i, c.v + at[Values::tile(i)], stride, v_off);
  };
  int blk = first + w;
  if (blk < last) {
    pages_of(blk, pg);
    place(blk);
    load_k();
    load_v();
    if (blk + kWaves < last) pages_of(blk + kWaves, pg);
  }

  floatx4 o[MT][NQ];   // O^T: row m = 4 g + r of tile mt, query 16 qt + col
  floatx4 ls[NQ];      // row sums of P, bf16: all rows hold the same; float32: those of the lane's keys in [0]
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

  for (; blk < last; blk += kWaves) {
    const bool more = blk + kWaves < last;
    const int key0 = blk * ROWS;
    bad = next_bad;
    wave_lds_order();   // the last reads of the block before
    kr.put(k_lds, lane);
    wave_lds_order();
    int64_t here[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) here[t] = at[t];
    if (more) {
      place(blk + kWaves);
      load_k();
      if (blk + 2 * kWaves < last) pages_of(blk + 2 * kWaves, pg);
    }
    floatx4 sc[TILES][NQ];
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      floatx4 some[SUMS][NQ];
#pragma unroll
      for (int i = 0; i < SUMS * NQ; ++i) some[i / NQ][i % NQ] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < PIECES; ++s) {
        const uintx4 k = Keys::get(k_lds, t, s, col, g);
        if constexpr (kBf16) {
#pragma unroll
          for (int qt = 0; qt < NQ; ++qt)
            some[0][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, qf[qt][s]), some[0][qt], 0, 0, 0);
        } else {
          const floatx4 x = __builtin_bit_cast(floatx4, k);
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int qt = 0; qt < NQ; ++qt) {
              const floatx4 y = __builtin_bit_cast(floatx4, qf[qt][s]);
              some[i % SUMS][qt] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], y[i], some[i % SUMS][qt], 0, 0, 0);
            }
        }
      }
#pragma unroll
      for (int qt = 0; qt < NQ; ++qt) {
        if constexpr (SUMS == 4) some[0][qt] = (some[0][qt] + some[1][qt]) + (some[2][qt] + some[3][qt]);
        sc[t][qt] = some[0][qt];
      }
    }
    const bool masked = key0 < lo || key0 + ROWS > fewest || bad != 0;
    bool apart = false;   // some queries see infinities or NaNs that others do not
    if (masked) {
#pragma unroll
      for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int key = key0 + 16 * t + 4 * g + r;
          const bool gone = key < lo || (bad >> t & 1);
#pragma unroll
          for (int qt = 0; qt < NQ; ++qt)
            if (gone || key >= sees[qt]) sc[t][qt][r] = -INFINITY;
        }
      // Rows that no query of the tile sees may hold anything: their probabilities are zero, and the product must not meet a NaN.
      bool strange = false;
#pragma unroll
      for (int i = 0; i < Values::kLoads; ++i) {
        const int t = Values::tile(i), key = key0 + 16 * t + Values::row(i, g, col);
        if (key < lo || key >= most || (bad >> t & 1)) vr.clear(i);
        strange |= key >= fewest && vr.strange(i);
      }
      apart = __any(strange);
    }
    // The reference is the largest score so far: the largest probabilities lie just below one, where bf16 rounds them finest.
    float m_new[NQ];
    bool moved = false;
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) {
      float mx = sc[0][qt][0];
#pragma unroll
      for (int j = 1; j < 4 * TILES; ++j) mx = maximum(mx, sc[j >> 2][qt][j & 3]);
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
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
      for (int qt = 0; qt < NQ; ++qt)
#pragma unroll
        for (int r = 0; r < 4; ++r) sc[t][qt][r] = __builtin_amdgcn_exp2f(fmaf(sc[t][qt][r], c2, -mc[qt]));
    if (__builtin_expect(apart, 0)) {
      // Each query takes what it sees: key by key, elements that are no numbers, and the product below goes without them.
      float* const p_sh = &ring[w][0];   // [key, query]
#pragma unroll
      for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int qt = 0; qt < NQ; ++qt)
#pragma unroll
          for (int r = 0; r < 4; ++r) p_sh[(16 * t + 4 * g + r) * QROWS + 16 * qt + col] = sc[t][qt][r];
      wave_lds_order();
#pragma unroll 1
      for (int x = 0; x < ROWS; ++x) {
        const int key = key0 + x, t = x >> 4;
        if (key < lo || key >= most || (bad >> t & 1)) continue;
        const T* v_row = reinterpret_cast<const T*>(c.v + (t ? here[TILES - 1] : here[0]) + (x & 15) * c.stride_row);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float y = (float)v_row[Values::dim(mt, 4 * g + r)];
            if ((__builtin_bit_cast(unsigned, y) & 0x7F800000u) != 0x7F800000u) continue;
#pragma unroll
            for (int qt = 0; qt < NQ; ++qt)
              if (key < sees[qt]) o[mt][qt][r] += p_sh[x * QROWS + 16 * qt + col] * y;
          }
      }
      wave_lds_order();
#pragma unroll
      for (int i = 0; i < Values::kLoads; ++i) vr.clear_strange(i);
    }
    if constexpr (kBf16) {
      bf16x8 pf[NQ];
#pragma unroll
      for (int qt = 0; qt < NQ; ++qt) {
#pragma unroll
        for (int j = 0; j < 8; ++j) pf[qt][j] = (__bf16)sc[j >> 2][qt][j & 3];
        ls[qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[qt], ls[qt], 0, 0, 0);   // sums over the numbers that the product below uses
      }
#pragma unroll
      for (int mt = 0; mt < MT; mt += 2) {
        bf16x8 vf[2];
        vr.operands(mt / 2, col, vf);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int qt = 0; qt < NQ; ++qt) o[mt + i][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[i], pf[qt], o[mt + i][qt], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int qt = 0; qt < NQ; ++qt) {
          ls[qt][0] += sc[0][qt][r];
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
            o[mt][qt] = __builtin_amdgcn_mfma_f32_16x16x4f32(vr.x[r][mt >> 2][mt & 3], sc[0][qt][r], o[mt][qt], 0, 0, 0);
        }
    }
    if (more) load_v();
  }
  if constexpr (!kBf16) {
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) {
      ls[qt][0] += __shfl_xor(ls[qt][0], 16, 64);
      ls[qt][0] += __shfl_xor(ls[qt][0], 32, 64);
    }
  }

  // ---- merge the waves' partial results; wave w finishes rows 4 g + w of all tiles ----
  wave_lds_order();
  float4* const mine = reinterpret_cast<float4*>(&ring[w][0]) + lane;
#pragma unroll
  for (int qt = 0; qt < NQ; ++qt)
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int m4 = 0; m4 < MT / 4; ++m4)
        mine[((r * NQ + qt) * (MT / 4) + m4) * 64] = make_float4(o[4 * m4][qt][r], o[4 * m4 + 1][qt][r], o[4 * m4 + 2][qt][r], o[4 * m4 + 3][qt][r]);
  if (g == 0) {
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) {
      m_sh[w][16 * qt + col] = mc[qt];
      l_sh[w][16 * qt + col] = ls[qt][0];
    }
  }
  __syncthreads();
  const bool whole = part == 1 && item.chunks == 1 && group < 0;
#pragma unroll
  for (int qt = 0; qt < NQ; ++qt) {
    float M = -FLT_MAX;
#pragma unroll
    for (int x = 0; x < kWaves; ++x) M = fmaxf(M, m_sh[x][16 * qt + col]);
    float fw[kWaves], L = 0.f;
#pragma unroll
    for (int x = 0; x < kWaves; ++x) {
      fw[x] = __builtin_amdgcn_exp2f(m_sh[x][16 * qt + col] - M);   // a wave without blocks has summed nothing
      L = fmaf(fw[x], l_sh[x][16 * qt + col], L);
    }
    float acc[MT];
#pragma unroll
    for (int m4 = 0; m4 < MT / 4; ++m4) {
      float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int x = 0; x < kWaves; ++x) {
        const float4 p = reinterpret_cast<const float4*>(&ring[x][0])[((w * NQ + qt) * (MT / 4) + m4) * 64 + lane];
        s.x = fmaf(fw[x], p.x, s.x);
        s.y = fmaf(fw[x], p.y, s.y);
        s.z = fmaf(fw[x], p.z, s.z);
        s.w = fmaf(fw[x], p.w, s.w);
      }
      acc[4 * m4] = s.x; acc[4 * m4 + 1] = s.y; acc[4 * m4 + 2] = s.z; acc[4 * m4 + 3] = s.w;
    }
    if (row[qt] < 0) continue;
    const float inv = sees[qt] > 0 ? 1.f / L : 0.f;
    const int64_t prow = item.row0 + 16 * qt + col;
    const bool some = MEND && !item.all;
    float f = 1.f;
    if (some && !whole) f = __builtin_amdgcn_exp2f(M - a.part_ml[2 * prow]);   // to the reference that stays
#pragma unroll
    for (int mt = 0; mt < MT; mt += SIDE) {
      const int d = Values::dim(mt, 4 * g + w);
      if (some && whole) mend_some(static_cast<T*>(a.out) + row[qt] * D + d, acc + mt, SIDE, inv);
      else if (some) mend_some(a.part_o + prow * D + d, acc + mt, SIDE, f);
      else if (whole) store_some(static_cast<T*>(a.out) + row[qt] * D + d, acc + mt, SIDE, inv);
      else store_some(a.part_o + prow * D + d, acc + mt, SIDE, 1.f);
    }
    if (!some && !whole && w == 0 && g == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * prow) = make_float2(M, L);
  }
}

// Work-group id of a part; lds: kFewLds bytes, 1024-byte aligned.
template <typename T, int D, int NQ, bool NT>
__device__ __forceinline__ void attn_pages_few(const AttnPagesArgs& a, int part, int id, unsigned char* lds) {
  constexpr int QROWS = 16 * NQ;
  const Pages& c = a.c;
  const int tiles = a.part[part].tiles;
  // The tiles of an entry, head and chunk follow each other on an XCD (work-group id mod 8).
  const int along = id >> 3, pair = (along / tiles) * 8 + (id & 7), tile = along % tiles;
  Work work;
  if (!find_work(a, part, pair, work)) return;
  const int chunk = work.local % work.chunks;
  if (work.local == 0 && tile == 0 && threadIdx.x == 0) a.plan[(part ? a.n_shared : 0) + work.entry] = make_int2(work.base, work.chunks);
  const int b0 = part == 0 ? a.shared[work.entry].first : c.by_head ? work.entry / c.heads : work.entry;   // the first (or only) batch element
  const int h = part == 1 && c.by_head ? work.entry % c.heads : work.local / work.chunks;
  const int group = part == 0 ? work.entry : group_of(a, b0), common = shared_rows(a, group);
  const int entry0 = c.by_head ? b0 * c.heads + h : b0;     // of the table
  const int lo = part ? common : 0;
  const int GN = a.G * c.n, n_rows = part ? GN : a.shared[work.entry].count * GN;
  if (tile * QROWS >= n_rows) return;
  few_queries<T, D, NQ, NT, false>(a, part, FewItem{b0, h, entry0, group, common, lo, n_rows, tile * QROWS, work.chunks, chunk,
                                                    a.part[part].row0 + ((int64_t)pair * tiles + tile) * QROWS, 0, 0, false}, lds);
}

}  // namespace dev
}  // namespace hack
