// Attention over caches in pages for many queries, bf16: work items of 128 queries, four waves of 32, or of 64, four waves of 16, which share every block of 32 keys through LDS (few
// queries, float32 contexts and the merge of partial results: kernels_attn_pages.hip).
//
// The stage is that of the 128-query kernel over contiguous rows: scores of block j + 1, probabilities of block j and PV product of block j - 1 side by
// side, in slots of one matrix instruction, an LDS read and a share of the vector work.  What pages add: a copy instruction takes rows of one
// 16-row tile, which lie in one page, so it has a base of its own, which is read a stage ahead out of a ring in LDS that the
// threads fill from the table, 256 blocks at a time.  Blocks with rows that some query of the item does not see (the last ones, causal; a first one that
// begins inside the shared rows) come first, their scores are masked, and rows that nobody sees are not copied: the nearest row that is seen stands in for them.
// A masked row's probability is zero, which keeps it out of the sums unless its value is an infinity or NaN (its own, or that of the seen row that stands in for
// it: zero times an infinity is NaN, whoever sees the row).  An item whose results are no numbers, and that finds values that are none in the rows of its masked
// blocks, does the queries of these waves again as few queries do it (attn_pages_few.h), and numbers among their results stand; one that met a page that is none
// does all of its queries again.  1000 causal queries of 72 heads of 64 over 3000 rows 94 us; with a NaN that some queries of an item see 234, with a page that is none 765
// (key by key in each wave, query after query: 42.5 ms).
//
// Bound by the matrix cores and the vector work beside them.  Measured, head_dim 128: 3000 causal queries of 32 heads over 4001 to 7001 rows of 8 caches 243 to 261 us (1.04 to 1.11
// PFLOP/s; a large library product reaches 1.2), without the mask 314 (1.10).  At head_dim 64 the exponentials of a block stand beside half the products: the same at 64, 160 to 163 us
// (0.83 to 0.84).  A third of the LDS' active cycles are the K reads' two-way bank conflicts, as in the kernel over contiguous rows, where a placement without them is no faster.  Places computed from the table in every stage, copies with scalar bases, masks in every stage: 479 us for the 310 that the form here took then; queries in the
// order number, head instead of head, number, so that an item's last blocks are few and items are in order of their lengths: 310 -> 270.
#include "attn_pages_few.h"

namespace hack {

namespace {

using namespace dev;

constexpr int kNW = 4;            // waves
constexpr int kNS = 4;            // LDS slots per tensor
constexpr int kRing = 512;        // blocks whose places LDS holds, filled by halves
constexpr float kHeadroom = 15.f; // the reference lies 2^15 above the running maximum: the exponent's top bit says that a probability reached 2

template <int I, int N, typename F>
__device__ __forceinline__ void for_each(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    for_each<I + 1, N>(f);
  }
}

// Vector work of a stage in the order of issue: E scores a lane become probabilities, dependent operations two elements apart.
struct Step {
  int kind, index;   // 0 multiply-add, 1 exponential, 2 conversion of elements index and index + 1
};
template <int E> constexpr Step softmax_step(int t) {
  int n = 0;
  for (int j = -2; j < E + 2; ++j) {
    if (j >= 0 && j < E && n++ == t) return Step{1, j};
    if (j + 2 < E && n++ == t) return Step{0, j + 2};
    if (j >= 2 && j % 2 == 0 && n++ == t) return Step{2, j - 2};
  }
  return Step{-1, 0};
}
template <int E> constexpr int steps_before(int s, int slots) {   // in front of slot s
  constexpr int kSteps = E + E + E / 2, kCycles = E * 4 + E * 8 + E / 2 * 4;
  if (s >= slots) return kSteps;
  int c = 0, t = 0;
  while (t < kSteps) {
    c += softmax_step<E>(t).kind == 1 ? 8 : 4;
    if (c * slots > kCycles * s) break;
    ++t;
  }
  return t;
}

template <int D> constexpr int kTileLds = 2 * kNS * kKeys * D * 2 + kRing * 16;   // bytes

// Work-group id of a part; lds: kTileLds bytes, 1024-byte aligned.  QT: tiles of 16 queries a wave, 2 (items of 128) or 1 (64; four work-groups a compute unit at
// head_dim 64, where LDS holds just as many.  64 queries of 480 units over 604 to 668 rows there: 19.6 us, by two waves of 32 22.7).
template <int D, int QT>
__device__ __forceinline__ void tile_part(const AttnPagesArgs& a, int part, int id, unsigned char* lds) {
  constexpr int KC = D / 32;        // MFMA steps over head_dim for S^T
  constexpr int MT = D / 16;        // 16-row tiles of O^T
  constexpr int IPW = D / 64;       // copy instructions per wave, block and tensor
  constexpr int BLK = kKeys * D;    // elements per block and tensor
  constexpr int QROWS = 64 * QT;
  const Pages& c = a.c;
  const int tiles = a.part[part].tiles;
  // The tiles of an entry, head and chunk follow each other on an XCD (work-group id mod 8), the last ones, which see the most rows, first.
  const int along = id >> 3, pair = (along / tiles) * 8 + (id & 7), tile = tiles - 1 - along % tiles;
  Work work;
  if (!find_work(a, part, pair, work)) return;
  const int chunk = work.local % work.chunks;
  if (work.local == 0 && tile == 0 && threadIdx.x == 0) a.plan[(part ? a.n_shared : 0) + work.entry] = make_int2(work.base, work.chunks);
  const int b0 = part == 0 ? a.shared[work.entry].first : c.by_head ? work.entry / c.heads : work.entry;
  const int h = part == 1 && c.by_head ? work.entry % c.heads : work.local / work.chunks;
  const int group = part == 0 ? work.entry : group_of(a, b0), common = shared_rows(a, group);
  const int entry0 = c.by_head ? b0 * c.heads + h : b0;     // of the table
  const int lo = part ? common : 0;
  const int GN = a.G * c.n, n_rows = part ? GN : a.shared[work.entry].count * GN;
  if (tile * QROWS >= n_rows) return;
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, g = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);

  __bf16 (&Ks)[kNS][BLK] = *reinterpret_cast<__bf16 (*)[kNS][BLK]>(lds);
  __bf16 (&Vs)[kNS][BLK] = *reinterpret_cast<__bf16 (*)[kNS][BLK]>(lds + sizeof Ks);
  int64_t (&place_sh)[kRing][2] = *reinterpret_cast<int64_t (*)[kRing][2]>(lds + 2 * sizeof Ks);   // where the two tiles of a block begin in k and v, bytes
  // In front of the first copies, and behind the last reads, the waves' words lie where K does.
  int* const most_sh = reinterpret_cast<int*>(lds);
  int* const fewest_sh = most_sh + kNW;
  int* const again_sh = fewest_sh + kNW;
  int* const strange_sh = again_sh + kNW;
  bool bad = false;   // this thread met a page that is none

  // ---- queries and the rows that they see ----
  struct Query {
    int64_t row;    // of q and out
    int sees;
    bool there;
  };
  const auto query = [&](int x) __attribute__((always_inline)) {
    const int j = tile * QROWS + x, jj = min(j, n_rows - 1), m = jj / GN, r = jj - m * GN, n = r / a.G, b = b0 + m;
    const int fresh = fresh_of(c, b), len = rows_of(c, c.by_head ? b * c.heads + h : b);
    Query q{((int64_t)b * c.heads + h) * GN + (r - n * a.G) * c.n + n, max(0, a.causal ? len - fresh + n + 1 : len), j < n_rows && n < fresh};
    if (part == 0) q.sees = min(q.sees, common);
    if (!q.there) q.sees = 0;
    return q;
  };
  int sees[QT];
  int most = 0, fewest = c.max_len;
  const __bf16* qrow[QT];
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    const Query q = query(16 * (QT * w + qt) + col);
    sees[qt] = q.sees;
    if (q.there) {
      most = max(most, q.sees);
      fewest = min(fewest, q.sees);
    }
    qrow[qt] = static_cast<const __bf16*>(a.q) + q.row * D + 8 * g;
  }
  most = row_most(most);
  fewest = row_fewest(fewest);
  if (lane == 0) {
    most_sh[w] = most;
    fewest_sh[w] = fewest;
  }
  __syncthreads();
  most = __builtin_amdgcn_readfirstlane(max(max(most_sh[0], most_sh[1]), max(most_sh[2], most_sh[3])));
  fewest = __builtin_amdgcn_readfirstlane(min(min(fewest_sh[0], fewest_sh[1]), min(fewest_sh[2], fewest_sh[3])));

  // ---- blocks of this chunk: [first, first + n_blocks), taken in the order of block_of ----
  const int all = blocks_between(lo, most), begin = lo / kKeys;
  const int first = begin + chunk_at(all, work.chunks, chunk), n_blocks = begin + chunk_at(all, work.chunks, chunk + 1) - first;
  const int end = first + n_blocks;
  const int full_end = max(first, min(end, fewest / kKeys));      // blocks from here on have rows that some query does not see
  const int n_tail = end - full_end, n_head = first < full_end && first * kKeys < lo ? 1 : 0, n_masked = n_tail + n_head;
  const auto block_of = [&](int j) __attribute__((always_inline)) { return j < n_tail ? end - 1 - j : j < n_masked ? first : first + j - n_tail; };

  floatx4 o[MT][QT];       // O^T: head-dim 16mt + 4g + r, query 16qt + col
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) o[mt][qt] = floatx4{0.f, 0.f, 0.f, 0.f};
  floatx4 ls[QT];   // row sums of P (equal in all four rows)
  float mc[QT];     // probabilities are 2^(c2 s - mc); finite from the start, so that keys whose score is -inf get 0
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    ls[qt] = floatx4{0.f, 0.f, 0.f, 0.f};
    mc[qt] = -FLT_MAX;
  }

  if (n_blocks > 0) {
    // ---- places of the blocks in the order in which they are taken, by halves of a ring; past the last block it is repeated ----
    const int row_lo = lo & ~15, row_hi = (most - 1) & ~15;   // first rows of the tiles that hold rows somebody sees
    const int32_t* const table = c.table + entry0 * c.table_stride;
    const auto tile_row = [&](int blk, int t) __attribute__((always_inline)) { return min(max(blk * kKeys + 16 * t, row_lo), row_hi); };
    const auto fill = [&](int j0) __attribute__((always_inline)) {   // those of blocks j0 .. j0 + kRing / 2, one a thread
      const int blk = block_of(min(j0 + tid, n_blocks - 1));
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int r = tile_row(blk, t);
        int p = table[r >> c.log2_rows];
        if ((unsigned)p >= (unsigned)c.pages) {
          report(c);
          bad = true;
          p = 0;
        }
        place_sh[(j0 + tid) % kRing][t] = p * c.stride_page + (r & ((1 << c.log2_rows) - 1)) * c.stride_row + h * c.stride_head;
      }
    };
    static_assert(kRing / 2 == 64 * kNW, "a thread a block");
    fill(0);
    fill(kRing / 2);
    __syncthreads();

    // LDS layout of a block: rows in groups of four, a group's 64-byte pieces row after row (piece x of row r at (r / 4) 8D + 256 x + 64 (r % 4)), the 16-byte
    // chunks of a piece permuted by the group: chunk y holds y ^ (group & 3) in K and y ^ 2 (group & 1) in V.  A copy instruction fills 1 KiB:
    // one group of rows at head_dim 128, two at 64; instruction i of a wave takes rows of tile i (128), or of tile w / 2 (64).
    constexpr int GPI = 2 / IPW;
    const int group_row = (GPI == 1 ? 4 * w : 4 * ((2 * w + (lane >> 5)) & 3)) + ((lane >> 2) & 3);   // row of this lane's piece within its tile
    const int cg = GPI == 1 ? w : 2 * w + (lane >> 5), piece = 4 * ((lane >> 4) & (KC - 1));
    const unsigned k_chunk = (piece + ((lane & 3) ^ (cg & 3))) * 16, v_chunk = (piece + ((lane & 3) ^ (2 * (cg & 1)))) * 16;
    const unsigned ks_lds = lds_addr_of(&Ks[0][0]), vs_lds = lds_addr_of(&Vs[0][0]);
    const uint8_t* const k_lane = c.k + group_row * c.stride_row + k_chunk;   // in a tile at place 0
    const uint8_t* const v_lane = c.v + group_row * c.stride_row + v_chunk;
    struct Places { int64_t at[IPW]; };   // of the tiles that this wave's copies take
    const auto places_of = [&](int j) __attribute__((always_inline)) {
      const int64_t* p = place_sh[j % kRing];
      Places x;
      if constexpr (IPW == 1) {
        x.at[0] = p[w >> 1];
      } else {
        x.at[0] = p[0];
        x.at[1] = p[1];
      }
      return x;
    };
    const auto copy = [&](const uint8_t* from, const Places& p, int slot, unsigned lds) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < IPW; ++i) load_to_lds(from + p.at[i], lds + (unsigned)((slot * BLK + (w + i * kNW) * 512) * 2));
    };
    // Block number j in the order of processing, masked or not: rows that nobody sees are not read.  Copies past the last block repeat it into slots that
    // nobody reads any more, so that every stage issues and awaits as many.
    const auto issue = [&](const uint8_t* from, const Places& p, int slot, int j, unsigned lds) __attribute__((always_inline)) {
      const int x = min(j, n_blocks - 1);
      if (x >= n_masked) return copy(from, p, slot, lds);
      const int blk = block_of(x);
#pragma unroll
      for (int i = 0; i < IPW; ++i) {
        const int r0 = tile_row(blk, IPW == 2 ? i : w >> 1), r = min(max(r0 + group_row, lo), most - 1) - r0;
        load_to_lds(from + p.at[i] + (r - group_row) * c.stride_row, lds + (unsigned)((slot * BLK + (w + i * kNW) * 512) * 2));
      }
    };
    {
      const Places p0 = places_of(0), p1 = places_of(1), p2 = places_of(2), p3 = places_of(3);
      issue(k_lane, p0, 0, 0, ks_lds);
      issue(v_lane, p0, 0, 0, vs_lds);
      if (n_blocks > 1) {
        issue(k_lane, p1, 1, 1, ks_lds);
        issue(k_lane, p2, 2, 2, ks_lds);
        issue(k_lane, p3, 3, 3, ks_lds);
        issue(v_lane, p1, 1, 1, vs_lds);
      }
    }
    Places next_k = places_of(kNS), next_v = places_of(2);   // of the copies of the next stage

    {
      // Q fragments (B operand of S^T = K Q^T): query 16 qt + col, head-dim slice [32kc + 8g, +8); consumed here, so that a wait for them does not drain the
      // copies that are meant to stay in flight later.
      bf16x8 qf[QT][KC];
#pragma unroll
      for (int qt = 0; qt < QT; ++qt)
#pragma unroll
        for (int kc = 0; kc < KC; ++kc) qf[qt][kc] = *reinterpret_cast<const bf16x8*>(qrow[qt] + 32 * kc);
#pragma unroll
      for (int kc = 0; kc < KC; ++kc) asm volatile("" ::"v"(qf[0][kc]), "v"(qf[QT - 1][kc]));

      const float c2 = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, a.scale * kLog2eF)));
      const int e = col >> 2, qd = col & 3;
      const int k_off = e * 4 * D + (col & 3) * 32 + (g ^ e) * 8;   // K operand: row 16kt + col, chunk 4kc + g
      // V^T operand: rows 4g + e and 16 + 4g + e, head-dim 16mt + 4qd; even and odd mt
      const int v_even = g * 4 * D + e * 32 + (2 * (g & 1) + (qd >> 1)) * 8 + 4 * (qd & 1), v_odd = v_even ^ 16;
      bf16x8 ones;
#pragma unroll
      for (int j = 0; j < 8; ++j) ones[j] = (__bf16)1.0f;
      asm volatile("" : "+v"(ones));   // stays in registers

      struct Scores { floatx4 t[2][QT]; };   // keys 16kt + 4g + r, query 16qt + col
      const auto mask = [&](Scores& sc, int blk) __attribute__((always_inline)) {
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int key = blk * kKeys + 16 * kt + 4 * g + r;
#pragma unroll
            for (int qt = 0; qt < QT; ++qt)
              if (key < lo || key >= sees[qt]) sc.t[kt][qt][r] = -INFINITY;
          }
      };
      const auto probs = [&](const Scores& sc, int qt, bf16x8& pf) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 8; ++j) pf[j] = (__bf16)__builtin_amdgcn_exp2f(fmaf(sc.t[j >> 2][qt][j & 3], c2, -mc[qt]));
      };
      const auto too_large = [&](const bf16x8 (&pf)[QT]) __attribute__((always_inline)) -> bool {
        const uintx4 x = __builtin_bit_cast(uintx4, pf[0]), y = __builtin_bit_cast(uintx4, pf[QT - 1]);
        return (((x[0] | x[1] | x[2]) | x[3] | y[0]) | y[1] | y[2] | y[3]) & 0x40004000u;
      };
      const auto rescale = [&](const Scores& sc, bf16x8 (&pf)[QT]) __attribute__((always_inline)) {
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
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
      const auto load_frag = [&](Frags& f, const __bf16* Kt, const __bf16* Vt, int i, int p) __attribute__((always_inline)) {   // one LDS read, p 0 .. 5
        if (p < 2) f.k[p] = *reinterpret_cast<const bf16x8*>(&Kt[16 * p * D + 128 * i + k_off]);
        else f.v[(p >> 1) - 1][p & 1] = lds_read_tr(&Vt[16 * (p & 1) * D + 128 * i + ((p >> 1) - 1 ? v_odd : v_even)]);
      };
      const auto joined = [](const bf16x4 (&v)[2]) __attribute__((always_inline)) { return bf16x8{v[0][0], v[0][1], v[0][2], v[0][3], v[1][0], v[1][1], v[1][2], v[1][3]}; };
      const auto qk = [&](Scores& sn, const Frags& f, int kc, int n) __attribute__((always_inline)) {
        const int kt = QT == 1 ? n : n >> 1, qt = QT == 1 ? 0 : kt ^ (n & 1);
        sn.t[kt][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.k[kt], qf[qt][kc], sn.t[kt][qt], 0, 0, 0);
      };
      const auto pv = [&](const Frags& f, const bf16x8 (&p)[QT], int i, int n) __attribute__((always_inline)) {
        const int m = QT == 1 ? n : n >> 1, qt = QT == 1 ? 0 : m ^ (n & 1);
        o[2 * i + m][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(joined(f.v[m]), p[qt], o[2 * i + m][qt], 0, 0, 0);
      };
      const auto row_sums = [&](const bf16x8 (&p)[QT], int qt) __attribute__((always_inline)) { ls[qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, p[qt], ls[qt], 0, 0, 0); };

      bf16x8 P[2][QT];  // probabilities of block j in P[j & 1]: those of the previous block wait for their PV product
      Frags pre;        // operands of the next stage's first step

      // Stage j, slot S = j % 4 (compile time).  On entry sc = scores of block j, on exit those of block j + 1.  FIRST: j = 0 (no previous block).
      // FULL: blocks from j + 1 on are not masked.
      auto stage = [&](auto slot_tag, auto first_tag, auto full_tag, int j, Scores& sc) __attribute__((always_inline)) {
        constexpr int S = decltype(slot_tag)::value;
        constexpr bool FIRST = decltype(first_tag)::value, FULL = decltype(full_tag)::value;
        const __bf16* const Kt = &Ks[(S + 1) % kNS][0];
        const __bf16* const Vt = &Vs[(S + 3) % kNS][0];
        Scores sn;
#pragma unroll
        for (int i = 0; i < 2 * QT; ++i) sn.t[i & 1][i >> 1] = floatx4{0.f, 0.f, 0.f, 0.f};
        bf16x8 (&pp)[QT] = P[(S + 1) & 1], (&pf)[QT] = P[S & 1];
        Frags f = pre, nx;
        constexpr int E = 8 * QT;
        float x[E];
        auto vec_op = [&](auto t_tag) __attribute__((always_inline)) {
          constexpr Step op = softmax_step<E>(decltype(t_tag)::value);
          constexpr int i = op.index, qt = (i >> 3) & 1, jj = i & 7;
          if constexpr (op.kind == 0) x[i] = fmaf(sc.t[jj >> 2][qt][jj & 3], c2, -mc[qt]);
          else if constexpr (op.kind == 1) x[i] = __builtin_amdgcn_exp2f(x[i]);
          else { pf[qt][jj] = (__bf16)x[i]; pf[qt][jj + 1] = (__bf16)x[i + 1]; }
        };
        constexpr int STEP = 4 * QT, SLOTS = STEP * KC + QT, VEC_SLOTS = SLOTS - 3 * KC / 4;   // the vector work ends early: its test travels beside the last MFMAs
        bool large = false;
        auto slot = [&](auto s_tag) __attribute__((always_inline)) {
          constexpr int T = decltype(s_tag)::value, I = T / STEP < KC ? T / STEP : KC - 1, N = T - STEP * I;   // the last step has QT more
          // one wait for both K operands (lgkmcnt(4)) and one for both of V^T (lgkmcnt(2)) instead of one for each
          if constexpr (N == 0) __builtin_amdgcn_s_waitcnt(0xC47F);
          if constexpr (N == 2 * QT) __builtin_amdgcn_s_waitcnt(0xC27F);
          if constexpr (N < 2 * QT) qk(sn, f, I, N);
          else if constexpr (N < STEP) { if (!FIRST) pv(f, pp, I, N - 2 * QT); }
          else { if (!FIRST) row_sums(pp, N - STEP); }
          for_each<steps_before<E>(T, VEC_SLOTS), steps_before<E>(T + 1, VEC_SLOTS)>(vec_op);
          if constexpr (T == VEC_SLOTS) large = __any(too_large(pf));
          if constexpr (N < 2 || (N >= 2 * QT && N < STEP)) {
            constexpr int READS = N < 2 ? 1 : 2 / QT, p = N < 2 ? N : 2 + READS * (N - 2 * QT);
#pragma unroll
            for (int i = 0; i < READS; ++i) {
              if constexpr (I + 1 < KC) load_frag(nx, Kt, Vt, I + 1, p + i);
              else load_frag(nx, &Ks[(S + 2) % kNS][0], &Vs[S][0], 0, p + i);
            }
          }
          if constexpr (N == STEP - 1 && I + 1 < KC) f = nx;
          __builtin_amdgcn_sched_barrier(0);
        };
        for_each<0, 2 * QT * KC>(slot);
        wait_and_sync<2 * IPW>();   // K(j + 2) and V(j) have landed: everything but what the previous stage issued
        if constexpr (FULL) {
          copy(k_lane, next_k, S, ks_lds);                   // K(j + 4)
          copy(v_lane, next_v, (S + 2) % kNS, vs_lds);       // V(j + 2)
        } else {
          issue(k_lane, next_k, S, j + kNS, ks_lds);
          issue(v_lane, next_v, (S + 2) % kNS, j + 2, vs_lds);
        }
        next_k = places_of(j + kNS + 1);
        next_v = places_of(j + 3);
        __builtin_amdgcn_sched_barrier(0);
        for_each<2 * QT * KC, SLOTS>(slot);
        pre = nx;
        if (__builtin_expect(large, 0)) rescale(sc, pf);
        if (!FULL && j + 1 < n_masked) mask(sn, block_of(j + 1));
        sc = sn;
      };

      dma_wait_but<0>();
      __syncthreads();
      Scores sc;
#pragma unroll
      for (int i = 0; i < 2 * QT; ++i) sc.t[i & 1][i >> 1] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kc = 0; kc < KC; ++kc) {
        Frags f;
        for (int n = 0; n < 2; ++n) load_frag(f, &Ks[0][0], nullptr, kc, n);
#pragma unroll
        for (int n = 0; n < 2 * QT; ++n) qk(sc, f, kc, n);
      }
      for (int n = 0; n < 2; ++n) load_frag(pre, &Ks[1][0], nullptr, 0, n);
      for (int n = 2; n < 6; ++n) load_frag(pre, nullptr, &Vs[0][0], 0, n);
      if (n_masked > 0) mask(sc, block_of(0));

      using No = std::false_type;
      using Yes = std::true_type;
      if (n_blocks > 1) {
        stage(std::integral_constant<int, 0>{}, Yes{}, No{}, 0, sc);
        int j = 1;
        const auto four = [&](auto full_tag) __attribute__((always_inline)) {   // stages j .. j + 3; whether there are more
          if (j >= n_blocks - 1) return false;
          stage(std::integral_constant<int, 1>{}, No{}, full_tag, j, sc);
          if (j + 1 >= n_blocks - 1) return false;
          stage(std::integral_constant<int, 2>{}, No{}, full_tag, j + 1, sc);
          if (j + 2 >= n_blocks - 1) return false;
          stage(std::integral_constant<int, 3>{}, No{}, full_tag, j + 2, sc);
          if (j + 3 >= n_blocks - 1) return false;
          if (__builtin_expect((j + 3) % (kRing / 2) == 0, 0)) fill(j + 3 + kRing / 2);   // over those of blocks that are done
          stage(std::integral_constant<int, 0>{}, No{}, full_tag, j + 3, sc);
          j += 4;
          return true;
        };
        bool more = true;
        while (more && j + 1 < n_masked) more = four(No{});
        while (more) more = four(Yes{});
      }
      // the last block: its probabilities, its PV product and the one of the block before
      const auto pv_block = [&](const __bf16* Vt, const bf16x8 (&p)[QT]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < KC; ++i) {
          Frags f;
          for (int n = 2; n < 6; ++n) load_frag(f, nullptr, Vt, i, n);
#pragma unroll
          for (int n = 0; n < 2 * QT; ++n) pv(f, p, i, n);
        }
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) row_sums(p, qt);
      };
      if (n_blocks > 1) {
        const bool odd = n_blocks & 1;   // the block before the last has an odd number
        bf16x8 pl[QT];
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
          const bf16x8 even_p = P[0][qt], odd_p = P[1][qt];
          pl[qt] = odd ? odd_p : even_p;
        }
        pv_block(&Vs[(n_blocks - 2) % kNS][0], pl);
      }
      wait_and_sync<0>();
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) probs(sc, qt, P[0][qt]);
      if (__any(too_large(P[0]))) rescale(sc, P[0]);
      pv_block(&Vs[(n_blocks - 1) % kNS][0], P[0]);
    }
  }

  // ---- normalise and store: a lane holds head-dim 16mt + 4g .. +4 of queries 16qt + col ----
  const bool whole = part == 1 && work.chunks == 1 && group < 0;
  const int64_t row0 = a.part[part].row0 + ((int64_t)pair * tiles + tile) * QROWS;   // of partial results
  bool odd = false;   // queries of the wave have results that are no numbers
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    const Query q = query(16 * (QT * w + qt) + col);
    if (n_masked > 0) {
      float x = 0.f;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int r = 0; r < 4; ++r) x = fmaf(o[mt][qt][r], 0.f, x);
      // NaN among the sums of rows, beside a number as the sum of probabilities, into which no row goes that is not seen: where that is none, the results are right.
      odd |= __any(q.there && x != 0.f && ls[qt][0] * 0.f == 0.f);
    }
    if (!q.there) continue;
    const float inv = q.sees > 0 ? 1.f / ls[qt][0] : 0.f;
    __bf16* const orow = static_cast<__bf16*>(a.out) + q.row * D;
    const int64_t prow = row0 + 16 * (QT * w + qt) + col;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      if (whole) {
        bf16x4 pk;
#pragma unroll
        for (int r = 0; r < 4; ++r) pk[r] = (__bf16)(o[mt][qt][r] * inv);
        *reinterpret_cast<bf16x4*>(orow + 16 * mt + 4 * g) = pk;
      } else {
        *reinterpret_cast<floatx4*>(a.part_o + prow * D + 16 * mt + 4 * g) = o[mt][qt];
      }
    }
    if (!whole && g == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * prow) = make_float2(mc[qt], ls[qt][0]);
  }
  // Results that are no numbers may be what the queries see: only rows of masked blocks can have brought them to queries that do not see these rows.
  const bool wave_bad = __any(bad);
  if (lane == 0) again_sh[w] = (wave_bad ? 15 : 0) | (odd ? 16 << w : 0);
  __syncthreads();
  const int found = again_sh[0] | again_sh[1] | again_sh[2] | again_sh[3];
  if (__builtin_expect(found == 0, 1)) return;
  const bool any_bad = found & 15;
  const int todo = any_bad ? 15 : found >> 4;   // waves
  if (!any_bad) {
    const int32_t* const table = c.table + entry0 * c.table_stride;
    constexpr int PIECES = D / 8;   // of 16 bytes in a row
    bool strange = false;
    for (int64_t x = tid; x < (int64_t)n_masked * (kKeys * PIECES); x += kNW * 64) {
      const int key = block_of((int)(x / (kKeys * PIECES))) * kKeys + (int)(x / PIECES % kKeys);
      if (key < lo || key >= most) continue;
      const int p = table[key >> c.log2_rows];
      if ((unsigned)p >= (unsigned)c.pages) continue;
      const uintx4 v = *reinterpret_cast<const uintx4*>(c.v + p * c.stride_page + (key & ((1 << c.log2_rows) - 1)) * c.stride_row + h * c.stride_head + x % PIECES * 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) strange |= (v[i] & 0x7F80u) == 0x7F80u || (v[i] & 0x7F800000u) == 0x7F800000u;
    }
    const bool wave_strange = __any(strange);
    if (lane == 0) strange_sh[w] = wave_strange;
    __syncthreads();
    if (!(strange_sh[0] | strange_sh[1] | strange_sh[2] | strange_sh[3])) return;
  }
  // 16 queries after the other, all waves at each (32 at a time: the kernels spill).
  static_assert(kFewLds<D, 1> <= kTileLds<D>, "few queries fit in a tile's LDS");
#pragma unroll 1
  for (int x = 0; x < QT * kNW; ++x) {
    if (!(todo >> x / QT & 1)) continue;
    __syncthreads();
    few_queries<__bf16, D, 1, false, true>(a, part, FewItem{b0, h, entry0, group, common, lo, n_rows, tile * QROWS + 16 * x, work.chunks, chunk, row0 + 16 * x, first, end,
                                                            any_bad}, lds);
  }
}

// Work-groups a compute unit: as many as LDS and the registers that they ask for allow.
template <int D, int QT>
__global__ __launch_bounds__(64 * kNW, D == 128 ? 2 : QT == 1 ? 4 : 3) void attn_pages_tiles(const AttnPagesArgs a) {
  __shared__ __attribute__((aligned(1024))) unsigned char lds[kTileLds<D>];
  const int grid0 = a.parts & 1 ? (a.part[0].pairs + 7) / 8 * 8 * a.part[0].tiles : 0, part = (int)blockIdx.x >= grid0 ? 1 : 0;
  tile_part<D, QT>(a, part, blockIdx.x - (part ? grid0 : 0), lds);
}

// Shared rows by tiles, own rows by few queries: the products of the one beside the loads of the other.
template <int D, int NQ, bool NT>
__global__ __launch_bounds__(64 * kNW, 2) void attn_pages_mixed(const AttnPagesArgs a) {
  __shared__ __attribute__((aligned(1024))) unsigned char lds[std::max(kTileLds<D>, kFewLds<D, NQ>)];
  const int grid0 = (a.part[0].pairs + 7) / 8 * 8 * a.part[0].tiles;
  if ((int)blockIdx.x < grid0) tile_part<D, 2>(a, 0, blockIdx.x, lds);
  else attn_pages_few<__bf16, D, NQ, NT>(a, 1, blockIdx.x - grid0, lds);
}

template <int D>
void launch_some(hipStream_t s, const AttnPagesArgs& a) {
  const dim3 grid((unsigned)(part_grid(a, 0) + part_grid(a, 1)));
  const bool once = reads_once(a);
#define HACK_ATTN_MIXED(NQ, NT) hipLaunchKernelGGL((attn_pages_mixed<D, NQ, NT>), grid, dim3(64 * kNW), 0, s, a)
  if (a.part[1].queries == 16 && once) HACK_ATTN_MIXED(1, true);
  else if (a.part[1].queries == 16) HACK_ATTN_MIXED(1, false);
  else if (a.part[1].queries == 32 && once) HACK_ATTN_MIXED(2, true);
  else if (a.part[1].queries == 32) HACK_ATTN_MIXED(2, false);
  else if (a.part[1].queries == kHalfTileQueries) hipLaunchKernelGGL((attn_pages_tiles<D, 1>), grid, dim3(64 * kNW), 0, s, a);
  else hipLaunchKernelGGL((attn_pages_tiles<D, 2>), grid, dim3(64 * kNW), 0, s, a);
#undef HACK_ATTN_MIXED
}

}  // namespace

void launch_attn_pages_tiles(hipStream_t s, int head_dim, const AttnPagesArgs& a) {
  if (head_dim == 64) launch_some<64>(s, a);
  else launch_some<128>(s, a);
}

}  // namespace hack
