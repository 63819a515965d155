// Work of attention over caches in pages: which entry, head, chunk and queries a work-group has, by the lengths in device memory.  HIP device code only.
//
// Every wave of a launch sums up the blocks of 32 keys of all entries (groups with shared rows; batch elements, or units, with their own), which gives the
// length of a chunk, and walks over the entries' chunks to its own.
#pragma once

#include <cfloat>

#include "pages_device.h"

namespace hack {
namespace dev {

constexpr int kWaves = 4, kThreads = 64 * kWaves;

struct Work {
  int entry, base, chunks, local;   // base: first pair of the entry; local: pair within it
};
// Whose shared rows batch element b has; -1: none.
__device__ __forceinline__ int group_of(const AttnPagesArgs& a, int b) {
  if (a.n_shared <= 8) {   // one after the other through the scalar cache: no chain of loads
    int g = -1;
    for (int i = 0; i < a.n_shared; ++i) {
      const Shared s = a.shared[i];
      if (b >= s.first && b < s.first + s.count) g = i;
    }
    return g;
  }
  int lo = 0, hi = a.n_shared;
  while (lo < hi) {   // the first group behind b
    const int mid = (lo + hi) >> 1;
    if (a.shared[mid].first <= b) lo = mid + 1;
    else hi = mid;
  }
  return lo > 0 && b < a.shared[lo - 1].first + a.shared[lo - 1].count ? lo - 1 : -1;
}
__device__ __forceinline__ int shared_rows(const AttnPagesArgs& a, int g) { return g < 0 ? 0 : min(a.shared[g].rows, a.c.max_len); }
// Blocks of an entry, and its heads.
__device__ __forceinline__ int entry_blocks(const AttnPagesArgs& a, int part, int e) {
  if (part == 0) return blocks_between(0, shared_rows(a, e));
  return blocks_between(a.n_shared == 0 ? 0 : shared_rows(a, group_of(a, a.c.by_head ? e / a.c.heads : e)), rows_of(a.c, e));
}
__device__ __forceinline__ int entries_of(const AttnPagesArgs& a, int part) { return part == 0 ? a.n_shared : a.c.by_head ? a.batch * a.c.heads : a.batch; }
__device__ __forceinline__ int entry_heads(const AttnPagesArgs& a, int part) { return part == 1 && a.c.by_head ? 1 : a.c.heads; }

// Sums over the lanes up to this one, without LDS.
template <int CTRL, int ROWS> __device__ __forceinline__ int dpp_zero(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xF, true); }
__device__ __forceinline__ int lanes_scan(int x) {
  x += dpp_zero<0x111, 0xF>(x);   // row_shr 1, 2, 4, 8
  x += dpp_zero<0x112, 0xF>(x);
  x += dpp_zero<0x114, 0xF>(x);
  x += dpp_zero<0x118, 0xF>(x);
  x += dpp_zero<0x142, 0xA>(x);   // row_bcast 15, 31
  x += dpp_zero<0x143, 0xC>(x);
  return x;
}
template <int CTRL, int ROWS> __device__ __forceinline__ float dpp_zero(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, ROWS, 0xF, true));
}
__device__ __forceinline__ float lanes_sum(float x) {   // in all lanes
  x += dpp_zero<0x111, 0xF>(x);
  x += dpp_zero<0x112, 0xF>(x);
  x += dpp_zero<0x114, 0xF>(x);
  x += dpp_zero<0x118, 0xF>(x);
  x += dpp_zero<0x142, 0xA>(x);
  x += dpp_zero<0x143, 0xC>(x);
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}
__device__ __forceinline__ int lanes_most(int x) {   // of numbers from 0 on, in all lanes
  x = max(x, dpp_zero<0x111, 0xF>(x));
  x = max(x, dpp_zero<0x112, 0xF>(x));
  x = max(x, dpp_zero<0x114, 0xF>(x));
  x = max(x, dpp_zero<0x118, 0xF>(x));
  x = max(x, dpp_zero<0x142, 0xA>(x));
  x = max(x, dpp_zero<0x143, 0xC>(x));
  return __builtin_amdgcn_readlane(x, 63);
}
// Over the 16 lanes of a row, in all of them.
template <int CTRL> __device__ __forceinline__ int dpp_mov(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, 0xF, 0xF, true); }
__device__ __forceinline__ int row_most(int x) {
  x = max(x, dpp_mov<0x121>(x));   // row_ror 1, 2, 4, 8
  x = max(x, dpp_mov<0x122>(x));
  x = max(x, dpp_mov<0x124>(x));
  return max(x, dpp_mov<0x128>(x));
}
__device__ __forceinline__ int row_fewest(int x) {
  x = min(x, dpp_mov<0x121>(x));
  x = min(x, dpp_mov<0x122>(x));
  x = min(x, dpp_mov<0x124>(x));
  return min(x, dpp_mov<0x128>(x));
}

// Every wave does it by itself.  Blocks of the first 256 entries stay in registers, those behind them are counted again.
__device__ __forceinline__ bool find_work(const AttnPagesArgs& a, int part, int pair, Work& w) {
  const int lane = threadIdx.x & 63, n = entries_of(a, part), heads = entry_heads(a, part);
  if (a.part[part].share == 0.f) {   // nothing is cut
    const int e = pair / heads;
    w = Work{e, e * heads, 1, pair - e * heads};
    return e < n;
  }
  constexpr int kHeld = 4;
  int held[kHeld];
  float sum = 0.f;
  int longest = 0;
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    held[i] = 64 * i + lane < n ? entry_blocks(a, part, 64 * i + lane) : 0;
    sum += held[i];
    longest = max(longest, held[i]);
  }
  for (int e = 64 * kHeld + lane; e < n; e += 64) {
    const int x = entry_blocks(a, part, e);
    sum += x;
    longest = max(longest, x);
  }
  sum *= (float)heads * a.part[part].tiles;
  if (a.parts == 3) {
    float other = 0.f;
    for (int e = lane; e < entries_of(a, 1 - part); e += 64) other += entry_blocks(a, 1 - part, e);
    sum = fmaf(other, (float)entry_heads(a, 1 - part) * a.part[1 - part].tiles, sum);
  }
  const int chunk = chunk_blocks(lanes_sum(sum), lanes_most(longest), a.part[part]);
  int carry = 0;
  const auto look = [&](int e0, int blocks) __attribute__((always_inline)) {
    const int e = e0 + lane, chunks = e < n ? entry_chunks(blocks, chunk) : 0, incl = lanes_scan(chunks * heads), base = carry + incl - chunks * heads;
    const uint64_t hit = __ballot(pair >= base && pair < base + chunks * heads);
    carry += __builtin_amdgcn_readlane(incl, 63);
    if (hit == 0) return false;
    const int at = __builtin_ctzll(hit), first = __builtin_amdgcn_readlane(base, at);
    w = Work{e0 + at, first, __builtin_amdgcn_readlane(chunks, at), pair - first};
    return true;
  };
#pragma unroll
  for (int i = 0; i < kHeld; ++i)
    if (64 * i < n && look(64 * i, held[i])) return true;
  for (int e0 = 64 * kHeld; e0 < n; e0 += 64)
    if (look(e0, e0 + lane < n ? entry_blocks(a, part, e0 + lane) : 0)) return true;
  return false;
}

}  // namespace dev
}  // namespace hack
