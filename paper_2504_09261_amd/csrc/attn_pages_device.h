// Work of attention over caches in pages: which entry, head, chunk and queries a work-group has, by the lengths in device memory.  HIP device code only.
//
// Every work-group of a launch sums up the blocks of 32 keys of all entries (groups with shared rows; batch elements, or units, with their own), which gives the
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
__device__ __forceinline__ int group_of(const AttnPagesArgs& a, int b) {   // whose shared rows batch element b has; -1: none
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
  return blocks_between(shared_rows(a, group_of(a, a.c.by_head ? e / a.c.heads : e)), rows_of(a.c, e));
}
__device__ __forceinline__ int entries_of(const AttnPagesArgs& a, int part) { return part == 0 ? a.n_shared : a.c.by_head ? a.batch * a.c.heads : a.batch; }
__device__ __forceinline__ int entry_heads(const AttnPagesArgs& a, int part) { return part == 1 && a.c.by_head ? 1 : a.c.heads; }

__device__ __forceinline__ bool find_work(const AttnPagesArgs& a, int part, int pair, Work& w) {
  __shared__ float total_sh[kWaves];
  __shared__ int scan_sh[kWaves];
  __shared__ Work work_sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  float sum = 0.f;
  if (a.part[part].share > 0.f) {
    for (int p = 0; p < 2; ++p) {
      if (!(a.parts >> p & 1)) continue;
      const float each = (float)entry_heads(a, p) * a.part[p].tiles;
      for (int e = tid; e < entries_of(a, p); e += kThreads) sum += each * entry_blocks(a, p, e);
    }
#pragma unroll
    for (int x = 1; x < 64; x *= 2) sum += __shfl_xor(sum, x, 64);
    if (lane == 0) total_sh[wave] = sum;
    __syncthreads();
    sum = total_sh[0] + total_sh[1] + total_sh[2] + total_sh[3];
  }
  const int chunk = chunk_blocks(sum, a.part[part].share, a.least);
  const int n = entries_of(a, part), heads = entry_heads(a, part);
  if (tid == 0) work_sh.entry = -1;
  int carry = 0;
  for (int e0 = 0; e0 < n && carry <= pair; e0 += kThreads) {
    const int e = e0 + tid;
    const int chunks = e < n ? entry_chunks(entry_blocks(a, part, e), chunk) : 0;
    int incl = chunks * heads;
#pragma unroll
    for (int x = 1; x < 64; x *= 2) {
      const int y = __shfl_up(incl, x, 64);
      if (lane >= x) incl += y;
    }
    __syncthreads();   // the sums of the round before have been read
    if (lane == 63) scan_sh[wave] = incl;
    __syncthreads();
    int all = 0, before = 0;
#pragma unroll
    for (int x = 0; x < kWaves; ++x) {
      if (x < wave) before += scan_sh[x];
      all += scan_sh[x];
    }
    const int base = carry + before + incl - chunks * heads;
    if (pair >= base && pair < base + chunks * heads) work_sh = Work{e, base, chunks, pair - base};
    carry += all;
  }
  __syncthreads();
  w = work_sh;
  w.entry = __builtin_amdgcn_readfirstlane(w.entry);
  w.base = __builtin_amdgcn_readfirstlane(w.base);
  w.chunks = __builtin_amdgcn_readfirstlane(w.chunks);
  w.local = __builtin_amdgcn_readfirstlane(w.local);
  return w.entry >= 0;
}

}  // namespace dev
}  // namespace hack
