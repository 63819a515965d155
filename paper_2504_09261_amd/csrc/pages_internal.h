// Internal declarations of the caches in pages: appending to them and attention over them (pages_api.cpp and the kernels behind it).  Nothing here is part
// of the C ABI.  Tables and lengths are device memory that the host never reads; everything else travels by value.
#pragma once

#include "ops_internal.h"

namespace hack {

struct Pages {
  uint8_t* k;
  uint8_t* v;
  int64_t stride_page, stride_row, stride_head;   // bytes
  const int32_t* table;
  int64_t table_stride;
  const int32_t* len;
  const int32_t* fresh;    // NULL: n for all
  int* fault;              // host-visible word that kernels raise
  int32_t pages;
  int32_t log2_rows;       // of a page
  int32_t max_len;
  int32_t heads;           // H
  int32_t by_head;
  int32_t n;               // N
};

// ---- appending --------------------------------------------------------------
// t[0]: q (no work-groups where there are none), t[1]: k, v beside them.
struct AppendArgs : RotateArgs {
  RotateTensor v;
  uint32_t all_groups;   // work-groups of a batch element
  int32_t own_rows;      // positions are the rows' numbers in the cache
  Pages c;
};
void launch_append(hipStream_t s, int elem_bytes, int head_dim, bool half_layout, int batch, AppendArgs a);

// ---- attention --------------------------------------------------------------
constexpr int kMostShared = 256;   // groups of a call
constexpr int kKeys = 32;          // of a block, in which work is counted and cut
struct Shared {
  int32_t first, count, rows;
};
// The shared rows of groups (0) and the rows that every batch element, or head of it, has alone (1).
struct AttnPart {
  int32_t queries;    // of a tile: 16 or 32 by few queries, kHalfTileQueries or kPageTileQueries by tiles
  int32_t tiles;      // of an entry's queries
  int32_t pairs;      // (entry, head, chunk) at most
  int32_t uncut;      // entries of up to so many blocks are not cut where none is longer
  int32_t least;      // blocks of a chunk at least
  float share;        // work-groups that the blocks of its launch are cut for; 0: no cuts
  float fill;         // work-groups that fill the device
  int64_t row0;       // first row of its partial results
};
constexpr int kHalfTileQueries = 64, kPageTileQueries = 128;
struct AttnPagesHead {
  Pages c;
  const void* q;
  void* out;
  float* part_o;      // [row0 of the part + (pair, tile, query of the tile), head_dim] unnormalised partial outputs
  float* part_ml;     // [.., 2] their references and normalisers
  int2* plan;         // [groups, then batch elements or units]: first pair and chunks of an entry
  AttnPart part[2];
  int32_t batch;
  int32_t G;          // query heads of a cache
  int32_t n_shared;
  int32_t causal;
  float scale;
  int32_t parts;      // of the launch, a bit each; set by launch_attn_pages
};
struct AttnPagesArgs : AttnPagesHead {
  Shared shared[kMostShared];
};
// How the kernels cut: blocks that hold rows lo to hi; blocks of a chunk where the launch has `total` (times heads and tiles of queries) and the part's longest entry
// `longest`; chunks of an entry.  Shorter chunks than kChunk only as far as compute units have no work-group.  A block counts the same in tiles of 16 queries and of 128.
// Us a call in a graph at kChunk 12 / 16 / 24 / 32 / 48: one long cache 99.6 / 99.4 / 99.5 / 99.8 / 104.3; one token of 64 elements behind 8192 shared rows, whose
// tiles of 128 stand beside own ones of 16, 46.4 / 46.3 / 46.1 / 45.3 / 46.9, behind 2048 36.6 / 36.8 / 36.5 / 36.3 / 36.3, behind 16384 54.6 / 54.5 / 54.5 / 52.2 / 49.5.
constexpr float kChunk = 32.f;
__host__ __device__ inline int blocks_between(int lo, int hi) { return hi > lo ? (hi + kKeys - 1) / kKeys - lo / kKeys : 0; }
__host__ __device__ inline int chunk_blocks(float total, int longest, const AttnPart& p) {
  if (p.share == 0.f || longest <= p.uncut) return 1 << 30;
  const float each = total / p.share, full = total / p.fill < kChunk ? total / p.fill : kChunk, most = each > full ? each : full;
  const int whole = (int)(most < 1e9f ? most : 1e9f);
  return whole < p.least ? p.least : whole + 1;
}
__host__ __device__ inline int entry_chunks(int blocks, int chunk) { return blocks > chunk ? chunks_of(blocks, chunk) : 1; }
constexpr int64_t pairs_grid(int64_t pairs, int64_t tiles) { return (pairs + 7) / 8 * 8 * tiles; }
// merge: partial results may have to be joined.
void launch_attn_pages(hipStream_t s, int elem_bytes, int head_dim, bool merge, AttnPagesArgs a);
void launch_attn_pages_tiles(hipStream_t s, int head_dim, const AttnPagesArgs& a);   // where a part has tiles of kHalfTileQueries or kPageTileQueries; bf16
// Whether every row of K and V is read by one work-group, whose loads then pass the caches by.
inline bool reads_once(const AttnPagesArgs& a) { return a.part[1].tiles == 1 && (!(a.parts & 1) || a.part[0].tiles == 1 || a.part[0].queries == kPageTileQueries); }
// Work-groups of part p in the launch.
inline int64_t part_grid(const AttnPagesArgs& a, int p) { return a.parts >> p & 1 ? pairs_grid(a.part[p].pairs, a.part[p].tiles) : 0; }

}  // namespace hack
