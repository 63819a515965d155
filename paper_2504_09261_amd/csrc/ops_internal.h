// Internal declarations of the operators around the cache: rotary positions, norms of queries and keys, the cache packed
// into 4 bits and attention over it (ops_api.cpp and the kernels behind it).  Nothing here is part of the C ABI.
// Everything a launch needs travels by value: lengths that grow by a token a call would fill a store of launch tables.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "hack_internal.h"

namespace hack {

// ---- rotary positions, norms ------------------------------------------------
constexpr int kMaxPairs = 64;   // rotating pairs of a head
enum : int32_t { kNormNone = 0, kNormRms = 1, kNormL2 = 2 };

struct RotateTensor {
  const void* x;        // element (b, h, n, i) at b sb + h sh + n sn + i
  void* out;            // [B, heads, N, head_dim]
  const float* w;       // weight of element i of head h at h w_stride + i, NULL: ones
  int64_t sb, sh, sn;
  int32_t heads;
  int32_t w_stride;
  // launch shape, set by shape_rotation
  int32_t tokens_log2;  // rows of one head a work-group takes (power of two)
  int32_t tiles;        // of rows: work-groups take one of them and a part of the heads
};
struct RotateArgs {
  RotateTensor t[2];
  const int32_t* pos;   // position of row n of batch element b on axis a at b pos_b + a N + n, NULL: pos0 + n
  int64_t pos_b;
  int32_t pos0;
  int32_t n;            // N
  int32_t rot_dim;      // rotating elements of a head, 0: none
  int32_t section;      // of an axis
  float gain, eps;
  int32_t norm;         // kNorm*
  float low;            // sums of squares below it, or not finite, are formed again from scaled rows; set by launch_rotate
  // launch shape, set by shape_rotation
  uint32_t groups[2];   // work-groups of a batch element: of t[0], of both
  int32_t steps;        // heads a thread takes, one after the other
  uint64_t turns[kMaxPairs];   // of a pair per position, in units of 2^-64 of a turn
};
constexpr int kRotateThreads = 256;   // of a work-group, 16 elements each
void launch_rotate(hipStream_t s, int elem_bytes, int head_dim, bool half_layout, int batch, int n_tensors, RotateArgs a);

// ---- rows in 4 bits ---------------------------------------------------------
constexpr int kPackRows = 64;    // rows of a block
constexpr int kPackGroup = 32;   // elements of a row that share a scale
inline int packed_block_bytes(int head_dim) { return kPackRows * (head_dim / 2 + head_dim / kPackGroup); }
struct PackUnit {
  int64_t row0;     // first row in the arrays of plain rows
  int32_t len_in;   // pack: cached rows there, which the new ones follow
  int32_t block;    // first block in the packed arrays
  int32_t first;    // row of the unit there
  int32_t n;        // rows
};
struct PackHead {
  CachePtrs plain;       // rows read (pack) or written (unpack)
  CachePtrs packed;
  const void* k_new;
  const void* v_new;
  const int32_t* kept;   // [unit, kept_stride], NULL: all rows in order
  int64_t kept_stride;
  int32_t n_new;         // rows of k_new / v_new of a unit
  int32_t pos_new;
  int32_t unit0;         // of the launch, set by the launchers
  int32_t row_at;        // row of each unit that the launch begins with, set by the launchers
};
void launch_pack(hipStream_t s, int elem_bytes, int head_dim, PackHead h, const PackUnit* units, int n_units);
void launch_unpack(hipStream_t s, int elem_bytes, int head_dim, PackHead h, const PackUnit* units, int n_units);

// ---- attention over them ----------------------------------------------------
struct AttnPackedUnit {
  int32_t block;   // first block
  int32_t len;     // rows
  int32_t unit;    // u = b*H + h
};
struct AttnPackedHead {
  const uint8_t* k;
  const uint8_t* v;
  const void* q;
  void* out;
  float* part_o;      // [slot, queries of a work-group, head_dim] unnormalised partial outputs
  float* part_ml;     // [slot, queries of a work-group, 2] their references and normalisers
  int32_t N_k;
  float scale;
  int32_t n_units;    // of the launch
  int32_t q_tiles;    // of a unit's queries
  int32_t n_chunks;   // most chunks that a unit's keys are cut into
  int32_t chunk;      // most blocks of kPackRows keys of one
};
// Chunks of a unit's blocks: how many of at most `most` blocks, where chunk c begins (as even as they can be), and the rows of a unit of len rows in blocks
// [lo, hi).  Unsigned: the last block of a unit may end at row 2^31.
__host__ __device__ inline int packed_blocks(int len) { return (int)(((unsigned)len + kPackRows - 1) / kPackRows); }
__host__ __device__ inline int chunks_of(int n, int most) { return (n + most - 1) / most; }
__host__ __device__ inline int chunk_at(int n, int chunks, int c) { return (int)((unsigned)n / chunks * c + ((unsigned)n % chunks) * c / chunks); }
__host__ __device__ inline int rows_in(int len, int lo, int hi) {
  const unsigned end = (unsigned)hi * kPackRows;
  return (int)((end < (unsigned)len ? end : (unsigned)len) - (unsigned)lo * kPackRows);
}
__host__ __device__ inline int stages_of(int rows, int each) { return (int)(((unsigned)rows + each - 1) / each); }
// Chunks of a unit at most: the merge keeps their factors in LDS.  (Two work-groups to each of 256 compute units make 512.)
constexpr int kMostChunks = 1024;
// Units of a launch.  They travel by value (a table in memory would be another copy each time a length grows), and as arguments are copied whole there is a short list
// too.  A call of 64 units and one of 65 take, with everything that the host does: packing 6.0 and 7.1 us, reading back 6.8 and 6.9, attention 5.8 and 6.5;
// of 512 units 8.5, 8.1 and 7.7, of one 6.4, 6.1 and 5.6.
constexpr int kFewUnits = 64, kPackUnits = 640, kAttnPackedUnits = 1024;
// queries: of a work-group, 16, 32 or kTileQueries; float32 (elem_bytes 4): 16
constexpr int kTileQueries = 128;
void launch_attn_packed(hipStream_t s, int elem_bytes, int head_dim, int queries, const AttnPackedHead& h, const AttnPackedUnit* units);
void launch_attn_packed_tiles(hipStream_t s, int head_dim, const AttnPackedHead& h, const AttnPackedUnit* units);   // without the merge
}  // namespace hack
