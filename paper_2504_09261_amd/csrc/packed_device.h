// Rows in 4 bits: layout and conversions.  HIP device code only.
//
// A row is cut into groups of 32 elements.  A group has an exponent s (8 bits) and 32 codes of 4 bits: sign, two exponent bits, one mantissa
// bit, for 0, 0.5, 1, 1.5, 2, 3, 4, 6; an element is its code times 2^(s - 127).  s is the smallest for which the group's largest magnitude is at
// most 7 of that unit, so no element is off by more than half of the step it lies in; codes are rounded to nearest, ties to even.  (Were s one lower
// where the largest lies between 6 and 7, it alone would be cut by up to an eighth more; were s one higher, all steps would double.)  s stays in [3, 252], so
// every value is a normal bf16 number or zero; s = 255 says that the group held an infinity or a NaN, and all of it reads as NaN.  Read rows
// packed again give the same bytes.
//
// Blocks of 64 rows hold the codes in the order in which the 16x16x32 matrix instruction takes its A operand, so that a wave's 16-byte loads are
// contiguous: lane l holds a quarter of the head, l / 16, of row l % 16 of a tile of 16 rows.  At head_dim 128 that is one group, 16 bytes; at 64
// half of one, 8 bytes, and two tiles lie side by side.  Behind the codes the exponents, one dword for group g and row r: rows r, r + 16, r + 32, r + 48.
#pragma once

#include "device_util.h"
#include "ops_internal.h"

namespace hack {
namespace dev {

template <int D> constexpr int kPackBytes = 34 * D;   // of a block

// Codes of a quarter of row `row` of a block.
template <int D> __device__ __forceinline__ int code_at(int row, int quarter) {
  const int t = row >> 4, r = row & 15;
  return D == 128 ? ((t * 4 + quarter) * 16 + r) * 16 : (((t >> 1) * 4 + quarter) * 16 + r) * 16 + (t & 1) * 8;
}
template <int D> __device__ __forceinline__ int exponent_at(int row, int group) { return 32 * D + (group * 16 + (row & 15)) * 4 + (row >> 4); }

__device__ __forceinline__ float scale_of(unsigned exponent) { return __builtin_bit_cast(float, exponent << 23); }

// Eight codes as bf16, exactly.
__device__ __forceinline__ bf16x8 codes_bf16(unsigned w, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1),
               c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// ---- attention: arguments, V in LDS -------------------------------------------
template <int N> struct AttnPackedArgs : AttnPackedHead { AttnPackedUnit unit[N]; };

// LDS layout of converted rows of V: groups of four, a group's 64-byte pieces row after row, the 16-byte chunks of a piece permuted by two bits of the row.
// All operands of the PV product stand at constant distances from two addresses, a lane's share of a row at constant distances from two others, and
// neither the writes (eight lanes at a time, 128 bytes: rows 0 to 7 or 8 to 15, one chunk) nor the transposing reads (8 rows, 32 bytes) meet a bank twice; counted:
// no conflict, where permuting by bits 2 and 3 of the row gave 8 cycles a write (64 tokens over 171 MB 37.8 -> 37.3 us, 32 units' 4096 queries 185.6 -> 184.2).
__device__ __forceinline__ int v_flip(int row) { return 2 * ((row >> 2) & 1) | ((row >> 1) & 1); }
template <int D> __device__ __forceinline__ int v_chunk(int row, int chunk) {   // element offset of a chunk
  return (row >> 2) * 4 * D + (chunk >> 2) * 128 + (row & 3) * 32 + ((chunk & 3) ^ v_flip(row)) * 8;
}

}  // namespace dev
}  // namespace hack
