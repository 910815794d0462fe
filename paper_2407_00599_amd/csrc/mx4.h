// Microscaled 4-bit floating point.  Along the index that a product sums over, values are cut into blocks of 32.  With a block's largest
// magnitude a in [2^x, 2^(x+1)) its scale is 2^(x-2), twice that where a / scale would round to 8; a value is kept as the one of
// 0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives (codes 0..7, and 8 more for the sign) that is nearest to value / scale, of two the one with the even code.
// The scale byte is b for 2^(b-127).  Edges: the smallest scale is 2^-127 (b = 0; a block of zeros has it too); the largest is 2^125, so that 6 of them
// are a number (magnitudes from 1.75 2^127 on, whose doubled scale would make 2^128 of them, stop there); a block that holds an infinity
// or a NaN has b = 255 and comes back, and goes into products, as NaN.
//
// A matrix with n rows of K summed values:
//   values  [n][ceil(K/32)][16]    two to a byte, the even index in the low half; behind the K-th value, zeros
//   scales  [ceil(K/512)][4][n][4] block 16 c + 4 s + q of row r at [c][q][r][s]; behind the last block, zeros
// The scaled matrix instruction v_mfma_scale_f32_16x16x128_f8f6f4 takes 32 values of one row from each lane, lane l those of block l / 16 of four,
// and their scale from a byte of a register.  16 bytes of a row are a lane's operand as they lie, and a dword of the scales is that lane's
// bytes for four instructions in a row, next to the neighbouring rows' for the neighbouring lanes.
#pragma once

#include "common.h"

namespace moe {

constexpr int MX4_BLOCK = 32, MX4_CHUNK = 512;     // values of a block, of the blocks whose scales lie together
inline int64_t mx4_blocks(int64_t K) { return (K + MX4_BLOCK - 1) / MX4_BLOCK; }
inline int64_t mx4_chunks(int64_t K) { return (K + MX4_CHUNK - 1) / MX4_CHUNK; }
inline size_t mx4_value_bytes(int64_t n, int64_t K) { return (size_t)n * mx4_blocks(K) * 16; }
inline size_t mx4_scale_bytes(int64_t n, int64_t K) { return (size_t)n * mx4_chunks(K) * 16; }

// scale byte of a block; top: the bits of its largest magnitude.  The carry out of the mantissa is the doubled scale: a / scale >= 7.
__device__ __forceinline__ int mx4_scale(uint32_t top) {
  return top >= 0x7F800000u ? 255 : min(max((int)((top + 0x200000u) >> 23) - 2, 0), 252);
}
// 8 values -> their codes in one register; the converter rounds to the nearest code, ties to the even one, and stops at 6
__device__ __forceinline__ uint32_t mx4_pack(const float (&v)[8], int b) {
  float t[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) t[e] = __builtin_amdgcn_ldexpf(v[e], 127 - b);
  uint32_t q = 0;
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, t[0], t[1], 1.0f, 0);
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, t[2], t[3], 1.0f, 1);
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, t[4], t[5], 1.0f, 2);
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, t[6], t[7], 1.0f, 3);
  return b == 255 ? 0u : q;
}
// 4 values -> 16 bits
__device__ __forceinline__ uint32_t mx4_pack4(const float (&v)[4], int b) {
  uint32_t q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, __builtin_amdgcn_ldexpf(v[0], 127 - b), __builtin_amdgcn_ldexpf(v[1], 127 - b), 1.0f, 0);
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, __builtin_amdgcn_ldexpf(v[2], 127 - b), __builtin_amdgcn_ldexpf(v[3], 127 - b), 1.0f, 1);
  return b == 255 ? 0u : q & 0xFFFFu;
}
__device__ __forceinline__ void mx4_values(uint32_t q, int b, float (&v)[8]) {
  typedef float f32x2_t __attribute__((ext_vector_type(2)));
  const f32x2_t t[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 1),
                        __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 3)};
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = b == 255 ? __uint_as_float(0x7FC00000u) : __builtin_amdgcn_ldexpf(t[e / 2][e % 2], b - 127);
}

// rows [rows, cols] of `dtype` to 4 bits along their columns (mx4.hip); G of them one after the other
void mx4_store_rows(const void* x, int dtype, int64_t G, int64_t rows, int cols, void* q, void* scales, hipStream_t st);

}  // namespace moe
