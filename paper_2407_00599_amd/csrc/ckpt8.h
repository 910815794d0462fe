// 8-bit form of an activation tensor: a row is cut into blocks of 32 columns; with the largest magnitude a of a block in
// [2^x, 2^(x+1)) its step is 2^(x - 6), or 2^(x - 5) where a / step would round to 128, and a value is kept as the whole number
// nearest to value / step (ties to even), within +-127: off by at most half a step.
// The scale byte is b = x + 127 (+ 1 for the doubled step), so the step is 2^(b - 133).  A power of two makes both directions exact
// but for the one rounding, and needs neither a divide nor a table.
// Edges: the smallest step is 2^-133, and 2^-132 takes over at 127 of them (subnormals have no binade); a step that would need
// b = 255 stays 2^121 and the values saturate at 127 steps; a block that holds an infinity or a NaN has b = 255 and comes back as NaN.
#pragma once

#include "common.h"

namespace moe {

constexpr int CKPT8_BLOCK = 32;

// scale byte of a block; top: the bits of its largest magnitude.  The carry out of the mantissa is the doubled step: a / step >= 127.5.
__device__ __forceinline__ int ckpt8_scale(uint32_t top) {
  return top >= 0x7F800000u ? 255 : (int)min((top + 0x10000u) >> 23, 254u);
}
// four values -> four bytes.  x + 1.5 * 2^23 has the whole number nearest to x in its low bits.
__device__ __forceinline__ uint32_t ckpt8_join(const uint32_t (&t)[4]) {
  return __builtin_amdgcn_perm(t[1], t[0], 0x0c0c0400u) | __builtin_amdgcn_perm(t[3], t[2], 0x04000c0cu);
}
__device__ __forceinline__ uint32_t ckpt8_pack(const float (&v)[4], int b) {
  uint32_t t[4];
#pragma unroll
  for (int e = 0; e < 4; ++e)
    t[e] = __float_as_uint(__builtin_amdgcn_fmed3f(__builtin_amdgcn_ldexpf(v[e], 133 - b), -127.f, 127.f) + 12582912.f);
  return ckpt8_join(t);
}
__device__ __forceinline__ uint32_t ckpt8_pack(const double (&v)[4], int b) {
  uint32_t t[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) t[e] = (uint32_t)(int)rint(fmin(fmax(ldexp(v[e], 133 - b), -127.0), 127.0));
  return ckpt8_join(t);
}
// value of byte e of q
__device__ __forceinline__ float ckpt8_value(uint32_t q, int e, int b) {
  const float v = __builtin_amdgcn_ldexpf((float)((int32_t)(q << (24 - 8 * e)) >> 24), b - 133);
  return b == 255 ? __uint_as_float(0x7FC00000u) : v;
}

}  // namespace moe
