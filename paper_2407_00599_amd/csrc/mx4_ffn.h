// What the products from microscaled 4-bit values share (mx4_few.hip: few rows; mx4_ffn.hip: the rest).
#pragma once

#include "mx4.h"
#include "ragged_tile.h"

namespace moe {

enum { MX4_STORE = 0, MX4_GLU = 1 };      // Y; act(g) u, brought to 4 bits

// Y [R, n] = X W of each row's expert, X [rows, K] (through a row map) and W [E, n, K] in 4 bits; or, of a gated first product, n = 2 half and 4 bits
// of act(g) u [R, half].
struct Mx4Args {
  const uint8_t* xq;
  const uint8_t* xs;
  const uint8_t* wq;
  const uint8_t* ws;
  const int32_t* off;              // [E + 1]
  const int32_t* gather;           // entries of the row map, or NULL: the rows as they lie
  int gather_k;
  uint32_t gather_magic;
  int64_t gather_rows;
  int R, E, n, K, blocks, chunks;  // blocks of 32 and chunks of 512 in K
  int64_t x_rows;                  // rows of X
  void* C;                         // Y, leading dimension n
  int f32;                         // Y (of a first product: the activations) in fp32, otherwise bf16
  int half, act;                   // gated first product: hidden columns
  uint8_t* aq;                     // its 4-bit results, of R rows
  uint8_t* as;
  int a_blocks;
  int tiles_n;
};

__device__ __forceinline__ int offset(const Mx4Args& p, int e) { return min(max(p.off[e], 0), p.R); }
__device__ __forceinline__ int token(const Mx4Args& p, int iv) {
  const uint32_t tok = p.gather_k == 1 ? (uint32_t)iv : __umulhi((uint32_t)iv, p.gather_magic);
  return iv >= 0 && (int64_t)tok < p.gather_rows ? (int)tok : -1;
}

// act(g) u on its way to 4 bits.  With fp32 activations in 64 bits, because a value next to the border between two codes decides which one is kept, and
// handed on rounded to odd: towards zero, with the last bit set where that was not exact, which any rounding to fewer bits decides as for the value
// itself.  With bf16 ones in fp32, SiLU by the exponential and the reciprocal of the hardware.
__device__ __forceinline__ float round_to_odd(double d) {
  const float f = (float)d;
  const uint32_t bits = __float_as_uint(f);
  return (double)f == d || d != d ? f : __uint_as_float((fabs((double)f) > fabs(d) ? bits - 1u : bits) | 1u);
}
template <int ACT, bool WIDE>
__device__ __forceinline__ float mx4_hidden(float g, float u) {
  if constexpr (WIDE) {
    const double z = (double)g;
    const double a = ACT == MOE_ACT_SILU ? z / (1.0 + exp(-z)) : 0.5 * z * erfc(z * -0.70710678118654752440);
    return round_to_odd(a * (double)u);
  }
  return gate_value<ACT, ACT == MOE_ACT_SILU>(g) * u;
}
// f(integral_constant<int, ACT>, bool_constant<WIDE>)
template <typename F>
__device__ __forceinline__ void with_hidden(int act, int wide, F&& f) {
  with_act(act, [&](auto a) {
    if (wide) f(a, std::true_type{});
    else f(a, std::false_type{});
  });
}

// 16 bytes at off + at, `at` the same in all lanes; OOB: zeros (the range is checked without `at`, against a range that is shorter by it)
__device__ __forceinline__ uint4 mx4_load16(__amdgpu_buffer_rsrc_t r, uint32_t off, int at) {
  const u32x4_t v = __builtin_amdgcn_raw_buffer_load_b128(r, (int)off, at, 0);
  return make_uint4(v.x, v.y, v.z, v.w);
}

typedef int i32x8_t __attribute__((ext_vector_type(8)));
// d += a b for 16 x 16 values and 128 k; the scales are bytes OPA of sa and OPB of sb
template <int OPA, int OPB = OPA>
__device__ __forceinline__ f32x4_t mx4_mfma(const uint4& a, const uint4& b, const f32x4_t& d, uint32_t sa, uint32_t sb) {
  const i32x8_t x = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0}, y = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, d, 4, 4, OPA, (int)sa, OPB, (int)sb);      // 4: e2m1
}
// Of a scale dword [c][q][row] the bytes of blocks that exist; the others may hold anything, also the byte of NaN, and are multiplied with zeros.
__device__ __forceinline__ uint32_t mx4_existing(const Mx4Args& p, uint32_t four, int c, int q) {
  const int have = (p.blocks - 16 * c - q + 3) >> 2;
  return have >= 4 ? four : have <= 0 ? 0u : four & ((1u << (8 * have)) - 1u);
}

int mx4_tile(int64_t R, int E, int64_t n, int K);      // which of the kernels takes a product: 0 few rows, otherwise the tile
void launch_mx4_few(Mx4Args a, int kind, hipStream_t st);
void launch_mx4_tile(const Mx4Args& m, int kind, int tile, hipStream_t st);      // tiles of 256 x 256 or 128 x 128

}  // namespace moe
