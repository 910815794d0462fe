// Activation checkpoints in 8 bits: a tensor to its 8-bit form (ckpt8.h) and back.
//
// Bound by memory: 2 (4) + 1 + 1/32 bytes a value in bf16 (fp32), each direction.  A lane takes 8 columns (16 bytes in bf16), so four
// neighbouring lanes hold a block and its largest magnitude takes two exchanges inside the quad.
#include <algorithm>

#include "ckpt8.h"

namespace moe {

constexpr int CKPT_THREADS = 256, CKPT_UNITS = 4;   // 8-column units of a thread, a workgroup's width apart: all requested before the first is used

struct CkptPlace {      // unit u of a tensor with `per_row` units a row (a multiple of 4: the last block of a row may be short)
  uint32_t row, col;
  bool ok;
};
template <bool WHOLE>   // WHOLE: cols is a multiple of 32, rows follow each other without a gap in the units
__device__ __forceinline__ CkptPlace ckpt_place(uint32_t u, uint32_t units, uint32_t per_row, int cols) {
  if (WHOLE) return CkptPlace{0u, u * 8u, u < units};
  const uint32_t row = u / per_row, col = (u - row * per_row) * 8u;
  return CkptPlace{row, col, u < units && col < (uint32_t)cols};
}

template <typename T>
struct Eight;
template <>
struct Eight<bf16_t> {
  uint4 v;
  __device__ __forceinline__ void load(const bf16_t* p) { v = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void none() { v = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ void get(float (&f)[8]) const { unpack_bf16x8(v, f); }
  static __device__ __forceinline__ void store(bf16_t* p, const float (&f)[8]) { *reinterpret_cast<uint4*>(p) = pack_bf16x8(f); }
};
template <>
struct Eight<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = *reinterpret_cast<const float4*>(p);
    b = *reinterpret_cast<const float4*>(p + 4);
  }
  __device__ __forceinline__ void none() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
  static __device__ __forceinline__ void store(float* p, const float (&f)[8]) {
    *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(f[4], f[5], f[6], f[7]);
  }
};

template <typename T, bool WHOLE>
__global__ __launch_bounds__(CKPT_THREADS) void ckpt8_store(const T* __restrict__ x, uint32_t units, uint32_t per_row, int cols,
                                                            uint8_t* __restrict__ q, uint8_t* __restrict__ s) {
  const uint32_t u0 = blockIdx.x * (CKPT_THREADS * CKPT_UNITS) + threadIdx.x;
  Eight<T> in[CKPT_UNITS];
  CkptPlace at[CKPT_UNITS];
#pragma unroll
  for (int n = 0; n < CKPT_UNITS; ++n) {
    at[n] = ckpt_place<WHOLE>(u0 + n * CKPT_THREADS, units, per_row, cols);
    if (at[n].ok) in[n].load(x + (int64_t)at[n].row * cols + at[n].col);
    else in[n].none();
  }
#pragma unroll
  for (int n = 0; n < CKPT_UNITS; ++n) {
    float v[8];
    in[n].get(v);
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[e]) & 0x7FFFFFFFu);
    top = max(top, (uint32_t)__shfl_xor((int)top, 1, 64));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2, 64));
    const int b = ckpt8_scale(top);
    if (!at[n].ok) continue;
    const float lo[4] = {v[0], v[1], v[2], v[3]}, hi[4] = {v[4], v[5], v[6], v[7]};
    *reinterpret_cast<uint2*>(q + (int64_t)at[n].row * cols + at[n].col) = make_uint2(ckpt8_pack(lo, b), ckpt8_pack(hi, b));
    const uint32_t u = u0 + n * CKPT_THREADS;
    if ((u & 3u) == 0) s[u >> 2] = (uint8_t)b;
  }
}

template <typename T, bool WHOLE>
__global__ __launch_bounds__(CKPT_THREADS) void ckpt8_load(const uint8_t* __restrict__ q, const uint8_t* __restrict__ s, uint32_t units,
                                                           uint32_t per_row, int cols, T* __restrict__ x) {
  const uint32_t u0 = blockIdx.x * (CKPT_THREADS * CKPT_UNITS) + threadIdx.x;
  uint2 in[CKPT_UNITS];
  int b[CKPT_UNITS];
  CkptPlace at[CKPT_UNITS];
#pragma unroll
  for (int n = 0; n < CKPT_UNITS; ++n) {
    const uint32_t u = u0 + n * CKPT_THREADS;
    at[n] = ckpt_place<WHOLE>(u, units, per_row, cols);
    if (!at[n].ok) continue;
    in[n] = *reinterpret_cast<const uint2*>(q + (int64_t)at[n].row * cols + at[n].col);
    b[n] = s[u >> 2];
  }
#pragma unroll
  for (int n = 0; n < CKPT_UNITS; ++n) {
    if (!at[n].ok) continue;
    float v[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = ckpt8_value(in[n].x, e, b[n]);
      v[4 + e] = ckpt8_value(in[n].y, e, b[n]);
    }
    Eight<T>::store(x + (int64_t)at[n].row * cols + at[n].col, v);
  }
}

namespace {

int check_ckpt(int dtype, int64_t rows, int cols) {
  MOE_REQUIRE(dtype == MOE_F32 || dtype == MOE_BF16, MOE_EINVAL);
  MOE_REQUIRE(rows >= 1 && cols >= 1, MOE_EINVAL);
  MOE_REQUIRE(cols % 8 == 0, MOE_EUNSUPPORTED);
  return MOE_OK;
}

// Launches over runs of rows whose units and columns 32 bits count; launch(first row, rows, units, units a row).
template <typename F>
void over_rows(int64_t rows, int cols, F&& launch) {
  const int64_t per_row = (int64_t)(cols + CKPT8_BLOCK - 1) / CKPT8_BLOCK * 4, most = std::max<int64_t>((1ll << 28) / per_row, 1);
  for (int64_t r = 0; r < rows; r += most) {
    const int64_t n = std::min(most, rows - r), units = n * per_row;
    launch(r, (uint32_t)units, (uint32_t)per_row,
           dim3((unsigned)((units + CKPT_THREADS * CKPT_UNITS - 1) / (CKPT_THREADS * CKPT_UNITS))));
  }
}

template <typename T>
void store_as(const void* x, int64_t rows, int cols, void* q, void* s, hipStream_t st) {
  over_rows(rows, cols, [&](int64_t r, uint32_t units, uint32_t per_row, dim3 grid) {
    const T* xr = (const T*)x + r * cols;
    uint8_t *qr = (uint8_t*)q + r * cols, *sr = (uint8_t*)s + r * (per_row / 4);
    if (cols % CKPT8_BLOCK == 0) hipLaunchKernelGGL((ckpt8_store<T, true>), grid, dim3(CKPT_THREADS), 0, st, xr, units, per_row, cols, qr, sr);
    else hipLaunchKernelGGL((ckpt8_store<T, false>), grid, dim3(CKPT_THREADS), 0, st, xr, units, per_row, cols, qr, sr);
  });
}
template <typename T>
void load_as(const void* q, const void* s, int64_t rows, int cols, void* x, hipStream_t st) {
  over_rows(rows, cols, [&](int64_t r, uint32_t units, uint32_t per_row, dim3 grid) {
    T* xr = (T*)x + r * cols;
    const uint8_t *qr = (const uint8_t*)q + r * cols, *sr = (const uint8_t*)s + r * (per_row / 4);
    if (cols % CKPT8_BLOCK == 0) hipLaunchKernelGGL((ckpt8_load<T, true>), grid, dim3(CKPT_THREADS), 0, st, qr, sr, units, per_row, cols, xr);
    else hipLaunchKernelGGL((ckpt8_load<T, false>), grid, dim3(CKPT_THREADS), 0, st, qr, sr, units, per_row, cols, xr);
  });
}

}  // namespace
}  // namespace moe

using namespace moe;

extern "C" int moe_ckpt8_store(const void* x, int dtype, int64_t rows, int cols, void* q, void* scales, void* stream) {
  if (int rc = check_ckpt(dtype, rows, cols)) return rc;
  MOE_REQUIRE_PTR(x); MOE_REQUIRE_PTR(q); MOE_REQUIRE_PTR(scales);
  if (dtype == MOE_BF16) store_as<bf16_t>(x, rows, cols, q, scales, (hipStream_t)stream);
  else store_as<float>(x, rows, cols, q, scales, (hipStream_t)stream);
  return check_launch();
}

extern "C" int moe_ckpt8_load(const void* q, const void* scales, int64_t rows, int cols, void* x, int dtype, void* stream) {
  if (int rc = check_ckpt(dtype, rows, cols)) return rc;
  MOE_REQUIRE_PTR(q); MOE_REQUIRE_PTR(scales); MOE_REQUIRE_PTR(x);
  if (dtype == MOE_BF16) load_as<bf16_t>(q, scales, rows, cols, x, (hipStream_t)stream);
  else load_as<float>(q, scales, rows, cols, x, (hipStream_t)stream);
  return check_launch();
}
