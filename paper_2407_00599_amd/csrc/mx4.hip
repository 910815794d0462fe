// A tensor to microscaled 4-bit floating point (mx4.h) and back, with the blocks along its rows or along its columns.
//
// Bound by memory: 2 (4) + 17/32 bytes a value in bf16 (fp32), each direction.  Along columns, bf16, 8 x 4096 x 28672 508 us to 4 bits (4.7 TB/s) and
// 447 back (5.3); along rows, bf16, 16384 x 4096 44 us (3.9 TB/s), fp32 of 1003 x 1544 4.2 and 4.5, the latency of one read and one write.
//   along rows      a lane takes 8 columns, four neighbouring lanes hold a block, and 64 lanes hold the 512 columns whose scales lie together: the
//                   four bytes of a dword meet by two exchanges.
//   along columns   (a weight [K, N] is summed over K)  a lane takes two columns and reads their 32 values of a block from 32 rows, a
//                   wave 256 (512) bytes of each; nothing is exchanged.  The four waves of a workgroup take a quarter of a chunk each; the chunk's
//                   256 bytes of each column meet in LDS and are written (read) as whole lines, and so are its scales.
#include <algorithm>

#include "mx4.h"

namespace moe {

constexpr int MX4_THREADS = 256, MX4_WAVES = MX4_THREADS / 64;

template <typename T> struct Values;       // 8 or 2 neighbouring values
template <> struct Values<bf16_t> {
  static __device__ __forceinline__ void load8(const bf16_t* p, float (&f)[8]) { unpack_bf16x8(*reinterpret_cast<const uint4*>(p), f); }
  static __device__ __forceinline__ void store8(bf16_t* p, const float (&f)[8]) { *reinterpret_cast<uint4*>(p) = pack_bf16x8(f); }
  typedef uint32_t Two;
  static __device__ __forceinline__ float2 get(Two t) { return make_float2(__uint_as_float(t << 16), __uint_as_float(t & 0xFFFF0000u)); }
  static __device__ __forceinline__ Two put(float a, float b) { return pack_bf16x2(a, b); }
};
template <> struct Values<float> {
  static __device__ __forceinline__ void load8(const float* p, float (&f)[8]) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
  static __device__ __forceinline__ void store8(float* p, const float (&f)[8]) {
    *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(f[4], f[5], f[6], f[7]);
  }
  typedef float2 Two;
  static __device__ __forceinline__ float2 get(Two t) { return t; }
  static __device__ __forceinline__ Two put(float a, float b) { return make_float2(a, b); }
};

struct Mx4Shape {
  int64_t n;             // rows of 4-bit values: of one matrix, summed over K
  int K, blocks, chunks;
};

// ---- blocks along rows ----
// LPR lanes to a row: 64, or as many as few columns need.  A workgroup takes consecutive rows of one chunk, so that their scales are whole lines.
constexpr int ROW_PASSES = 4;
template <typename T, int LPR>
__global__ __launch_bounds__(MX4_THREADS) void mx4_rows_store(const T* __restrict__ x, const Mx4Shape sh, int64_t groups, uint8_t* __restrict__ q,
                                                              uint32_t* __restrict__ s) {
  constexpr int RPW = 64 / LPR, ROWS = MX4_WAVES * RPW;      // rows of a wave, of a workgroup's pass
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane % LPR;
  const int64_t unit = blockIdx.x, g = unit / (groups * sh.chunks), rest = unit - g * groups * sh.chunks;
  const int c = (int)(rest / groups);
  const int64_t r0 = (rest - c * groups) * (ROWS * ROW_PASSES) + wave * RPW + lane / LPR;
  const int col = c * MX4_CHUNK + 8 * l;
  float v[ROW_PASSES][8];
#pragma unroll
  for (int p = 0; p < ROW_PASSES; ++p) {
    const int64_t row = r0 + p * ROWS;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[p][e] = 0.f;
    if (row < sh.n && col < sh.K) Values<T>::load8(x + (g * sh.n + row) * sh.K + col, v[p]);
  }
#pragma unroll
  for (int p = 0; p < ROW_PASSES; ++p) {
    const int64_t row = r0 + p * ROWS;
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[p][e]) & 0x7FFFFFFFu);
    top = max(top, (uint32_t)__shfl_xor((int)top, 1, 64));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2, 64));
    const int b = mx4_scale(top);
    uint32_t four = (uint32_t)b << (8 * (l / 16));           // block 4 s + q of the chunk, s = l / 16
    if (LPR >= 32) four |= (uint32_t)__shfl_xor((int)four, 16, 64);
    if (LPR >= 64) four |= (uint32_t)__shfl_xor((int)four, 32, 64);
    if (row >= sh.n) continue;
    const int block = c * 16 + l / 4;
    if (block < sh.blocks) *reinterpret_cast<uint32_t*>(q + ((g * sh.n + row) * sh.blocks + block) * 16 + (l & 3) * 4) = mx4_pack(v[p], b);
    if (l < 16 && (l & 3) == 0) s[((g * sh.chunks + c) * 4 + l / 4) * sh.n + row] = four;
  }
}

template <typename T, int LPR>
__global__ __launch_bounds__(MX4_THREADS) void mx4_rows_load(const uint8_t* __restrict__ q, const uint8_t* __restrict__ s, const Mx4Shape sh,
                                                             int64_t groups, T* __restrict__ x) {
  constexpr int RPW = 64 / LPR, ROWS = MX4_WAVES * RPW;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane % LPR;
  const int64_t unit = blockIdx.x, g = unit / (groups * sh.chunks), rest = unit - g * groups * sh.chunks;
  const int c = (int)(rest / groups);
  const int64_t r0 = (rest - c * groups) * (ROWS * ROW_PASSES) + wave * RPW + lane / LPR;
  const int col = c * MX4_CHUNK + 8 * l;
  uint32_t codes[ROW_PASSES];
  int b[ROW_PASSES];
#pragma unroll
  for (int p = 0; p < ROW_PASSES; ++p) {
    const int64_t row = r0 + p * ROWS;
    codes[p] = 0;
    b[p] = 0;
    if (row < sh.n && col < sh.K) {
      codes[p] = *reinterpret_cast<const uint32_t*>(q + ((g * sh.n + row) * sh.blocks + c * 16 + l / 4) * 16 + (l & 3) * 4);
      b[p] = s[(((g * sh.chunks + c) * 4 + l / 4 % 4) * sh.n + row) * 4 + l / 16];
    }
  }
#pragma unroll
  for (int p = 0; p < ROW_PASSES; ++p) {
    const int64_t row = r0 + p * ROWS;
    if (row >= sh.n || col >= sh.K) continue;
    float v[8];
    mx4_values(codes[p], b[p], v);
    Values<T>::store8(x + (g * sh.n + row) * sh.K + col, v);
  }
}

// ---- blocks along columns: n columns, K rows ----
constexpr int COLS = 128;      // columns of a workgroup
constexpr int COL_PITCH = MX4_CHUNK / 2 + 16;      // bytes of a column's chunk in LDS
template <typename T>
__global__ __launch_bounds__(MX4_THREADS) void mx4_cols_store(const T* __restrict__ x, const Mx4Shape sh, int64_t groups, uint8_t* __restrict__ q,
                                                              uint32_t* __restrict__ s) {
  using Two = typename Values<T>::Two;
  __shared__ __attribute__((aligned(16))) uint8_t codes[COLS * COL_PITCH];
  __shared__ __attribute__((aligned(4))) uint8_t bytes[4][COLS][4];      // [q][column][s]
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t unit = blockIdx.x, g = unit / (groups * sh.chunks), rest = unit - g * groups * sh.chunks;
  const int c = (int)(rest / groups);
  const int64_t c0 = (rest - c * groups) * COLS, col = c0 + 2 * lane;
  const T* from = x + g * sh.n * sh.K + (col < sh.n ? col : 0);
  Two in[2][MX4_BLOCK];
  auto fetch = [&](int i, Two (&d)[MX4_BLOCK]) {      // rows behind the last one: that one, zeroed below
    const int k0 = (c * 16 + 4 * wave + i) * MX4_BLOCK;
#pragma unroll
    for (int k = 0; k < MX4_BLOCK; ++k) d[k] = *reinterpret_cast<const Two*>(from + (int64_t)min(k0 + k, sh.K - 1) * sh.n);
  };
  fetch(0, in[0]);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (i < 3) fetch(i + 1, in[(i + 1) & 1]);
    const int left = sh.K - (c * 16 + 4 * wave + i) * MX4_BLOCK;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float v[MX4_BLOCK];
      uint32_t top = 0;
#pragma unroll
      for (int k = 0; k < MX4_BLOCK; ++k) {
        const float2 f = Values<T>::get(in[i & 1][k]);
        v[k] = k < left ? (h ? f.y : f.x) : 0.f;
        top = max(top, __float_as_uint(v[k]) & 0x7FFFFFFFu);
      }
      const int b = left > 0 ? mx4_scale(top) : 0;
      uint32_t w[4];
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        float t[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = v[8 * d + e];
        w[d] = mx4_pack(t, b);
      }
      *reinterpret_cast<uint4*>(codes + (2 * lane + h) * COL_PITCH + (4 * wave + i) * 16) = make_uint4(w[0], w[1], w[2], w[3]);
      bytes[i][2 * lane + h][wave] = (uint8_t)b;
    }
  }
  __syncthreads();
  const int blocks = min(16, sh.blocks - c * 16);     // of this chunk
#pragma unroll
  for (int u = tid; u < COLS * 16; u += MX4_THREADS) {
    const int k = u / 16, block = u % 16;
    if (c0 + k < sh.n && block < blocks)
      *reinterpret_cast<uint4*>(q + ((g * sh.n + c0 + k) * sh.blocks + c * 16 + block) * 16) = *reinterpret_cast<const uint4*>(codes + k * COL_PITCH + block * 16);
  }
#pragma unroll
  for (int u = tid; u < 4 * COLS; u += MX4_THREADS) {
    const int i = u / COLS, k = u % COLS;
    if (c0 + k < sh.n) s[((g * sh.chunks + c) * 4 + i) * sh.n + c0 + k] = *reinterpret_cast<const uint32_t*>(bytes[i][k]);
  }
}

template <typename T>
__global__ __launch_bounds__(MX4_THREADS) void mx4_cols_load(const uint8_t* __restrict__ q, const uint32_t* __restrict__ s, const Mx4Shape sh,
                                                             int64_t groups, T* __restrict__ x) {
  using Two = typename Values<T>::Two;
  __shared__ __attribute__((aligned(16))) uint8_t codes[COLS * COL_PITCH];
  __shared__ __attribute__((aligned(4))) uint8_t bytes[4][COLS][4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t unit = blockIdx.x, g = unit / (groups * sh.chunks), rest = unit - g * groups * sh.chunks;
  const int c = (int)(rest / groups);
  const int64_t c0 = (rest - c * groups) * COLS, col = c0 + 2 * lane;
  const int blocks = min(16, sh.blocks - c * 16);
  uint4 in[COLS * 16 / MX4_THREADS];
#pragma unroll
  for (int r = 0; r < COLS * 16 / MX4_THREADS; ++r) {
    const int u = tid + r * MX4_THREADS, k = u / 16, block = u % 16;
    in[r] = make_uint4(0, 0, 0, 0);
    if (c0 + k < sh.n && block < blocks) in[r] = *reinterpret_cast<const uint4*>(q + ((g * sh.n + c0 + k) * sh.blocks + c * 16 + block) * 16);
  }
#pragma unroll
  for (int u = tid; u < 4 * COLS; u += MX4_THREADS) {
    const int i = u / COLS, k = u % COLS;
    if (c0 + k < sh.n) *reinterpret_cast<uint32_t*>(bytes[i][k]) = s[((g * sh.chunks + c) * 4 + i) * sh.n + c0 + k];
  }
#pragma unroll
  for (int r = 0; r < COLS * 16 / MX4_THREADS; ++r) {
    const int u = tid + r * MX4_THREADS;
    *reinterpret_cast<uint4*>(codes + u / 16 * COL_PITCH + u % 16 * 16) = in[r];
  }
  __syncthreads();
  if (col >= sh.n) return;
  T* to = x + g * sh.n * sh.K + col;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int block = 4 * wave + i, k0 = (c * 16 + block) * MX4_BLOCK, left = sh.K - k0;
    if (left <= 0) break;
    const uint4 a = *reinterpret_cast<const uint4*>(codes + 2 * lane * COL_PITCH + block * 16);
    const uint4 d = *reinterpret_cast<const uint4*>(codes + (2 * lane + 1) * COL_PITCH + block * 16);
    const int ba = bytes[i][2 * lane][wave], bd = bytes[i][2 * lane + 1][wave];
    const uint32_t wa[4] = {a.x, a.y, a.z, a.w}, wd[4] = {d.x, d.y, d.z, d.w};
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      float va[8], vd[8];
      mx4_values(wa[p], ba, va);
      mx4_values(wd[p], bd, vd);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (8 * p + e < left) *reinterpret_cast<Two*>(to + (int64_t)(k0 + 8 * p + e) * sh.n) = Values<T>::put(va[e], vd[e]);
    }
  }
}

namespace {

Mx4Shape shape_of(int64_t n, int K) { return Mx4Shape{n, K, (int)mx4_blocks(K), (int)mx4_chunks(K)}; }
constexpr int rows_of_group(int lpr) { return MX4_WAVES * (64 / lpr) * ROW_PASSES; }
template <typename F>
void with_lanes(int K, F&& f) {
  if (K <= 128) f(std::integral_constant<int, 16>{});
  else if (K <= 256) f(std::integral_constant<int, 32>{});
  else f(std::integral_constant<int, 64>{});
}
double grid_of(int64_t G, int64_t n, int K, int transposed) {      // workgroups of a call (sizes that do not exist would overflow 64 bits)
  int64_t groups = (n + COLS - 1) / COLS;
  if (!transposed) with_lanes(K, [&](auto lanes) { groups = (n + rows_of_group(decltype(lanes)::value) - 1) / rows_of_group(decltype(lanes)::value); });
  return (double)G * (double)mx4_chunks(K) * (double)groups;
}

template <typename T>
void load_rows(const void* q, const void* s, int64_t G, int64_t rows, int cols, void* x, hipStream_t st) {
  const Mx4Shape sh = shape_of(rows, cols);
  with_lanes(cols, [&](auto lanes) {
    constexpr int LPR = decltype(lanes)::value;
    const int64_t groups = (rows + rows_of_group(LPR) - 1) / rows_of_group(LPR);
    hipLaunchKernelGGL((mx4_rows_load<T, LPR>), dim3((unsigned)(G * sh.chunks * groups)), dim3(MX4_THREADS), 0, st, (const uint8_t*)q, (const uint8_t*)s,
                       sh, groups, (T*)x);
  });
}
template <typename T>
void store_rows(const void* x, int64_t G, int64_t rows, int cols, void* q, void* s, hipStream_t st) {
  const Mx4Shape sh = shape_of(rows, cols);
  with_lanes(cols, [&](auto lanes) {
    constexpr int LPR = decltype(lanes)::value;
    const int64_t groups = (rows + rows_of_group(LPR) - 1) / rows_of_group(LPR);
    hipLaunchKernelGGL((mx4_rows_store<T, LPR>), dim3((unsigned)(G * sh.chunks * groups)), dim3(MX4_THREADS), 0, st, (const T*)x, sh, groups, (uint8_t*)q,
                       (uint32_t*)s);
  });
}
template <typename T>
void store_cols(const void* x, int64_t G, int rows, int64_t cols, void* q, void* s, hipStream_t st) {
  const Mx4Shape sh = shape_of(cols, rows);
  const int64_t groups = (cols + COLS - 1) / COLS;
  hipLaunchKernelGGL((mx4_cols_store<T>), dim3((unsigned)(G * sh.chunks * groups)), dim3(MX4_THREADS), 0, st, (const T*)x, sh, groups, (uint8_t*)q, (uint32_t*)s);
}
template <typename T>
void load_cols(const void* q, const void* s, int64_t G, int rows, int64_t cols, void* x, hipStream_t st) {
  const Mx4Shape sh = shape_of(cols, rows);
  const int64_t groups = (cols + COLS - 1) / COLS;
  hipLaunchKernelGGL((mx4_cols_load<T>), dim3((unsigned)(G * sh.chunks * groups)), dim3(MX4_THREADS), 0, st, (const uint8_t*)q, (const uint32_t*)s, sh, groups,
                     (T*)x);
}

int check_mx4(int dtype, int64_t G, int64_t rows, int cols, int transposed) {
  MOE_REQUIRE(dtype == MOE_F32 || dtype == MOE_BF16, MOE_EINVAL);
  MOE_REQUIRE(G >= 1 && rows >= 1 && cols >= 1 && (transposed == 0 || transposed == 1), MOE_EINVAL);
  MOE_REQUIRE(cols % 8 == 0 && (!transposed || rows % 8 == 0), MOE_EUNSUPPORTED);
  MOE_REQUIRE(G <= 1 << 20 && rows <= 1ll << 31 && (!transposed || rows < 1ll << 31), MOE_EUNSUPPORTED);
  // a launch has fewer than 2^32 threads
  MOE_REQUIRE((transposed ? grid_of(G, cols, (int)rows, 1) : grid_of(G, rows, cols, 0)) * MX4_THREADS < 4294967296.0, MOE_EUNSUPPORTED);
  return MOE_OK;
}

}  // namespace

void mx4_store_rows(const void* x, int dtype, int64_t G, int64_t rows, int cols, void* q, void* scales, hipStream_t st) {
  if (dtype == MOE_BF16) store_rows<bf16_t>(x, G, rows, cols, q, scales, st);
  else store_rows<float>(x, G, rows, cols, q, scales, st);
}

}  // namespace moe

using namespace moe;

extern "C" int moe_mx4_store(const void* x, int dtype, int64_t G, int64_t rows, int cols, int transposed, void* q, void* scales, void* stream) {
  if (int rc = check_mx4(dtype, G, rows, cols, transposed)) return rc;
  MOE_REQUIRE_PTR(x); MOE_REQUIRE_PTR(q); MOE_REQUIRE_PTR(scales);
  hipStream_t st = (hipStream_t)stream;
  if (!transposed) mx4_store_rows(x, dtype, G, rows, cols, q, scales, st);
  else if (dtype == MOE_BF16) store_cols<bf16_t>(x, G, (int)rows, cols, q, scales, st);
  else store_cols<float>(x, G, (int)rows, cols, q, scales, st);
  return check_launch();
}

extern "C" int moe_mx4_load(const void* q, const void* scales, int64_t G, int64_t rows, int cols, int transposed, void* x, int dtype, void* stream) {
  if (int rc = check_mx4(dtype, G, rows, cols, transposed)) return rc;
  MOE_REQUIRE_PTR(q); MOE_REQUIRE_PTR(scales); MOE_REQUIRE_PTR(x);
  hipStream_t st = (hipStream_t)stream;
  if (transposed) {
    if (dtype == MOE_BF16) load_cols<bf16_t>(q, scales, G, (int)rows, cols, x, st);
    else load_cols<float>(q, scales, G, (int)rows, cols, x, st);
  } else {
    if (dtype == MOE_BF16) load_rows<bf16_t>(q, scales, G, rows, cols, x, st);
    else load_rows<float>(q, scales, G, rows, cols, x, st);
  }
  return check_launch();
}
