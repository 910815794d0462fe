// What the kernels over ragged rows share: their arguments, the rows of an expert, the bf16 activation.
#pragma once

#include "ffn_tile.h"

namespace moe {

enum { EPI_ACT = 16, EPI_GELU8 = 17, EPI_DGELU8 = 18 };   // GeLU alone; GeLU and the 8-bit form; dZ and GeLU from the 8-bit form

struct RaggedArgs : GemmArgs {     // G = E experts, Cc = R = rows of the buffers, Mdim = R in row-tiled GEMMs, C2 / Zin = the 8-bit values
  const int32_t* off;              // [E + 1]
  uint8_t* Zs;                     // [R, ldz] scales of the 8-bit values
  int ldz;
  int grid;                        // workgroups of this problem (of a part, where its reduction is split)
};

struct RaggedPlace {
  int g, tm, tn;
  int lo, n;        // first row and number of rows of expert g
};

// first row of expert e, whatever the caller's offsets hold
__device__ __forceinline__ int offset(const RaggedArgs& p, int e) { return min(max(p.off[e], 0), p.R); }
// token of an entry of the row map; -1: none, a row of zeros
__device__ __forceinline__ int token(const RaggedArgs& p, int iv) {
  const uint32_t tok = p.gather_k == 1 ? (uint32_t)iv : __umulhi((uint32_t)iv, p.gather_magic);
  return iv >= 0 && (int64_t)tok < p.gather_rows ? (int)tok : -1;
}
// share `at` of `shares` of the rows behind the last expert's
template <int ESZ>
__device__ __forceinline__ void fill_behind(const RaggedArgs& p, int at, int shares) {
  const int64_t row_units = p.ldc * ESZ / 16, r0 = offset(p, p.G), units = (p.R - r0) * row_units;
  if (units <= 0 || at >= shares) return;
  const int64_t per = (units + shares - 1) / shares, u1 = min(per * (at + 1), units);
  u32x4_t* c = reinterpret_cast<u32x4_t*>(p.C) + r0 * row_units;
  const u32x4_t z = {0u, 0u, 0u, 0u};
  for (int64_t u = per * at + threadIdx.x; u < u1; u += blockDim.x) __builtin_nontemporal_store(z, c + u);
}

// Tiles of a row-tiled GEMM in linear order expert by expert, each with ceil(n / TM) row tiles; XCDs and patches as in the padded
// calls.  The grid is made for the most tiles that R rows can have, and the workgroups behind the last tile store the rows
// behind offsets[E] as zeros, an equal share each.
template <int KIND, int EPI, int ESZ, int TM, int TN>
__device__ __forceinline__ bool find_tile(const RaggedArgs& p, int vb, RaggedPlace& at) {
  const int x = vb & 7, i = vb >> 3, lane = threadIdx.x & 63;
  if (KIND == KIND_TN) {
    const int per_xcd = (p.total_tiles + 7) / 8, tile = xcd_tile(p, x, i, per_xcd), per_g = p.tiles_m * p.tiles_n;
    if (i >= per_xcd || tile >= p.total_tiles) return false;
    at.g = tile / per_g;
    patch_order(tile - at.g * per_g, p.tiles_m, p.tiles_n, at.tm, at.tn);
    at.lo = __builtin_amdgcn_readfirstlane(offset(p, at.g));
    at.n = __builtin_amdgcn_readfirstlane(max(offset(p, at.g + 1) - at.lo, 0));
    return true;
  }
  // 64 experts at a time, a lane each
  int lo = 0, n = 0, m = 0, incl = 0;
  auto scan = [&](int e0) {
    const int e = e0 + lane;
    lo = offset(p, min(e, p.G));
    n = e < p.G ? max(offset(p, min(e + 1, p.G)) - lo, 0) : 0;
    m = (n + TM - 1) / TM;
    incl = m;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int v = __shfl_up(incl, d, 64);
      if (lane >= d) incl += v;
    }
    return __builtin_amdgcn_readlane(incl, 63);
  };
  int all = 0;
  for (int e0 = 0; e0 < p.G; e0 += 64) all += scan(e0);
  const int T = all * p.tiles_n, per_t = (T + 7) / 8;
  if (i >= per_t) {
    if (EPI == EPI_STORE) fill_behind<ESZ>(p, (i - per_t) * 8 + x, p.grid - 8 * per_t);
    return false;
  }
  const int tile = xcd_tile(p, x, i, per_t);
  if (tile >= T) return false;
  int run = 0;
  for (int e0 = 0; e0 < p.G; e0 += 64) {
    if (p.G > 64) scan(e0);
    const unsigned long long hit = __ballot((run + incl) * p.tiles_n > tile);
    if (hit) {
      const int l = __ffsll((long long)hit) - 1;
      at.g = e0 + l;
      at.lo = __builtin_amdgcn_readlane(lo, l);
      at.n = __builtin_amdgcn_readlane(n, l);
      patch_order(tile - (run + __builtin_amdgcn_readlane(incl - m, l)) * p.tiles_n, __builtin_amdgcn_readlane(m, l), p.tiles_n,
                  at.tm, at.tn);
      return true;
    }
    run += __builtin_amdgcn_readlane(incl, 63);
  }
  return false;
}

// GeLU(z) = z Phi(z) and GeLU'(z) = Phi(z) + z phi(z).  Phi(z) - 1/2 is the odd minimax polynomial of fit_gelu_poly.py on |z| <= 4.25
// (absolute error 1.2e-5), clamped outside; phi is exp2 of the hardware.
__device__ constexpr float PHI_ODD[9] = {3.989023268e-01f, -6.634449214e-02f, 9.815968573e-03f, -1.108560129e-03f,
                                         9.341852274e-05f, -5.626405255e-06f, 2.255412426e-07f, -5.327701835e-09f,
                                         5.564777111e-11f};
__device__ __forceinline__ float normal_cdf(float z) {
  const float zc = __builtin_amdgcn_fmed3f(z, -4.25f, 4.25f), u = zc * zc;
  float q = fmaf(PHI_ODD[8], u, PHI_ODD[7]);
#pragma unroll
  for (int i = 6; i >= 0; --i) q = fmaf(q, u, PHI_ODD[i]);
  return __builtin_amdgcn_fmed3f(fmaf(zc, q, 0.5f), 0.0f, 1.0f);
}
__device__ __forceinline__ float gelu_fast(float z) { return z * normal_cdf(z); }
__device__ __forceinline__ void gelu_and_grad_fast(float z, float& g, float& dg) {
  const float cdf = normal_cdf(z);
  g = z * cdf;
  dg = fmaf(z * 0.39894228040143267794f, __builtin_amdgcn_exp2f(z * z * -0.72134752044448170368f), cdf);   // (1/2) log2(e)
}

// The FFN of few rows (ragged_few.hip): bf16, nothing kept for a backward pass; ws of few_rows_bytes().
size_t few_rows_bytes(int64_t R, int E, int M, int Hl);
void launch_few_rows(const RaggedArgs& first, const RaggedArgs& second, void* ws, hipStream_t st);

// fp32 products on the fp32 matrix cores (ragged_f32.hip); EPI_PART: the reduction in a.splits parts, which go to a.part
constexpr int F32_TILE = 64, KC = 32;      // tile, k chunk
template <int KIND, int EPI>
void launch_f32(RaggedArgs a, hipStream_t st);
void launch_trio_f32(RaggedArgs dx, RaggedArgs w2, RaggedArgs w1, hipStream_t st);

// ---- host side ----
// Row tiles that R rows of E experts are priced at: half a tile of each expert's last one is empty.  How the rows are spread is not
// known here.
inline double priced_row_tiles(int R, int E, int tile_m) {
  const double rows = (double)R / E;
  return E * (rows < 1.0 ? rows : std::max(1.0, rows / tile_m + 0.45));
}
// the most row tiles that R rows of E experts can have
inline int64_t most_row_tiles(int R, int E, int tile_m) {
  const int64_t used = std::min(R, E);
  return ((int64_t)R + used * (tile_m - 1)) / tile_m;
}

constexpr int ZERO_SHARES = 64;    // workgroups at least that can store rows behind the last expert's
// tile counts and grid of a row-tiled GEMM, and of a weight gradient
inline dim3 size_rows(RaggedArgs& a, int tile_m, int tile_n, bool zeros) {
  const int64_t row_tiles = most_row_tiles(a.R, a.G, tile_m);
  a.tiles_m = (int)row_tiles;
  a.tiles_n = (a.Ndim + tile_n - 1) / tile_n;
  a.total_tiles = (int)(row_tiles * a.tiles_n);
  a.grid = (a.total_tiles + 7) / 8 * 8 + (zeros ? ZERO_SHARES : 0);
  a.run_mask = ~31;
  return dim3((unsigned)a.grid);
}
inline dim3 size_weights(RaggedArgs& a, int tile) {
  a.tiles_m = (a.Mdim + tile - 1) / tile;
  a.tiles_n = (a.Ndim + tile - 1) / tile;
  a.total_tiles = a.G * a.tiles_m * a.tiles_n;
  a.run_mask = ~31;
  a.grid = (a.total_tiles + 7) / 8 * 8;
  return dim3((unsigned)a.grid);
}

}  // namespace moe
