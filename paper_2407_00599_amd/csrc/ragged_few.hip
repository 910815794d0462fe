// The expert FFN of few rows (bf16, nothing kept): a decoding step, whose time is that of reading the weights once.
//
// The tiles of ffn_tile.h bring operands through LDS in k tiles behind a barrier each, and a matrix of few columns gives them few workgroups,
// while a compute unit draws no more than some 20 GB/s from HBM: the second product of 2 rows over 2 experts x 4096 x 1024 took 15.5 us on
// 32 of them.  Here nothing is shared in the k loop.  A wave reads 32 k x 16 NCL columns of the weights straight into registers, a lane 8
// k-rows of NCL columns, so that it holds whole fragments: fragment i of v_mfma_f32_16x16x32_bf16 is column NCL (l % 16) + i, eight k of it
// in each lane, put together from pairs of k-rows by one v_perm each.  The rows of X are fragments as they lie in memory (16 bytes a lane),
// from L2, where every workgroup of an expert finds them.  The waves of a workgroup take the steps over k in turn, some requested ahead,
// and their sums meet in LDS in a fixed order.
//   first product   a workgroup for every 128 columns of every expert, or 64 where those are fewer than the compute units
//   second product  its k is long and its columns are few: cut into as many parts as the chip has room for beside the experts that have
//                   rows.  A part leaves fp32 sums in the workspace; the last one of a tile to arrive adds all of them in their order,
//                   so the result does not depend on who it is.  The first product's launch clears the tiles' counters.
// Bound by HBM with large experts, by launches and the first loads' latency with small ones.  Forward call, tiles and this: 2 rows, 8 experts x 1024
// x 4096 28.5 -> 17.6 us; 64 rows 44.0 -> 38.5; 64 rows, 8 x 4096 x 14336 375 -> 334 (5.6 TB/s).  Wide rows of weights matter more than many
// workgroups: 32, 64 and 128 columns a wave, the last of these shapes 487, 382 and 345 us.
#include "ragged.h"

namespace moe {

constexpr int few_ahead(int rg) { return rg == 1 ? 4 : rg == 2 ? 3 : 2; }     // steps requested ahead, by the registers there are
constexpr int FEW_GRID = 512;         // workgroups of the second product (1024: both products of 64 rows x 8 experts x 1024 x 4096 41.8 us, 512: 38.8)
constexpr int FEW_PART_STEPS = 8;     // steps of a part at least

template <int NCL> struct Cols;
template <> struct Cols<4> {
  u32x2_t v;
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, uint32_t off) { v = __builtin_amdgcn_raw_buffer_load_b64(r, (int)off, 0, 0); }
  __device__ __forceinline__ uint32_t pair(int i) const { return v[i]; }
};
template <> struct Cols<8> {
  u32x4_t v;
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, uint32_t off) { v = __builtin_amdgcn_raw_buffer_load_b128(r, (int)off, 0, 0); }
  __device__ __forceinline__ uint32_t pair(int i) const { return v[i]; }
};

struct FewArgs : RaggedArgs {
  float* sums;            // [parts, R, Ndim] of a split product
  int32_t* arrived;       // [G, tiles_n]
  int n_arrived, max_parts;
};

// Sums of steps s0 .. s1 - 1 for rows m0 .. m0 + 16 RG - 1 of an expert and 16 NCL columns, handed on in pairs of columns: out(row, column, two sums).
template <int NCL, int RG, int WAVES, typename F>
__device__ __forceinline__ void few_rows(const FewArgs& p, float* red, int g, int lo, int n, int m0, int n0, int s0, int s1, F&& out) {
  constexpr int TN = 16 * NCL, PITCH = TN + 4, FEW_PF = few_ahead(RG);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c16 = lane & 15, kg = lane >> 4;
  const __amdgpu_buffer_rsrc_t rX = make_rsrc(p.A, (uint32_t)p.a_bytes);
  const uint32_t ldb2 = (uint32_t)p.ldb * 2u;      // the weights' descriptor ends with the shard's last row
  const __amdgpu_buffer_rsrc_t rW = make_rsrc(reinterpret_cast<const bf16_t*>(p.B) + ((int64_t)g * p.b_goff + p.b_off),
                                              (uint32_t)(p.Kdim - 1) * ldb2 + (uint32_t)p.Ndim * 2u);
  const int col = n0 + NCL * c16;
  const uint32_t w_off = col < p.Ndim ? (uint32_t)(8 * kg) * ldb2 + (uint32_t)col * 2u : OOB;
  int entry[RG];                                  // of the row map; asked for first, waited for behind the weights' requests
  bool here[RG];
#pragma unroll
  for (int q = 0; q < RG; ++q) {
    const int r = m0 + 16 * q + c16;
    here[q] = r < n;
    entry[q] = lo + min(r, n - 1);
    if (p.gather != nullptr) entry[q] = p.gather[entry[q]];
  }
  Cols<NCL> w[FEW_PF][8];
  uint4 x[FEW_PF][RG];
  uint32_t x_off[RG];                             // byte offset of this lane's row at its first k, or OOB: zeros
  auto request_w = [&](int slot, int s) {         // past the end: zeros
    const bool in = s < s1 && 32 * s + 8 * kg < p.Kdim && w_off != OOB;     // Kdim is a multiple of 8: a lane's 8 k exist together
#pragma unroll
    for (int j = 0; j < 8; ++j) w[slot][j].load(rW, in ? w_off + (uint32_t)(32 * s + j) * ldb2 : OOB);
  };
  auto request_x = [&](int slot, int s) {
    const bool in = s < s1 && 32 * s + 8 * kg < p.Kdim;
#pragma unroll
    for (int q = 0; q < RG; ++q) x[slot][q] = ldb16(rX, in && x_off[q] != OOB ? x_off[q] + 64u * (uint32_t)s : OOB);
  };
  f32x4_t acc[RG][NCL];
#pragma unroll
  for (int q = 0; q < RG; ++q)
#pragma unroll
    for (int i = 0; i < NCL; ++i) acc[q][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int u = 0; u < FEW_PF; ++u) {
    request_w(u, s0 + wave + WAVES * u);
    __builtin_amdgcn_sched_barrier(0);            // in this order: the first step's are waited for first
  }
#pragma unroll
  for (int q = 0; q < RG; ++q) {
    int row = here[q] ? entry[q] : -1;
    if (p.gather != nullptr && here[q]) row = token(p, row);
    x_off[q] = row >= 0 ? (uint32_t)row * (uint32_t)p.lda * 2u + (uint32_t)kg * 16u : OOB;
  }
#pragma unroll
  for (int u = 0; u < FEW_PF; ++u) {
    request_x(u, s0 + wave + WAVES * u);
    __builtin_amdgcn_sched_barrier(0);
  }
  for (int s = s0 + wave; s < s1; s += WAVES * FEW_PF) {
#pragma unroll
    for (int u = 0; u < FEW_PF; ++u) {
      if (s + WAVES * u >= s1) break;             // (uniform)
      Frag fx[RG];
#pragma unroll
      for (int q = 0; q < RG; ++q) fx[q].q = u32x4_t{x[u][q].x, x[u][q].y, x[u][q].z, x[u][q].w};
#pragma unroll
      for (int i = 0; i < NCL; ++i) {
        Frag fw;
#pragma unroll
        for (int d = 0; d < 4; ++d)
          fw.q[d] = __builtin_amdgcn_perm(w[u][2 * d + 1].pair(i / 2), w[u][2 * d].pair(i / 2), (i & 1) ? 0x07060302u : 0x05040100u);
#pragma unroll
        for (int q = 0; q < RG; ++q) acc[q][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fx[q].v, fw.v, acc[q][i], 0, 0, 0);
      }
      if (s + WAVES * (u + FEW_PF) < s1) {
        request_w(u, s + WAVES * (u + FEW_PF));
        request_x(u, s + WAVES * (u + FEW_PF));
      }
    }
  }
#pragma unroll
  for (int q = 0; q < RG; ++q) {
    if (m0 + 16 * q >= n) break;                  // (uniform)
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NCL; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) red[(wave * 16 + 4 * kg + r) * PITCH + NCL * c16 + i] = acc[q][i][r];
    __syncthreads();
    for (int u = tid; u < 16 * TN / 2; u += 64 * WAVES) {
      const int row = u / (TN / 2), c = u % (TN / 2) * 2;
      float2 v = make_float2(0.f, 0.f);
#pragma unroll
      for (int t = 0; t < WAVES; ++t) {
        const float2 a = *reinterpret_cast<const float2*>(&red[(t * 16 + row) * PITCH + c]);
        v.x += a.x;
        v.y += a.y;
      }
      if (m0 + 16 * q + row < n && n0 + c < p.Ndim) out(lo + m0 + 16 * q + row, n0 + c, v);
    }
  }
}
template <int NCL, int WAVES>
constexpr int few_floats() { return WAVES * 16 * (16 * NCL + 4); }
__device__ __forceinline__ void store_pair(const FewArgs& p, int row, int col, const float2& v) {
  *reinterpret_cast<uint32_t*>(reinterpret_cast<bf16_t*>(p.C) + (int64_t)row * p.ldc + col) = pack_bf16x2(v.x, v.y);
}

// RG: groups of 16 rows that go along with one reading of the weights; an expert with more rows takes another one.
constexpr int FIRST_WAVES = 8, SECOND_WAVES = 4;
template <int NCL, int RG>
__global__ __launch_bounds__(64 * FIRST_WAVES) void ragged_few_first(const FewArgs p) {
  __shared__ float red[few_floats<NCL, FIRST_WAVES>()];
  const int cleared = (int)blockIdx.x * 64 * FIRST_WAVES + (int)threadIdx.x;
  if (cleared < p.n_arrived) p.arrived[cleared] = 0;
  const int tile = (int)blockIdx.x;
  if (tile >= p.total_tiles) return;
  const int g = tile / p.tiles_n, n0 = (tile - g * p.tiles_n) * 16 * NCL;
  const int lo = __builtin_amdgcn_readfirstlane(offset(p, g)), n = __builtin_amdgcn_readfirstlane(offset(p, g + 1)) - lo;
  for (int m0 = 0; m0 < n; m0 += 16 * RG)
    few_rows<NCL, RG, FIRST_WAVES>(p, red, g, lo, n, m0, n0, 0, (p.Kdim + 31) / 32, [&](int row, int col, const float2& v) {
      store_pair(p, row, col, make_float2(gelu_fast(v.x), gelu_fast(v.y)));
    });
}

template <int RG>
__global__ __launch_bounds__(64 * SECOND_WAVES) void ragged_few_second(const FewArgs p) {
  constexpr int NCL = 8, TN = 16 * NCL;
  __shared__ float red[few_floats<NCL, SECOND_WAVES>()];
  __shared__ int last;
  const int tid = threadIdx.x, lane = tid & 63;
  int used = 0;                                     // experts that have rows
  for (int e0 = 0; e0 < p.G; e0 += 64)
    used += __popcll(__ballot(e0 + lane < p.G && offset(p, min(e0 + lane + 1, p.G)) > offset(p, min(e0 + lane, p.G))));
  const int tiles = used * p.tiles_n, steps = (p.Kdim + 31) / 32;
  const int parts = tiles == 0 ? 1 : max(min(FEW_GRID / tiles, p.max_parts), 1);
  for (int unit = (int)blockIdx.x; unit < tiles * parts; unit += FEW_GRID) {
    const int part = unit / tiles, tile = unit - part * tiles, nth = tile / p.tiles_n, tn = tile - nth * p.tiles_n;
    int g = 0, before = 0;                          // the nth expert that has rows
    for (int e0 = 0; e0 < p.G; e0 += 64) {
      const unsigned long long has = __ballot(e0 + lane < p.G && offset(p, min(e0 + lane + 1, p.G)) > offset(p, min(e0 + lane, p.G)));
      const int count = __popcll(has);
      if (nth < before + count) {
        const bool mine = ((has >> lane) & 1ull) && __popcll(has & ((1ull << lane) - 1ull)) == nth - before;
        g = e0 + __ffsll((long long)__ballot(mine)) - 1;
        break;
      }
      before += count;
    }
    g = __builtin_amdgcn_readfirstlane(g);
    const int lo = __builtin_amdgcn_readfirstlane(offset(p, g)), n = __builtin_amdgcn_readfirstlane(offset(p, g + 1)) - lo;
    const int s0 = steps * part / parts, s1 = steps * (part + 1) / parts, n0 = tn * TN;
    for (int m0 = 0; m0 < n; m0 += 16 * RG)
      few_rows<NCL, RG, SECOND_WAVES>(p, red, g, lo, n, m0, n0, s0, s1, [&](int row, int col, const float2& v) {
        if (parts == 1) store_pair(p, row, col, v);
        else __hip_atomic_store(reinterpret_cast<uint64_t*>(p.sums + ((int64_t)part * p.R + row) * p.Ndim + col), __builtin_bit_cast(uint64_t, v),
                                __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      });
    if (parts == 1) continue;
    // The sums are written past the caches that the XCDs do not share, and read past them: once a wave's stores are complete they are
    // where every reader looks, and no cache has to be written back or invalidated (fences in 1024 workgroups: 50 us).
    __builtin_amdgcn_s_waitcnt(0x0070);             // vmcnt(0), lgkmcnt(0)
    __syncthreads();
    if (tid == 0) last = __hip_atomic_fetch_add(&p.arrived[g * p.tiles_n + tn], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == parts - 1;
    __syncthreads();
    if (!last) continue;
    const int cols = min(TN, p.Ndim - n0) / 2;      // pairs; Ndim is a multiple of 8
    for (int u = tid; u < n * cols; u += 64 * SECOND_WAVES) {
      const int r = u / cols, row = lo + r, col = n0 + 2 * (u - r * cols);
      const float* src = p.sums + (int64_t)row * p.Ndim + col;
      float2 v = make_float2(0.f, 0.f);
#pragma unroll 8
      for (int q = 0; q < parts; ++q) {
        const float2 a = __builtin_bit_cast(float2, __hip_atomic_load(reinterpret_cast<const uint64_t*>(src + (int64_t)q * p.R * p.Ndim),
                                                                      __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
        v.x += a.x;
        v.y += a.y;
      }
      store_pair(p, row, col, v);
    }
  }
  fill_behind<2>(p, (int)blockIdx.x, FEW_GRID);
}

namespace {
int second_parts(int N, int K) {      // the most parts that the second product is cut into
  const int tiles_n = (N + 127) / 128, steps = (K + 31) / 32;
  return std::max(1, std::min(FEW_GRID / tiles_n, steps / FEW_PART_STEPS));
}
}  // namespace

// counters, and the second product's partial sums
size_t few_rows_bytes(int64_t R, int E, int M, int Hl) {
  return align_up((size_t)E * ((M + 127) / 128) * 4, 256) + align_up((size_t)second_parts(M, Hl) * R * M * 4, 256);
}

void launch_few_rows(const RaggedArgs& first, const RaggedArgs& second, void* ws, hipStream_t st) {
  FewArgs a{}, y{};
  static_cast<RaggedArgs&>(a) = first;
  static_cast<RaggedArgs&>(y) = second;
  y.tiles_n = (y.Ndim + 127) / 128;
  a.n_arrived = y.G * y.tiles_n;
  a.arrived = y.arrived = (int32_t*)ws;
  y.sums = (float*)((char*)ws + align_up((size_t)a.n_arrived * 4, 256));
  y.max_parts = second_parts(y.Ndim, y.Kdim);
  using std::integral_constant;
  auto with_groups = [&](auto&& f) {    // mean rows of an expert, with room for some more of them
    if (a.R <= 8 * (int64_t)a.G || a.R <= 16) f(integral_constant<int, 1>{});
    else f(integral_constant<int, 2>{});
  };
  auto launch = [&](auto ncl, auto rg) {
    constexpr int NCL = decltype(ncl)::value, RG = decltype(rg)::value;
    a.tiles_n = (a.Ndim + 16 * NCL - 1) / (16 * NCL);
    a.total_tiles = a.G * a.tiles_n;
    const int grid = std::max(a.total_tiles, (a.n_arrived + 64 * FIRST_WAVES - 1) / (64 * FIRST_WAVES));
    hipLaunchKernelGGL((ragged_few_first<NCL, RG>), dim3((unsigned)grid), dim3(64 * FIRST_WAVES), 0, st, a);
  };
  const int64_t tiles128 = std::min<int64_t>(a.R, a.G) * ((a.Ndim + 127) / 128);
  with_groups([&](auto rg) {
    if (tiles128 >= num_cus()) launch(integral_constant<int, 8>{}, rg);
    else launch(integral_constant<int, 4>{}, rg);
    hipLaunchKernelGGL((ragged_few_second<decltype(rg)::value>), dim3(FEW_GRID), dim3(64 * SECOND_WAVES), 0, st, y);
  });
}

}  // namespace moe
