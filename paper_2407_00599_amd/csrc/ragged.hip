// Expert products over ragged rows: the chosen rows of all experts lie expert by expert in one [R, .] buffer with no capacity padding
// between them.  With the kept rows n_e = min(counts[e], C) of expert e,
//   offsets[e] = n_0 + ... + n_(e-1),   row of choice (t, j) = offsets[idx[t, j]] + slot[t, j],
// and rows at or behind offsets[E] hold zeros.  Here are the plan of the rows, the three grouped products
//   Y = X W,  dX = dY W^T,  dW = X^T dY       (X optionally read from the token matrix through the plan's row map)
// and the expert FFN of an ESP shard forward and backward, whose pre-activation is kept for the backward pass in 8 bits (ckpt8.h):
//   forward   Z = X W1, A = GeLU(Z), Y = A W2;  Zq, Zs <- 8-bit form of Z
//   backward  z = the value that (Zq, Zs) stand for:  A' = GeLU(z), dZ = (dY W2^T) GeLU'(z), dW2 = A'^T dY, dW1 = X^T dZ, dX = dZ W1^T
// against the padded FFN's Z and A in the storage type, 4 bytes a value in bf16, the backward pass reads 1 + 1/32.
// In bf16, A, A' and dZ are rounded to bf16 between two products, as the padded FFN's: they are operands of bf16 matrix instructions, and fp32 ones
// run at a ninth of the rate.  That takes Y and the gradients from 1.66e-3 of their size off the exact ones (the last rounding alone) to 2.35e-3.
//
// The tiles are those of the capacity-padded calls (ffn_tile.h).  The offsets are read on the device: a workgroup finds the expert of
// its tile by a scan over the experts' tile counts, so no count crosses to the host and a call can be captured into a graph.
#include <math.h>

#include "ragged_tile.h"

namespace moe {

// ------------------------------------------------------------------------------------------
// plan
// ------------------------------------------------------------------------------------------
constexpr int PLAN_THREADS = 256;
static_assert(MOE_MAX_E <= PLAN_THREADS, "a thread per expert");

// Every workgroup scans the kept rows of all experts for itself (at most 256, 8 shuffles and two barriers), so the plan is one launch;
// it reads and writes 20 bytes a choice and is bound by that launch.
__global__ __launch_bounds__(PLAN_THREADS) void ragged_plan(const int32_t* __restrict__ idx, const int32_t* __restrict__ slot,
                                                            const int32_t* __restrict__ counts, int R, int S, int E, int k, int C,
                                                            int32_t* __restrict__ offsets, int32_t* __restrict__ row_idx,
                                                            int32_t* __restrict__ row_slot, int32_t* __restrict__ row_inv) {
  __shared__ int off[MOE_MAX_E + 1], wave_sum[PLAN_THREADS / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int c = (int)blockIdx.x * PLAN_THREADS + tid;     // choice t k + j; and, for the empty rows, a row
  const int e = idx[min(c, R - 1)], s = slot[min(c, R - 1)];      // requested with the counts, not behind their scan
  const int kept = tid < E ? min(max(counts[tid], 0), C) : 0;
  int incl = kept;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int v = __shfl_up(incl, d, 64);
    if (lane >= d) incl += v;
  }
  if (lane == 63) wave_sum[wave] = incl;
  __syncthreads();
  for (int w = 0; w < wave; ++w) incl += wave_sum[w];
  if (tid < E) off[tid + 1] = min(incl, R);
  if (tid == 0) off[0] = 0;
  __syncthreads();
  if (blockIdx.x == 0)
    for (int q = tid; q <= E; q += PLAN_THREADS) offsets[q] = off[q];
  const int end = off[E];
  if (c >= R) return;
  int row = -1;
  if (s >= 0 && (unsigned)e < (unsigned)E && s < off[e + 1] - off[e]) row = off[e] + s;
  row_idx[c] = row >= 0 ? (int)((unsigned)row / (unsigned)S) : 0;
  row_slot[c] = row >= 0 ? (int)((unsigned)row % (unsigned)S) : -1;
  if (row >= 0) row_inv[row] = c;
  if (c >= end) row_inv[c] = -1;
}

// The pre-activation that is kept: on the fp64 matrix cores, because a sum next to the border between two steps decides which one is kept.
template <int T, bool WIDE>   // T x T tiles
__global__ __launch_bounds__(256, 4) void ragged_kept_f32(const RaggedArgs p) {
  __shared__ __attribute__((aligned(16))) double smem[f32_lds<T, T>() / 8];
  gemm_f32_tile<KIND_NN, EPI_GELU8, T, T, WIDE, Ragged>(p, smem, (int)blockIdx.x);
}

// dX = dZ W1^T and the two weight gradients, which only depend on dZ, in one launch; the third problem gathers its rows
template <typename CFX, typename CFW, int EPI>
__global__ __launch_bounds__(512) void ragged_ffn_bwd_trio(const RaggedArgs px, const RaggedArgs pw2, const RaggedArgs pw1, int nbx, int nb2) {
  static_assert(CFX::NW == 8 && CFW::NW == 8, "one block size");
  __shared__ __attribute__((aligned(1024))) char smem[CFX::LDS > CFW::LDS ? CFX::LDS : CFW::LDS];
  const int b = (int)blockIdx.x;
  if (b < nbx) gemm_dma_tile<KIND_NT, EPI_STORE, CFX, ROWS_PLAIN, Ragged>(px, smem, b);
  else if (b < nbx + nb2) gemm_dma_tile<KIND_TN, EPI, CFW, ROWS_PLAIN, Ragged>(pw2, smem, b - nbx);
  else gemm_dma_tile<KIND_TN, EPI, CFW, ROWS_GATHER, Ragged>(pw1, smem, b - nbx - nb2);
}

// Adds the parts of one or two split weight gradients in order and stores them: a thread owns 4 columns of a row.
template <typename T>
__global__ __launch_bounds__(256) void ragged_add_parts(const RaggedArgs p2, const RaggedArgs p1, int64_t n2, int64_t n) {
  int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (u >= n) return;
  const RaggedArgs& p = u < n2 ? p2 : p1;
  if (u >= n2) u -= n2;
  const int64_t size = (int64_t)p.G * p.Mdim * p.Ndim, at = u * 4;
  const float* src = p.part + at;
  f32x4_t v = *reinterpret_cast<const f32x4_t*>(src);
#pragma unroll 8
  for (int q = 1; q < p.splits; ++q) v += *reinterpret_cast<const f32x4_t*>(src + q * size);
  const int64_t row = at / p.Ndim, g = row / p.Mdim;
  T* dst = reinterpret_cast<T*>(p.C) + g * p.c_goff + p.c_off + (row - g * p.Mdim) * p.ldc + (at - row * p.Ndim);
  if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
  else *reinterpret_cast<f32x4_t*>(dst) = v;
}

// The same for a split product over rows (fp32), whose rows behind the last expert's are zeros.
__global__ __launch_bounds__(256) void ragged_add_rows(const RaggedArgs p) {
  const int64_t size = (int64_t)p.R * p.Ndim, at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (at >= size) return;
  const int row = (int)(at / p.Ndim);
  f32x4_t v = {0.f, 0.f, 0.f, 0.f};
  if (row < offset(p, p.G)) {
#pragma unroll 4
    for (int q = 0; q < p.splits; ++q) v += *reinterpret_cast<const f32x4_t*>(p.part + q * size + at);
  }
  *reinterpret_cast<f32x4_t*>(reinterpret_cast<float*>(p.C) + (int64_t)row * p.ldc + (at - (int64_t)row * p.Ndim)) = v;
}

// ------------------------------------------------------------------------------------------
// host side
// ------------------------------------------------------------------------------------------
namespace {

void launch_kept_f32(RaggedArgs a, hipStream_t st) {
  auto launch = [&](auto tile, auto wide) {
    constexpr int T = decltype(tile)::value;
    const dim3 grid = size_rows(a, T, T, false);
    hipLaunchKernelGGL((ragged_kept_f32<T, decltype(wide)::value>), grid, dim3(256), 0, st, a);
  };
  using std::integral_constant;
  if (std::max(a.lda, a.ldb) >= 1 << 24) launch(integral_constant<int, 32>{}, std::true_type{});
  else if (priced_row_tiles(a.R, a.G, 64) * ((a.Ndim + 63) / 64) >= 3.0 * num_cus()) launch(integral_constant<int, 64>{}, std::false_type{});
  else launch(integral_constant<int, 32>{}, std::false_type{});
}

template <int KIND>
void launch_row_parts(RaggedArgs a, int parts, void* ws, hipStream_t st) {
  a.splits = parts;
  a.part = (float*)ws;
  launch_f32<KIND, EPI_PART>(a, st);
  hipLaunchKernelGGL(ragged_add_rows, dim3((unsigned)(((int64_t)a.R * a.Ndim / 4 + 255) / 256)), dim3(256), 0, st, a);
}

template <int KIND, int EPI>
void launch_rows(RaggedArgs a, int dtype, hipStream_t st) {
  if (dtype == MOE_F32) {
    if constexpr (EPI == EPI_GELU8) launch_kept_f32(a, st);
    else launch_f32<KIND, EPI>(a, st);
    return;
  }
  buffer_sizes(a, false);
  auto launch = [&](auto cfg) {
    using CF = decltype(cfg);
    const dim3 grid = size_rows(a, CF::TM, CF::TN, EPI == EPI_STORE);
    hipLaunchKernelGGL((ragged_ffn_gemm_dma<KIND, EPI, CF>), grid, dim3(64 * CF::NW), 0, st, a);
  };
  const TilePlan t = plan_rows(a);
  if (t.tile_m == 256) launch(Tile256{});
  else if (t.tile_m == 192) launch(Tile192{});
  else if (t.tile_m == 128) launch(Tile128{});
  else if (t.tile_m == 64 && t.tile_n == 128) launch(Tile64x128{});
  else if (t.tile_m == 64) launch(Tile64{});
  else launch(Tile32x64{});
}


// one weight gradient; parts: room for a.splits of them
void launch_weights(RaggedArgs a, int dtype, float* parts, hipStream_t st) {
  a.part = parts;
  if (dtype == MOE_F32) {
    if (a.splits > 1) launch_f32<KIND_TN, EPI_PART>(a, st);
    else launch_f32<KIND_TN, EPI_STORE>(a, st);
  } else {
    buffer_sizes(a, true);
    auto launch = [&](auto cfg, auto epi) {
      using CF = decltype(cfg);
      constexpr int EPI = decltype(epi)::value;
      const dim3 grid(size_weights(a, CF::TM).x * a.splits);
      if (a.gather) hipLaunchKernelGGL((ragged_ffn_gemm_dma<KIND_TN, EPI, CF, ROWS_GATHER>), grid, dim3(64 * CF::NW), 0, st, a);
      else hipLaunchKernelGGL((ragged_ffn_gemm_dma<KIND_TN, EPI, CF>), grid, dim3(64 * CF::NW), 0, st, a);
    };
    using Store = std::integral_constant<int, EPI_STORE>;
    if (!small_weights(a.G, a.Mdim, a.Ndim)) launch(Tile256{}, Store{});
    else if (a.splits > 1) launch(Tile128{}, std::integral_constant<int, EPI_PART>{});
    else launch(Tile128{}, Store{});
  }
  if (a.splits > 1) add_parts(a, a, 1, dtype, st);
}

// dX and the two weight gradients of the FFN
void launch_backward(RaggedArgs dx, RaggedArgs w2, RaggedArgs w1, int dtype, float* parts, hipStream_t st) {
  w2.part = parts;
  w1.part = w2.splits > 1 ? parts + (size_t)w2.splits * w2.G * w2.Mdim * w2.Ndim : nullptr;
  if (dtype == MOE_F32) {
    launch_trio_f32(dx, w2, w1, st);
  } else if (w1.gather == nullptr) {
    launch_rows<KIND_NT, EPI_STORE>(dx, dtype, st);
    launch_weights(w2, dtype, w2.part, st);
    launch_weights(w1, dtype, w1.part, st);
    return;
  } else {
    buffer_sizes(dx, false); buffer_sizes(w2, true); buffer_sizes(w1, true);
    auto launch = [&](auto cfx, auto cfw, auto epi) {
      using CFX = decltype(cfx);
      using CFW = decltype(cfw);
      const unsigned nbx = size_rows(dx, CFX::TM, CFX::TN, true).x;
      const unsigned nb2 = size_weights(w2, CFW::TM).x * w2.splits, nb1 = size_weights(w1, CFW::TM).x * w1.splits;
      hipLaunchKernelGGL((ragged_ffn_bwd_trio<CFX, CFW, decltype(epi)::value>), dim3(nbx + nb2 + nb1), dim3(512), 0, st, dx, w2, w1, (int)nbx, (int)nb2);
    };
    using Store = std::integral_constant<int, EPI_STORE>;
    if (small_weights(w2.G, w2.Mdim, w2.Ndim)) {
      if (w2.splits > 1) launch(Tile64x128{}, Tile128{}, std::integral_constant<int, EPI_PART>{});
      else launch(Tile64x128{}, Tile128{}, Store{});
    } else {
      const TilePlan t = plan_rows(dx, true);
      if (t.tile_m == 256) launch(Tile256{}, Tile256{}, Store{});
      else if (t.tile_m == 192) launch(Tile192{}, Tile256{}, Store{});
      else if (t.tile_m == 128) launch(Tile128{}, Tile256{}, Store{});
      else launch(Tile64x128{}, Tile256{}, Store{});
    }
  }
  if (w2.splits > 1) add_parts(w2, w1, 2, dtype, st);
}

// The FFN of few rows (ragged_few.hip), where weights of a million values and more outweigh its launches and the second product's reduction is at
// least twice as long as its rows are wide, which gives the tiles few workgroups.  Forward call, tiles and this: 8 experts x 1024 x 4096, 2 rows 23.2
// and 16.2 us, 64 rows 42.9 and 38.1; 8 x 2048 x 8192, 2 rows 54.2 and 39.4; 8 x 256 x 1024, 64 rows 12.6 and 15.9; 8 x 1024 x 1024, 64 rows 18.4 and
// 21.5; 32 x 4096 x 2048, 4 rows 32.3 and 39.4.
// An expert's weights are read again for every 16 rows, and how the rows are spread is not known here, so their number has a bound: up to 32 rows
// this is the faster one or even under any routing, up to 64 it gains up to 12 % if the experts get equal shares and loses as much (8 x 1024 x 4096,
// 64 rows) if their logits differ by N(0, 1) or N(0, 2), beyond it gains nothing and loses the more (E x 1024 x 4096, tiles and this, equal and skewed by N(0, 2): 16
// experts, 128 rows 64.1 and 64.0, 40.7 and 66.2; 64 experts, 256 rows 195 and 196, 64 and 129; 512 rows 204 and 210, 78 and 258; one expert of 64 with all 512
// rows 36 and 354).
bool few_rows(int dtype, int64_t R, int E, int M, int Hl) {
  return dtype == MOE_BF16 && (R <= 32 || (R <= 64 && R <= 8 * (int64_t)E)) && Hl >= 2 * (int64_t)M && (int64_t)M * Hl >= 1 << 20;
}

}  // namespace

// The tile of a bf16 row-tiled GEMM: the prices of the padded calls' tiles (ffn_tile.h) for what is multiplied, against the time of reading the
// weights, 4.9 TB/s, priced as if a second row tile of an expert found half of them in a cache.  Weights bound the launch where experts have few rows, and a tile that
// all rows of most experts fit in is then the fastest: 8 experts of 64 rows x 4096 x 14336 and x 14336 x 4096, tiles of 128 x 128 189 and 188 us,
// 64 x 128 198 and 243, 64 x 64 227 and 249; of 1024 x 1024 x 4096 102 and 128, 192 x 256 82.
TilePlan rows_tile(int R, int E, int K, int N, bool wide) {
  const float nk = (float)((K + DK - 1) / DK), cu = (float)num_cus(), used = (float)std::min(R, E);
  const float weights = used * (float)K * (float)N * 2.f / 4.9e6f;
  TilePlan best{256, 256};
  float best_t = 0.f;
  for (const TileCost& c : ROW_TILES) {
    if (wide && c.tile.tile_n == 64) continue;
    const float row_tiles = (float)priced_row_tiles(R, E, c.tile.tile_m);
    const float n = row_tiles * (float)((N + c.tile.tile_n - 1) / c.tile.tile_n);
    const float busy = c.per_cu == 1 ? n / cu : (n - cu) / cu;
    const float k = c.k_few + (c.k_all - c.k_few) * fminf(fmaxf(busy, 0.f), 1.f);
    const float products = ceilf(n / (cu * c.per_cu)) * (nk * k + c.fixed), reads = weights * 0.5f * (1.f + fmaxf(row_tiles / used, 1.f));
    const float t = fmaxf(products, reads) + 0.2f * fminf(products, reads);
    if (best_t == 0.f || t < best_t) { best_t = t; best = c.tile; }
  }
  return best;
}

void launch_second(const RaggedArgs& y, int dtype, void* ws, size_t ws_bytes, hipStream_t st) {
  const int parts = row_parts(dtype, y.R, y.G, y.Kdim, y.Ndim);
  if (parts > 1 && ws != nullptr && ws_bytes >= row_part_bytes(parts, y.R, y.Ndim)) launch_row_parts<KIND_NN>(y, parts, ws, st);
  else launch_rows<KIND_NN, EPI_STORE>(y, dtype, st);
}

void add_parts(const RaggedArgs& p2, const RaggedArgs& p1, int problems, int dtype, hipStream_t st) {
  const int64_t n = (int64_t)p2.G * p2.Mdim * p2.Ndim / 4;       // sizes are multiples of 8
  const dim3 grid((unsigned)((problems * n + 255) / 256));
  if (dtype == MOE_BF16) hipLaunchKernelGGL((ragged_add_parts<bf16_t>), grid, dim3(256), 0, st, p2, p1, n, problems * n);
  else hipLaunchKernelGGL((ragged_add_parts<float>), grid, dim3(256), 0, st, p2, p1, n, problems * n);
}

}  // namespace moe

using namespace moe;

extern "C" int moe_ragged_plan(const int32_t* idx, const int32_t* slot, const int32_t* counts, int64_t S, int E, int k, int64_t C,
                               int32_t* offsets, int32_t* row_idx, int32_t* row_slot, int32_t* row_inv, void* stream) {
  if (int rc = common_shape_check(S, 8, E, k, C)) return rc;
  MOE_REQUIRE_PTR(idx); MOE_REQUIRE_PTR(slot); MOE_REQUIRE_PTR(counts); MOE_REQUIRE_PTR(offsets);
  MOE_REQUIRE_PTR(row_idx); MOE_REQUIRE_PTR(row_slot); MOE_REQUIRE_PTR(row_inv);
  const int64_t R = S * k;
  MOE_REQUIRE(R <= (1ll << 29), MOE_EUNSUPPORTED);
  hipLaunchKernelGGL(ragged_plan, dim3((unsigned)((R + PLAN_THREADS - 1) / PLAN_THREADS)), dim3(PLAN_THREADS), 0, (hipStream_t)stream,
                     idx, slot, counts, (int)R, (int)S, E, k, (int)C, offsets, row_idx, row_slot, row_inv);
  return check_launch();
}

extern "C" size_t moe_ragged_gemm_workspace_bytes(int dtype, int64_t R, int E, int K, int N) {
  if (check_product(dtype, R, E, K, N) != MOE_OK) return 0;
  return row_part_bytes(row_parts(dtype, R, E, K, N), R, N);
}

extern "C" int moe_ragged_gemm(const void* x, int dtype, int64_t S, const int32_t* inv, int k, const void* W, int transposed,
                               const int32_t* offsets, int64_t R, int E, int K, int N, void* Y, void* ws, size_t ws_bytes,
                               void* stream) {
  if (int rc = check_product(dtype, R, E, K, N)) return rc;
  MOE_REQUIRE(transposed == 0 || transposed == 1, MOE_EINVAL);
  if (int rc = check_source(x, dtype, S, inv, k, K)) return rc;
  MOE_REQUIRE_PTR(W); MOE_REQUIRE_PTR(offsets); MOE_REQUIRE_PTR(Y);
  const int parts = row_parts(dtype, R, E, K, N);
  MOE_REQUIRE(parts == 1 || (ws != nullptr && ws_bytes >= row_part_bytes(parts, R, N)), MOE_EWORKSPACE);
  MOE_OPTIONAL_PTR(ws);
  RaggedArgs a = base_args(offsets, R, E);
  set_gather(a, inv, k, S);
  a.A = x; a.lda = K;
  a.B = W; a.ldb = transposed ? K : N; a.b_goff = (int64_t)K * N;
  a.C = Y; a.ldc = N;
  a.Mdim = a.R; a.Ndim = N; a.Kdim = K;
  if (parts > 1) transposed ? launch_row_parts<KIND_NT>(a, parts, ws, (hipStream_t)stream) : launch_row_parts<KIND_NN>(a, parts, ws, (hipStream_t)stream);
  else if (transposed) launch_rows<KIND_NT, EPI_STORE>(a, dtype, (hipStream_t)stream);
  else launch_rows<KIND_NN, EPI_STORE>(a, dtype, (hipStream_t)stream);
  return check_launch();
}

extern "C" size_t moe_ragged_wgrad_workspace_bytes(int dtype, int64_t R, int E, int K, int N) {
  if (check_product(dtype, R, E, K, N) != MOE_OK) return 0;
  return part_bytes(weight_parts(dtype, R, E, K, N, 1), E, K, N);
}

extern "C" int moe_ragged_wgrad(const void* x, int dtype, int64_t S, const int32_t* inv, int k, const void* dY, const int32_t* offsets,
                                int64_t R, int E, int K, int N, void* dW, void* ws, size_t ws_bytes, void* stream) {
  if (int rc = check_product(dtype, R, E, K, N)) return rc;
  if (int rc = check_source(x, dtype, S, inv, k, K)) return rc;
  MOE_REQUIRE_PTR(dY); MOE_REQUIRE_PTR(offsets); MOE_REQUIRE_PTR(dW);
  const int parts = weight_parts(dtype, R, E, K, N, 1);
  MOE_REQUIRE(parts == 1 || (ws != nullptr && ws_bytes >= part_bytes(parts, E, K, N)), MOE_EWORKSPACE);
  MOE_OPTIONAL_PTR(ws);
  RaggedArgs a = base_args(offsets, R, E);
  a.splits = parts;
  set_gather(a, inv, k, S);
  a.A = x; a.lda = K;
  a.B = dY; a.ldb = N;
  a.C = dW; a.ldc = N; a.c_goff = (int64_t)K * N;
  a.Mdim = K; a.Ndim = N; a.Kdim = a.R;
  launch_weights(a, dtype, (float*)ws, (hipStream_t)stream);
  return check_launch();
}

extern "C" size_t moe_ragged_ffn_workspace_bytes(int dtype, int64_t R, int E, int M, int H, int n_esp, int backward) {
  if (check_ffn(dtype, R, E, M, H, 0, n_esp) != MOE_OK) return 0;
  const int Hl = H / n_esp;
  if (backward) return 2 * hidden_bytes(dtype, R, Hl) + 2 * part_bytes(weight_parts(dtype, R, E, M, Hl, 2), E, M, Hl);
  return few_rows(dtype, R, E, M, Hl) ? few_rows_bytes(R, E, M, Hl) : row_part_bytes(row_parts(dtype, R, E, Hl, M), R, M);
}

extern "C" int moe_ragged_ffn_fwd(const void* x, int dtype, int64_t S, const int32_t* inv, int k, const void* W1, const void* W2,
                                  const int32_t* offsets, int64_t R, int E, int M, int H, int esp_idx, int n_esp, void* Zq, void* Zs,
                                  void* A, void* Y, void* ws, size_t ws_bytes, void* stream) {
  if (int rc = check_ffn(dtype, R, E, M, H, esp_idx, n_esp)) return rc;
  if (int rc = check_source(x, dtype, S, inv, k, M)) return rc;
  MOE_REQUIRE_PTR(W1); MOE_REQUIRE_PTR(W2); MOE_REQUIRE_PTR(offsets); MOE_REQUIRE_PTR(A); MOE_REQUIRE_PTR(Y);
  MOE_REQUIRE((Zq == nullptr) == (Zs == nullptr), MOE_ENULL);
  MOE_OPTIONAL_PTR(Zq); MOE_OPTIONAL_PTR(Zs); MOE_OPTIONAL_PTR(ws);
  hipStream_t st = (hipStream_t)stream;
  const int Hl = H / n_esp;
  const int64_t h0 = (int64_t)esp_idx * Hl;
  RaggedArgs a = base_args(offsets, R, E);
  set_gather(a, inv, k, S);
  a.A = x; a.lda = M;
  a.B = W1; a.ldb = H; a.b_goff = (int64_t)M * H; a.b_off = h0;
  a.C = A; a.C2 = Zq; a.Zs = (uint8_t*)Zs; a.ldc = Hl; a.ldz = (Hl + 31) / 32;
  a.Mdim = a.R; a.Ndim = Hl; a.Kdim = M;
  RaggedArgs y = base_args(offsets, R, E);
  y.A = A; y.lda = Hl;
  y.B = W2; y.ldb = M; y.b_goff = (int64_t)H * M; y.b_off = h0 * M;
  y.C = Y; y.ldc = M;
  y.Mdim = y.R; y.Ndim = M; y.Kdim = Hl;
  if (Zq == nullptr && few_rows(dtype, R, E, M, Hl) && ws != nullptr && ws_bytes >= few_rows_bytes(R, E, M, Hl)) {
    buffer_sizes(a, false);
    buffer_sizes(y, false);
    launch_few_rows(a, y, false, ws, st);
    return check_launch();
  }
  if (Zq) launch_rows<KIND_NN, EPI_GELU8>(a, dtype, st);
  else launch_rows<KIND_NN, EPI_ACT>(a, dtype, st);
  launch_second(y, dtype, ws, ws_bytes, st);
  return check_launch();
}

extern "C" int moe_ragged_ffn_bwd(const void* dY, const void* x, int dtype, int64_t S, const int32_t* inv, int k, const void* Zq,
                                  const void* Zs, const void* W1, const void* W2, const int32_t* offsets, int64_t R, int E, int M,
                                  int H, int esp_idx, int n_esp, void* dX, void* dW1, void* dW2, void* ws, size_t ws_bytes,
                                  void* stream) {
  if (int rc = check_ffn(dtype, R, E, M, H, esp_idx, n_esp)) return rc;
  MOE_REQUIRE_PTR(dY);
  if (int rc = check_source(x, dtype, S, inv, k, M)) return rc;
  MOE_REQUIRE_PTR(Zq); MOE_REQUIRE_PTR(Zs); MOE_REQUIRE_PTR(W1); MOE_REQUIRE_PTR(W2); MOE_REQUIRE_PTR(offsets);
  MOE_REQUIRE_PTR(dX); MOE_REQUIRE_PTR(dW1); MOE_REQUIRE_PTR(dW2);
  const int Hl = H / n_esp;
  const size_t hidden = hidden_bytes(dtype, R, Hl);
  const int parts = weight_parts(dtype, R, E, M, Hl, 2);
  MOE_REQUIRE(ws != nullptr && ws_bytes >= 2 * hidden + 2 * part_bytes(parts, E, M, Hl), MOE_EWORKSPACE);
  MOE_REQUIRE(aligned16(ws), MOE_EALIGN);
  hipStream_t st = (hipStream_t)stream;
  const int64_t h0 = (int64_t)esp_idx * Hl;
  void* dZ = ws;
  void* Act = (char*)ws + hidden;

  // dZ = (dY W2^T) GeLU'(z), Act = GeLU(z)
  RaggedArgs a = base_args(offsets, R, E);
  a.A = dY; a.lda = M;
  a.B = W2; a.ldb = M; a.b_goff = (int64_t)H * M; a.b_off = h0 * M;
  a.C = dZ; a.C2 = Act; a.Zin = Zq; a.Zs = (uint8_t*)const_cast<void*>(Zs); a.ldc = Hl; a.ldz = (Hl + 31) / 32;
  a.Mdim = a.R; a.Ndim = Hl; a.Kdim = M;
  launch_rows<KIND_NT, EPI_DGELU8>(a, dtype, st);
  // dX = dZ W1^T
  RaggedArgs dx = base_args(offsets, R, E);
  dx.A = dZ; dx.lda = Hl;
  dx.B = W1; dx.ldb = H; dx.b_goff = (int64_t)M * H; dx.b_off = h0;
  dx.C = dX; dx.ldc = M;
  dx.Mdim = dx.R; dx.Ndim = M; dx.Kdim = Hl;
  // dW2[h0:h0+Hl, :] = Act^T dY
  RaggedArgs w2 = base_args(offsets, R, E);
  w2.A = Act; w2.lda = Hl;
  w2.B = dY; w2.ldb = M;
  w2.C = dW2; w2.ldc = M; w2.c_goff = (int64_t)H * M; w2.c_off = h0 * M;
  w2.Mdim = Hl; w2.Ndim = M; w2.Kdim = w2.R;
  w2.splits = parts;
  // dW1[:, h0:h0+Hl] = X^T dZ
  RaggedArgs w1 = base_args(offsets, R, E);
  set_gather(w1, inv, k, S);
  w1.A = x; w1.lda = M;
  w1.B = dZ; w1.ldb = Hl;
  w1.C = dW1; w1.ldc = H; w1.c_goff = (int64_t)M * H; w1.c_off = h0;
  w1.Mdim = M; w1.Ndim = Hl; w1.Kdim = w1.R;
  w1.splits = parts;
  launch_backward(dx, w2, w1, dtype, (float*)((char*)ws + 2 * hidden), st);
  return check_launch();
}
