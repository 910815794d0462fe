// Expert products and the gated expert FFN over ragged rows from microscaled 4-bit values (mx4.h):
//   Y = X W of each row's expert, both in 4 bits, fp32 sums of exact products;
//   the FFN: token rows to 4 bits, G and U from the two halves of W1, A = act(G) U to 4 bits, Y = A W2.
#include <math.h>

#include "mx4_ffn.h"

namespace moe {
namespace {

void set_source(Mx4Args& a, const int32_t* inv, int k, int64_t S) {
  a.gather = inv;
  a.gather_k = inv ? k : 0;
  a.gather_rows = inv ? S : 0;
  a.gather_magic = inv ? magic_of(k) : 0u;
  a.x_rows = inv ? S : a.R;
}
void set_summed(Mx4Args& a, int K) {
  a.K = K;
  a.blocks = (int)mx4_blocks(K);
  a.chunks = (int)mx4_chunks(K);
}
size_t tensor_bytes(int64_t n, int K) { return align_up(mx4_value_bytes(n, K), 256) + align_up(mx4_scale_bytes(n, K), 256); }

// How a product is computed: 0, the kernel for few rows; 128 or 256, square tiles.  Experts of few rows are bound by their weights' bytes, which the kernel
// for few rows reads fastest, but again for every 16 rows of an expert (32 where more than 16 rows are of three experts or fewer), one reading after the
// other in one workgroup.  How the rows are spread is not known here, so their number has a bound: up to 32 rows this is the faster one or nearly even
// under any routing, beyond it it gains little with equal shares and loses the more if the experts' logits differ.  us of a product, this and tiles of 128, with equal
// shares, logits that differ by N(0, 1) and by N(0, 2), and one expert with all rows:
//    1 x 4096 x 14336   16 rows 9 and 16, 32 rows 10 and 16, 64 rows 18 and 18
//    8 x 4096 x 14336   32 rows 49 and 55, 42 and 45, 41 and 49, 15 and 16;  64 rows 51 and 54, 70 and 53, 35 and 23, 26 and 18;
//                      128 rows 56 and 55, 82 and 56, 67 and 52, 59 and 17
//   64 x 2048 x 2048    16 rows 9 and 12, 10 and 10, 8 and 9, 8 and 9;  32 rows 15 and 16, 13 and 10, 10 and 10, 8 and 9;
//                       64 rows 28 and 31, 15 and 14, 13 and 10, 14 and 9;  1024 rows 31 and 32, 55 and 24, 95 and 15, 132 and 10
//  256 x 7168 x 2048    32 rows 49 and 52, 44 and 47, 27 and 30, 21 and 24;  64 rows 95 and 99, 69 and 54, 44 and 30, 38 and 24;
//                      1024 rows 378 and 416, 267 and 147, 297 and 85, 557 and 30
// Of the tiles the small ones waste less of experts with few rows and fill the chip with fewer of them: rounds of tiles on the chip, each of k tiles of
// 256 and what is outside the k loop (us, measured; with few and with all compute units busy).  8 x 4096 x 14336 with 64, 256, 1024 and 4096 rows each, tiles of
// 128 64, 124, 376 and 1353 us, of 256 76, 111, 290 and 1092; 1 x 2048 x 8192 with 1024 and 4096 rows 18 and 55, 22 and 44.  Tiles of 64 x 128 were nowhere the fastest.
struct Mx4TileCost {
  int tile, per_cu;
  float k_few, k_all, fixed;
};
constexpr Mx4TileCost MX4_TILES[] = {{256, 1, 1.25f, 1.75f, 8.f}, {128, 2, 0.75f, 1.10f, 6.f}};
constexpr int MX4_FEW_ROWS = 32;
// workgroups of `threads` threads each: a launch has fewer than 2^32 threads
bool launches(int64_t groups, int threads) { return groups * threads < 1ll << 32; }
int64_t few_groups(int E, int64_t n) { return E * ((n + 63) / 64) + ZERO_SHARES; }
}  // namespace
int mx4_tile(int64_t R, int E, int64_t n, int K) {
  if (R <= MX4_FEW_ROWS && launches(few_groups(E, n), 256)) return 0;
  const float nk = (float)((K + 255) / 256), cu = (float)num_cus();
  int best = 0;
  float best_t = 0.f;
  for (const Mx4TileCost& c : MX4_TILES) {
    const double rows = E == 1 ? (double)((R + c.tile - 1) / c.tile) : priced_row_tiles((int)R, E, c.tile);
    const float tiles = (float)rows * (float)((n + c.tile - 1) / c.tile);
    const float busy = c.per_cu == 1 ? tiles / cu : (tiles - cu) / cu;
    const float k = c.k_few + (c.k_all - c.k_few) * fminf(fmaxf(busy, 0.f), 1.f);
    const float t = ceilf(tiles / (cu * c.per_cu)) * (nk * k + c.fixed);
    if (best == 0 || t < best_t) { best_t = t; best = c.tile; }
  }
  return best;
}
namespace {
void launch(const Mx4Args& a, int kind, hipStream_t st) {
  const int tile = mx4_tile(a.R, a.E, a.n, a.K);
  if (tile == 0) launch_mx4_few(a, kind, st);
  else launch_mx4_tile(a, kind, tile, st);
}

// rows of X, of one expert's W and of Y: 32-bit byte offsets
int check_mx4_product(int64_t R, int E, int K, int64_t n) {
  MOE_REQUIRE(R >= 1 && E >= 1 && K >= 1 && n >= 1, MOE_EINVAL);
  MOE_REQUIRE(E <= MOE_MAX_E && K % 8 == 0 && n % 8 == 0, MOE_EUNSUPPORTED);
  MOE_REQUIRE(R <= 1ll << 29 && K <= 1 << 28 && n <= 1ll << 29, MOE_EUNSUPPORTED);
  MOE_REQUIRE(std::max(mx4_value_bytes(n, K), mx4_scale_bytes(n, K)) <= 0xFFFFFFF0ull, MOE_EUNSUPPORTED);
  MOE_REQUIRE(R * n <= 1ll << 37 && (int64_t)E * n <= 1ll << 34, MOE_EUNSUPPORTED);
  if (const int tile = mx4_tile(R, E, n, K))
    MOE_REQUIRE(launches(most_row_tiles((int)R, E, tile) * ((n + tile - 1) / tile) + 8 + ZERO_SHARES, 2 * tile), MOE_EUNSUPPORTED);
  return MOE_OK;
}
int check_mx4_rows(int64_t rows, int K) {
  MOE_REQUIRE(std::max(mx4_value_bytes(rows, K), mx4_scale_bytes(rows, K)) <= 0xFFFFFFF0ull, MOE_EUNSUPPORTED);
  return MOE_OK;
}
// rows through the plan's map, or as they lie
int check_map(int64_t S, const int32_t* inv, int k) {
  MOE_OPTIONAL_PTR(inv);
  if (inv == nullptr) {
    MOE_REQUIRE(k == 1, MOE_EINVAL);
    return MOE_OK;
  }
  MOE_REQUIRE(S >= 1 && k >= 1, MOE_EINVAL);
  MOE_REQUIRE(k <= MOE_MAX_K && S * (int64_t)k <= (1ll << 29), MOE_EUNSUPPORTED);
  return MOE_OK;
}
int check_mx4_glu(int64_t R, int E, int M, int H) {
  MOE_REQUIRE(R >= 1 && E >= 1 && M >= 1 && H >= 1, MOE_EINVAL);
  MOE_REQUIRE(H <= 1 << 28, MOE_EUNSUPPORTED);
  if (int rc = check_mx4_product(R, E, M, 2 * (int64_t)H)) return rc;
  if (int rc = check_mx4_product(R, E, H, M)) return rc;
  return check_mx4_rows(R, H);
}

}  // namespace
}  // namespace moe

using namespace moe;

extern "C" size_t moe_ragged_gemm_mx4_workspace_bytes(int64_t R, int E, int K, int N) {
  (void)R; (void)E; (void)K; (void)N;
  return 0;
}

extern "C" int moe_ragged_gemm_mx4(const void* xq, const void* xs, int64_t S, const int32_t* inv, int k, const void* Wq, const void* Ws,
                                   const int32_t* offsets, int64_t R, int E, int K, int N, void* Y, int dtype, void* ws, size_t ws_bytes,
                                   void* stream) {
  MOE_REQUIRE(dtype == MOE_F32 || dtype == MOE_BF16, MOE_EINVAL);
  if (int rc = check_mx4_product(R, E, K, N)) return rc;
  if (int rc = check_map(S, inv, k)) return rc;
  if (int rc = check_mx4_rows(inv ? S : R, K)) return rc;
  MOE_REQUIRE_PTR(xq); MOE_REQUIRE_PTR(xs); MOE_REQUIRE_PTR(Wq); MOE_REQUIRE_PTR(Ws); MOE_REQUIRE_PTR(offsets); MOE_REQUIRE_PTR(Y);
  MOE_OPTIONAL_PTR(ws);
  (void)ws_bytes;
  Mx4Args a{};
  a.xq = (const uint8_t*)xq; a.xs = (const uint8_t*)xs; a.wq = (const uint8_t*)Wq; a.ws = (const uint8_t*)Ws;
  a.off = offsets; a.R = (int)R; a.E = E; a.n = N;
  set_summed(a, K);
  set_source(a, inv, k, S);
  a.C = Y; a.f32 = dtype == MOE_F32;
  launch(a, MX4_STORE, (hipStream_t)stream);
  return check_launch();
}

extern "C" size_t moe_ragged_glu_mx4_workspace_bytes(int64_t S, int64_t R, int E, int M, int H) {
  if (S < 0 || check_mx4_glu(R, E, M, H) != MOE_OK || check_mx4_rows(std::max(S, R), M) != MOE_OK) return 0;
  return tensor_bytes(std::max(S, R), M) + tensor_bytes(R, H);
}

extern "C" int moe_ragged_glu_mx4(const void* x, int dtype, int64_t S, const int32_t* inv, int k, const void* W1q, const void* W1s, const void* W2q,
                                  const void* W2s, const int32_t* offsets, int64_t R, int E, int M, int H, int act, void* Y, void* ws,
                                  size_t ws_bytes, void* stream) {
  MOE_REQUIRE(dtype == MOE_F32 || dtype == MOE_BF16, MOE_EINVAL);
  MOE_REQUIRE(act == MOE_ACT_SILU || act == MOE_ACT_GELU, MOE_EINVAL);
  if (int rc = check_mx4_glu(R, E, M, H)) return rc;
  if (int rc = check_map(S, inv, k)) return rc;
  const int64_t rows = inv ? S : R;
  if (int rc = check_mx4_rows(rows, M)) return rc;
  MOE_REQUIRE_PTR(x); MOE_REQUIRE_PTR(W1q); MOE_REQUIRE_PTR(W1s); MOE_REQUIRE_PTR(W2q); MOE_REQUIRE_PTR(W2s); MOE_REQUIRE_PTR(offsets); MOE_REQUIRE_PTR(Y);
  const size_t x_bytes = tensor_bytes(rows, M), a_bytes = tensor_bytes(R, H);
  MOE_REQUIRE(ws != nullptr && ws_bytes >= x_bytes + a_bytes, MOE_EWORKSPACE);
  MOE_REQUIRE(aligned16(ws), MOE_EALIGN);
  hipStream_t st = (hipStream_t)stream;
  uint8_t* xq = (uint8_t*)ws;
  uint8_t* xs = xq + align_up(mx4_value_bytes(rows, M), 256);
  uint8_t* aq = xq + x_bytes;
  uint8_t* as = aq + align_up(mx4_value_bytes(R, H), 256);
  mx4_store_rows(x, dtype, 1, rows, M, xq, xs, st);

  Mx4Args a{};
  a.xq = xq; a.xs = xs; a.wq = (const uint8_t*)W1q; a.ws = (const uint8_t*)W1s;
  a.off = offsets; a.R = (int)R; a.E = E; a.n = 2 * H;
  set_summed(a, M);
  set_source(a, inv, k, S);
  a.half = H; a.act = act; a.f32 = dtype == MOE_F32; a.aq = aq; a.as = as; a.a_blocks = (int)mx4_blocks(H);
  launch(a, MX4_GLU, st);

  Mx4Args y{};
  y.xq = aq; y.xs = as; y.wq = (const uint8_t*)W2q; y.ws = (const uint8_t*)W2s;
  y.off = offsets; y.R = (int)R; y.E = E; y.n = M;
  set_summed(y, H);
  set_source(y, nullptr, 1, 0);
  y.C = Y; y.f32 = dtype == MOE_F32;
  launch(y, MX4_STORE, st);
  return check_launch();
}
