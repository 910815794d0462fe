// Gated expert FFN of an ESP shard over ragged rows, forward and backward.  W1 [E, M, 2 H] holds the gate's columns and behind them the up
// projection's; with the shard's columns of both halves
//   forward   G = X W1g, U = X W1u, A = act(G) U, Y = A W2;   Z = [G | U] rounded to the storage type, or nothing
//   backward  g, u = the values in Z:  dA = dY W2^T, dG = dA u act'(g), dU = dA act(g), A' = act(g) u,
//             dX = [dG | dU] W1^T,  dW1 = X^T [dG | dU],  dW2 = A'^T dY
// Both projections, the activation and the product are one launch: the tile's columns are 16 of the gate and the 16 of the up projection that belong
// to them in turn, so that a lane's accumulators hold both of a hidden value, and neither of them goes to memory unless it is kept.  The
// interleaving is in the addresses of the requests alone (Glu::column): 256 tile columns are 256 bytes of either half of a row of W1, whole lines.
// dX is one product over 2 H_l: of a shard the second half's k indexes lie elsewhere in W1 (Glu::k_skip).
// In bf16, A, A', dG and dU are rounded between two products, as in the FFN with one projection.
//
// Bound by the matrix instructions in training and by reading the weights in serving.  bf16, us of the launches: 4096 tokens top-2 of 8 experts x 1024 x 4096
// (16 k tiles a tile, so what is outside the k loop weighs: a third) first product with Z kept 187 (0.74 PFLOP/s), A W2 91, dA and its epilogue 129, dX and the
// weight gradients 407 (0.84); 16384 tokens top-2 of 8 experts x 4096 x half of 14336, under the power limit, 3018, 1571, 1752 and 8077 (1.2 to 1.28 PFLOP/s
// where the launch is a product alone); 256 tokens top-2 of 8 experts x 4096 x 14336, A kept alone, 425 and 208 (4.4 and 4.5 TB/s of weights).
#include "ragged_tile.h"

namespace moe {

struct Glu : Ragged {
  template <int EPI>
  static __device__ __forceinline__ int column(const Args& p, int n0, int c) {
    if constexpr (EPI == EPI_GLU || EPI == EPI_GLU_KEEP) return glu_column(p, n0, c);
    else return Ragged::column<EPI>(p, n0, c);
  }
  template <int EPI>
  static __device__ __forceinline__ uint32_t k_skip(const Args& p, int row0, uint32_t at) {
    if constexpr (EPI == EPI_GLU_DX) return (uint32_t)row0 + (at >> 1) >= (uint32_t)p.half ? (uint32_t)(p.up - p.half) * 2u : 0u;
    else return 0u;
  }
  // a map that is not there reads as zeros: the rows as they lie
  static __device__ __forceinline__ int in_order(const Args& p, int row) { return p.gather == nullptr ? row : 0; }
  static __device__ __forceinline__ uint32_t map_bytes(const Args& p) { return p.gather == nullptr ? 0u : Ragged::map_bytes(p); }

  // Epilogues, staged through the wave's slice of LDS 32 rows at a time as in the other calls: images [32][CW] of up to three tensors, written in
  // accumulator order, read back row by row and stored 16 bytes a lane.  Of a piece of 32 tile columns a lane holds 4 (two times 4) values of the
  // gate and the up projection's of the same hidden columns.
  static constexpr int pieces_of_step(int mr, int nbk) { return mr == 16 ? nbk : 1; }      // store_backward
  template <int KIND, int EPI, int MR, int NBK>
  static constexpr int staged_bytes() {
    if (EPI == EPI_DGLU) return 3 * 32 * (64 * pieces_of_step(MR, NBK) + 16);
    if (EPI == EPI_GLU || EPI == EPI_GLU_KEEP) return (EPI == EPI_GLU ? 1 : 3) * 32 * (32 * NBK + 16);
    return Ragged::staged_bytes<KIND, EPI_STORE, MR, NBK>();
  }
  template <int KIND, int EPI, int MR, int MB, int NBK, int AM, int AN>
  static __device__ __forceinline__ void store(const Args& p, typename AccBlock<MR>::type (&acc)[AM][AN], char* wave_lds, int g, int mwave,
                                               int mshift, int nbase, const uint32_t (&out_off)[2], int lane) {
    if constexpr (EPI == EPI_STORE || EPI == EPI_GLU_DX) {
      Ragged::store<KIND, EPI_STORE, MR, MB, NBK>(p, acc, wave_lds, g, mwave, mshift, nbase, out_off, lane);
    } else {
      with_act(p.act, [&](auto act) {
        constexpr int ACT = decltype(act)::value;
        if constexpr (EPI == EPI_DGLU) store_backward<ACT, MR, MB, NBK>(p, acc, wave_lds, mshift, nbase, out_off, lane);
        else store_forward<ACT, EPI == EPI_GLU_KEEP, MR, MB, NBK>(p, acc, wave_lds, mshift, nbase, out_off, lane);
      });
    }
  }

  // values 4 q4 .. 4 q4 + 3 of a lane in piece (i, j): row MR (q4 / QG) + lane % MR of the piece's 32
  template <int MR, int AM, int AN>
  static __device__ __forceinline__ float value(typename AccBlock<MR>::type (&acc)[AM][AN], int i, int j, int q4, int e) {
    if constexpr (MR == 32) return acc[i][j][q4 * 4 + e];
    else return acc[2 * i + (q4 >> 1)][2 * j + (q4 & 1)][e];
  }
  // byte offset in the output of a row of the piece (and bit 0: a row of zeros), or OOB
  static __device__ __forceinline__ uint32_t row_offset(const uint32_t (&out_off)[2], int d, int rl) {
    return (uint32_t)__shfl((int)(d < 64 ? out_off[0] : out_off[1]), (d & 63) + rl, 64);
  }

  template <int ACT, bool KEEP, int MR, int MB, int NBK, int AM, int AN>
  static __device__ __forceinline__ void store_forward(const Args& p, typename AccBlock<MR>::type (&acc)[AM][AN], char* wave_lds, int mshift,
                                                       int nbase, const uint32_t (&out_off)[2], int lane) {
    constexpr int CW = 16 * NBK, PITCH = 2 * CW + 16, IMAGE = 32 * PITCH;
    constexpr int LPR = CW / 8, RPI = 64 / LPR, NT = 32 / RPI;
    constexpr int RG = 32 / MR, QG = 4 / RG;
    const int rl = lane / LPR, cc = lane % LPR, ncol = nbase / 2 + cc * 8;
    const uint64_t values = (uint64_t)p.R * (uint64_t)p.half;
    const __amdgpu_buffer_rsrc_t rA = make_rsrc(p.C, (uint32_t)(values * 2)), rZ = make_rsrc(KEEP ? p.C2 : p.C, KEEP ? (uint32_t)(values * 4) : 0u);
#pragma unroll
    for (int i = 0; i < MB; ++i) {
#pragma unroll
      for (int j = 0; j < NBK; ++j)
#pragma unroll
        for (int h = 0; h < RG; ++h)
#pragma unroll
          for (int u = 0; u < QG / 2; ++u) {
            float a[4], gv[4], uv[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              gv[e] = value<MR>(acc, i, j, h * QG + u, e);
              uv[e] = value<MR>(acc, i, j, h * QG + QG / 2 + u, e);
              a[e] = gate_value<ACT, true>(gv[e]) * uv[e];
            }
            char* at = wave_lds + (MR * h + (lane & (MR - 1))) * PITCH + (16 * j + 8 * u + 4 * (lane / MR)) * 2;
            *reinterpret_cast<uint2*>(at) = make_uint2(pack_bf16x2(a[0], a[1]), pack_bf16x2(a[2], a[3]));
            if constexpr (KEEP) {
              *reinterpret_cast<uint2*>(at + IMAGE) = make_uint2(pack_bf16x2(gv[0], gv[1]), pack_bf16x2(gv[2], gv[3]));
              *reinterpret_cast<uint2*>(at + 2 * IMAGE) = make_uint2(pack_bf16x2(uv[0], uv[1]), pack_bf16x2(uv[2], uv[3]));
            }
          }
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const uint32_t o = row_offset(out_off, mshift + i * 32 + RPI * t, rl);
        const bool zero = o != OOB && (o & 1u), ok = o != OOB && ncol < p.half;
        const uint32_t row = o & ~1u;
        const char* at = wave_lds + (RPI * t + rl) * PITCH + cc * 16;
        auto put = [&](const __amdgpu_buffer_rsrc_t& r, uint32_t off, const char* from, auto stream) {
          const uint4 v = *reinterpret_cast<const uint4*>(from);
          stb16<decltype(stream)::value>(r, ok ? off : OOB, zero ? make_uint4(0, 0, 0, 0) : v);
        };
        put(rA, row + (uint32_t)ncol * 2u, at, std::false_type{});
        if constexpr (KEEP) {
          put(rZ, 2u * row + (uint32_t)ncol * 2u, at + IMAGE, std::true_type{});
          put(rZ, 2u * row + (uint32_t)(p.half + ncol) * 2u, at + 2 * IMAGE, std::true_type{});
        }
      }
    }
  }

  // JB pieces at a time: three images of 64 columns are more than a wave's slice of LDS in the tiles with two wave groups
  template <int ACT, int MR, int MB, int NBK, int AM, int AN>
  static __device__ __forceinline__ void store_backward(const Args& p, typename AccBlock<MR>::type (&acc)[AM][AN], char* wave_lds, int mshift,
                                                        int nbase, const uint32_t (&out_off)[2], int lane) {
    constexpr int JB = pieces_of_step(MR, NBK), STEPS = MB * (NBK / JB);
    constexpr int CW = 32 * JB, PITCH = 2 * CW + 16, IMAGE = 32 * PITCH;
    constexpr int LPR = CW / 8, RPI = 64 / LPR, NT = 32 / RPI;
    constexpr int RG = 32 / MR, QG = 4 / RG;
    static_assert(NBK % JB == 0, "pieces of a step");
    const int rl = lane / LPR, cc = lane % LPR;
    const uint64_t values = (uint64_t)p.R * (uint64_t)p.half;
    const __amdgpu_buffer_rsrc_t rA = make_rsrc(p.C, (uint32_t)(values * 2)), rD = make_rsrc(p.C2, (uint32_t)(values * 4)),
                                 rZ = make_rsrc(p.Zin, (uint32_t)(values * 4));
    uint32_t wide[NT];          // byte offset of this lane's 8 columns of g (dG) in the step at hand, or OOB
    uint4 zg[NT], zu[NT];
    auto request = [&](int s) {
      const int i = s / (NBK / JB), ncol = nbase + 32 * JB * (s % (NBK / JB)) + cc * 8;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const uint32_t o = row_offset(out_off, mshift + i * 32 + RPI * t, rl);
        wide[t] = o != OOB && ncol < p.half ? 2u * o + (uint32_t)ncol * 2u : OOB;
        zg[t] = ldb16<true>(rZ, wide[t]);
        zu[t] = ldb16<true>(rZ, wide[t] == OOB ? OOB : wide[t] + (uint32_t)p.half * 2u);
      }
    };
    request(0);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int i = s / (NBK / JB), j0 = JB * (s % (NBK / JB));
      uint32_t to[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        char* at = wave_lds + (RPI * t + rl) * PITCH + cc * 16;
        *reinterpret_cast<uint4*>(at) = zg[t];
        *reinterpret_cast<uint4*>(at + IMAGE) = zu[t];
        to[t] = wide[t];
      }
      if (s + 1 < STEPS) request(s + 1);
#pragma unroll
      for (int j = 0; j < JB; ++j)
#pragma unroll
        for (int h = 0; h < RG; ++h)
#pragma unroll
          for (int u = 0; u < QG; ++u) {
            char* at = wave_lds + (MR * h + (lane & (MR - 1))) * PITCH + (32 * j + (MR == 32 ? 8 : 16) * u + 4 * (lane / MR)) * 2;
            const uint2 gb = *reinterpret_cast<const uint2*>(at), ub = *reinterpret_cast<const uint2*>(at + IMAGE);
            const float gv[4] = {__uint_as_float(gb.x << 16), __uint_as_float(gb.x & 0xFFFF0000u), __uint_as_float(gb.y << 16), __uint_as_float(gb.y & 0xFFFF0000u)};
            const float uv[4] = {__uint_as_float(ub.x << 16), __uint_as_float(ub.x & 0xFFFF0000u), __uint_as_float(ub.y << 16), __uint_as_float(ub.y & 0xFFFF0000u)};
            float dg[4], du[4], av[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float d = value<MR>(acc, i, j0 + j, h * QG + u, e);
              float a, da;
              gate_and_slope<ACT, true>(gv[e], a, da);
              dg[e] = d * uv[e] * da;
              du[e] = d * a;
              av[e] = a * uv[e];
            }
            *reinterpret_cast<uint2*>(at) = make_uint2(pack_bf16x2(dg[0], dg[1]), pack_bf16x2(dg[2], dg[3]));
            *reinterpret_cast<uint2*>(at + IMAGE) = make_uint2(pack_bf16x2(du[0], du[1]), pack_bf16x2(du[2], du[3]));
            *reinterpret_cast<uint2*>(at + 2 * IMAGE) = make_uint2(pack_bf16x2(av[0], av[1]), pack_bf16x2(av[2], av[3]));
          }
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const char* at = wave_lds + (RPI * t + rl) * PITCH + cc * 16;
        const uint32_t ncol2 = (uint32_t)(nbase + 32 * j0 + cc * 8) * 2u;
        stb16(rD, to[t], *reinterpret_cast<const uint4*>(at));
        stb16(rD, to[t] == OOB ? OOB : to[t] + (uint32_t)p.half * 2u, *reinterpret_cast<const uint4*>(at + IMAGE));
        stb16(rA, to[t] == OOB ? OOB : (to[t] - ncol2) / 2u + ncol2, *reinterpret_cast<const uint4*>(at + 2 * IMAGE));
      }
    }
  }
};

template <int KIND, int EPI, typename CF>
__global__ __launch_bounds__(64 * CF::NW) void glu_gemm_dma(const RaggedArgs p) {
  __shared__ __attribute__((aligned(1024))) char smem[CF::LDS];
  gemm_dma_tile<KIND, EPI, CF, ROWS_PLAIN, Glu>(p, smem, (int)blockIdx.x);
}

using Tile256Brief = TileCfg<256, 256, 2, 4, 1, 3, 2, 32>;

// dX, dW2 and the gate's and the up projection's half of dW1, which only depend on dG, dU and A', in one launch; the last two read X's rows
template <typename CFX, typename CFW, int EPI>
__global__ __launch_bounds__(512) void glu_bwd_quad(const RaggedArgs px, const RaggedArgs pw2, const RaggedArgs pwg, const RaggedArgs pwu, int nbx, int nb2,
                                                    int nb1) {
  static_assert(CFX::NW == 8 && CFW::NW == 8, "one block size");
  __shared__ __attribute__((aligned(1024))) char smem[CFX::LDS > CFW::LDS ? CFX::LDS : CFW::LDS];
  const int b = (int)blockIdx.x;
  if (b < nbx) {
    gemm_dma_tile<KIND_NT, EPI_GLU_DX, CFX, ROWS_PLAIN, Glu>(px, smem, b);
  } else if (b < nbx + nb2) {
    gemm_dma_tile<KIND_TN, EPI, CFW, ROWS_PLAIN, Glu>(pw2, smem, b - nbx);
  } else {
    const int c = b - nbx - nb2;
    gemm_dma_tile<KIND_TN, EPI, CFW, ROWS_GATHER, Glu>(c < nb1 ? pwg : pwu, smem, c < nb1 ? c : c - nb1);
  }
}

namespace {

template <int KIND, int EPI>
void launch_glu(RaggedArgs a, int dtype, hipStream_t st) {
  if (dtype == MOE_F32) {
    launch_f32<KIND, EPI>(a, st);
    return;
  }
  buffer_sizes(a, false);
  auto launch = [&](auto cfg) {
    using CF = decltype(cfg);
    const dim3 grid = size_rows(a, CF::TM, CF::TN, false);
    hipLaunchKernelGGL((glu_gemm_dma<KIND, EPI, CF>), grid, dim3(64 * CF::NW), 0, st, a);
  };
  const TilePlan t = plan_rows(a);
  if (t.tile_m == 256) launch(Tile256{});
  else if (t.tile_m == 192) launch(Tile192{});
  else if (t.tile_m == 128) launch(Tile128{});
  else if (t.tile_m == 64 && t.tile_n == 128) launch(Tile64x128{});
  else if (t.tile_m == 64) launch(Tile64{});
  else launch(Tile32x64{});
}

// parts of the three weight gradients' reductions: dW2 and the halves of dW1 are of one size
int glu_parts(int dtype, int64_t R, int E, int M, int Hl) { return weight_parts(dtype, R, E, M, Hl, 3); }
size_t glu_part_bytes(int parts, int E, int M, int Hl) { return 3 * part_bytes(parts, E, M, Hl); }

void launch_glu_backward(RaggedArgs dx, RaggedArgs w2, RaggedArgs wg, RaggedArgs wu, int dtype, float* parts, hipStream_t st) {
  if (w2.splits > 1) {
    const size_t size = part_bytes(w2.splits, w2.G, w2.Mdim, w2.Ndim) / 4;
    w2.part = parts;
    wg.part = parts + size;
    wu.part = parts + 2 * size;
  }
  if (dtype == MOE_F32) {
    launch_glu_bwd_f32(dx, w2, wg, wu, st);
  } else {
    buffer_sizes(dx, false); buffer_sizes(w2, true); buffer_sizes(wg, true); buffer_sizes(wu, true);
    wu.b_bytes -= (uint64_t)wu.half * 2;      // B starts behind the first row's dG
    auto launch = [&](auto cfx, auto cfw, auto epi) {
      using CFX = decltype(cfx);
      using CFW = decltype(cfw);
      const unsigned nbx = size_rows(dx, CFX::TM, CFX::TN, true).x;
      const unsigned nb2 = size_weights(w2, CFW::TM).x * w2.splits, nb1 = size_weights(wg, CFW::TM).x * wg.splits;
      size_weights(wu, CFW::TM);
      hipLaunchKernelGGL((glu_bwd_quad<CFX, CFW, decltype(epi)::value>), dim3(nbx + nb2 + 2 * nb1), dim3(512), 0, st, dx, w2, wg, wu, (int)nbx, (int)nb2,
                         (int)nb1);
    };
    using Store = std::integral_constant<int, EPI_STORE>;
    if (small_weights(w2.G, w2.Mdim, w2.Ndim)) {
      if (w2.splits > 1) launch(Tile64x128{}, Tile128{}, std::integral_constant<int, EPI_PART>{});
      else launch(Tile64x128{}, Tile128{}, Store{});
    } else {
      // A compute unit holds one workgroup of this launch whatever its tile (the LDS of a 256 x 256 one), so the tile of 192 rows gains nothing: dX in tiles of
      // 192 and of 256 rows, 8 experts of 1024 rows x 1024 x 4096 475 and 437 us, 2 of 2048 x 2048 x 8192 728 and 666.  The weight gradients take 32 x 32 x 16
      // instructions; with 16 x 16 x 32 ones the call is within 2 % of it either way, us with these and with those: 8 experts x 1024 x 4096 of 1024, 4096, 8192
      // and 16384 rows each 490 and 481, 1560 and 1555, 3005 and 3041, 6014 and 6010; 4 x 4096 x 7168 of 2048, 4096, 8192 and 16384 2437 and 2418, 4606 and
      // 4624, 8957 and 9022, 17961 and 18053; 8 x 4096 x 7168 of 4096 9216 and 9307; 1 x 1024 x 2816 of 4096 and 32768 208 and 210, 1852 and 1858.
      const TilePlan t = plan_rows(dx, true);
      if (t.tile_m >= 192) launch(Tile256{}, Tile256Brief{}, Store{});
      else if (t.tile_m == 128) launch(Tile128{}, Tile256Brief{}, Store{});
      else launch(Tile64x128{}, Tile256Brief{}, Store{});
    }
  }
  if (w2.splits > 1) {
    add_parts(w2, wg, 2, dtype, st);
    add_parts(wu, wu, 1, dtype, st);
  }
}

// The kernels for few rows: as for the FFN with one projection, their number has a bound because an expert's weights are read again for every 16 of them.
// Tiles and this, forward call: 2 rows, 8 experts x 1024 x 4096 26.4 and 19.9 us, 8 x 4096 x 14336 166 and 131; 64 rows 57.5 and 50.1, 567 and 509; but with
// few weights the tiles' two launches are shorter, 2 rows of 64 x 2048 x 2048 24.0 and 24.6, 16 rows of 1 x 1024 x 2816 21.0 and 23.2, 32 rows of
// 8 x 512 x 1536 18.9 and 19.3.  With fewer hidden columns there is less to gain than to lose: tiles and this, equal shares, and one expert with all rows, 2 rows of
// 16 x 7168 x 2048 74 and 76, 45 and 45, 32 rows 281 and 246, 50 and 128; 2 and 32 rows of 64 x 4096 x 1536 32 and 35, 31 and 33, 242 and 230, 35 and 95;
// 32 rows of 64 x 2048 x 1024 89 and 81, 22 and 48, of 8 x 4096 x 4096 170 and 146, 42 and 90.  Within the rule the widest loss of this kind, 64 rows of
// 8 x 1024 x 4096, is 57 and 48, 26 and 67.
bool few_rows_glu(int dtype, int64_t R, int E, int M, int Hl) {
  return dtype == MOE_BF16 && (R <= 32 || (R <= 64 && R <= 8 * (int64_t)E)) && Hl >= 2 * (int64_t)M && std::min<int64_t>(R, E) * M * Hl >= 1 << 23;
}

int check_glu(int dtype, int64_t R, int E, int M, int H, int esp_idx, int n_esp) {
  MOE_REQUIRE(M >= 1 && H >= 1 && n_esp >= 1 && esp_idx >= 0 && esp_idx < n_esp && H % n_esp == 0, MOE_EINVAL);
  MOE_REQUIRE(H <= 1 << 28, MOE_EUNSUPPORTED);      // 2 H and its tiles are counted in 32 bits
  const int Hl = H / n_esp;
  if (int rc = check_rows(dtype, R, E, std::max(M, 2 * Hl))) return rc;
  MOE_REQUIRE(M % 8 == 0 && Hl % 8 == 0, MOE_EUNSUPPORTED);
  if (dtype == MOE_BF16) MOE_REQUIRE((uint64_t)M * H * 4 <= 0xFFFFFFF0ull, MOE_EUNSUPPORTED);
  return MOE_OK;
}
size_t dz_bytes(int dtype, int64_t R, int Hl) { return hidden_bytes(dtype, R, 2 * Hl); }

}  // namespace
}  // namespace moe

using namespace moe;

extern "C" size_t moe_ragged_glu_workspace_bytes(int dtype, int64_t R, int E, int M, int H, int n_esp, int backward) {
  if (check_glu(dtype, R, E, M, H, 0, n_esp) != MOE_OK) return 0;
  const int Hl = H / n_esp;
  if (backward) return dz_bytes(dtype, R, Hl) + hidden_bytes(dtype, R, Hl) + glu_part_bytes(glu_parts(dtype, R, E, M, Hl), E, M, Hl);
  return few_rows_glu(dtype, R, E, M, Hl) ? few_rows_bytes(R, E, M, Hl) : row_part_bytes(row_parts(dtype, R, E, Hl, M), R, M);
}

extern "C" int moe_ragged_glu_fwd(const void* x, int dtype, int64_t S, const int32_t* inv, int k, const void* W1, const void* W2,
                                  const int32_t* offsets, int64_t R, int E, int M, int H, int esp_idx, int n_esp, int act, void* Z,
                                  void* A, void* Y, void* ws, size_t ws_bytes, void* stream) {
  if (int rc = check_glu(dtype, R, E, M, H, esp_idx, n_esp)) return rc;
  MOE_REQUIRE(act == MOE_ACT_SILU || act == MOE_ACT_GELU, MOE_EINVAL);
  if (int rc = check_source(x, dtype, S, inv, k, M)) return rc;
  MOE_REQUIRE_PTR(W1); MOE_REQUIRE_PTR(W2); MOE_REQUIRE_PTR(offsets); MOE_REQUIRE_PTR(A); MOE_REQUIRE_PTR(Y);
  MOE_OPTIONAL_PTR(Z); MOE_OPTIONAL_PTR(ws);
  hipStream_t st = (hipStream_t)stream;
  const int Hl = H / n_esp;
  const int64_t h0 = (int64_t)esp_idx * Hl;
  RaggedArgs a = base_args(offsets, R, E);
  set_gather(a, inv, k, S);
  a.A = x; a.lda = M;
  a.B = W1; a.ldb = 2 * (int64_t)H; a.b_goff = (int64_t)M * 2 * H; a.b_off = h0;
  a.C = A; a.C2 = Z; a.ldc = Hl;
  a.Mdim = a.R; a.Ndim = 2 * Hl; a.Kdim = M;
  a.half = Hl; a.up = H; a.act = act;
  RaggedArgs y = base_args(offsets, R, E);
  y.A = A; y.lda = Hl;
  y.B = W2; y.ldb = M; y.b_goff = (int64_t)H * M; y.b_off = h0 * M;
  y.C = Y; y.ldc = M;
  y.Mdim = y.R; y.Ndim = M; y.Kdim = Hl;
  if (Z == nullptr && few_rows_glu(dtype, R, E, M, Hl) && ws != nullptr && ws_bytes >= few_rows_bytes(R, E, M, Hl)) {
    buffer_sizes(a, false);
    buffer_sizes(y, false);
    launch_few_rows(a, y, true, ws, st);
    return check_launch();
  }
  if (Z) launch_glu<KIND_NN, EPI_GLU_KEEP>(a, dtype, st);
  else launch_glu<KIND_NN, EPI_GLU>(a, dtype, st);
  launch_second(y, dtype, ws, ws_bytes, st);
  return check_launch();
}

extern "C" int moe_ragged_glu_bwd(const void* dY, const void* x, int dtype, int64_t S, const int32_t* inv, int k, const void* Z, const void* W1,
                                  const void* W2, const int32_t* offsets, int64_t R, int E, int M, int H, int esp_idx, int n_esp, int act,
                                  void* dX, void* dW1, void* dW2, void* ws, size_t ws_bytes, void* stream) {
  if (int rc = check_glu(dtype, R, E, M, H, esp_idx, n_esp)) return rc;
  MOE_REQUIRE(act == MOE_ACT_SILU || act == MOE_ACT_GELU, MOE_EINVAL);
  MOE_REQUIRE_PTR(dY);
  if (int rc = check_source(x, dtype, S, inv, k, M)) return rc;
  MOE_REQUIRE_PTR(Z); MOE_REQUIRE_PTR(W1); MOE_REQUIRE_PTR(W2); MOE_REQUIRE_PTR(offsets);
  MOE_REQUIRE_PTR(dX); MOE_REQUIRE_PTR(dW1); MOE_REQUIRE_PTR(dW2);
  const int Hl = H / n_esp, parts = glu_parts(dtype, R, E, M, Hl);
  const size_t dz = dz_bytes(dtype, R, Hl), hidden = hidden_bytes(dtype, R, Hl);
  MOE_REQUIRE(ws != nullptr && ws_bytes >= dz + hidden + glu_part_bytes(parts, E, M, Hl), MOE_EWORKSPACE);
  MOE_REQUIRE(aligned16(ws), MOE_EALIGN);
  hipStream_t st = (hipStream_t)stream;
  const int64_t h0 = (int64_t)esp_idx * Hl, esz = dtype == MOE_BF16 ? 2 : 4;
  void* dZ = ws;
  void* Act = (char*)ws + dz;

  // dZ = [dG | dU] and Act = act(g) u, from dA = dY W2^T
  RaggedArgs a = base_args(offsets, R, E);
  a.A = dY; a.lda = M;
  a.B = W2; a.ldb = M; a.b_goff = (int64_t)H * M; a.b_off = h0 * M;
  a.C = Act; a.C2 = dZ; a.Zin = Z; a.ldc = Hl;
  a.Mdim = a.R; a.Ndim = Hl; a.Kdim = M;
  a.half = Hl; a.up = H; a.act = act;
  launch_glu<KIND_NT, EPI_DGLU>(a, dtype, st);
  // dX = dZ W1^T
  RaggedArgs dx = base_args(offsets, R, E);
  dx.A = dZ; dx.lda = 2 * (int64_t)Hl;
  dx.B = W1; dx.ldb = 2 * (int64_t)H; dx.b_goff = (int64_t)M * 2 * H; dx.b_off = h0;
  dx.C = dX; dx.ldc = M;
  dx.Mdim = dx.R; dx.Ndim = M; dx.Kdim = 2 * Hl;
  dx.half = Hl; dx.up = H;
  // dW2[h0:h0+Hl, :] = Act^T dY
  RaggedArgs w2 = base_args(offsets, R, E);
  w2.A = Act; w2.lda = Hl;
  w2.B = dY; w2.ldb = M;
  w2.C = dW2; w2.ldc = M; w2.c_goff = (int64_t)H * M; w2.c_off = h0 * M;
  w2.Mdim = Hl; w2.Ndim = M; w2.Kdim = w2.R;
  w2.splits = parts;
  // the gate's half of dW1, X^T dG, and the up projection's, X^T dU
  RaggedArgs wg = base_args(offsets, R, E);
  set_gather(wg, inv, k, S);
  if (inv == nullptr) { wg.gather_k = 1; wg.gather_rows = R; }      // Glu::in_order
  wg.A = x; wg.lda = M;
  wg.B = dZ; wg.ldb = 2 * (int64_t)Hl;
  wg.C = dW1; wg.ldc = 2 * (int64_t)H; wg.c_goff = (int64_t)M * 2 * H; wg.c_off = h0;
  wg.Mdim = M; wg.Ndim = Hl; wg.Kdim = wg.R;
  wg.splits = parts;
  wg.half = Hl;
  RaggedArgs wu = wg;
  wu.B = (const char*)dZ + Hl * esz;
  wu.c_off = H + h0;
  launch_glu_backward(dx, w2, wg, wu, dtype, (float*)((char*)ws + dz + hidden), st);
  return check_launch();
}
