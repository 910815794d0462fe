// Layout of the tiles over ragged rows (ragged.hip: the products and the GeLU FFN; glu.hip: the gated FFN), and what their host sides share.
#pragma once

#include "ckpt8.h"
#include "ragged.h"

namespace moe {

// ------------------------------------------------------------------------------------------
// layout of the tiles
// ------------------------------------------------------------------------------------------
struct Ragged : PlainOrder {
  using Args = RaggedArgs;
  using Place = RaggedPlace;

  template <int KIND, int EPI, int ESZ, int TM, int TN>
  static __device__ __forceinline__ bool find(const Args& p, int vb, Place& at) { return find_tile<KIND, EPI, ESZ, TM, TN>(p, vb, at); }
  template <int TM, int RA>
  static __device__ __forceinline__ void rows(const Args& p, const Place& at, int q0, int w0, int (&q_row)[RA], uint32_t (&out_off)[2]) {
    int r[RA + 2], row[RA + 2];
#pragma unroll
    for (int j = 0; j < RA + 2; ++j) {
      r[j] = j < RA ? q0 + 8 * j : w0 + 64 * (j - RA);
      row[j] = r[j] < at.n ? at.lo + r[j] : -1;
    }
    bool zero[2] = {false, false};
    if (p.gather != nullptr) {
      int iv[RA + 2];
#pragma unroll
      for (int j = 0; j < RA + 2; ++j) iv[j] = p.gather[at.lo + min(r[j], at.n - 1)];
#pragma unroll
      for (int j = 0; j < RA + 2; ++j) {
        const int tok = token(p, iv[j]);
        if (j < RA) row[j] = row[j] >= 0 ? tok : -1;
        else zero[j - RA] = tok < 0;
      }
    }
#pragma unroll
    for (int j = 0; j < RA; ++j) q_row[j] = max(row[j], 0);      // no row: any row of the tensor
#pragma unroll
    for (int j = 0; j < 2; ++j)
      if (row[RA + j] >= 0) out_off[j] = (uint32_t)row[RA + j] * (uint32_t)p.ldc * 2u + (zero[j] ? 1u : 0u);
  }
  template <int TM>
  static __device__ __forceinline__ void rows_f32(const Args& p, const Place& at, int, int ra, int ro, int& a_row, int& o_row,
                                                  bool& o_zero) {
    a_row = at.lo + min(ra, at.n - 1);     // a row behind the expert's last one: that one, its results are not stored
    o_row = ro < at.n ? at.lo + ro : -1;
    o_zero = false;
    if (p.gather != nullptr) {
      a_row = max(token(p, p.gather[a_row]), 0);
      o_zero = token(p, p.gather[at.lo + min(ro, at.n - 1)]) < 0;
    }
  }
  // The reduction of a weight gradient: the expert's rows, which lie together.  Parts of a split reduction are consecutive runs of k tiles.
  template <bool PARTS>
  struct Walk {
    int row, left, part, splits;
    __device__ __forceinline__ Walk(const Args& p, const Place& at, int part_) : row(at.lo), left(at.n), part(part_), splits(p.splits) {}
    __device__ __forceinline__ int start(int step, bool) {
      int nk = (left + step - 1) / step;
      if (PARTS) {
        const int t0 = (int)((int64_t)nk * part / splits), t1 = (int)((int64_t)nk * (part + 1) / splits);
        row += t0 * step;
        left = min(left - t0 * step, (t1 - t0) * step);
        nk = t1 - t0;
      }
      return nk;
    }
    __device__ __forceinline__ void skip(int) {}
    __device__ __forceinline__ KTile next(int step) {
      if (left <= 0) return KTile{0, 0};
      const KTile t{row, min(left, step)};
      row += step;
      left -= step;
      return t;
    }
  };
  static __device__ __forceinline__ uint32_t map_bytes(const Args& p) { return (uint32_t)p.R * 4u; }

  // Epilogue of the bf16 tile, staged through the wave's slice of LDS as in the padded calls: 32 rows at a time in accumulator order
  // into [32][CW] images of the outputs, read back row by row and stored 16 bytes (8-bit values: 8 bytes) a lane.  The 32 columns of a
  // block of the 8-bit form are 32 columns of one wave's tile: their largest magnitude is 8 or 16 values of a lane and one or
  // two exchanges between lanes.
  template <int KIND, int EPI, int MR, int NBK>
  static constexpr int staged_bytes() { return 32 * (64 * NBK + 16) * (EPI == EPI_GELU8 || EPI == EPI_DGELU8 ? 2 : 1); }
  template <int KIND, int EPI, int MR, int MB, int NBK, int AM, int AN>
  static __device__ __forceinline__ void store(const Args& p, typename AccBlock<MR>::type (&acc)[AM][AN], char* wave_lds, int g,
                                               int mwave, int mshift, int nbase, const uint32_t (&out_off)[2], int lane) {
    constexpr bool Q_OUT = EPI == EPI_GELU8, Q_IN = EPI == EPI_DGELU8;
    constexpr int CW = 32 * NBK, PITCH = 2 * CW + 16, PITCH8 = CW + 8;
    constexpr int LPR = CW / 8, RPI = 64 / LPR, NT = 32 / RPI;   // lanes per row, rows per instruction, instructions (row-wise phase)
    constexpr int RG = 32 / MR, QG = 4 / RG;                     // row groups of a 32 x 32 piece, a lane's groups of 4 columns in each
    char* buf0 = wave_lds;                    // first output (8-bit values on their way in)
    char* buf1 = wave_lds + 32 * PITCH;       // second output
    const int rl = lane / LPR, cc = lane % LPR, ncol = nbase + cc * 8;
    const bool col_ok = ncol < p.Ndim;
    __amdgpu_buffer_rsrc_t rC, rQ, rS, rC2;
    if (KIND == KIND_TN) {
      rC = make_rsrc(reinterpret_cast<bf16_t*>(p.C) + ((int64_t)g * p.c_goff + p.c_off),
                     (uint32_t)(((int64_t)(p.Mdim - 1) * p.ldc + p.Ndim) * 2));
      rQ = rS = rC2 = rC;
    } else {
      const uint64_t values = (uint64_t)p.R * (uint64_t)p.ldc;
      rC = make_rsrc(p.C, (uint32_t)(values * 2));
      rQ = make_rsrc(Q_OUT ? p.C2 : Q_IN ? p.Zin : p.C, Q_OUT || Q_IN ? (uint32_t)values : 0u);
      rS = make_rsrc(p.Zs, Q_OUT || Q_IN ? (uint32_t)p.R * (uint32_t)p.ldz : 0u);
      rC2 = make_rsrc(p.C2, Q_IN ? (uint32_t)(values * 2) : 0u);
    }
    uint32_t off[MB][NT];      // bf16 byte offset of this lane's 8 columns (row-wise phase), or OOB; even: bit 0 marks a row of zeros
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const int d = mshift + i * 32 + RPI * t;
        if (KIND == KIND_TN) {
          off[i][t] = mwave + d + rl < p.Mdim && col_ok ? ((uint32_t)(mwave + d + rl) * (uint32_t)p.ldc + (uint32_t)ncol) * 2u : OOB;
        } else {
          const uint32_t o = (uint32_t)__shfl((int)(d < 64 ? out_off[0] : out_off[1]), (d & 63) + rl, 64);
          off[i][t] = o != OOB && col_ok ? o + (uint32_t)ncol * 2u : OOB;
        }
      }
    auto half = [](uint32_t o) { return o == OOB ? OOB : o >> 1; };       // the same place in the 8-bit values
    // scales of this lane's row (accumulator order, group h of block i): offset of the first of its NBK blocks (+ S_ZERO: a row of zeros, whose
    // accumulators are another row's), or OOB; offsets are under 2^28, a block being 8 columns at least
    constexpr uint32_t S_ZERO = 1u << 30;
    uint32_t s_off[Q_OUT || Q_IN ? MB : 1][RG];
    if constexpr (Q_OUT || Q_IN) {
      uint32_t mine[2];
#pragma unroll
      for (int u = 0; u < 2; ++u)
        mine[u] = out_off[u] == OOB ? OOB
                                    : ((out_off[u] >> 1) / (uint32_t)p.ldc * (uint32_t)p.ldz + (uint32_t)(nbase >> 5)) | (Q_OUT && (out_off[u] & 1u) ? S_ZERO : 0u);
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int h = 0; h < RG; ++h) {
          const int d = mshift + i * 32 + MR * h;
          s_off[i][h] = (uint32_t)__shfl((int)(d < 64 ? mine[0] : mine[1]), (d & 63) + (lane & (MR - 1)), 64);
        }
    }
    auto s_at = [&](int i, int h, int j) -> uint32_t {
      return s_off[i][h] != OOB && nbase + 32 * j < p.Ndim ? (Q_OUT ? s_off[i][h] & ~S_ZERO : s_off[i][h]) + j : OOB;
    };
    u32x2_t q_next[Q_IN ? NT : 1];
    uint32_t s_next[RG][NBK];
    auto request = [&](int i) {
#pragma unroll
      for (int t = 0; t < NT; ++t) q_next[Q_IN ? t : 0] = __builtin_amdgcn_raw_buffer_load_b64(rQ, (int)half(off[i][t]), 0, 2);
#pragma unroll
      for (int h = 0; h < RG; ++h)
#pragma unroll
        for (int j = 0; j < NBK; ++j) s_next[h][j] = __builtin_amdgcn_raw_buffer_load_b8(rS, (int)s_at(i, h, j), 0, 0);
    };
    if constexpr (Q_IN) request(0);
    static_assert(AM == MB * 32 / MR && AN == NBK * 32 / MR, "accumulator blocks of the wave tile");
    auto value = [&](int i, int j, int q4, int e) -> float {
      if constexpr (MR == 32) return acc[i][j][q4 * 4 + e];
      else return acc[2 * i + (q4 >> 1)][2 * j + (q4 & 1)][e];
    };
    // row group h, group u of 4 columns: row MR h + lane % MR, columns col_of(u) + 0..3 of the piece
    auto col_of = [&](int u) { return (MR == 32 ? 8 : 16) * u + 4 * (lane / MR); };
#pragma unroll
    for (int i = 0; i < MB; ++i) {
      uint32_t qv[NBK][4], sv[RG][NBK];
      if constexpr (Q_IN) {
#pragma unroll
        for (int t = 0; t < NT; ++t) *reinterpret_cast<u32x2_t*>(buf0 + (RPI * t + rl) * PITCH8 + cc * 8) = q_next[t];
#pragma unroll
        for (int h = 0; h < RG; ++h)
#pragma unroll
          for (int j = 0; j < NBK; ++j) sv[h][j] = s_next[h][j];
        if (i + 1 < MB) request(i + 1);
#pragma unroll
        for (int j = 0; j < NBK; ++j)
#pragma unroll
          for (int h = 0; h < RG; ++h)
#pragma unroll
            for (int u = 0; u < QG; ++u)
              qv[j][h * QG + u] = *reinterpret_cast<const uint32_t*>(buf0 + (MR * h + (lane & (MR - 1))) * PITCH8 + 32 * j + col_of(u));
      }
#pragma unroll
      for (int j = 0; j < NBK; ++j)
#pragma unroll
        for (int h = 0; h < RG; ++h) {
          const int row = MR * h + (lane & (MR - 1));
          int b = 0;
          if constexpr (Q_OUT) {
            uint32_t top = 0;
#pragma unroll
            for (int u = 0; u < QG; ++u) {
              uint32_t t = 0;
#pragma unroll
              for (int e = 0; e < 4; ++e) t = max(t, __float_as_uint(value(i, j, h * QG + u, e)) & 0x7FFFFFFFu);
              top = max(top, nbase + 32 * j + col_of(u) < p.Ndim ? t : 0u);    // a column outside the problem counts for nothing
            }
#pragma unroll
            for (int d = MR; d < 64; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d, 64));
            b = s_off[i][h] & S_ZERO ? 0 : ckpt8_scale(top);
            if (lane < MR) __builtin_amdgcn_raw_buffer_store_b8((unsigned char)b, rS, (int)s_at(i, h, j), 0, 2);
          } else if constexpr (Q_IN) {
            b = (int)sv[h][j];
          }
#pragma unroll
          for (int u = 0; u < QG; ++u) {
            const int q4 = h * QG + u;
            const float v[4] = {value(i, j, q4, 0), value(i, j, q4, 1), value(i, j, q4, 2), value(i, j, q4, 3)};
            char* a0 = buf0 + row * PITCH + (32 * j + col_of(u)) * 2;
            float w[4];
            if constexpr (EPI == EPI_STORE) {
#pragma unroll
              for (int e = 0; e < 4; ++e) w[e] = v[e];
            } else if constexpr (EPI == EPI_ACT || Q_OUT) {
#pragma unroll
              for (int e = 0; e < 4; ++e) w[e] = gelu_fast(v[e]);
              if constexpr (Q_OUT) *reinterpret_cast<uint32_t*>(buf1 + row * PITCH8 + 32 * j + col_of(u)) = ckpt8_pack(v, b);
            } else {
              float a[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                float dg;
                gelu_and_grad_fast(ckpt8_value(qv[j][q4], e, b), a[e], dg);
                w[e] = v[e] * dg;
              }
              *reinterpret_cast<uint2*>(buf1 + row * PITCH + (32 * j + col_of(u)) * 2) = make_uint2(pack_bf16x2(a[0], a[1]), pack_bf16x2(a[2], a[3]));
            }
            *reinterpret_cast<uint2*>(a0) = make_uint2(pack_bf16x2(w[0], w[1]), pack_bf16x2(w[2], w[3]));
          }
        }
      // row-wise read-back and store (LDS operations of one wave complete in program order)
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const bool zero = KIND != KIND_TN && (off[i][t] & 1u) && off[i][t] != OOB;
        const uint32_t o = off[i][t] & ~1u;
        const uint4 none = make_uint4(0, 0, 0, 0);
        const uint4 v = *reinterpret_cast<const uint4*>(buf0 + (RPI * t + rl) * PITCH + cc * 16);
        stb16<KIND == KIND_TN>(rC, o, zero ? none : v);
        if constexpr (Q_OUT) {
          u32x2_t q = *reinterpret_cast<const u32x2_t*>(buf1 + (RPI * t + rl) * PITCH8 + cc * 8);
          if (zero) q = u32x2_t{0u, 0u};
          __builtin_amdgcn_raw_buffer_store_b64(q, rQ, (int)half(off[i][t]), 0, 2);
        } else if constexpr (Q_IN) {
          stb16(rC2, o, *reinterpret_cast<const uint4*>(buf1 + (RPI * t + rl) * PITCH + cc * 16));
        }
      }
    }
  }

  // Bits of |z| rounded towards zero: ckpt8_scale's borders are fp32 values, so it decides them as for z itself.  What fp32's own
  // rounding makes an infinity stays one.
  static __device__ __forceinline__ uint32_t magnitude_below(double z) {
    const float f = fabsf((float)z);
    const uint32_t bits = __float_as_uint(f);
    return bits < 0x7F800000u && (double)f > fabs(z) ? bits - 1u : bits;
  }
  // Epilogue of the fp32 tile: lane l holds D[4 r + l / 16][l % 16] of its blocks of 16 columns, in fp64.  For the 8-bit form the tile
  // goes through LDS, because two waves share a row where the k halves are split; values and scales are formed from the fp64 sums, whose rounding to
  // fp32 could move one across the border between two steps.
  template <int KIND, int EPI, int TM, int TN, int KW>
  static __device__ __forceinline__ void store_f32(const Args& p, const f64x4_t (&acc)[TN / 16], double* Bs, int g, int m0, int n0,
                                                   int rw, int kw, int lane, int o_row, bool o_zero) {
    constexpr int NJ = TN / 16;
    float* __restrict__ C = reinterpret_cast<float*>(p.C);
    constexpr int PITCH = TN + 1, UNITS = TM * TN / 32, TPU = 256 / UNITS, CPT = 32 / TPU;   // blocks; threads and columns of each
    static_assert(EPI == EPI_GELU8, "the other products are on the fp32 matrix cores");
    static_assert(TM * PITCH * 8 <= f32_lds<TM, TN>() && CPT % 4 == 0, "the tile fits in the buffers");
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int j = 0; j < NJ / KW; ++j) Bs[(rw * 16 + 4 * r + (lane >> 4)) * PITCH + 16 * (KW * j + kw) + (lane & 15)] = acc[j][r];
    __syncthreads();
    const int tid = threadIdx.x, unit = tid / TPU, ml = unit / (TN / 32), c0 = unit % (TN / 32) * 32 + tid % TPU * CPT;
    const int row = __shfl(o_row, ml & 63, 64), n = n0 + c0;
    const bool zero = __shfl((int)o_zero, ml & 63, 64) != 0;
    double z[CPT];
    uint32_t top = 0;
#pragma unroll
    for (int u = 0; u < CPT; ++u) {
      z[u] = zero || n + u >= p.Ndim ? 0.0 : Bs[ml * PITCH + c0 + u];
      top = max(top, magnitude_below(z[u]));
    }
#pragma unroll
    for (int d = 1; d < TPU; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d, 64));
    const int b = ckpt8_scale(top);
    if (row < 0) return;
#pragma unroll
    for (int u = 0; u < CPT; u += 4) {
      if (n + u >= p.Ndim) break;
      float4 a;
      a.x = gelu_f((float)z[u]); a.y = gelu_f((float)z[u + 1]); a.z = gelu_f((float)z[u + 2]); a.w = gelu_f((float)z[u + 3]);
      *reinterpret_cast<float4*>(C + (int64_t)row * p.ldc + n + u) = a;
      const double q[4] = {z[u], z[u + 1], z[u + 2], z[u + 3]};
      *reinterpret_cast<uint32_t*>(reinterpret_cast<uint8_t*>(p.C2) + (int64_t)row * p.ldc + n + u) = ckpt8_pack(q, b);
    }
    if (tid % TPU == 0 && n < p.Ndim) p.Zs[(int64_t)row * p.ldz + (n >> 5)] = (uint8_t)b;
  }
};

template <int KIND, int EPI, typename CF, int ROWS = ROWS_PLAIN>
__global__ __launch_bounds__(64 * CF::NW) void ragged_ffn_gemm_dma(const RaggedArgs p) {
  __shared__ __attribute__((aligned(1024))) char smem[CF::LDS];
  gemm_dma_tile<KIND, EPI, CF, ROWS, Ragged>(p, smem, (int)blockIdx.x);
}

// ---- host side ----
inline void buffer_sizes(RaggedArgs& a, bool weights) {
  a.a_bytes = (a.gather ? (uint64_t)a.gather_rows : (uint64_t)a.R) * (uint64_t)a.lda * 2;
  a.b_bytes = weights ? (uint64_t)a.R * (uint64_t)a.ldb * 2 : (uint64_t)a.G * (uint64_t)a.b_goff * 2;
}

// the tile of a bf16 row-tiled GEMM (ragged.hip); wide: only tiles of eight waves
TilePlan rows_tile(int R, int E, int K, int N, bool wide);
inline TilePlan plan_rows(const RaggedArgs& a, bool wide = false) { return rows_tile(a.R, a.G, a.Kdim, a.Ndim, wide); }

// An fp32 product over rows with few tiles and a long reduction is cut into parts too, of at least ROW_PART_CHUNKS chunks of 32 k: 8 experts of
// 256 rows x 2048 x 512 96 us whole, 68 in parts and 5 for adding them.
constexpr int CHIP_CUS = 256;   // compute units of an MI355X
constexpr int ROW_PART_CHUNKS = 8;
inline int row_parts(int dtype, int64_t R, int E, int K, int N) {
  if (dtype != MOE_F32) return 1;
  const double tiles = priced_row_tiles((int)R, E, F32_TILE) * ((N + F32_TILE - 1) / F32_TILE);
  const int parts = std::min({(int)(4 * CHIP_CUS / std::max(tiles, 1.0)), K / KC / ROW_PART_CHUNKS, 16});
  return parts < 2 ? 1 : parts;
}
inline size_t row_part_bytes(int parts, int64_t R, int N) { return parts > 1 ? align_up((size_t)parts * R * N * 4, 256) : 0; }

// Weight gradients.  Tiles of 128 x 128 where those of 256 x 256 would be fewer than 64; of fp32, 64 x 64.  With few tiles a reduction over
// thousands of rows is what a launch waits for: it is cut into parts of at least PART_TILES k tiles of an expert's mean share of the
// rows, as many as the chip has room for (two workgroups of 128 x 128, four of fp32, to a compute unit).  Whole and in parts, bf16 (fp32): 4 experts of
// 4096 rows x 256 x 512 50 and 22 us (134 and 72), 2 of 16384 x 512 x 128 178 and 23 (512 and 69), 1 of 8192 x 1024 x 1024 92 and 38 (266 and
// 192), 8 of 2048 x 128 x 256 23 and 19 (67 and 39).  Arithmetic on the shape: the parts are a part of the workspace's size.
constexpr int PART_TILES = 12;
inline bool small_weights(int E, int M, int N) { return (int64_t)E * ((M + 255) / 256) * ((N + 255) / 256) < 64; }
inline int weight_parts(int dtype, int64_t R, int E, int M, int N, int problems) {
  if (dtype == MOE_BF16 && !small_weights(E, M, N)) return 1;
  const int tile = dtype == MOE_BF16 ? 128 : F32_TILE, room = (dtype == MOE_BF16 ? 2 : 4) * CHIP_CUS;
  const int64_t tiles = (int64_t)problems * E * ((M + tile - 1) / tile) * ((N + tile - 1) / tile), nk = R / E / DK;
  const int64_t parts = std::min<int64_t>({room / tiles, nk / PART_TILES, 64});
  return parts < 2 ? 1 : (int)parts;
}
inline size_t part_bytes(int parts, int E, int M, int N) { return parts > 1 ? align_up((size_t)parts * E * M * N * 4, 256) : 0; }

inline uint32_t magic_of(int k) { return k > 1 ? (uint32_t)((0x100000000ull + (uint64_t)k - 1) / (uint64_t)k) : 0u; }
inline void set_gather(RaggedArgs& a, const int32_t* inv, int k, int64_t S) {
  a.gather = inv;
  a.gather_k = inv ? k : 0;
  a.gather_rows = inv ? S : 0;
  a.gather_magic = inv ? magic_of(k) : 0u;
}
inline RaggedArgs base_args(const int32_t* offsets, int64_t R, int E) {
  RaggedArgs a{};
  a.off = offsets;
  a.G = E; a.n_src = 1; a.Cc = a.R = (int)R;
  a.splits = 1;
  return a;
}

inline int check_rows(int dtype, int64_t R, int E, int64_t widest) {
  MOE_REQUIRE(dtype == MOE_F32 || dtype == MOE_BF16, MOE_EINVAL);
  MOE_REQUIRE(R >= 1 && E >= 1, MOE_EINVAL);
  MOE_REQUIRE(E <= MOE_MAX_E, MOE_EUNSUPPORTED);
  MOE_REQUIRE(R <= (1ll << 29), MOE_EUNSUPPORTED);    // 32-bit byte offsets into the row map
  if (dtype == MOE_BF16) MOE_REQUIRE((uint64_t)R * (uint64_t)widest * 2 <= 0xFFFFFFF0ull, MOE_EUNSUPPORTED);
  else MOE_REQUIRE(R * widest <= 1ll << 37, MOE_EUNSUPPORTED);     // tiles are counted in 32 bits
  return MOE_OK;
}
// the row operand: the token matrix and the plan's row map, or rows in the experts' order
inline int check_source(const void* x, int dtype, int64_t S, const int32_t* inv, int k, int M) {
  MOE_REQUIRE_PTR(x); MOE_OPTIONAL_PTR(inv);
  if (inv == nullptr) {
    MOE_REQUIRE(k == 1, MOE_EINVAL);
    return MOE_OK;
  }
  MOE_REQUIRE(S >= 1 && k >= 1, MOE_EINVAL);
  MOE_REQUIRE(k <= MOE_MAX_K && S * (int64_t)k <= (1ll << 29), MOE_EUNSUPPORTED);   // entries t k + j are divided by multiplication
  if (dtype == MOE_BF16) MOE_REQUIRE((uint64_t)S * (uint64_t)M * 2 <= 0xFFFFFFF0ull, MOE_EUNSUPPORTED);
  return MOE_OK;
}
inline int check_product(int dtype, int64_t R, int E, int K, int N) {
  MOE_REQUIRE(K >= 1 && N >= 1, MOE_EINVAL);
  if (int rc = check_rows(dtype, R, E, std::max(K, N))) return rc;
  MOE_REQUIRE(K % 8 == 0 && N % 8 == 0, MOE_EUNSUPPORTED);
  if (dtype == MOE_BF16) MOE_REQUIRE((uint64_t)K * N * 2 <= 0xFFFFFFF0ull, MOE_EUNSUPPORTED);
  return MOE_OK;
}
inline int check_ffn(int dtype, int64_t R, int E, int M, int H, int esp_idx, int n_esp) {
  MOE_REQUIRE(M >= 1 && H >= 1 && n_esp >= 1 && esp_idx >= 0 && esp_idx < n_esp && H % n_esp == 0, MOE_EINVAL);
  const int Hl = H / n_esp;
  if (int rc = check_rows(dtype, R, E, std::max(M, Hl))) return rc;
  MOE_REQUIRE(M % 8 == 0 && Hl % 8 == 0, MOE_EUNSUPPORTED);
  if (dtype == MOE_BF16) MOE_REQUIRE((uint64_t)M * H * 2 <= 0xFFFFFFF0ull, MOE_EUNSUPPORTED);
  return MOE_OK;
}
inline size_t hidden_bytes(int dtype, int64_t R, int Hl) { return align_up((size_t)R * Hl * (dtype == MOE_BF16 ? 2 : 4), 256); }

}  // namespace moe
