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

#include "ckpt8.h"
#include "ragged.h"

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

// ------------------------------------------------------------------------------------------
// layout of the tiles
// ------------------------------------------------------------------------------------------
struct Ragged {
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

void buffer_sizes(RaggedArgs& a, bool weights) {
  a.a_bytes = (a.gather ? (uint64_t)a.gather_rows : (uint64_t)a.R) * (uint64_t)a.lda * 2;
  a.b_bytes = weights ? (uint64_t)a.R * (uint64_t)a.ldb * 2 : (uint64_t)a.G * (uint64_t)a.b_goff * 2;
}

// The tile of a bf16 row-tiled GEMM: the prices of the padded calls' tiles (ffn_tile.h) for what is multiplied, against the time of reading the
// weights, 4.9 TB/s, priced as if a second row tile of an expert found half of them in a cache.  Weights bound the launch where experts have few rows, and a tile that
// all rows of most experts fit in is then the fastest: 8 experts of 64 rows x 4096 x 14336 and x 14336 x 4096, tiles of 128 x 128 189 and 188 us,
// 64 x 128 198 and 243, 64 x 64 227 and 249; of 1024 x 1024 x 4096 102 and 128, 192 x 256 82.
// wide: only tiles of eight waves.
TilePlan plan_rows(const RaggedArgs& a, bool wide = false) {
  const float nk = (float)((a.Kdim + DK - 1) / DK), cu = (float)num_cus(), used = (float)std::min(a.R, a.G);
  const float weights = used * (float)a.Kdim * (float)a.Ndim * 2.f / 4.9e6f;
  TilePlan best{256, 256};
  float best_t = 0.f;
  for (const TileCost& c : ROW_TILES) {
    if (wide && c.tile.tile_n == 64) continue;
    const float row_tiles = (float)priced_row_tiles(a.R, a.G, c.tile.tile_m);
    const float n = row_tiles * (float)((a.Ndim + c.tile.tile_n - 1) / c.tile.tile_n);
    const float busy = c.per_cu == 1 ? n / cu : (n - cu) / cu;
    const float k = c.k_few + (c.k_all - c.k_few) * fminf(fmaxf(busy, 0.f), 1.f);
    const float products = ceilf(n / (cu * c.per_cu)) * (nk * k + c.fixed), reads = weights * 0.5f * (1.f + fmaxf(row_tiles / used, 1.f));
    const float t = fmaxf(products, reads) + 0.2f * fminf(products, reads);
    if (best_t == 0.f || t < best_t) { best_t = t; best = c.tile; }
  }
  return best;
}

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

// An fp32 product over rows with few tiles and a long reduction is cut into parts too, of at least ROW_PART_CHUNKS chunks of 32 k: 8 experts of
// 256 rows x 2048 x 512 96 us whole, 68 in parts and 5 for adding them.
constexpr int CHIP_CUS = 256;   // compute units of an MI355X
constexpr int ROW_PART_CHUNKS = 8;
int row_parts(int dtype, int64_t R, int E, int K, int N) {
  if (dtype != MOE_F32) return 1;
  const double tiles = priced_row_tiles((int)R, E, F32_TILE) * ((N + F32_TILE - 1) / F32_TILE);
  const int parts = std::min({(int)(4 * CHIP_CUS / std::max(tiles, 1.0)), K / KC / ROW_PART_CHUNKS, 16});
  return parts < 2 ? 1 : parts;
}
size_t row_part_bytes(int parts, int64_t R, int N) { return parts > 1 ? align_up((size_t)parts * R * N * 4, 256) : 0; }
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

// Weight gradients.  Tiles of 128 x 128 where those of 256 x 256 would be fewer than 64; of fp32, 64 x 64.  With few tiles a reduction over
// thousands of rows is what a launch waits for: it is cut into parts of at least PART_TILES k tiles of an expert's mean share of the
// rows, as many as the chip has room for (two workgroups of 128 x 128, four of fp32, to a compute unit).  Whole and in parts, bf16 (fp32): 4 experts of
// 4096 rows x 256 x 512 50 and 22 us (134 and 72), 2 of 16384 x 512 x 128 178 and 23 (512 and 69), 1 of 8192 x 1024 x 1024 92 and 38 (266 and
// 192), 8 of 2048 x 128 x 256 23 and 19 (67 and 39).  Arithmetic on the shape: the parts are a part of the workspace's size.
constexpr int PART_TILES = 12;
bool small_weights(int E, int M, int N) { return (int64_t)E * ((M + 255) / 256) * ((N + 255) / 256) < 64; }
int weight_parts(int dtype, int64_t R, int E, int M, int N, int problems) {
  if (dtype == MOE_BF16 && !small_weights(E, M, N)) return 1;
  const int tile = dtype == MOE_BF16 ? 128 : F32_TILE, room = (dtype == MOE_BF16 ? 2 : 4) * CHIP_CUS;
  const int64_t tiles = (int64_t)problems * E * ((M + tile - 1) / tile) * ((N + tile - 1) / tile), nk = R / E / DK;
  const int64_t parts = std::min<int64_t>({room / tiles, nk / PART_TILES, 64});
  return parts < 2 ? 1 : (int)parts;
}
size_t part_bytes(int parts, int E, int M, int N) { return parts > 1 ? align_up((size_t)parts * E * M * N * 4, 256) : 0; }

void add_parts(const RaggedArgs& p2, const RaggedArgs& p1, int problems, int dtype, hipStream_t st) {
  const int64_t n = (int64_t)p2.G * p2.Mdim * p2.Ndim / 4;       // sizes are multiples of 8
  const dim3 grid((unsigned)((problems * n + 255) / 256));
  if (dtype == MOE_BF16) hipLaunchKernelGGL((ragged_add_parts<bf16_t>), grid, dim3(256), 0, st, p2, p1, n, problems * n);
  else hipLaunchKernelGGL((ragged_add_parts<float>), grid, dim3(256), 0, st, p2, p1, n, problems * n);
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

uint32_t magic_of(int k) { return k > 1 ? (uint32_t)((0x100000000ull + (uint64_t)k - 1) / (uint64_t)k) : 0u; }
void set_gather(RaggedArgs& a, const int32_t* inv, int k, int64_t S) {
  a.gather = inv;
  a.gather_k = inv ? k : 0;
  a.gather_rows = inv ? S : 0;
  a.gather_magic = inv ? magic_of(k) : 0u;
}
RaggedArgs base_args(const int32_t* offsets, int64_t R, int E) {
  RaggedArgs a{};
  a.off = offsets;
  a.G = E; a.n_src = 1; a.Cc = a.R = (int)R;
  a.splits = 1;
  return a;
}

int check_rows(int dtype, int64_t R, int E, int64_t widest) {
  MOE_REQUIRE(dtype == MOE_F32 || dtype == MOE_BF16, MOE_EINVAL);
  MOE_REQUIRE(R >= 1 && E >= 1, MOE_EINVAL);
  MOE_REQUIRE(E <= MOE_MAX_E, MOE_EUNSUPPORTED);
  MOE_REQUIRE(R <= (1ll << 29), MOE_EUNSUPPORTED);    // 32-bit byte offsets into the row map
  if (dtype == MOE_BF16) MOE_REQUIRE((uint64_t)R * (uint64_t)widest * 2 <= 0xFFFFFFF0ull, MOE_EUNSUPPORTED);
  else MOE_REQUIRE(R * widest <= 1ll << 37, MOE_EUNSUPPORTED);     // tiles are counted in 32 bits
  return MOE_OK;
}
// the row operand: the token matrix and the plan's row map, or rows in the experts' order
int check_source(const void* x, int dtype, int64_t S, const int32_t* inv, int k, int M) {
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
int check_product(int dtype, int64_t R, int E, int K, int N) {
  MOE_REQUIRE(K >= 1 && N >= 1, MOE_EINVAL);
  if (int rc = check_rows(dtype, R, E, std::max(K, N))) return rc;
  MOE_REQUIRE(K % 8 == 0 && N % 8 == 0, MOE_EUNSUPPORTED);
  if (dtype == MOE_BF16) MOE_REQUIRE((uint64_t)K * N * 2 <= 0xFFFFFFF0ull, MOE_EUNSUPPORTED);
  return MOE_OK;
}
int check_ffn(int dtype, int64_t R, int E, int M, int H, int esp_idx, int n_esp) {
  MOE_REQUIRE(M >= 1 && H >= 1 && n_esp >= 1 && esp_idx >= 0 && esp_idx < n_esp && H % n_esp == 0, MOE_EINVAL);
  const int Hl = H / n_esp;
  if (int rc = check_rows(dtype, R, E, std::max(M, Hl))) return rc;
  MOE_REQUIRE(M % 8 == 0 && Hl % 8 == 0, MOE_EUNSUPPORTED);
  if (dtype == MOE_BF16) MOE_REQUIRE((uint64_t)M * H * 2 <= 0xFFFFFFF0ull, MOE_EUNSUPPORTED);
  return MOE_OK;
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
size_t hidden_bytes(int dtype, int64_t R, int Hl) { return align_up((size_t)R * Hl * (dtype == MOE_BF16 ? 2 : 4), 256); }

}  // namespace
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
    launch_few_rows(a, y, ws, st);
    return check_launch();
  }
  if (Zq) launch_rows<KIND_NN, EPI_GELU8>(a, dtype, st);
  else launch_rows<KIND_NN, EPI_ACT>(a, dtype, st);
  const int parts = row_parts(dtype, R, E, Hl, M);
  if (parts > 1 && ws != nullptr && ws_bytes >= row_part_bytes(parts, R, M)) launch_row_parts<KIND_NN>(y, parts, ws, st);
  else launch_rows<KIND_NN, EPI_STORE>(y, dtype, st);
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
