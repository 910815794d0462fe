// Expert products over ragged rows: the chosen rows of all experts lie expert by expert in one [R, .] buffer with no capacity padding
// between them.  With the kept rows n_e = min(counts[e], C) of expert e,
//   offsets[e] = n_0 + ... + n_(e-1),   row of choice (t, j) = offsets[idx[t, j]] + slot[t, j],
// and rows at or behind offsets[E] hold zeros.  Here are the plan of the rows, the three grouped products
//   Y = X W,  dX = dY W^T,  dW = X^T dY       (X optionally read from the token matrix through the plan's row map)
// and the expert FFN of an ESP shard forward and backward, whose pre-activation is kept for the backward pass in 8 bits (ckpt8.h):
//   forward   Z = X W1, A = GeLU(Z), Y = A W2;  Zq, Zs <- 8-bit form of Z
//   backward  z = the value that (Zq, Zs) stand for:  A' = GeLU(z), dZ = (dY W2^T) GeLU'(z), dW2 = A'^T dY, dW1 = X^T dZ, dX = dZ W1^T
// against the padded FFN's Z and A in the storage type, 4 bytes a value in bf16, the backward pass reads 1 + 1/32.
//
// The tiles are those of the capacity-padded calls (ffn_tile.h).  The offsets are read on the device: a workgroup finds the expert of
// its tile by a scan over the experts' tile counts, so no count crosses to the host and a call can be captured into a graph.
#include <math.h>

#include "ckpt8.h"
#include "ffn_tile.h"

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
    for (int e = tid; e <= E; e += PLAN_THREADS) offsets[e] = off[e];
  const int end = off[E];
  const int c = (int)blockIdx.x * PLAN_THREADS + tid;     // choice t k + j; and, for the empty rows, a row
  if (c >= R) return;
  const int e = idx[c], s = slot[c];
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
enum { EPI_ACT = 16, EPI_GELU8 = 17, EPI_DGELU8 = 18 };   // GeLU alone; GeLU and the 8-bit form; dZ and GeLU from the 8-bit form

struct RaggedArgs : GemmArgs {     // G = E experts, Cc = R = rows of the buffers, Mdim = R in row-tiled GEMMs, C2 / Zin = the 8-bit values
  const int32_t* off;              // [E + 1]
  uint8_t* Zs;                     // [R, ldz] scales of the 8-bit values
  int ldz;
  int grid;                        // workgroups of this problem
};

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

struct Ragged {
  using Args = RaggedArgs;
  struct Place {
    int g, tm, tn;
    int lo, n;        // first row and number of rows of expert g
  };
  static __device__ __forceinline__ int offset(const Args& p, int e) { return min(max(p.off[e], 0), p.R); }

  // Tiles of a row-tiled GEMM in linear order expert by expert, each with ceil(n / TM) row tiles; XCDs and patches as in the padded
  // calls.  The grid is made for the most tiles that R rows can have, and the workgroups behind the last tile store the rows
  // behind offsets[E] as zeros, an equal share each.
  template <int KIND, int EPI, int ESZ, int TM, int TN>
  static __device__ __forceinline__ bool find(const Args& p, int vb, Place& at) {
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
  // share `at` of `shares` of the rows behind the last expert's
  template <int ESZ>
  static __device__ __forceinline__ void fill_behind(const Args& p, int at, int shares) {
    const int64_t row_units = p.ldc * ESZ / 16, r0 = offset(p, p.G), units = (p.R - r0) * row_units;
    if (units <= 0 || at >= shares) return;
    const int64_t per = (units + shares - 1) / shares, u1 = min(per * (at + 1), units);
    u32x4_t* c = reinterpret_cast<u32x4_t*>(p.C) + r0 * row_units;
    const u32x4_t z = {0u, 0u, 0u, 0u};
    for (int64_t u = per * at + threadIdx.x; u < u1; u += blockDim.x) __builtin_nontemporal_store(z, c + u);
  }
  static __device__ __forceinline__ int token(const Args& p, int iv) {   // -1: no token, a row of zeros
    const uint32_t tok = p.gather_k == 1 ? (uint32_t)iv : __umulhi((uint32_t)iv, p.gather_magic);
    return iv >= 0 && (int64_t)tok < p.gather_rows ? (int)tok : -1;
  }
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
    // scales of this lane's row (accumulator order, group h of block i): offset of the first of its NBK blocks, or OOB
    uint32_t s_off[Q_OUT || Q_IN ? MB : 1][RG];
    if constexpr (Q_OUT || Q_IN) {
      uint32_t mine[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) mine[u] = out_off[u] == OOB ? OOB : (out_off[u] >> 1) / (uint32_t)p.ldc * (uint32_t)p.ldz + (uint32_t)(nbase >> 5);
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int h = 0; h < RG; ++h) {
          const int d = mshift + i * 32 + MR * h;
          s_off[i][h] = (uint32_t)__shfl((int)(d < 64 ? mine[0] : mine[1]), (d & 63) + (lane & (MR - 1)), 64);
        }
    }
    auto s_at = [&](int i, int h, int j) -> uint32_t {
      return s_off[i][h] != OOB && nbase + 32 * j < p.Ndim ? s_off[i][h] + j : OOB;
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
            b = ckpt8_scale(top);
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

  // Epilogue of the fp32 tile: lane l holds D[4 r + l / 16][l % 16] of its blocks of 16 columns, in fp64.  For the 8-bit form the tile
  // goes through LDS, because two waves share a row where the k halves are split; it is formed from the fp64 sums, whose rounding to
  // fp32 could move a value across the border between two steps.
  template <int KIND, int EPI, int TM, int TN, int KW>
  static __device__ __forceinline__ void store_f32(const Args& p, const f64x4_t (&acc)[TN / 16], double* Bs, int g, int m0, int n0,
                                                   int rw, int kw, int lane, int o_row, bool o_zero) {
    constexpr int NJ = TN / 16;
    float* __restrict__ C = reinterpret_cast<float*>(p.C);
    if constexpr (EPI == EPI_GELU8) {
      constexpr int PITCH = TN + 1, UNITS = TM * TN / 32, TPU = 256 / UNITS, CPT = 32 / TPU;   // blocks; threads and columns of each
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
        top = max(top, __float_as_uint((float)z[u]) & 0x7FFFFFFFu);
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
      return;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int ml = rw * 16 + 4 * r + (lane >> 4);
      int64_t crow;
      int row = 0;
      bool zero = false;
      if (KIND == KIND_TN) {
        if (m0 + ml >= p.Mdim) continue;
        crow = (int64_t)g * p.c_goff + p.c_off + (int64_t)(m0 + ml) * p.ldc;
      } else {
        row = __shfl(o_row, ml, 64);
        zero = __shfl((int)o_zero, ml, 64) != 0;
        if (row < 0) continue;
        crow = (int64_t)row * p.ldc;
      }
#pragma unroll
      for (int j = 0; j < NJ / KW; ++j) {
        const int n = n0 + 16 * (KW * j + kw) + (lane & 15);
        if (n >= p.Ndim) continue;
        const float v = zero ? 0.f : (float)acc[j][r];
        if (EPI == EPI_STORE) {
          C[crow + n] = v;
        } else if (EPI == EPI_ACT) {
          C[crow + n] = gelu_f(v);
        } else {
          float ge, dg;
          const uint32_t q = reinterpret_cast<const uint8_t*>(p.Zin)[crow + n];
          gelu_and_grad(ckpt8_value(q, 0, p.Zs[(int64_t)row * p.ldz + (n >> 5)]), ge, dg);
          C[crow + n] = v * dg;
          reinterpret_cast<float*>(p.C2)[crow + n] = ge;
        }
      }
    }
  }
};

template <int KIND, int EPI, typename CF, int ROWS = ROWS_PLAIN>
__global__ __launch_bounds__(64 * CF::NW) void ragged_ffn_gemm_dma(const RaggedArgs p) {
  __shared__ __attribute__((aligned(1024))) char smem[CF::LDS];
  gemm_dma_tile<KIND, EPI, CF, ROWS, Ragged>(p, smem, (int)blockIdx.x);
}

template <int KIND, int EPI, int T, bool WIDE>   // T x T tiles
__global__ __launch_bounds__(256, 4) void ragged_ffn_gemm_f32(const RaggedArgs p) {
  __shared__ __attribute__((aligned(16))) double smem[f32_lds<T, T>() / 8];
  gemm_f32_tile<KIND, EPI, T, T, WIDE, Ragged>(p, smem, (int)blockIdx.x);
}

// ------------------------------------------------------------------------------------------
// host side
// ------------------------------------------------------------------------------------------
namespace {

// Row tiles that R rows of E experts are priced at: half a tile of each expert's last one is empty.  How the rows are spread is not
// known here.
double priced_row_tiles(int R, int E, int tile_m) {
  const double rows = (double)R / E;
  return E * (rows < 1.0 ? rows : std::max(1.0, rows / tile_m + 0.45));
}
// the most row tiles that R rows of E experts can have
int64_t most_row_tiles(int R, int E, int tile_m) {
  const int64_t used = std::min(R, E);
  return ((int64_t)R + used * (tile_m - 1)) / tile_m;
}

TilePlan plan_rows(const RaggedArgs& a) {
  const float nk = (float)((a.Kdim + DK - 1) / DK), cu = (float)num_cus();
  TilePlan best{256, 256};
  float best_t = 0.f;
  for (const TileCost& c : ROW_TILES) {
    const float n = (float)(priced_row_tiles(a.R, a.G, c.tile.tile_m) * ((a.Ndim + c.tile.tile_n - 1) / c.tile.tile_n));
    const float busy = c.per_cu == 1 ? n / cu : (n - cu) / cu;
    const float k = c.k_few + (c.k_all - c.k_few) * fminf(fmaxf(busy, 0.f), 1.f);
    const float t = ceilf(n / (cu * c.per_cu)) * (nk * k + c.fixed);
    if (best_t == 0.f || t < best_t) { best_t = t; best = c.tile; }
  }
  return best;
}

constexpr int ZERO_SHARES = 64;    // workgroups at least that can store rows behind the last expert's
template <int KIND, int EPI>
void launch_rows(RaggedArgs a, int dtype, hipStream_t st) {
  auto sizes = [&](int tile_m, int tile_n) {
    const int64_t row_tiles = most_row_tiles(a.R, a.G, tile_m);
    a.tiles_m = (int)row_tiles;
    a.tiles_n = (a.Ndim + tile_n - 1) / tile_n;
    a.total_tiles = (int)(row_tiles * a.tiles_n);
    a.grid = (a.total_tiles + 7) / 8 * 8 + (EPI == EPI_STORE ? ZERO_SHARES : 0);
    a.run_mask = ~31;
    return dim3((unsigned)a.grid);
  };
  if (dtype == MOE_F32) {
    auto launch = [&](auto tile, auto wide) {
      constexpr int T = decltype(tile)::value;
      const dim3 grid = sizes(T, T);
      hipLaunchKernelGGL((ragged_ffn_gemm_f32<KIND, EPI, T, decltype(wide)::value>), grid, dim3(256), 0, st, a);
    };
    const bool wide = std::max(a.lda, a.ldb) >= 1 << 24;
    const double tiles64 = priced_row_tiles(a.R, a.G, 64) * ((a.Ndim + 63) / 64);
    if (wide) launch(std::integral_constant<int, 32>{}, std::true_type{});
    else if (tiles64 >= 3.0 * num_cus()) launch(std::integral_constant<int, 64>{}, std::false_type{});
    else launch(std::integral_constant<int, 32>{}, std::false_type{});
    return;
  }
  a.a_bytes = (a.gather ? (uint64_t)a.gather_rows : (uint64_t)a.R) * (uint64_t)a.lda * 2;
  a.b_bytes = (uint64_t)a.G * (uint64_t)a.b_goff * 2;
  auto launch = [&](auto cfg) {
    using CF = decltype(cfg);
    const dim3 grid = sizes(CF::TM, CF::TN);
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

void launch_weights(RaggedArgs a, int dtype, hipStream_t st) {
  auto sizes = [&](int tile) {
    a.tiles_m = (a.Mdim + tile - 1) / tile;
    a.tiles_n = (a.Ndim + tile - 1) / tile;
    a.total_tiles = a.G * a.tiles_m * a.tiles_n;
    a.run_mask = ~31;
    a.grid = (a.total_tiles + 7) / 8 * 8;
    return dim3((unsigned)a.grid);
  };
  if (dtype == MOE_F32) {
    const bool wide = std::max(a.lda, a.ldb) >= 1 << 24;
    const int64_t tiles64 = (int64_t)a.G * ((a.Mdim + 63) / 64) * ((a.Ndim + 63) / 64);
    auto launch = [&](auto tile, auto w) {
      constexpr int T = decltype(tile)::value;
      const dim3 grid = sizes(T);
      hipLaunchKernelGGL((ragged_ffn_gemm_f32<KIND_TN, EPI_STORE, T, decltype(w)::value>), grid, dim3(256), 0, st, a);
    };
    if (wide) launch(std::integral_constant<int, 32>{}, std::true_type{});
    else if (tiles64 >= 3 * (int64_t)num_cus()) launch(std::integral_constant<int, 64>{}, std::false_type{});
    else launch(std::integral_constant<int, 32>{}, std::false_type{});
    return;
  }
  a.a_bytes = (a.gather ? (uint64_t)a.gather_rows : (uint64_t)a.R) * (uint64_t)a.lda * 2;
  a.b_bytes = (uint64_t)a.R * (uint64_t)a.ldb * 2;
  auto launch = [&](auto cfg) {
    using CF = decltype(cfg);
    const dim3 grid = sizes(CF::TM);
    if (a.gather) hipLaunchKernelGGL((ragged_ffn_gemm_dma<KIND_TN, EPI_STORE, CF, ROWS_GATHER>), grid, dim3(64 * CF::NW), 0, st, a);
    else hipLaunchKernelGGL((ragged_ffn_gemm_dma<KIND_TN, EPI_STORE, CF>), grid, dim3(64 * CF::NW), 0, st, a);
  };
  const int64_t tiles256 = (int64_t)a.G * ((a.Mdim + 255) / 256) * ((a.Ndim + 255) / 256);
  if (tiles256 >= 64) launch(Tile256{});
  else launch(Tile128{});
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

extern "C" size_t moe_ragged_gemm_workspace_bytes(int, int64_t, int, int, int) { return 0; }

extern "C" int moe_ragged_gemm(const void* x, int dtype, int64_t S, const int32_t* inv, int k, const void* W, int transposed,
                               const int32_t* offsets, int64_t R, int E, int K, int N, void* Y, void*, size_t, void* stream) {
  if (int rc = check_product(dtype, R, E, K, N)) return rc;
  MOE_REQUIRE(transposed == 0 || transposed == 1, MOE_EINVAL);
  if (int rc = check_source(x, dtype, S, inv, k, K)) return rc;
  MOE_REQUIRE_PTR(W); MOE_REQUIRE_PTR(offsets); MOE_REQUIRE_PTR(Y);
  RaggedArgs a = base_args(offsets, R, E);
  set_gather(a, inv, k, S);
  a.A = x; a.lda = K;
  a.B = W; a.ldb = transposed ? K : N; a.b_goff = (int64_t)K * N;
  a.C = Y; a.ldc = N;
  a.Mdim = a.R; a.Ndim = N; a.Kdim = K;
  if (transposed) launch_rows<KIND_NT, EPI_STORE>(a, dtype, (hipStream_t)stream);
  else launch_rows<KIND_NN, EPI_STORE>(a, dtype, (hipStream_t)stream);
  return check_launch();
}

extern "C" size_t moe_ragged_wgrad_workspace_bytes(int, int64_t, int, int, int) { return 0; }

extern "C" int moe_ragged_wgrad(const void* x, int dtype, int64_t S, const int32_t* inv, int k, const void* dY, const int32_t* offsets,
                                int64_t R, int E, int K, int N, void* dW, void*, size_t, void* stream) {
  if (int rc = check_product(dtype, R, E, K, N)) return rc;
  if (int rc = check_source(x, dtype, S, inv, k, K)) return rc;
  MOE_REQUIRE_PTR(dY); MOE_REQUIRE_PTR(offsets); MOE_REQUIRE_PTR(dW);
  RaggedArgs a = base_args(offsets, R, E);
  set_gather(a, inv, k, S);
  a.A = x; a.lda = K;
  a.B = dY; a.ldb = N;
  a.C = dW; a.ldc = N; a.c_goff = (int64_t)K * N;
  a.Mdim = K; a.Ndim = N; a.Kdim = a.R;
  launch_weights(a, dtype, (hipStream_t)stream);
  return check_launch();
}

extern "C" size_t moe_ragged_ffn_workspace_bytes(int dtype, int64_t R, int E, int M, int H, int n_esp, int backward) {
  if (check_ffn(dtype, R, E, M, H, 0, n_esp) != MOE_OK) return 0;
  return backward ? 2 * hidden_bytes(dtype, R, H / n_esp) : 0;
}

extern "C" int moe_ragged_ffn_fwd(const void* x, int dtype, int64_t S, const int32_t* inv, int k, const void* W1, const void* W2,
                                  const int32_t* offsets, int64_t R, int E, int M, int H, int esp_idx, int n_esp, void* Zq, void* Zs,
                                  void* A, void* Y, void*, size_t, void* stream) {
  if (int rc = check_ffn(dtype, R, E, M, H, esp_idx, n_esp)) return rc;
  if (int rc = check_source(x, dtype, S, inv, k, M)) return rc;
  MOE_REQUIRE_PTR(W1); MOE_REQUIRE_PTR(W2); MOE_REQUIRE_PTR(offsets); MOE_REQUIRE_PTR(A); MOE_REQUIRE_PTR(Y);
  MOE_REQUIRE((Zq == nullptr) == (Zs == nullptr), MOE_ENULL);
  MOE_OPTIONAL_PTR(Zq); MOE_OPTIONAL_PTR(Zs);
  hipStream_t st = (hipStream_t)stream;
  const int Hl = H / n_esp;
  const int64_t h0 = (int64_t)esp_idx * Hl;
  RaggedArgs a = base_args(offsets, R, E);
  set_gather(a, inv, k, S);
  a.A = x; a.lda = M;
  a.B = W1; a.ldb = H; a.b_goff = (int64_t)M * H; a.b_off = h0;
  a.C = A; a.C2 = Zq; a.Zs = (uint8_t*)Zs; a.ldc = Hl; a.ldz = (Hl + 31) / 32;
  a.Mdim = a.R; a.Ndim = Hl; a.Kdim = M;
  if (Zq) launch_rows<KIND_NN, EPI_GELU8>(a, dtype, st);
  else launch_rows<KIND_NN, EPI_ACT>(a, dtype, st);
  RaggedArgs y = base_args(offsets, R, E);
  y.A = A; y.lda = Hl;
  y.B = W2; y.ldb = M; y.b_goff = (int64_t)H * M; y.b_off = h0 * M;
  y.C = Y; y.ldc = M;
  y.Mdim = y.R; y.Ndim = M; y.Kdim = Hl;
  launch_rows<KIND_NN, EPI_STORE>(y, dtype, st);
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
  MOE_REQUIRE(ws != nullptr && ws_bytes >= 2 * hidden, MOE_EWORKSPACE);
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
  launch_rows<KIND_NT, EPI_STORE>(dx, dtype, st);
  // dW2[h0:h0+Hl, :] = Act^T dY
  RaggedArgs w2 = base_args(offsets, R, E);
  w2.A = Act; w2.lda = Hl;
  w2.B = dY; w2.ldb = M;
  w2.C = dW2; w2.ldc = M; w2.c_goff = (int64_t)H * M; w2.c_off = h0 * M;
  w2.Mdim = Hl; w2.Ndim = M; w2.Kdim = w2.R;
  launch_weights(w2, dtype, st);
  // dW1[:, h0:h0+Hl] = X^T dZ
  RaggedArgs w1 = base_args(offsets, R, E);
  set_gather(w1, inv, k, S);
  w1.A = x; w1.lda = M;
  w1.B = dZ; w1.ldb = Hl;
  w1.C = dW1; w1.ldc = H; w1.c_goff = (int64_t)M * H; w1.c_off = h0;
  w1.Mdim = M; w1.Ndim = Hl; w1.Kdim = w1.R;
  launch_weights(w1, dtype, st);
  return check_launch();
}
