// Norms around an MoE block, with what stands beside them fused in, forward and backward:
//   in front    u = n(x)
//   behind      y = x + alpha gate n(h)           gate: per channel [M], per token [S] or none
//   n(v) = (v - mean) rstd w + b  ("layer", rstd = 1 / sqrt(var + eps))   or   v rstd w  ("rms", rstd = 1 / sqrt(mean(v^2) + eps))
// Backward of n for an upstream g = dL/dn:  with hat = n's normalised value and gw = g w,
//   dv = rstd (gw - hat mean(gw hat) [- mean(gw) for "layer"]),   dw = sum_t g hat,   db = sum_t g.
// Behind the block g = alpha gate dy; with A = sum_t alpha dy hat and B = sum_t alpha dy (times the token's gate, if that is per token)
// a gate per channel gives dw = gate A, db = gate B and dgate = w A + b B, so two column sums serve all three gradients.
//
// Bound by memory: every row is read once into registers, where both passes of the statistics run (sum, then squares of the centred
// values: no cancellation), in fp32.  TPR threads hold a row, NV pieces of 8 values each; a workgroup walks over rows with the weights
// in registers, because weights read again for every row would be more L2 traffic than the rows themselves (4 + 4 bytes a column
// against 2).  Column sums stay in a thread's registers over all of its workgroup's rows, and the workgroups' sums are added in a
// launch of their own in a fixed order: no atomics, the same bits every time.  A workgroup's next row is requested before the current
// one's sums, or 8 waves on a compute unit that stand at a barrier leave the memory idle.  bf16, 32768 rows of 4096, without and with that: n(x) 125 and 103 us
// (5.2 TB/s), behind the block 155 and 149 (5.4), backward 219 and 195 (5.5), behind the block 208 and 170 (4.7); a copy runs at 4.9.
#include <algorithm>
#include <type_traits>

#include "common.h"

namespace moe {

enum { GATE_NONE = MOE_GATE_NONE, GATE_CHANNEL = MOE_GATE_CHANNEL, GATE_TOKEN = MOE_GATE_TOKEN };

struct NormArgs {
  const void *v, *res, *up;        // normalised tensor; residual (forward) or gradient added to the result (backward); upstream gradient
  const float *w, *b, *gate;
  const float *mean_in, *rstd_in;
  float *mean, *rstd;
  void* out;
  float *dw, *db, *dgate, *part;   // part: [2, blocks, M] column sums
  int64_t S;
  int M, layer, gate_kind;
  float alpha, eps;
};

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void load8(const float* p, float (&f)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
// eight values as they lie in memory: requested a row ahead, converted when they are used
template <typename T>
struct Raw8 {
  u32x4_t q[sizeof(T) / 2];
  __device__ __forceinline__ void load(const void* base, int64_t at) {
#pragma unroll
    for (int h = 0; h < (int)sizeof(T) / 2; ++h) q[h] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>((const T*)base + at) + h);
  }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f[2 * e] = __uint_as_float(q[0][e] << 16);
        f[2 * e + 1] = __uint_as_float(q[0][e] & 0xFFFF0000u);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(q[e / 4][e % 4]);
    }
  }
};
template <typename T>
__device__ __forceinline__ void store8(void* base, int64_t at, const float (&f)[8]) {
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<uint4*>((bf16_t*)base + at) = pack_bf16x8(f);
  } else {
    *reinterpret_cast<float4*>((float*)base + at) = make_float4(f[0], f[1], f[2], f[3]);
    *reinterpret_cast<float4*>((float*)base + at + 4) = make_float4(f[4], f[5], f[6], f[7]);
  }
}

constexpr int block_of(int tpr) { return tpr > 256 ? tpr : 256; }

// Sums of N values over the TPR threads of a row, in every one of them.  `turn` alternates between two buffers, so that one
// barrier a sum is enough.
template <int TPR>
constexpr int red_floats() { return TPR > 64 ? 2 * (block_of(TPR) / 64) * 4 : 1; }
template <int TPR, int N>
__device__ __forceinline__ void row_sums(float (&s)[N], float* red, int& turn) {
  constexpr int IN_WAVE = TPR < 64 ? TPR : 64, WAVES = TPR / 64;
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int d = 1; d < IN_WAVE; d <<= 1) s[n] += __shfl_xor(s[n], d, 64);
  if constexpr (WAVES > 1) {
    float* r = red + turn * (block_of(TPR) / 64 * 4);
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int n = 0; n < N; ++n) r[(threadIdx.x >> 6) * 4 + n] = s[n];
    }
    __syncthreads();
    const int first = threadIdx.x / TPR * WAVES;      // the row's first wave
#pragma unroll
    for (int n = 0; n < N; ++n) {
      s[n] = 0.f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) s[n] += r[(first + w) * 4 + n];
    }
  }
}

// RES: the norm behind the block
template <typename T, int TPR, int NV, bool RES>
__global__ __launch_bounds__(block_of(TPR)) void norm_fwd(const NormArgs p) {
  constexpr int GROUPS = block_of(TPR) / TPR;
  constexpr bool AHEAD = TPR < 1024;     // the next row's requests go out before this row's sums; 1024 threads have no registers for that
  __shared__ float red[red_floats<TPR>()];
  const int lane = threadIdx.x % TPR, M = p.M;
  int turn = 0;
  float w[NV][8], b[NV][8], gc[RES ? NV : 1][8];
  bool in[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * TPR + lane) * 8;
    in[i] = c < M;
#pragma unroll
    for (int e = 0; e < 8; ++e) { w[i][e] = 0.f; b[i][e] = 0.f; if (RES) gc[RES ? i : 0][e] = 1.f; }
    if (in[i]) {
      load8(p.w + c, w[i]);
      if (p.b) load8(p.b + c, b[i]);
      if (RES && p.gate_kind == GATE_CHANNEL) load8(p.gate + c, gc[RES ? i : 0]);
    }
  }
  const float rm = 1.f / (float)M;
  // The rows of a workgroup's groups end together (barriers): a group behind the last row works on that one and stores nothing.
  const int64_t step = (int64_t)gridDim.x * GROUPS, end = (p.S + GROUPS - 1) / GROUPS * GROUPS;
  Raw8<T> nv[NV], nr[RES ? NV : 1];
  auto request = [&](int64_t row) {      // a piece behind the row's end is fetched from its beginning
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int64_t at = min(row, p.S - 1) * M + (in[i] ? (i * TPR + lane) * 8 : 0);
      nv[i].load(p.v, at);
      if (RES) nr[RES ? i : 0].load(p.res, at);
    }
  };
  int64_t row = (int64_t)blockIdx.x * GROUPS + threadIdx.x / TPR;
  if (AHEAD) request(row);
  for (; row < end; row += step) {
    if (!AHEAD) request(row);
    const bool here = row < p.S;
    const int64_t base = row * M + lane * 8;
    float v[NV][8], r[RES ? NV : 1][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      nv[i].get(v[i]);
      if (RES) nr[RES ? i : 0].get(r[RES ? i : 0]);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = in[i] ? v[i][e] : 0.f;
    }
    if (AHEAD) request(row + step);
    float mean = 0.f;
    if (p.layer) {
      float s[1] = {0.f};
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) s[0] += v[i][e];
      row_sums<TPR, 1>(s, red, turn);
      mean = s[0] * rm;
    }
    float q[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[i][e] = in[i] ? v[i][e] - mean : 0.f;
        q[0] = fmaf(v[i][e], v[i][e], q[0]);
      }
    row_sums<TPR, 1>(q, red, turn);
    const float rstd = 1.f / sqrtf(fmaf(q[0], rm, p.eps));
    if (!here) continue;
    if (lane == 0) {
      if (p.mean) p.mean[row] = mean;
      if (p.rstd) p.rstd[row] = rstd;
    }
    const float ag = !RES ? 1.f : p.gate_kind == GATE_TOKEN ? p.alpha * p.gate[row] : p.alpha;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (!in[i]) continue;
      float o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        o[e] = fmaf(v[i][e] * rstd, w[i][e], b[i][e]);
        if (RES) o[e] = fmaf(ag * gc[RES ? i : 0][e], o[e], r[RES ? i : 0][e]);
      }
      store8<T>(p.out, base + (int64_t)i * TPR * 8, o);
    }
  }
}

// gradients of the weights of column c from its two sums
__device__ __forceinline__ void weight_grads(const NormArgs& p, int c, float a, float b) {
  if (p.gate_kind == GATE_CHANNEL) {
    if (p.dgate) p.dgate[c] = fmaf(p.w[c], a, p.b ? p.b[c] * b : 0.f);
    a *= p.gate[c];
    b *= p.gate[c];
  }
  p.dw[c] = a;
  if (p.db) p.db[c] = b;
}

template <typename T, int TPR, int NV, bool RES>
__global__ __launch_bounds__(block_of(TPR)) void norm_bwd(const NormArgs p) {
  constexpr int GROUPS = block_of(TPR) / TPR;
  constexpr bool AHEAD = TPR < 1024;
  __shared__ float red[GROUPS > 1 ? GROUPS * TPR * 8 : red_floats<TPR>()];
  const int lane = threadIdx.x % TPR, group = threadIdx.x / TPR, M = p.M;
  int turn = 0;
  float w[NV][8], wb[RES ? NV : 1][8], gc[RES ? NV : 1][8], ca[NV][8], cb[NV][8];
  bool in[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * TPR + lane) * 8;
    in[i] = c < M;
#pragma unroll
    for (int e = 0; e < 8; ++e) { w[i][e] = 0.f; ca[i][e] = cb[i][e] = 0.f; if (RES) { wb[RES ? i : 0][e] = 0.f; gc[RES ? i : 0][e] = 1.f; } }
    if (in[i]) {
      load8(p.w + c, w[i]);
      if (RES && p.gate_kind == GATE_TOKEN && p.b) load8(p.b + c, wb[RES ? i : 0]);
      if (RES && p.gate_kind == GATE_CHANNEL) load8(p.gate + c, gc[RES ? i : 0]);
    }
  }
  const float rm = 1.f / (float)M;
  const int64_t step = (int64_t)gridDim.x * GROUPS, end = (p.S + GROUPS - 1) / GROUPS * GROUPS;
  Raw8<T> nv[NV], ng[NV], nr[RES ? 1 : NV];
  float next_mean = 0.f, next_rstd = 0.f;
  auto request = [&](int64_t row) {      // as in the forward pass
    row = min(row, p.S - 1);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int64_t at = row * M + (in[i] ? (i * TPR + lane) * 8 : 0);
      nv[i].load(p.v, at);
      ng[i].load(p.up, at);
      if (!RES && p.res) nr[RES ? 0 : i].load(p.res, at);
    }
    if (p.layer) next_mean = p.mean_in[row];
    next_rstd = p.rstd_in[row];
  };
  int64_t row = (int64_t)blockIdx.x * GROUPS + group;
  if (AHEAD) request(row);
  for (; row < end; row += step) {
    if (!AHEAD) request(row);
    const bool here = row < p.S;
    const int64_t base = row * M + lane * 8;
    float v[NV][8], g[NV][8], r[RES ? 1 : NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      nv[i].get(v[i]);
      ng[i].get(g[i]);
      if (!RES && p.res) nr[RES ? 0 : i].get(r[RES ? 0 : i]);
#pragma unroll
      for (int e = 0; e < 8; ++e) g[i][e] = here && in[i] ? g[i][e] : 0.f;
    }
    const float mean = next_mean, rstd = next_rstd;
    if (AHEAD) request(row + step);
    const float tg = RES && p.gate_kind == GATE_TOKEN && here ? p.gate[row] : 1.f;
    float s[3] = {0.f, 0.f, 0.f};     // sums of gw hat, of gw, and (gate per token) of alpha dy n
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float hat = here && in[i] ? (v[i][e] - mean) * rstd : 0.f;
        float up = g[i][e];
        if (RES) {
          up *= p.alpha;
          if (p.gate_kind == GATE_TOKEN) s[2] = fmaf(up, fmaf(hat, w[i][e], wb[RES ? i : 0][e]), s[2]);
          up *= tg;
        }
        ca[i][e] = fmaf(up, hat, ca[i][e]);
        cb[i][e] += up;
        const float gw = (RES ? up * gc[RES ? i : 0][e] : up) * w[i][e];
        s[0] = fmaf(gw, hat, s[0]);
        s[1] += gw;
        v[i][e] = hat;
        g[i][e] = gw;
      }
    row_sums<TPR, 3>(s, red, turn);
    if (!here) continue;
    if (RES && p.gate_kind == GATE_TOKEN && p.dgate && lane == 0) p.dgate[row] = s[2];
    const float c1 = s[0] * rm, c2 = p.layer ? s[1] * rm : 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (!in[i]) continue;
      float o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        o[e] = rstd * (fmaf(-v[i][e], c1, g[i][e]) - c2);
        if (!RES && p.res) o[e] += r[RES ? 0 : i][e];
      }
      store8<T>(p.out, base + (int64_t)i * TPR * 8, o);
    }
  }
  // the groups' column sums, in order
#pragma unroll
  for (int i = 0; i < NV; ++i) {
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      float sum[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] = which ? cb[i][e] : ca[i][e];
      if constexpr (GROUPS > 1) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) red[(group * TPR + lane) * 8 + e] = sum[e];
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          sum[e] = 0.f;
#pragma unroll
          for (int q = 0; q < GROUPS; ++q) sum[e] += red[(q * TPR + lane) * 8 + e];
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) (which ? cb : ca)[i][e] = sum[e];
    }
    if (group != 0 || !in[i]) continue;
    const int c = (i * TPR + lane) * 8;
    if (gridDim.x == 1) {
#pragma unroll
      for (int e = 0; e < 8; ++e) weight_grads(p, c + e, ca[i][e], cb[i][e]);
    } else {
      store8<float>(p.part, (int64_t)blockIdx.x * M + c, ca[i]);
      store8<float>(p.part, ((int64_t)gridDim.x + blockIdx.x) * M + c, cb[i]);
    }
  }
}

constexpr int SUM_COLS = 16, SUM_LINES = 64;     // columns and parts side by side of a workgroup
__global__ __launch_bounds__(SUM_COLS * SUM_LINES) void norm_add_parts(const NormArgs p, int blocks) {
  __shared__ float red[2][SUM_LINES][SUM_COLS + 1];
  const int cl = threadIdx.x % SUM_COLS, line = threadIdx.x / SUM_COLS, c = blockIdx.x * SUM_COLS + cl;
  float a = 0.f, b = 0.f;
  if (c < p.M) {
#pragma unroll 8
    for (int q = line; q < blocks; q += SUM_LINES) {
      a += p.part[(int64_t)q * p.M + c];
      b += p.part[((int64_t)blocks + q) * p.M + c];
    }
  }
  red[0][line][cl] = a;
  red[1][line][cl] = b;
#pragma unroll
  for (int d = SUM_LINES / 2; d >= 1; d >>= 1) {
    __syncthreads();
    if (line < d) {
      red[0][line][cl] += red[0][line + d][cl];
      red[1][line][cl] += red[1][line + d][cl];
    }
  }
  if (line == 0 && c < p.M) weight_grads(p, c, red[0][0][cl], red[1][0][cl]);
}

namespace {

constexpr int MAX_M = 32768;
constexpr int BWD_BLOCKS = 512;      // two workgroups to a compute unit

// Threads to a row, and pieces to a thread (with_shape): as few threads as leave a thread two pieces up to 4096 columns (weights, column sums and the
// next row: two waves to a SIMD and more) and four up to 8192 (one or two; the backward kernels reach into the accumulation registers), for what a row
// costs beside its bytes.  bf16, 32768 rows, the four calls: 1536 columns on 64 threads 39 / 57 / 102 / 99 us,
// 128 39 / 55 / 88 / 78, 256 41 / 68 / 125 / 104; 1024 on 64 28 / 38 / 53 / 46, on 256 38 / 57 / 119 / 99; 8192 202 / 307 / 381 / 417 (5.3, 5.2, 5.6 and
// 3.9 TB/s).
// Wider rows take 1024 threads, which have 128 registers each.  The forward kernels fit up to 16384 columns (behind the block 328 us for 16384 rows,
// 4.9 TB/s); behind the block from there on, and the backward kernels from 8193 columns, keep weights and sums in scratch memory and are bound by that:
// bf16, 16384 x 16384 backward 1060 and 1133 us (2.0 and 1.4 TB/s), 8192 x 32768 behind the block 785 (2.1), backward 2388 and 2720 (0.9 and 0.6).
int threads_per_row(int M) { return M <= 128 ? 16 : M <= 1024 ? 64 : M <= 2048 ? 128 : M <= 8192 ? 256 : 1024; }
int groups_of(int M) { return block_of(threads_per_row(M)) / threads_per_row(M); }
int64_t fwd_blocks(int64_t S, int M) { return std::min<int64_t>((S + groups_of(M) - 1) / groups_of(M), 2048); }
// a workgroup has at least 4 rows to a group, or its column sums would be as much traffic as its rows
int bwd_blocks(int64_t S, int M) { return (int)std::min<int64_t>((S + 4 * groups_of(M) - 1) / (4 * groups_of(M)), BWD_BLOCKS); }

template <typename F>
void with_shape(int M, F&& f) {
  auto go = [&](auto tpr, auto nv) { f(tpr, nv); };
  using std::integral_constant;
  if (M <= 128) go(integral_constant<int, 16>{}, integral_constant<int, 1>{});
  else if (M <= 512) go(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  else if (M <= 1024) go(integral_constant<int, 64>{}, integral_constant<int, 2>{});
  else if (M <= 2048) go(integral_constant<int, 128>{}, integral_constant<int, 2>{});
  else if (M <= 4096) go(integral_constant<int, 256>{}, integral_constant<int, 2>{});
  else if (M <= 8192) go(integral_constant<int, 256>{}, integral_constant<int, 4>{});
  else if (M <= 16384) go(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
  else go(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
}

template <bool RES>
int run_fwd(const NormArgs& p, int dtype, hipStream_t st) {
  with_shape(p.M, [&](auto tpr, auto nv) {
    constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value;
    const dim3 grid((unsigned)fwd_blocks(p.S, p.M)), block(block_of(TPR));
    if (dtype == MOE_BF16) hipLaunchKernelGGL((norm_fwd<bf16_t, TPR, NV, RES>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((norm_fwd<float, TPR, NV, RES>), grid, block, 0, st, p);
  });
  return check_launch();
}
template <bool RES>
int run_bwd(const NormArgs& p, int dtype, hipStream_t st) {
  const int blocks = bwd_blocks(p.S, p.M);
  with_shape(p.M, [&](auto tpr, auto nv) {
    constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value;
    const dim3 grid((unsigned)blocks), block(block_of(TPR));
    if (dtype == MOE_BF16) hipLaunchKernelGGL((norm_bwd<bf16_t, TPR, NV, RES>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((norm_bwd<float, TPR, NV, RES>), grid, block, 0, st, p);
  });
  if (blocks > 1)
    hipLaunchKernelGGL(norm_add_parts, dim3((unsigned)((p.M + SUM_COLS - 1) / SUM_COLS)), dim3(SUM_COLS * SUM_LINES), 0, st, p, blocks);
  return check_launch();
}

int check_norm(int dtype, int64_t S, int M, int kind) {
  MOE_REQUIRE(dtype == MOE_F32 || dtype == MOE_BF16, MOE_EINVAL);
  MOE_REQUIRE(S >= 1 && M >= 1, MOE_EINVAL);
  MOE_REQUIRE(kind == MOE_NORM_LAYER || kind == MOE_NORM_RMS, MOE_EINVAL);
  MOE_REQUIRE(M % 8 == 0 && M <= MAX_M, MOE_EUNSUPPORTED);
  return MOE_OK;
}
int check_gate(int gate_kind, const float* gate) {
  MOE_REQUIRE(gate_kind >= MOE_GATE_NONE && gate_kind <= MOE_GATE_TOKEN, MOE_EINVAL);
  MOE_REQUIRE((gate_kind == MOE_GATE_NONE) == (gate == nullptr), gate ? MOE_EINVAL : MOE_ENULL);
  MOE_OPTIONAL_PTR(gate);
  return MOE_OK;
}

}  // namespace
}  // namespace moe

using namespace moe;

extern "C" int moe_norm_fwd(const void* x, int dtype, int64_t S, int M, int kind, const float* w, const float* b, float eps, void* u,
                            float* mean, float* rstd, void* stream) {
  if (int rc = check_norm(dtype, S, M, kind)) return rc;
  MOE_REQUIRE(eps >= 0.f, MOE_EINVAL);
  MOE_REQUIRE(kind == MOE_NORM_LAYER || (b == nullptr && mean == nullptr), MOE_EINVAL);
  MOE_REQUIRE_PTR(x); MOE_REQUIRE_PTR(w); MOE_OPTIONAL_PTR(b); MOE_REQUIRE_PTR(u); MOE_OPTIONAL_PTR(mean); MOE_OPTIONAL_PTR(rstd);
  NormArgs p{};
  p.v = x; p.w = w; p.b = b; p.out = u; p.mean = mean; p.rstd = rstd;
  p.S = S; p.M = M; p.layer = kind == MOE_NORM_LAYER; p.eps = eps; p.alpha = 1.f;
  return run_fwd<false>(p, dtype, (hipStream_t)stream);
}

extern "C" int moe_norm_residual_fwd(const void* h, const void* x, int dtype, int64_t S, int M, int kind, const float* w, const float* b,
                                     const float* gate, int gate_kind, float alpha, float eps, void* y, float* mean, float* rstd,
                                     void* stream) {
  if (int rc = check_norm(dtype, S, M, kind)) return rc;
  MOE_REQUIRE(eps >= 0.f, MOE_EINVAL);
  MOE_REQUIRE(kind == MOE_NORM_LAYER || (b == nullptr && mean == nullptr), MOE_EINVAL);
  if (int rc = check_gate(gate_kind, gate)) return rc;
  MOE_REQUIRE_PTR(h); MOE_REQUIRE_PTR(x); MOE_REQUIRE_PTR(w); MOE_OPTIONAL_PTR(b); MOE_REQUIRE_PTR(y);
  MOE_OPTIONAL_PTR(mean); MOE_OPTIONAL_PTR(rstd);
  NormArgs p{};
  p.v = h; p.res = x; p.w = w; p.b = b; p.gate = gate; p.gate_kind = gate_kind; p.out = y; p.mean = mean; p.rstd = rstd;
  p.S = S; p.M = M; p.layer = kind == MOE_NORM_LAYER; p.eps = eps; p.alpha = alpha;
  return run_fwd<true>(p, dtype, (hipStream_t)stream);
}

extern "C" size_t moe_norm_bwd_workspace_bytes(int64_t S, int M) {
  if (check_norm(MOE_F32, S, M, MOE_NORM_LAYER) != MOE_OK) return 0;
  const int blocks = bwd_blocks(S, M);
  return blocks > 1 ? align_up((size_t)2 * blocks * M * sizeof(float), 256) : 0;
}

static int check_ws(int64_t S, int M, const void* ws, size_t ws_bytes) {
  const size_t need = moe_norm_bwd_workspace_bytes(S, M);
  MOE_REQUIRE(need == 0 || (ws != nullptr && ws_bytes >= need), MOE_EWORKSPACE);
  MOE_OPTIONAL_PTR(ws);
  return MOE_OK;
}

extern "C" int moe_norm_bwd(const void* du, const void* x, int dtype, int64_t S, int M, int kind, const float* w, const float* mean,
                            const float* rstd, const void* dres, void* dx, float* dw, float* db, void* ws, size_t ws_bytes,
                            void* stream) {
  if (int rc = check_norm(dtype, S, M, kind)) return rc;
  const bool layer = kind == MOE_NORM_LAYER;
  MOE_REQUIRE(layer || (mean == nullptr && db == nullptr), MOE_EINVAL);
  MOE_REQUIRE_PTR(du); MOE_REQUIRE_PTR(x); MOE_REQUIRE_PTR(w); MOE_REQUIRE_PTR(rstd); MOE_OPTIONAL_PTR(dres); MOE_REQUIRE_PTR(dx);
  MOE_REQUIRE_PTR(dw); MOE_OPTIONAL_PTR(db);
  if (layer) MOE_REQUIRE_PTR(mean);
  if (int rc = check_ws(S, M, ws, ws_bytes)) return rc;
  NormArgs p{};
  p.v = x; p.up = du; p.res = dres; p.w = w; p.mean_in = mean; p.rstd_in = rstd; p.out = dx; p.dw = dw; p.db = db;
  p.part = (float*)ws; p.S = S; p.M = M; p.layer = layer; p.alpha = 1.f;
  return run_bwd<false>(p, dtype, (hipStream_t)stream);
}

extern "C" int moe_norm_residual_bwd(const void* dy, const void* h, int dtype, int64_t S, int M, int kind, const float* w, const float* b,
                                     const float* gate, int gate_kind, float alpha, const float* mean, const float* rstd, void* dh,
                                     float* dw, float* db, float* dgate, void* ws, size_t ws_bytes, void* stream) {
  if (int rc = check_norm(dtype, S, M, kind)) return rc;
  const bool layer = kind == MOE_NORM_LAYER;
  MOE_REQUIRE(layer || (b == nullptr && mean == nullptr && db == nullptr), MOE_EINVAL);
  if (int rc = check_gate(gate_kind, gate)) return rc;
  MOE_REQUIRE(gate != nullptr || dgate == nullptr, MOE_EINVAL);
  MOE_REQUIRE_PTR(dy); MOE_REQUIRE_PTR(h); MOE_REQUIRE_PTR(w); MOE_OPTIONAL_PTR(b); MOE_REQUIRE_PTR(rstd); MOE_REQUIRE_PTR(dh);
  MOE_REQUIRE_PTR(dw); MOE_OPTIONAL_PTR(db); MOE_OPTIONAL_PTR(dgate);
  if (layer) MOE_REQUIRE_PTR(mean);
  if (int rc = check_ws(S, M, ws, ws_bytes)) return rc;
  NormArgs p{};
  p.v = h; p.up = dy; p.w = w; p.b = b; p.gate = gate; p.gate_kind = gate_kind; p.mean_in = mean; p.rstd_in = rstd; p.out = dh;
  p.dw = dw; p.db = db; p.dgate = dgate; p.part = (float*)ws; p.S = S; p.M = M; p.layer = layer; p.alpha = alpha;
  return run_bwd<true>(p, dtype, (hipStream_t)stream);
}
