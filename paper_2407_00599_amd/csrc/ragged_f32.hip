// fp32 products over ragged rows on the fp32 matrix cores (v_mfma_f32_32x32x2_f32: lane l supplies A[l % 32][l / 32] and B[l / 32][l % 32] and
// receives D[8 (r / 4) + 4 (l / 32) + r % 4][l % 32], r = 0..15), fp32 accumulation.
//
// T x T tile, four waves of T/2 x T/2, k chunks of 32 in two LDS buffers, one barrier a chunk: a chunk is requested two chunks ahead and stored
// behind the products of the chunk in between.  Which k a half of the lanes feeds in which step is free as long as both operands agree:
// in step t of 8 k the halves take k = t and k = 4 + t, so that an operand with k contiguous in memory is read from LDS 16 bytes a lane,
// four steps at once ([k / 4][row][4], a row of them one piece longer: the writes of a row's pieces hit different banks).  An operand with k as
// the slow index lies as it does in memory ([k][T + 8]: the rows the two halves read are 4 apart, half the banks).
// A wave multiplies 64 cycles for every 256 bytes that it reads from LDS, without bank conflicts, so the matrix units are what bounds a busy compute
// unit: for 1003 tokens with 3 choices x 520 x 1544 over 12 experts they work 63 % of the cycles in which it holds a workgroup.  The launch has 1.3 rounds of tiles,
// which leaves the units idle a quarter of the time: 47 % of all cycles, 70 of 151 TFLOP/s; HBM traffic is 1.3 TB/s.
#include "ckpt8.h"
#include "ragged.h"

namespace moe {

constexpr int FLUSH = 4;

template <int T, bool SLOW>
struct Operand {       // one operand of a tile in LDS, and a thread's part in bringing it there
  static constexpr int U = T * KC / 4 / 256;                                  // 16-byte pieces a thread
  static constexpr int FLOATS = SLOW ? KC * (T + 8) : KC / 4 * (T + 1) * 4;
  // piece u of thread t: k index (slow: of all four values; contiguous: of the first) and row / first column
  static __device__ __forceinline__ int k_of(int t, int u) { return SLOW ? t / (T / 4) + 1024 / T * u : t % (KC / 4) * 4; }
  static __device__ __forceinline__ int at_of(int t, int u) { return SLOW ? t % (T / 4) * 4 : t / (KC / 4) + 256 / (KC / 4) * u; }
  static __device__ __forceinline__ void put(float* lds, int t, int u, const f32x4_t& v) {
    *reinterpret_cast<f32x4_t*>(lds + (SLOW ? k_of(t, u) * (T + 8) + at_of(t, u) : (k_of(t, u) / 4 * (T + 1) + at_of(t, u)) * 4)) = v;
  }
  // the four steps' values of k group s (8 k), of row / column c, for the lanes' half h
  static __device__ __forceinline__ void get(const float* lds, int s, int h, int c, float (&v)[4]) {
    if (SLOW) {
#pragma unroll
      for (int t = 0; t < 4; ++t) v[t] = lds[(8 * s + 4 * h + t) * (T + 8) + c];
    } else {
      const float4 q = *reinterpret_cast<const float4*>(lds + ((2 * s + h) * (T + 1) + c) * 4);
      v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
    }
  }
};

template <int KIND, int T>
constexpr int f32_floats() { return 2 * (Operand<T, KIND == KIND_TN>::FLOATS + Operand<T, KIND != KIND_NT>::FLOATS); }

// Epilogues of the gated FFN.  Forward: 16 lanes hold g of a row and the 16 next to them its u; real: which of the tile's rows have a token, of the
// others g and u are zeros, also with weights that are not finite.
template <int EPI, int T, int ACT>
__device__ __forceinline__ void store_glu(const RaggedArgs& p, const f32x16_t (&total)[T / 64][T / 64], const RaggedPlace& at, int m0, int n0,
                                          int wm, int wn, int lane, const float* real) {
  constexpr int W = T / 2, NB = W / 32;
  const int l32 = lane & 31, half = lane >> 5;
  float* __restrict__ A = reinterpret_cast<float*>(p.C);      // act(g) u
  float* __restrict__ Z = reinterpret_cast<float*>(p.C2);     // [g | u], or their gradients
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int m = m0 + wm * W + 32 * i + 8 * (r >> 2) + 4 * half + (r & 3);
      const int64_t row = at.lo + m;
      const bool none = EPI != EPI_DGLU && real[m - m0] == 0.f;
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        const float v = none ? 0.f : total[i][j][r];
        const int c = n0 + wn * W + 32 * j + l32;
        if constexpr (EPI == EPI_DGLU) {
          if (m >= at.n || c >= p.half) continue;
          const float* __restrict__ z = reinterpret_cast<const float*>(p.Zin) + row * 2 * p.half + c;
          const float u = z[p.half];
          float a, da;
          gate_and_slope<ACT, false>(z[0], a, da);
          A[row * p.half + c] = a * u;
          Z[row * 2 * p.half + c] = v * u * da;
          Z[row * 2 * p.half + p.half + c] = v * a;
        } else {
          const float w = __shfl_xor(v, 16, 64);
          const int h = glu_hidden(c);
          if (m >= at.n || h >= p.half) continue;
          if (l32 < 16) A[row * p.half + h] = gate_value<ACT, false>(v) * w;
          if (EPI == EPI_GLU_KEEP) Z[row * 2 * p.half + (l32 < 16 ? h : p.half + h)] = v;
        }
      }
    }
}

template <int KIND, int EPI, int T>
__device__ __forceinline__ void f32_tile(const RaggedArgs& p, float* smem, int vb) {
  constexpr bool A_SLOW = KIND == KIND_TN, B_SLOW = KIND != KIND_NT;
  constexpr bool GLU = EPI == EPI_GLU || EPI == EPI_GLU_KEEP;
  using OA = Operand<T, A_SLOW>;
  using OB = Operand<T, B_SLOW>;
  constexpr int UA = OA::U, UB = OB::U, W = T / 2, NB = W / 32;
  constexpr int BUF = OA::FLOATS + OB::FLOATS;
  int part = 0;                                      // of a split reduction; the parts of a tile are a grid apart
  if (EPI == EPI_PART) {
    part = vb / p.grid;
    vb -= part * p.grid;
  }
  RaggedPlace at;
  if (!find_tile<KIND, EPI, 4, T, T>(p, vb, at)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1, l32 = lane & 31, half = lane >> 5;
  const int m0 = at.tm * T, n0 = at.tn * T;
  const float* __restrict__ A = reinterpret_cast<const float*>(p.A);
  const float* __restrict__ B = reinterpret_cast<const float*>(p.B) + (KIND == KIND_TN ? 0 : (int64_t)at.g * p.b_goff + p.b_off);
  const int K = KIND == KIND_TN ? at.n : p.Kdim;     // k indexes that exist
  int c0 = 0, nk = (K + KC - 1) / KC;                // chunks c0 .. nk - 1
  if (EPI == EPI_PART) {
    c0 = (int)((int64_t)nk * part / p.splits);
    nk = (int)((int64_t)nk * (part + 1) / p.splits);
  }

  // ---- this thread's pieces: where they start and whether they exist beside their k ----
  const float* pa[UA];
  const float* pb[UB];
  bool oka[UA], okb[UB];
#pragma unroll
  for (int u = 0; u < UA; ++u) {
    const int c = OA::at_of(tid, u);
    if (A_SLOW) {                                    // column m of the rows of a chunk, which follow from the chunk
      oka[u] = m0 + c < p.Mdim;
      pa[u] = A + (oka[u] ? m0 + c : 0);
    } else {
      oka[u] = m0 + c < at.n;
      int row = oka[u] ? at.lo + m0 + c : at.lo;
      if (p.gather != nullptr) {
        row = token(p, p.gather[row]);
        oka[u] = oka[u] && row >= 0;
        row = max(row, 0);
      }
      pa[u] = A + (int64_t)row * p.lda;
    }
  }
#pragma unroll
  for (int u = 0; u < UB; ++u) {
    const int c = OB::at_of(tid, u);
    okb[u] = GLU ? glu_hidden(n0 + c) < p.half : n0 + c < p.Ndim;
    if (GLU) pb[u] = B + glu_column(p, n0, c);
    else pb[u] = B + (B_SLOW ? (int64_t)(okb[u] ? n0 + c : 0) : (int64_t)(okb[u] ? n0 + c : 0) * p.ldb);
  }
  // token rows of a reduction: map entries of the chunk that is requested next
  int entry[A_SLOW ? UA : 1];
  auto fetch_map = [&](int c) {
    if constexpr (A_SLOW) {
#pragma unroll
      for (int u = 0; u < UA; ++u) entry[u] = p.gather[at.lo + min(c * KC + OA::k_of(tid, u), K - 1)];
    }
  };
  const bool gathered = A_SLOW && p.gather != nullptr;
  struct Chunk {
    f32x4_t a[UA], b[UB];
    uint32_t keep_a, keep_b;                         // pieces that exist; the others are fetched from somewhere in the tensor and zeroed
  };
  Chunk ch[2];
  auto fetch = [&](int c, Chunk& d) {
    d.keep_a = d.keep_b = 0;
#pragma unroll
    for (int u = 0; u < UA; ++u) {
      const int k = c * KC + OA::k_of(tid, u);
      bool ok = oka[u] && k < K;
      int64_t off;
      if (A_SLOW) {
        int row = at.lo + min(k, K - 1);
        if (gathered) {
          row = token(p, entry[A_SLOW ? u : 0]);
          ok = ok && row >= 0;
          row = max(row, 0);
        }
        off = (int64_t)row * p.lda;
      } else {
        off = k < K ? k : 0;
      }
      d.a[u] = *reinterpret_cast<const f32x4_t*>(pa[u] + off);
      d.keep_a |= (uint32_t)ok << u;
    }
#pragma unroll
    for (int u = 0; u < UB; ++u) {
      const int k = c * KC + OB::k_of(tid, u), kk = k < K ? k : 0;
      const int64_t off = KIND == KIND_TN ? (int64_t)(at.lo + kk) * p.ldb : B_SLOW ? (int64_t)kk * p.ldb : kk + (EPI == EPI_GLU_DX && kk >= p.half ? p.up - p.half : 0);
      d.b[u] = *reinterpret_cast<const f32x4_t*>(pb[u] + off);
      d.keep_b |= (uint32_t)(okb[u] && k < K) << u;
    }
  };
  auto kept = [](const f32x4_t& v, uint32_t keep) {
    f32x4_t r;
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = keep & 1u ? v[e] : 0.f;
    return r;
  };
  auto put = [&](int buf, const Chunk& d) {
#pragma unroll
    for (int u = 0; u < UA; ++u) OA::put(smem + buf * BUF, tid, u, kept(d.a[u], d.keep_a >> u));
#pragma unroll
    for (int u = 0; u < UB; ++u) OB::put(smem + buf * BUF + OA::FLOATS, tid, u, kept(d.b[u], d.keep_b >> u));
  };

  // Sums over FLUSH chunks are added to the totals: a rounding is then that of a sum of 128 products or of one of K / 128 such sums, not of one
  // of K (5000 k: 1.5e-6 of a row's size without, twice that of a library's product).
  f32x16_t acc[NB][NB], total[NB][NB];
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = total[i][j][r] = 0.f;
  auto flush = [&]() {
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          total[i][j][r] += acc[i][j][r];
          acc[i][j][r] = 0.f;
        }
  };
  // One chunk: the one after the next is requested into set SET, and the next one, which the other set holds, is stored behind the products.
  // No fetch stands in a branch, or its values would be copied, and waited for, where the branches meet; behind the last chunk that one is
  // fetched again.
  auto step = [&](int c, auto set_tag) {
    constexpr int SET = decltype(set_tag)::value;
    __syncthreads();                                 // chunk c is in its buffer, and the other one is consumed
    fetch(min(c + 2, nk - 1), ch[SET]);
    if (gathered) fetch_map(min(c + 3, nk - 1));
    const float* a = smem + SET * BUF;
    const float* b = a + OA::FLOATS;
    float va[2][NB][4], vb[2][NB][4];
    auto get = [&](int s) {
#pragma unroll
      for (int i = 0; i < NB; ++i) OA::get(a, s, half, wm * W + 32 * i + l32, va[s & 1][i]);
#pragma unroll
      for (int j = 0; j < NB; ++j) OB::get(b, s, half, wn * W + 32 * j + l32, vb[s & 1][j]);
    };
    get(0);
#pragma unroll
    for (int s = 0; s < KC / 8; ++s) {
      if (s + 1 < KC / 8) get(s + 1);                // under the products of this group
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
          for (int j = 0; j < NB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(va[s & 1][i][t], vb[s & 1][j][t], acc[i][j], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
    put(SET ^ 1, ch[SET ^ 1]);
  };
  if (nk > c0) {
    if (gathered) fetch_map(c0);
    fetch(c0, ch[0]);
    if (gathered) fetch_map(min(c0 + 1, nk - 1));
    fetch(min(c0 + 1, nk - 1), ch[1]);
    if (gathered) fetch_map(min(c0 + 2, nk - 1));
    put(0, ch[0]);
    for (int c = c0;;) {
      step(c, std::integral_constant<int, 0>{});
      if (++c >= nk) break;
      step(c, std::integral_constant<int, 1>{});
      if (++c >= nk) break;
      if (((c - c0) & (FLUSH - 1)) == 0) flush();
    }
    flush();
  }

  if constexpr (GLU || EPI == EPI_DGLU) {
    if constexpr (GLU) {
      __syncthreads();
#pragma unroll
      for (int u = 0; u < UA; ++u) smem[OA::at_of(tid, u)] = oka[u] ? 1.f : 0.f;      // (the threads of a row write the same)
      __syncthreads();
    }
    with_act(p.act, [&](auto act) { store_glu<EPI, T, decltype(act)::value>(p, total, at, m0, n0, wm, wn, lane, smem); });
    return;
  }
  float* __restrict__ C = EPI == EPI_PART ? p.part : reinterpret_cast<float*>(p.C);
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int m = m0 + wm * W + 32 * i + 8 * (r >> 2) + 4 * half + (r & 3);
      int64_t row;
      if (KIND == KIND_TN) {
        if (m >= p.Mdim) continue;
        row = EPI == EPI_PART ? (((int64_t)part * p.G + at.g) * p.Mdim + m) * p.Ndim : (int64_t)at.g * p.c_goff + p.c_off + (int64_t)m * p.ldc;
      } else {
        if (m >= at.n) continue;
        row = EPI == EPI_PART ? ((int64_t)part * p.R + at.lo + m) * p.Ndim : (int64_t)(at.lo + m) * p.ldc;
      }
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        const int n = n0 + wn * W + 32 * j + l32;
        if (n >= p.Ndim) continue;
        const float v = total[i][j][r];
        if constexpr (EPI == EPI_STORE || EPI == EPI_PART || EPI == EPI_GLU_DX) {
          C[row + n] = v;
        } else if constexpr (EPI == EPI_ACT) {
          C[row + n] = gelu_f(v);
        } else if constexpr (EPI == EPI_DGELU8) {
          float ge, dg;
          const uint32_t q = reinterpret_cast<const uint8_t*>(p.Zin)[row + n];
          gelu_and_grad(ckpt8_value(q, 0, p.Zs[(int64_t)(at.lo + m) * p.ldz + (n >> 5)]), ge, dg);
          C[row + n] = v * dg;
          reinterpret_cast<float*>(p.C2)[row + n] = ge;
        }
      }
    }
}

template <int KIND, int EPI>
__global__ __launch_bounds__(256, 2) void ragged_gemm_f32(const RaggedArgs p) {
  __shared__ __attribute__((aligned(16))) float smem[f32_floats<KIND, F32_TILE>()];
  f32_tile<KIND, EPI, F32_TILE>(p, smem, (int)blockIdx.x);
}
// the three products of the backward pass that only depend on dZ, dX first
template <int EPI>
__global__ __launch_bounds__(256, 2) void ragged_bwd_trio_f32(const RaggedArgs px, const RaggedArgs pw2, const RaggedArgs pw1, int nbx, int nb2) {
  __shared__ __attribute__((aligned(16))) float smem[f32_floats<KIND_TN, F32_TILE>()];
  static_assert(f32_floats<KIND_TN, F32_TILE>() >= f32_floats<KIND_NT, F32_TILE>(), "one buffer");
  const int b = (int)blockIdx.x;
  if (b < nbx) f32_tile<KIND_NT, EPI_STORE, F32_TILE>(px, smem, b);
  else f32_tile<KIND_TN, EPI, F32_TILE>(b < nbx + nb2 ? pw2 : pw1, smem, b < nbx + nb2 ? b - nbx : b - nbx - nb2);
}

// the four of the gated FFN: dX over [dG | dU], dW2, and the gate's and the up projection's half of dW1
template <int EPI>
__global__ __launch_bounds__(256, 2) void ragged_glu_bwd_f32(const RaggedArgs px, const RaggedArgs pw2, const RaggedArgs pwg, const RaggedArgs pwu,
                                                             int nbx, int nbw) {
  __shared__ __attribute__((aligned(16))) float smem[f32_floats<KIND_TN, F32_TILE>()];
  const int b = (int)blockIdx.x;
  if (b < nbx) f32_tile<KIND_NT, EPI_GLU_DX, F32_TILE>(px, smem, b);
  else f32_tile<KIND_TN, EPI, F32_TILE>(b < nbx + nbw ? pw2 : b < nbx + 2 * nbw ? pwg : pwu, smem, (b - nbx) % nbw);
}

template <int KIND, int EPI>
void launch_f32(RaggedArgs a, hipStream_t st) {
  const dim3 grid = KIND == KIND_TN ? size_weights(a, F32_TILE) : size_rows(a, F32_TILE, F32_TILE, EPI == EPI_STORE);
  hipLaunchKernelGGL((ragged_gemm_f32<KIND, EPI>), dim3(grid.x * (EPI == EPI_PART ? a.splits : 1)), dim3(256), 0, st, a);
}
template void launch_f32<KIND_NN, EPI_STORE>(RaggedArgs, hipStream_t);
template void launch_f32<KIND_NN, EPI_PART>(RaggedArgs, hipStream_t);
template void launch_f32<KIND_NN, EPI_ACT>(RaggedArgs, hipStream_t);
template void launch_f32<KIND_NT, EPI_STORE>(RaggedArgs, hipStream_t);
template void launch_f32<KIND_NT, EPI_PART>(RaggedArgs, hipStream_t);
template void launch_f32<KIND_NT, EPI_DGELU8>(RaggedArgs, hipStream_t);
template void launch_f32<KIND_NN, EPI_GLU>(RaggedArgs, hipStream_t);
template void launch_f32<KIND_NN, EPI_GLU_KEEP>(RaggedArgs, hipStream_t);
template void launch_f32<KIND_NT, EPI_DGLU>(RaggedArgs, hipStream_t);
template void launch_f32<KIND_TN, EPI_STORE>(RaggedArgs, hipStream_t);
template void launch_f32<KIND_TN, EPI_PART>(RaggedArgs, hipStream_t);

void launch_trio_f32(RaggedArgs dx, RaggedArgs w2, RaggedArgs w1, hipStream_t st) {
  const unsigned nbx = size_rows(dx, F32_TILE, F32_TILE, true).x;
  const unsigned nb2 = size_weights(w2, F32_TILE).x * w2.splits, nb1 = size_weights(w1, F32_TILE).x * w1.splits;
  const dim3 grid(nbx + nb2 + nb1);
  if (w2.splits > 1) hipLaunchKernelGGL((ragged_bwd_trio_f32<EPI_PART>), grid, dim3(256), 0, st, dx, w2, w1, (int)nbx, (int)nb2);
  else hipLaunchKernelGGL((ragged_bwd_trio_f32<EPI_STORE>), grid, dim3(256), 0, st, dx, w2, w1, (int)nbx, (int)nb2);
}

void launch_glu_bwd_f32(RaggedArgs dx, RaggedArgs w2, RaggedArgs wg, RaggedArgs wu, hipStream_t st) {
  const unsigned nbx = size_rows(dx, F32_TILE, F32_TILE, true).x;
  const unsigned nbw = size_weights(w2, F32_TILE).x * w2.splits;       // the three have as many tiles each
  size_weights(wg, F32_TILE);
  size_weights(wu, F32_TILE);
  const dim3 grid(nbx + 3 * nbw);
  if (w2.splits > 1) hipLaunchKernelGGL((ragged_glu_bwd_f32<EPI_PART>), grid, dim3(256), 0, st, dx, w2, wg, wu, (int)nbx, (int)nbw);
  else hipLaunchKernelGGL((ragged_glu_bwd_f32<EPI_STORE>), grid, dim3(256), 0, st, dx, w2, wg, wu, (int)nbx, (int)nbw);
}

}  // namespace moe
