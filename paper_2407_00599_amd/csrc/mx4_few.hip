// Products from microscaled 4-bit values of few rows: a decoding step, whose time is that of reading the weights once.
//
// As in ragged_few.hip nothing is shared in the k loop: a lane's 16 bytes of a weight row are its operand of the scaled matrix instruction as they lie
// in memory, and so are those of a row of X, from L2.  A wave takes units of 256 k, in which 16 rows give it whole 128-byte lines, for NC groups of 16
// columns; the waves of a workgroup take the units in turn, the next one requested behind the products, and their sums meet in LDS in a fixed order.
// Of a gated first product the groups are the gate's and the up projection's of the same hidden columns in turn, and 32 hidden columns, one block
// of A, meet in one row of the sums, so A goes to memory in 4 bits.
//
// Bound by HBM: 8 tokens top-2 of 8 experts x 4096 x 14336 83 to 85 us for the first product (499 MB of weights and scales, 5.9 TB/s) and 47 to 49
// for the second (5.1 to 5.3).
#include "mx4_ffn.h"

namespace moe {

constexpr int MX4_NC = 4, MX4_FEW_WAVES = 4;      // groups of 16 columns and waves of a workgroup

template <int KIND, int RG>      // groups of 16 rows that go along with one reading of the weights
__global__ __launch_bounds__(64 * MX4_FEW_WAVES, 2) void mx4_few(const Mx4Args p) {
  constexpr int NC = MX4_NC, WAVES = MX4_FEW_WAVES, TN = 16 * NC, PITCH = TN + 4;
  __shared__ float red[WAVES * 16 * PITCH];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c16 = lane & 15, kg = lane >> 4;
  const int tile = (int)blockIdx.x;
  if (tile >= p.E * p.tiles_n) {                   // rows behind the last expert's: zeros
    if (KIND == MX4_STORE) {
      const int64_t r0 = offset(p, p.E), total = (int64_t)(p.R - r0) * p.n * (p.f32 ? 4 : 2) / 16, at = tile - p.E * p.tiles_n;
      u32x4_t* c = reinterpret_cast<u32x4_t*>(p.C) + r0 * p.n * (p.f32 ? 4 : 2) / 16;
      for (int64_t u = at * (64 * WAVES) + tid; u < total; u += (int64_t)ZERO_SHARES * 64 * WAVES) c[u] = u32x4_t{0u, 0u, 0u, 0u};
    }
    return;
  }
  const int g = tile / p.tiles_n, tn = tile - g * p.tiles_n;
  const int lo = __builtin_amdgcn_readfirstlane(offset(p, g)), n = __builtin_amdgcn_readfirstlane(offset(p, g + 1)) - lo;
  if (n <= 0) return;
  const int units = (p.blocks + 7) / 8;
  const uint32_t pitch = (uint32_t)p.blocks * 16u, w_scales = (uint32_t)p.n * 4u, x_scales = (uint32_t)p.x_rows * 4u;
  const __amdgpu_buffer_rsrc_t rX = make_rsrc(p.xq, (uint32_t)p.x_rows * pitch), rXS = make_rsrc(p.xs, (uint32_t)p.chunks * 4u * x_scales),
                               rW = make_rsrc(p.wq + (int64_t)g * p.n * pitch, (uint32_t)p.n * pitch),
                               rWS = make_rsrc(p.ws + (int64_t)g * p.chunks * 4 * w_scales, (uint32_t)p.chunks * 4u * w_scales);
  uint32_t w_off[NC], ws_off[NC];      // this lane's column in W and its scales, or OOB: zeros
#pragma unroll
  for (int j = 0; j < NC; ++j) {
    const int col = KIND == MX4_GLU ? tn * (TN / 2) + 16 * (j / 2) + c16 : tn * TN + 16 * j + c16;
    const bool ok = col < (KIND == MX4_GLU ? p.half : p.n);
    const uint32_t row = (uint32_t)(KIND == MX4_GLU && (j & 1) ? p.half + col : col);
    w_off[j] = ok ? row * pitch + (uint32_t)kg * 16u : OOB;
    ws_off[j] = ok ? (uint32_t)kg * w_scales + row * 4u : OOB;
  }
  for (int m0 = 0; m0 < n; m0 += 16 * RG) {
    int entry[RG];             // of the row map; asked for first, waited for behind the weights' requests
#pragma unroll
    for (int q = 0; q < RG; ++q) {
      entry[q] = lo + min(m0 + 16 * q + c16, n - 1);
      if (p.gather != nullptr) entry[q] = p.gather[entry[q]];
    }
    uint32_t x_off[RG], xs_off[RG];
    struct Unit {
      uint4 w[NC][2], x[RG][2];
      uint32_t ws[NC], xs[RG];
    };
    Unit d;
    // Offsets of this lane's rows are fixed, the unit's part of an address is in a scalar register.
    // No request and no product stands in a branch: their registers would be copied, and waited for, where the branches meet.
    auto request_w = [&](int s) {         // blocks behind the last one: zeros
      const int at = min(s, units - 1);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < NC; ++j) d.w[j][h] = mx4_load16(rW, 8 * s + 4 * h + kg < p.blocks ? w_off[j] : OOB, at * 128 + h * 64);
#pragma unroll
      for (int j = 0; j < NC; ++j) d.ws[j] = __builtin_amdgcn_raw_buffer_load_b32(rWS, (int)ws_off[j], (int)((uint32_t)at / 2u * 4u * w_scales), 0);
    };
    auto request_x = [&](int s) {
      const int at = min(s, units - 1);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int q = 0; q < RG; ++q) d.x[q][h] = mx4_load16(rX, 8 * s + 4 * h + kg < p.blocks ? x_off[q] : OOB, at * 128 + h * 64);
#pragma unroll
      for (int q = 0; q < RG; ++q) d.xs[q] = __builtin_amdgcn_raw_buffer_load_b32(rXS, (int)xs_off[q], (int)((uint32_t)at / 2u * 4u * x_scales), 0);
    };
    f32x4_t acc[RG][NC];
#pragma unroll
    for (int q = 0; q < RG; ++q)
#pragma unroll
      for (int j = 0; j < NC; ++j) acc[q][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    request_w(wave);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int q = 0; q < RG; ++q) {
      int row = m0 + 16 * q + c16 < n ? entry[q] : -1;
      if (p.gather != nullptr && row >= 0) row = token(p, row);
      x_off[q] = row >= 0 ? (uint32_t)row * pitch + (uint32_t)kg * 16u : OOB;
      xs_off[q] = row >= 0 ? (uint32_t)kg * x_scales + (uint32_t)row * 4u : OOB;
    }
    request_x(wave);
    __builtin_amdgcn_sched_barrier(0);
    for (int s = wave; s < units; s += WAVES) {
      const int c = s >> 1, sh = 16 * (s & 1);
      uint32_t xs[RG];
#pragma unroll
      for (int q = 0; q < RG; ++q) xs[q] = mx4_existing(p, d.xs[q], c, kg) >> sh;
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        const uint32_t ws = mx4_existing(p, d.ws[j], c, kg) >> sh;
#pragma unroll
        for (int q = 0; q < RG; ++q) {
          acc[q][j] = mx4_mfma<0>(d.x[q][0], d.w[j][0], acc[q][j], xs[q], ws);
          acc[q][j] = mx4_mfma<1>(d.x[q][1], d.w[j][1], acc[q][j], xs[q], ws);
        }
      }
      __builtin_amdgcn_sched_barrier(0);           // or the next unit's registers are taken before these are free
      request_w(s + WAVES);
      request_x(s + WAVES);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int q = 0; q < RG; ++q) {
      if (m0 + 16 * q >= n) break;                 // (uniform)
      // rows of the group that have a token: of the others the products are zeros, also with weights that are not finite
      const uint32_t real = (uint32_t)__ballot(x_off[q] != OOB);
      __syncthreads();
#pragma unroll
      for (int j = 0; j < NC; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) red[(wave * 16 + 4 * kg + r) * PITCH + 16 * j + c16] = acc[q][j][r];
      __syncthreads();
      if constexpr (KIND == MX4_STORE) {
        for (int v = tid; v < 16 * TN / 2; v += 64 * WAVES) {
          const int row = v / (TN / 2), c = v % (TN / 2) * 2, r = m0 + 16 * q + row, col = tn * TN + c;
          float2 t = make_float2(0.f, 0.f);
#pragma unroll
          for (int w = 0; w < WAVES; ++w) {
            const float2 a = *reinterpret_cast<const float2*>(&red[(w * 16 + row) * PITCH + c]);
            t.x += a.x;
            t.y += a.y;
          }
          if (r >= n || col >= p.n) continue;
          if (!(real >> row & 1u)) t = make_float2(0.f, 0.f);
          const int64_t at = (int64_t)(lo + r) * p.n + col;
          if (p.f32) *reinterpret_cast<float2*>(reinterpret_cast<float*>(p.C) + at) = t;
          else *reinterpret_cast<uint32_t*>(reinterpret_cast<bf16_t*>(p.C) + at) = pack_bf16x2(t.x, t.y);
        }
      } else if (tid < 64) {                       // four lanes a row, 8 hidden columns each; columns 16 .. 31 are those of the next two groups
        const int row = tid >> 2, h0 = 8 * (tid & 3), r = m0 + 16 * q + row, from = (h0 >> 4) * 32 + (h0 & 15), hidden = tn * (TN / 2) + h0;
        float gv[8], uv[8], a[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) gv[e] = uv[e] = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            gv[e] += red[(w * 16 + row) * PITCH + from + e];
            uv[e] += red[(w * 16 + row) * PITCH + from + 16 + e];
          }
        uint32_t top = 0;
        with_hidden(p.act, p.f32, [&](auto act, auto wide) {
#pragma unroll
          for (int e = 0; e < 8; ++e) a[e] = hidden < p.half && (real >> row & 1u) ? mx4_hidden<decltype(act)::value, decltype(wide)::value>(gv[e], uv[e]) : 0.f;
        });
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(a[e]) & 0x7FFFFFFFu);
        top = max(top, (uint32_t)__shfl_xor((int)top, 1, 64));
        top = max(top, (uint32_t)__shfl_xor((int)top, 2, 64));
        const int b = mx4_scale(top), block = tn;  // TN / 2 = 32
        if (r < n) {
          *reinterpret_cast<uint32_t*>(p.aq + ((int64_t)(lo + r) * p.a_blocks + block) * 16 + (tid & 3) * 4) = mx4_pack(a, b);
          if ((tid & 3) == 0) p.as[(((int64_t)(block >> 4) * 4 + (block & 3)) * p.R + lo + r) * 4 + (block >> 2 & 3)] = (uint8_t)b;
        }
      }
    }
  }
}
static_assert(16 * MX4_NC / 2 == MX4_BLOCK, "a tile's hidden columns are one block");

void launch_mx4_few(Mx4Args a, int kind, hipStream_t st) {
  a.tiles_n = kind == MX4_GLU ? (a.half + 8 * MX4_NC - 1) / (8 * MX4_NC) : (a.n + 16 * MX4_NC - 1) / (16 * MX4_NC);
  const dim3 grid((unsigned)(a.E * a.tiles_n + (kind == MX4_STORE ? ZERO_SHARES : 0)));
  auto launch = [&](auto k, auto rg) {
    hipLaunchKernelGGL((mx4_few<decltype(k)::value, decltype(rg)::value>), grid, dim3(64 * MX4_FEW_WAVES), 0, st, a);
  };
  using std::integral_constant;
  auto with_kind = [&](auto rg) {
    if (kind == MX4_GLU) launch(integral_constant<int, MX4_GLU>{}, rg);
    else launch(integral_constant<int, MX4_STORE>{}, rg);
  };
  if (a.R <= 8 * (int64_t)a.E || a.R <= 16) with_kind(integral_constant<int, 1>{});
  else with_kind(integral_constant<int, 2>{});
}

}  // namespace moe
