// Products from microscaled 4-bit values of many rows: the bf16 tile of ffn_tile.h with other matrix instructions.
//
// 16 bytes of a row are a lane's operand of v_mfma_scale_f32_16x16x128_f8f6f4 (32 k) as they are of v_mfma_f32_16x16x32_bf16 (8 k), and a k tile is
// 128 bytes of a row either way, 256 k here: requests, LDS, fragment reads and waits are the same code, in which "k" counts pairs of bytes, and each
// instruction does four times the products in the time of one.  What is added are the scales: a byte for every 16 bytes.  Two k tiles' are a dword a row
// and lane group ([c][q][row][s], mx4.h); a request brings those of 64 rows to LDS (rows of X through the row map), and a lane reads
// the two bytes of its rows for a k tile, which the two steps of the tile select.
// Tiles have two ring slots for either operand: the scales take the LDS of the third.
//
// Bound by power, and with short reductions by what stands outside the k loop: 8 experts of 4096 rows x 4096 x 14336, gated, 2090 us and 960 back (3.68 and
// 4.0 PFLOP/s; the matrix pipes busy 54 % of the cycles at the 1.6 GHz that the power limit leaves): 1.7 to 1.85 us a k tile of 256 x 256 and 8 us a round
// of tiles, a chain of offsets, row map and first k tile (4 to 7, cold) and the epilogue (2 to 4).  64 experts of 512 rows x 2048 x 2048, 8 k tiles, 139 us (2.0 PFLOP/s).
// Requests spread over less of the k tile, or over all of it, measured the same; four waves of 128 x 128, which read a third less
// from LDS, with their accumulators in the other half of the register file 136 -> 144 us and 935 -> 1000; tiles of 64 x 128 were nowhere faster.
#include "mx4_ffn.h"

namespace moe {

struct Mx4TileArgs : RaggedArgs {      // A, B: 4-bit values, lda, ldb, Kdim in pairs of bytes; ldc: row pitch of Y in pairs of bytes
  const uint8_t* xs;
  const uint8_t* ws;
  int64_t x_rows;
  int n, blocks, chunks, f32;
  uint8_t* aq;                         // of a gated first product
  uint8_t* as;
  int a_blocks;
};

struct Mx4 : Ragged {
  using Args = Mx4TileArgs;
  static constexpr bool SCALED = true;

  template <int EPI>
  static __device__ __forceinline__ int row(const Args& p, int n0, int c) {
    if constexpr (EPI == EPI_GLU) return min(glu_hidden(n0 + c), p.half - 1) + (((n0 + c) & 16) ? p.half : 0);
    else return min(n0 + c, p.n - 1);
  }
  // Entry of the row map for row r of an expert (behind its last one: that one's).  Without a map nothing is read, and no branch stands
  // around the read, so that those of a tile's operand and output rows are requested before the first is waited for (one after the other they took
  // 2 us).  The entry of the row whose scales a lane brings (Scales) is one more read behind them.
  static __device__ __forceinline__ int entry(const Args& p, const Place& at, int r) {
    const __amdgpu_buffer_rsrc_t map = make_rsrc(p.gather, p.gather == nullptr ? 0u : (uint32_t)p.R * 4u);
    return (int)__builtin_amdgcn_raw_buffer_load_b32(map, (at.lo + min(r, at.n - 1)) * 4, 0, 0);
  }
  // row of X that row r of an expert reads, or -1: none
  static __device__ __forceinline__ int x_row(const Args& p, const Place& at, int r, int entry) {
    return p.gather == nullptr ? at.lo + min(r, at.n - 1) : token(p, entry);
  }
  // physical rows as in Ragged::rows; of rows lane, lane + 64 of the wave tile twice the row (+ 1: a row of zeros), or OOB
  template <int TM, int RA>
  static __device__ __forceinline__ void rows(const Args& p, const Place& at, int q0, int w0, int (&q_row)[RA], uint32_t (&out)[2]) {
    int e[RA + 2];
#pragma unroll
    for (int j = 0; j < RA + 2; ++j) e[j] = entry(p, at, j < RA ? q0 + 8 * j : w0 + 64 * (j - RA));
#pragma unroll
    for (int j = 0; j < RA; ++j) q_row[j] = max(x_row(p, at, q0 + 8 * j, e[j]), 0);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int r = w0 + 64 * j;
      if (r < at.n) out[j] = 2u * (uint32_t)(at.lo + r) + (x_row(p, at, r, e[RA + j]) < 0 ? 1u : 0u);
    }
  }

  template <typename CF>
  struct Scales {
    static constexpr int TM = CF::TM, TN = CF::TN, NW = CF::NW, MB = CF::MB, NB = CF::NB;
    static constexpr int PA = TM * 4 + 64, PB = TN * 4 + 64, SLOT = 4 * (PA + PB);    // planes of one q, apart so that they fall on different banks
    // A wave requests 64 rows of either operand, PLANES planes of a chunk, every other one of them with each of two refill sets: every set has the same
    // requests, and no branch stands between the products.
    static constexpr int PARTS_A = TM / 64, PARTS_B = TN / 64, PLANES_A = 4 * PARTS_A / NW, PLANES_B = 4 * PARTS_B / NW;
    static_assert(NW % PARTS_A == 0 && NW % PARTS_B == 0 && PLANES_A % 2 == 0 && PLANES_B % 2 == 0 && CF::MR == 16, "requests are dealt evenly");
    __amdgpu_buffer_rsrc_t rA, rB;
    uint32_t off_a, off_b, plane_a, plane_b;            // of this lane's row in a plane; bytes of a plane
    char* to_a;                     // this wave's place in its first plane
    char* to_b;
    int first_a, first_b, chunks, blocks, q;
    uint32_t a[MB], b[NB], next_b[NB], keep;      // a block's two bytes of a k tile; which bytes' blocks exist
    uint32_t lds_a, lds_b;

    __device__ __forceinline__ Scales(const Args& p, const Place& at, int g, int n0, char* smem, int lane, int wave, int wm, int wn)
        : chunks(p.chunks), blocks(p.blocks), q(lane >> 4) {
      plane_a = (uint32_t)p.x_rows * 4u;
      plane_b = (uint32_t)p.n * 4u;
      rA = make_rsrc(p.xs, plane_a * 4u * (uint32_t)chunks);
      rB = make_rsrc(p.ws + (int64_t)g * chunks * 16 * p.n, plane_b * 4u * (uint32_t)chunks);
      const int r = at.tm * TM + 64 * (wave % PARTS_A) + lane;
      off_a = (uint32_t)max(x_row(p, at, r, entry(p, at, r)), 0) * 4u;
      const int c = 64 * (wave % PARTS_B) + lane;
      off_b = (uint32_t)(p.half ? row<EPI_GLU>(p, n0, c) : row<EPI_STORE>(p, n0, c)) * 4u;
      first_a = wave / PARTS_A * PLANES_A;
      first_b = wave / PARTS_B * PLANES_B;
      char* lds = smem + CF::LDS;
      to_a = lds + wave % PARTS_A * 256;
      to_b = lds + 4 * PA + wave % PARTS_B * 256;
      const uint32_t base = (uint32_t)(uintptr_t)(LDS_AS char*)lds;
      lds_a = base + q * PA + (wm * (TM / CF::WM) + (lane & 15)) * 4;
      lds_b = base + 4 * PA + q * PB + (wn * (TN / CF::WN) + (lane & 15)) * 4;
    }

    // half h of this wave's share of chunk c into the chunk's slot; behind the last chunk that one, which nobody reads there
    __device__ __forceinline__ void request(int c, int h) {
      const int slot = (c & 1) * SLOT;
      const uint32_t from = 4u * (uint32_t)min(c, chunks - 1);
#pragma unroll
      for (int r = 0; r < PLANES_A / 2; ++r) {
        const int plane = first_a + 2 * r + h;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rA, (LDS_AS void*)(to_a + slot + plane * PA), 4, (int)off_a, (int)((from + plane) * plane_a), 0, 0);
      }
#pragma unroll
      for (int r = 0; r < PLANES_B / 2; ++r) {
        const int plane = first_b + 2 * r + h;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rB, (LDS_AS void*)(to_b + slot + plane * PB), 4, (int)off_b, (int)((from + plane) * plane_b), 0, 0);
      }
    }
    template <int OFF>
    static __device__ __forceinline__ void lds_read(uint32_t& d, uint32_t addr) {
      asm volatile("ds_read_u16 %0, %1 offset:%2" : "=v"(d) : "v"(addr), "n"(OFF));
    }
    static __device__ __forceinline__ uint32_t tile_at(int t) { return (uint32_t)((t >> 1) & 1) * SLOT + 2u * (uint32_t)(t & 1); }
    // The bytes of k tile t.  Those of rows [FROM, TO) of blocks of A go where the tile before had them, once it has multiplied the row; B's, which
    // every row uses, wait beside them.
    template <int FROM, int TO>
    __device__ __forceinline__ void read_a(int t) {
      const uint32_t at = lds_a + tile_at(t);
      unrolled<FROM, TO>([&](auto i) { lds_read<decltype(i)::value * 64>(a[decltype(i)::value], at); });
    }
    __device__ __forceinline__ void read_b(int t) {
      const uint32_t at = lds_b + tile_at(t);
      unrolled<0, NB>([&](auto j) { lds_read<decltype(j)::value * 64>(next_b[decltype(j)::value], at); });
    }
    // B's, and row 0's of A, have landed.  B's are moved by an instruction of its own behind the wait: as an assignment the compiler is free to copy them
    // in front of it, and does (it takes them as written at the read).  Bytes of blocks that do not exist, which may be the byte of NaN, are taken as
    // 2^-127: whatever the fragments hold there, the products with two of them are under 2^-240, zero in fp32.
    // A product reads a register two instructions behind the vector instruction that wrote it at the earliest, and of an asm the compiler need not know that
    // it is one: the first product reads b[0], NB - 1 moves behind its own.
    template <bool LAST>
    __device__ __forceinline__ void take_b(int t) {
      static_assert(NB >= 3, "two wait states");
      if constexpr (LAST) keep = (8 * t + q < blocks ? 0xFFu : 0u) | (8 * t + 4 + q < blocks ? 0xFF00u : 0u);
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        asm volatile("v_mov_b32 %0, %1" : "=v"(b[j]) : "v"(next_b[j]));
        if constexpr (LAST) b[j] &= keep;
      }
    }
    template <bool LAST, int I>
    __device__ __forceinline__ void take_a() {
      asm volatile("" : "+v"(a[I]));
      if constexpr (LAST) a[I] &= keep;
    }
    // Behind the last tile, whose reads for a next one nobody takes: every read has landed, and until then its register stayed taken.
    __device__ __forceinline__ void landed() {
#pragma unroll
      for (int i = 0; i < MB; ++i) asm volatile("" : "+v"(a[i]));
#pragma unroll
      for (int j = 0; j < NB; ++j) asm volatile("" : "+v"(next_b[j]));
    }
    template <int ST, int I, int J>
    __device__ __forceinline__ void product(f32x4_t& acc, const Frag& fb, const Frag& fa) {
      acc = mx4_mfma<ST>(make_uint4(fb.q[0], fb.q[1], fb.q[2], fb.q[3]), make_uint4(fa.q[0], fa.q[1], fa.q[2], fa.q[3]), acc, b[J], a[I]);
    }
  };

  // Lane l has row l % 16 and columns 4 (l / 16) .. + 3 of each block of 16 x 16.
  template <int KIND, int EPI, int MR, int MB, int NBK, int AM, int AN>
  static __device__ __forceinline__ void store(const Args& p, f32x4_t (&acc)[AM][AN], char* wave_lds, int, int, int mshift, int nbase,
                                               const uint32_t (&out)[2], int lane) {
    static_assert(AM == 2 * MB && AN == 2 * NBK, "blocks of 16 x 16");
    auto row_of = [&](int d, int rl) { return (uint32_t)__shfl((int)(d < 64 ? out[0] : out[1]), (d & 63) + rl, 64); };
    const int l16 = lane & 15, kg = lane >> 4;
    if constexpr (EPI == EPI_GLU) {
      // pieces of 32 columns are 16 of the gate and 16 of the up projection: two of them are 32 hidden columns, one block of A
      static_assert(NBK == 2, "a wave's hidden columns are one block");
      const int h0 = nbase / 2, block = h0 / MX4_BLOCK;
      // Nothing stands in a branch, and lane groups meet without LDS: 8 values of a lane go through the exponential and the reciprocal side by side.
      const bool is[2] = {h0 + 4 * kg < p.half, h0 + 16 + 4 * kg < p.half};
      const __amdgpu_buffer_rsrc_t rQ = make_rsrc(p.aq, (uint32_t)p.R * (uint32_t)p.a_blocks * 16u),
                                   rS = make_rsrc(p.as, (uint32_t)p.R * 16u * ((uint32_t)(p.a_blocks + 15) / 16u));
      const uint32_t q_at = (uint32_t)block * 16u + 8u * (kg & 1) + 4u * (kg >> 1);
      const uint32_t s_at = (uint32_t)((block >> 4) * 4 + (block & 3)) * (uint32_t)p.R * 4u + (uint32_t)((block >> 2) & 3);
      with_hidden(p.act, p.f32, [&](auto act, auto wide) {
#pragma unroll
        for (int i = 0; i < AM; ++i) {
          const uint32_t o = row_of(mshift + 16 * i, l16);
          float v[2][4];
          uint32_t top = 0;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            uint32_t t = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              v[j][e] = mx4_hidden<decltype(act)::value, decltype(wide)::value>(acc[i][2 * j][e], acc[i][2 * j + 1][e]);
              t = max(t, __float_as_uint(v[j][e]) & 0x7FFFFFFFu);
            }
            top = max(top, is[j] ? t : 0u);
          }
          const auto t16 = __builtin_amdgcn_permlane16_swap(top, top, false, false);
          top = max(t16[0], t16[1]);
          const auto t32 = __builtin_amdgcn_permlane32_swap(top, top, false, false);
          top = max(t32[0], t32[1]);
          const bool zero = o & 1u;
          const int b = zero ? 0 : mx4_scale(top);
          const uint32_t c0 = is[0] ? mx4_pack4(v[0], b) : 0u, c1 = is[1] ? mx4_pack4(v[1], b) : 0u;
          // neighbouring lane groups make dwords: the even one of columns 0..15, the odd one of 16..31
          const auto c = __builtin_amdgcn_permlane16_swap(c0, c1, false, false);
          const bool stored = o != OOB && h0 < p.half;
          const uint32_t r = o >> 1;
          __builtin_amdgcn_raw_buffer_store_b32(zero ? 0u : c[0] | c[1] << 16, rQ, (int)(stored ? r * ((uint32_t)p.a_blocks * 16u) + q_at : OOB), 0, 0);
          __builtin_amdgcn_raw_buffer_store_b8((uint8_t)b, rS, (int)(stored && kg == 0 ? r * 4u + s_at : OOB), 0, 0);
        }
      });
    } else if (p.f32) {
#pragma unroll
      for (int i = 0; i < AM; ++i) {
        const uint32_t o = row_of(mshift + 16 * i, l16);
        float* c = reinterpret_cast<float*>(p.C) + (int64_t)(o >> 1) * p.n;
#pragma unroll
        for (int j = 0; j < AN; ++j) {
          const int n = nbase + 16 * j + 4 * kg;
          if (o != OOB && n < p.n) *reinterpret_cast<f32x4_t*>(c + n) = o & 1u ? f32x4_t{0.f, 0.f, 0.f, 0.f} : acc[i][j];
        }
      }
    } else {            // through the wave's slice of LDS, 32 rows at a time
      constexpr int CW = 32 * NBK, PITCH = 2 * CW + 16, LPR = CW / 8, RPI = 64 / LPR, NT = 32 / RPI;
      const int rl = lane / LPR, cc = lane % LPR, n = nbase + cc * 8;
#pragma unroll
      for (int i = 0; i < MB; ++i) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int j = 0; j < AN; ++j) {
            const f32x4_t v = acc[2 * i + h][j];
            *reinterpret_cast<uint2*>(wave_lds + (16 * h + l16) * PITCH + (16 * j + 4 * kg) * 2) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
          }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const uint32_t o = row_of(mshift + 32 * i + RPI * t, rl);
          const uint4 v = *reinterpret_cast<const uint4*>(wave_lds + (RPI * t + rl) * PITCH + cc * 16);
          if (o != OOB && n < p.n) *reinterpret_cast<uint4*>(reinterpret_cast<bf16_t*>(p.C) + (int64_t)(o >> 1) * p.n + n) = o & 1u ? make_uint4(0, 0, 0, 0) : v;
        }
      }
    }
  }
};

template <int EPI, typename CF>
__global__ __launch_bounds__(64 * CF::NW, 2) void mx4_gemm(const Mx4TileArgs p) {
  __shared__ __attribute__((aligned(1024))) char smem[CF::LDS + 2 * Mx4::Scales<CF>::SLOT];
  gemm_dma_tile<KIND_NT, EPI, CF, ROWS_PLAIN, Mx4>(p, smem, (int)blockIdx.x);
}

using Mx4Tile256 = TileCfg<256, 256, 2, 4, 1, 2, 2>;
using Mx4Tile128 = TileCfg<128, 128, 2, 2, 1, 2, 2>;

void launch_mx4_tile(const Mx4Args& m, int kind, int tile, hipStream_t st) {
  Mx4TileArgs a{};
  a.off = m.off;
  a.G = m.E; a.n_src = 1; a.Cc = a.R = m.R;
  a.splits = 1;
  a.gather = m.gather; a.gather_k = m.gather_k; a.gather_magic = m.gather_magic; a.gather_rows = m.gather_rows;
  a.A = m.xq; a.lda = 8 * (int64_t)m.blocks;
  a.B = m.wq; a.ldb = 8 * (int64_t)m.blocks; a.b_goff = (int64_t)m.n * a.ldb;
  a.a_bytes = (uint64_t)m.x_rows * (uint64_t)a.lda * 2;
  a.b_bytes = (uint64_t)m.E * (uint64_t)a.b_goff * 2;
  a.C = m.C; a.ldc = (int64_t)m.n * (m.f32 ? 2 : 1);
  a.Mdim = m.R; a.Ndim = m.n; a.Kdim = 8 * m.blocks;
  a.half = m.half; a.act = m.act;
  a.xs = m.xs; a.ws = m.ws; a.x_rows = m.x_rows;
  a.n = m.n; a.blocks = m.blocks; a.chunks = m.chunks; a.f32 = m.f32;
  a.aq = m.aq; a.as = m.as; a.a_blocks = m.a_blocks;
  auto launch = [&](auto cfg) {
    using CF = decltype(cfg);
    const dim3 grid = size_rows(a, CF::TM, CF::TN, kind == MX4_STORE);
    if (kind == MX4_GLU) hipLaunchKernelGGL((mx4_gemm<EPI_GLU, CF>), grid, dim3(64 * CF::NW), 0, st, a);
    else hipLaunchKernelGGL((mx4_gemm<EPI_STORE, CF>), grid, dim3(64 * CF::NW), 0, st, a);
  };
  if (tile == 256) launch(Mx4Tile256{});
  else launch(Mx4Tile128{});
}

}  // namespace moe
