// Matrix tiles of the expert FFN's grouped GEMMs, shared by the calls over capacity-padded rows (ffn.hip) and over ragged rows
// (ragged.hip): the bf16 MFMA tile with an LDS-DMA pipeline, the fp32 tile on the fp64 matrix cores, and what plans them.
//
// A tile is written against a layout L, which says what differs between the two: L::Args (a GemmArgs), L::Place with the expert g
// and the tile (tm, tn), and the static functions
//   find       workgroup -> Place; false: there is no tile to multiply (what has to be stored as zeros has been stored)
//   rows, rows_f32   where a row-tiled GEMM reads and stores the rows of a tile
//   Walk       the k tiles of a weight gradient, whose reduction runs over the expert's rows
//   store, store_f32 the epilogue
//   map_bytes  size of the row map of a gathered operand
#pragma once

#include <algorithm>
#include <type_traits>

#include "common.h"

namespace moe {

enum { KIND_NN = 1, KIND_NT = 2, KIND_TN = 3 };
enum { EPI_STORE = 0, EPI_GELU = 1, EPI_DGELU = 2, EPI_PART = 3 };   // EPI_PART: fp32 partial sums of a split reduction

struct GemmArgs {
  const void* A;
  const void* B;
  void* C;
  void* C2;         // second output (the activation GeLU(Z)) for EPI_GELU
  const void* Zin;  // saved pre-activation for EPI_DGELU
  const int32_t* cnt;  // optional [n_src, G]: rows of chunk (s, g) at or beyond min(cnt, Cc) are zero padding
  // fused dispatch (NN GEMMs, n_src = 1): A is the token matrix and row r of expert g is the token
  // gather[g * Cc + r] / gather_k (the gate's inverse slot map; negative = empty slot, a zero row)
  const int32_t* gather;
  int gather_k;
  uint32_t gather_magic;  // ceil(2^32 / gather_k): v / gather_k = umulhi(v, magic) for v < 2^29 (gather_k <= 8)
  int64_t gather_rows;    // rows of the token matrix
  int G, n_src;
  int Cc;           // rows per chunk (capacity C)
  int R;            // n_src * Cc: virtual rows per expert
  int Mdim, Ndim, Kdim;
  int64_t lda, ldb, ldc;             // leading dimensions, elements
  int64_t b_goff, c_goff;            // per-expert stride of weight-type operands, elements
  int64_t b_off, c_off;              // constant offset of the ESP slice, elements
  int tiles_m, tiles_n, total_tiles;
  int run_mask;                      // tile order (xcd_tile): ~31: the XCDs take runs of 32 tiles in turn; 0: a range each
  uint64_t a_bytes, b_bytes;         // bf16 path: byte sizes of the A and B tensors (buffer descriptors)
  int splits;                        // EPI_PART: parts of the reduction; part q of every expert's matrix in
  float* part;                       // [splits, G, Mdim, Ndim]
};

// ------------------------------------------------------------------------------------------
// bf16 MFMA kernel
// ------------------------------------------------------------------------------------------
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

// The epilogue's 16-byte accesses go through buffer descriptors: a lane that must not load or store passes an offset
// beyond num_records, which reads as zeros and stores nothing, without a branch.  (The requests of the k loop go through
// descriptors too, but always lie inside their tensor: see gemm_dma_tile.)
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
constexpr uint32_t OOB = 0xFFFFFFF0u;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(const void* base, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, bytes, 0x00020000);
}
template <bool STREAM = false>   // STREAM: non-temporal hint, for data read here for the last time
__device__ __forceinline__ uint4 ldb16(__amdgpu_buffer_rsrc_t r, uint32_t byte_off) {
  const u32x4_t v = __builtin_amdgcn_raw_buffer_load_b128(r, (int)byte_off, 0, STREAM ? 2 : 0);
  return make_uint4(v.x, v.y, v.z, v.w);
}

// STREAM = the non-temporal hint, for tensors that are not read again soon (the saved pre-activation,
// the weight gradients): they then do not push the weights and the live activations out of the
// last-level cache, which the next GEMMs read their operands from.
template <bool STREAM = false>
__device__ __forceinline__ void stb16(__amdgpu_buffer_rsrc_t r, uint32_t byte_off, const uint4& v) {
  const u32x4_t q = {v.x, v.y, v.z, v.w};
  __builtin_amdgcn_raw_buffer_store_b128(q, r, (int)byte_off, 0, STREAM ? 2 : 0);
}
// The accumulators come in MFMA blocks of MR x MR; a 32 x 32 piece of the wave tile is four groups of 4 consecutive
// columns per lane either way (quad()).
template <int MR> struct AccBlock;
template <> struct AccBlock<32> { typedef f32x16_t type; };
template <> struct AccBlock<16> { typedef f32x4_t type; };

// ------------------------------------------------------------------------------------------
// bf16 MFMA tile with an LDS-DMA pipeline.
//
// TM x TN output tile, k tile 64, WM x WN waves over the tile times WK waves over the MFMA steps of a k tile (two
// of 32 k or four of 16 k; WK = 2: two of the four per group, whose sums are added through LDS at the end).  Global memory
// goes straight to LDS (buffer_load ... lds, 16 bytes per lane, no VGPR staging, no ds_write) into two rings of whole k
// tiles, SA tiles of the A operand and SB of the B operand.  A k tile is 64 wide so that every request of a k-contiguous
// operand covers whole 128-byte lines.  A wave instruction fills 1 KiB of consecutive 16-byte slots in lane
// order, so a tile is stored unpadded and bank conflicts are avoided by permuting WHICH 16-byte chunk of a row
// each lane fetches (an XOR swizzle that the fragment reads undo).  Every lane of a request fetches from inside the
// tensor: the zero fill of an out-of-range request can reach LDS after the wait for it is over, and would then
// destroy what the slot was refilled with.  Rows and columns outside the problem and padding rows are fetched
// from another row / column (what they yield is not stored, or stored as zeros), k indexes behind the end of a k tile
// from its first one (the fragments of both operands are masked).
//   operand with k contiguous in memory : [row][64 k] (128-byte rows, 8 chunks), chunk c of row r in slot
//       c ^ ((r >> 1) & 7); fragments are read with ds_read_b128.
//   operand with k as the slow index    : [64 k][T cols], chunk c of k-row k in slot c ^ 4 (k & 3) (T = 64:
//       c ^ 4 ((k >> 1) & 1); 16 x 16 MFMAs: also ^ 2 ((k >> 3) & 1), because the 16-lane groups then differ in k);
//       fragments are read with the transposing LDS load ds_read_b64_tr_b16: a
//       16-lane group reads a 4(k) x 16(col) patch (lane s: k-row s/4, 8-byte piece s%4) and lane i receives
//       the 4 k-values of column i.
// Pipeline: the fragments of MFMA step s+1 are read under step s, each between two MFMAs (Reads).  Once per k tile, inside its
// last step (when the fragments of that step are in registers, so nobody needs the tile's LDS any more), each wave waits until
// its own requests for the next tile have landed, all waves meet at a barrier, the fragments of the next tile's
// first step are read, and the freed slots are refilled: tile t+SB of B, then tile t+SA of A, one request
// between MFMA rows.  The last SA tiles have nothing to request behind them; they are a loop of their own, in which a
// wave waits for all of its requests instead of for the older ones by count.
// What bounds it: with every compute unit busy, the power limit (the clock falls to 1.7 - 1.8 GHz) and the delivery
// of tiles from L2; with few tiles, the latency of a k tile.  k tiles of 64 instead of 32 (64-byte pieces of
// k-contiguous rows fetch half a cache line and look every line up twice): 8 experts of 16384 x 4096 x 7168, per
// GEMM, 6.83 / 6.44 (forward) and 6.90 / 7.59 (backward) -> 6.3 / 5.9 and 6.1 / 6.1 ms, 1.1 - 1.2 -> 1.2 - 1.35
// PFLOP/s.  Four waves of 128 x 128 and rows padded off a power of two measured no better.
// Which MFMA: under the power limit 16x16x32 costs less energy per flop than 32x32x16 (on random operands in registers 2.05
// against 1.81 PFLOP/s, operands from LDS 1.80 against 1.55).  In this kernel it buys clock, 1.74 against 1.51 GHz, and
// pays only with the reads spread between the MFMAs: reads behind every fourth MFMA, 65 % of the cycles busy and no
// gain; spread, 69 %: the three launches of the GEMMs above and the merged backward launch 6.74 / 6.27 / 6.45 / 18.99 ->
// 6.57 / 6.11 / 6.25 / 18.39 ms.  The tiles with two wave groups over k keep 32x32x16, which gives each group two steps
// per k tile, and so do weight gradients with few k tiles (Tile256Brief), which are not under the power limit.  Tried
// without gain: rows of the last step in front of the barrier 2 -> 3 or 4 (to 4 % slower at 12 k tiles), s_setprio for half
// of the waves, a second barrier that frees B's slot in the first step (-1 to +3 % in single launches).
// ------------------------------------------------------------------------------------------
#define LDS_AS __attribute__((address_space(3)))
constexpr int DK = 64;   // k tile
// s_waitcnt immediate that waits until at most n vector-memory operations are outstanding (gfx9 encoding)
constexpr int vmcnt_imm(int n) { return 0x0F70 | (n & 15) | ((n >> 4) << 14); }
constexpr int lgkmcnt_imm(int n) { return 0xC07F | (n << 8); }   // LDS operations of a wave end in order

template <int TM_, int TN_, int WM_, int WN_, int WK_, int SA_, int SB_, int MR_ = WK_ == 1 ? 16 : 32>
struct TileCfg {
  static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_, WK = WK_, SA = SA_, SB = SB_;
  static constexpr int NW = WM * WN * WK;             // waves
  static constexpr int MR = MR_;                      // MFMA: MR x MR x KS
  static constexpr int KS = 512 / MR;
  static constexpr int MB = TM / WM / MR, NB = TN / WN / MR;   // MFMA blocks per wave
  static constexpr int RA = TM / 8 / NW, RB = TN / 8 / NW;     // requests (1 KiB) per wave and k tile
  static constexpr int SPT = DK / KS / WK;            // MFMA steps per wave and k tile
  static constexpr int A_UNIT = TM * DK * 2, B_UNIT = TN * DK * 2;
  static constexpr int LDS = SA * A_UNIT + SB * B_UNIT;
  static_assert(SPT % 2 == 0, "the steps take turns with the two register sets of B fragments");
  static_assert(TM / 8 % NW == 0 && TN / 8 % NW == 0, "requests are dealt evenly");
  static_assert(SA == SB || SA == SB + 1, "ring depths");
};

__device__ __forceinline__ void dma16(__amdgpu_buffer_rsrc_t r, char* lds_wave_base, uint32_t byte_off) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (LDS_AS void*)lds_wave_base, 16, (int)byte_off, 0, 0, 0);
}
// Fragment reads are issued as volatile asm: the compiler then neither reorders them nor guards
// them with conservative waits against the LDS-DMA requests in flight.  The kernel waits for them
// itself (s_waitcnt lgkmcnt(0)) and passes the registers through ready() before the MFMAs use them.  Every read is
// waited for like that, also one that is not used: the compiler takes the registers as written at the read.
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
union Frag {
  bf16x8_t v;
  u32x4_t q;
  u32x2_t h[2];
};
template <int OFF>
__device__ __forceinline__ void lds_read_kc(Frag& f, uint32_t addr) {
  asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(f.q) : "v"(addr), "n"(OFF));
}
template <int OFF, int HOFF>   // HOFF: distance of the second half's k-rows
__device__ __forceinline__ void lds_read_nc(Frag& f, uint32_t addr) {
  asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(f.h[0]) : "v"(addr), "n"(OFF));
  asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(f.h[1]) : "v"(addr), "n"(OFF + HOFF));
}
__device__ __forceinline__ void ready(Frag& f) { asm volatile("" : "+v"(f.q)); }

template <int I, int N, typename F>
__device__ __forceinline__ void unrolled(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    unrolled<I + 1, N>(f);
  }
}

// Workgroup -> output tile.  Workgroup ids are dealt round-robin to the 8 XCDs, so id % 8 names the XCD (problems
// of a merged launch start at multiples of 8).  Linear tile order: expert by expert, blocks of 16 row tiles, in a block
// strips of 4 tile columns, in a strip row by row.  32 consecutive tiles (what an XCD's 32 CUs run at the same time) then
// form an 8 x 4 patch, which shares 8 + 4 operand slices per k step in that XCD's L2 instead of 1 + 32, and the XCDs take
// consecutive patches: the whole chip is in one 16 x 16 block, whose operands the last-level cache can hold until the
// block is done (what misses L2 stays the same).  (With a contiguous range of the order per XCD the eight XCDs were in
// eight experts, whose strips together do not fit that cache: 8 experts of 16384 x 4096 x 7168, two forward GEMMs,
// dZ, merged backward: 6.57 / 6.11 / 6.25 / 18.39 -> 6.12 / 5.50 / 5.91 / 17.11 ms on one card.)
// Where an expert's operands fit in an XCD's L2 (tile_runs) a row-tiled GEMM keeps the contiguous ranges: an XCD then reads
// those of few experts, and every strip but the first finds them in its L2.
// t = index within an expert of tm_n row tiles.
__device__ __forceinline__ void patch_order(int t, int tm_n, int tiles_n, int& tm, int& tn) {
  constexpr int SW = 4, RB = 16;
  int m0 = 0;                           // first row tile of the block
  if (tm_n > RB) {                      // (a division that few rows do without)
    m0 = t / (RB * tiles_n) * RB;
    t -= m0 * tiles_n;
    tm_n = min(RB, tm_n - m0);
  }
  const int full = tiles_n / SW, strip = tm_n * SW;
  if (t < full * strip) {
    const int sn = t / strip, r = t - sn * strip;
    tm = r / SW;
    tn = sn * SW + (r - tm * SW);
  } else {
    const int w = tiles_n - full * SW, r = t - full * strip;
    tm = r / w;
    tn = full * SW + (r - tm * w);
  }
  tm += m0;
}
// the i-th of n tiles (n = 8 per_xcd, rounded up) that XCD x takes: runs of 32 in turn, or one range
__device__ __forceinline__ int xcd_tile(const GemmArgs& p, int x, int i, int per_xcd) {
  const int full = per_xcd & p.run_mask;
  return i < full ? ((i & ~31) * 8 + x * 32) + (i & 31) : full * 8 + x * (per_xcd - full) + (i - full);
}

struct KTile {
  int row0, lim;   // first row of the k tile in the operand (row-tiled GEMMs: first k), rows (k values) that exist
};

// The fragment reads of a tile's k loop.  A row's A fragment is replaced by the next step's once the row has been
// multiplied, the B fragments, which every row uses, have two register sets.  The next step's reads are taken in
// the order B0 A0 B1 A1 ... and spread between the MFMAs (place: behind which MFMA of the step), so that
// they do not queue up in front of the multiplications.  A row waits for its own fragments by count: the LDS reads of a
// wave return in order.
template <int KIND, typename CF>
struct Reads {
  static constexpr int MB = CF::MB, NB = CF::NB, N = MB + NB;
  static constexpr int BR = MB > 4 ? 2 : 1;          // rows of a k tile's last step in front of the barrier
  static_assert(MB >= NB, "the order of the reads");
  static constexpr bool is_b(int op) { return op < 2 * NB && op % 2 == 0; }
  static constexpr int of(int op) { return op < 2 * NB ? op / 2 : op - NB; }     // which fragment
  static constexpr int ins(int op) { return (is_b(op) ? KIND != KIND_NT : KIND == KIND_TN) ? 2 : 1; }   // LDS instructions
  static constexpr int place(int st, int op) {
    if (st == CF::SPT - 1) return BR * NB - 1 + op * (MB * NB - BR * NB) / (N - 1);   // behind the barrier
    return is_b(op) ? of(op) * NB + NB / 2 : of(op) + 1 < MB ? (of(op) + 1) * NB : MB * NB - 1;
  }
  static constexpr bool in_place() {                 // no A fragment is replaced before its row has been multiplied
    for (int op = 0; op < N; ++op)
      if (!is_b(op) && (place(0, op) < of(op) * NB + NB - 1 || place(CF::SPT - 1, op) < of(op) * NB + NB - 1)) return false;
    return true;
  }
  static_assert(in_place(), "the order of the reads");
  // LDS instructions that may still be in flight when row `row` of step st is about to be multiplied
  static constexpr int newer(int st, int row) {
    int n = 0;
    const int need = row == 0 ? (NB > 1 ? 2 * NB - 2 : 1) : row < NB ? 2 * row + 1 : row + NB;   // row 0: every B fragment
    for (int op = need + 1; op < N; ++op) n += ins(op);
    for (int op = 0; op < N; ++op) n += place(st, op) < row * NB ? ins(op) : 0;
    return n < 15 ? n : 15;
  }
};


// How a weight-gradient GEMM finds its k-rows.  GATHER: the k-slow A operand (X^T dZ) is the token matrix read through the
// inverse slot map (row r of the chunk is token gather[g C + r] / gather_k); n_src = 1.  PACKED: k tiles of pieces of
// several chunks (ChunkWalk).
enum { ROWS_PLAIN = 0, ROWS_GATHER = 1, ROWS_PACKED = 2 };
template <int KIND, int EPI, typename CF, int ROWS, typename L>
__device__ __forceinline__ void gemm_dma_tile(const typename L::Args& p, char* smem, int vb) {
  constexpr bool GATHER = ROWS == ROWS_GATHER, PIECES = ROWS == ROWS_PACKED;
  constexpr bool A_NC = (KIND == KIND_TN);                     // A has k as the slow index
  constexpr bool B_NC = (KIND == KIND_NN || KIND == KIND_TN);  // B has k as the slow index
  constexpr int TM = CF::TM, TN = CF::TN, WM = CF::WM, WN = CF::WN, WK = CF::WK, SA = CF::SA, SB = CF::SB;
  constexpr int MB = CF::MB, NB = CF::NB, RA = CF::RA, RB = CF::RB, SPT = CF::SPT, MR = CF::MR, KS = CF::KS;
  constexpr int WTM = TM / WM, WTN = TN / WN;   // wave tile
  static_assert(!A_NC || TM == 64 || TM == 128 || TM == 256, "k-slow tiles are a power of two wide");
  static_assert(ROWS == ROWS_PLAIN || KIND == KIND_TN, "rows of a reduction");
  static_assert(!GATHER || (KIND == KIND_TN && CF::NW == 8), "row gather in the reduction: eight k-rows per wave");

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);   // uniform: keeps LDS bases in SGPRs
  const int wk = WK == 1 ? 0 : wave / (WM * WN);
  const int wm = (wave / WN) % WM, wn = wave % WN;

  int part = 0;   // EPI_PART: which part of the reduction; the parts of a tile are total_tiles apart
  if (EPI == EPI_PART) {
    const int per = (p.total_tiles + 7) / 8 * 8;
    part = vb / per;
    vb -= part * per;
  }
  typename L::Place at;
  if (!L::template find<KIND, EPI, 2, TM, TN>(p, vb, at)) return;
  const int g = at.g, m0 = at.tm * TM, n0 = at.tn * TN;

  const int64_t b_base = (int64_t)g * p.b_goff + p.b_off;
  const __amdgpu_buffer_rsrc_t rA = make_rsrc(p.A, (uint32_t)p.a_bytes);
  const uint64_t b_rem = p.b_bytes - (uint64_t)b_base * 2;
  const __amdgpu_buffer_rsrc_t rB =
      (KIND == KIND_TN) ? make_rsrc(p.B, (uint32_t)p.b_bytes)
                        : make_rsrc(reinterpret_cast<const bf16_t*>(p.B) + b_base, b_rem > OOB ? OOB : (uint32_t)b_rem);

  // physical rows of the requests' A rows (row-tiled GEMMs) and of rows lane, lane + 64 of the wave tile
  int q_row[RA];
  uint32_t out_off[2] = {OOB, OOB};   // byte offset of the row in the output (+ 1: a row of zeros), or OOB
  if (KIND != KIND_TN) L::template rows<TM, RA>(p, at, m0 + wave * RA * 8 + (lane >> 3), m0 + wm * WTM + lane, q_row, out_off);
  // 32 x 32 pieces a wave finishes (WK = 2: MR = 32, a piece is an MFMA block)
  constexpr int EMB = (WK == 2 && MB >= 2) ? MB / 2 : WTM / 32;
  constexpr int ENB = (WK == 2 && MB < 2 && NB >= 2) ? NB / 2 : WTN / 32;
  constexpr bool ONE = WK == 2 && MB < 2 && NB < 2;            // a single block: the second group's waves finish nothing
  const int e_i = (WK == 2 && MB >= 2) ? wk * EMB : 0, e_j = (WK == 2 && MB < 2 && NB >= 2) ? wk * ENB : 0;
  const int e_n = n0 + wn * WTN + 32 * e_j;
  char* e_lds = smem + wave * (CF::LDS / CF::NW / 64 * 64);

  // ---- k tiles: Kdim / 64 of a row-tiled GEMM, the walk over the expert's chunks for a weight gradient ----
  typename L::template Walk<EPI == EPI_PART && !PIECES> walk(p, at, part);
  int nk = KIND == KIND_TN ? walk.start(DK, PIECES) : (p.Kdim + DK - 1) / DK;
  int k_left = nk;               // packed parts: k tiles that the walk has not been asked for
  if (EPI == EPI_PART && PIECES) {
    const int t0 = (int)((int64_t)nk * part / p.splits), t1 = (int)((int64_t)nk * (part + 1) / p.splits);
    walk.skip(t0 * DK);
    k_left = nk = t1 - t0;
  }

  // ---- per-lane request coordinates: byte offset of the lane's row / column, the k index within the tile that the
  // request covers (k-slow) or starts at (k-contiguous), and the byte offset of that k index ----
  uint32_t a_req[RA], b_req[RB], a_ko[RA], b_ko[RB];
  int a_k[RA], b_k[RB];
  constexpr int ACPR = TM / 8, BCPR = TN / 8;   // k-slow: 16-byte chunks per k-row
  const uint32_t lda2 = (uint32_t)p.lda * 2u, ldb2 = (uint32_t)p.ldb * 2u;
  auto swz_nc = [](int k, int cpr) {
    return cpr >= 16 ? 4 * (k & 3) + (MR == 16 ? 2 * ((k >> 3) & 1) : 0) : 4 * ((k >> 1) & 1);
  };
#pragma unroll
  for (int j = 0; j < RA; ++j) {
    const int q = wave * RA + j;
    if (!A_NC) {
      a_k[j] = ((lane & 7) ^ ((4 * q + (lane >> 4)) & 7)) * 8;
      a_req[j] = (uint32_t)q_row[j] * lda2;
      a_ko[j] = (uint32_t)a_k[j] * 2u;
    } else {
      a_k[j] = q * (64 / ACPR) + lane / ACPR;
      const int col = m0 + (((lane % ACPR) ^ swz_nc(a_k[j], ACPR)) * 8);
      a_req[j] = (uint32_t)(col < p.Mdim ? col : m0) * 2u;
      a_ko[j] = GATHER ? 0u : (uint32_t)a_k[j] * lda2;
    }
  }
#pragma unroll
  for (int j = 0; j < RB; ++j) {
    const int q = wave * RB + j;
    if (!B_NC) {
      b_k[j] = ((lane & 7) ^ ((4 * q + (lane >> 4)) & 7)) * 8;
      b_req[j] = (uint32_t)min(n0 + q * 8 + (lane >> 3), p.Ndim - 1) * ldb2;
      b_ko[j] = (uint32_t)b_k[j] * 2u;
    } else {
      b_k[j] = q * (64 / BCPR) + lane / BCPR;
      const int col = n0 + (((lane % BCPR) ^ swz_nc(b_k[j], BCPR)) * 8);
      b_req[j] = (uint32_t)(col < p.Ndim ? col : n0) * 2u;
      b_ko[j] = (uint32_t)b_k[j] * ldb2;
    }
  }

  // GATHER: the k-rows of a k tile are token rows.  Lane l loads the slot-map entry of k-row l, one request set ahead of
  // the A requests that use it and before that set's own requests: the wait for tile t+1 at the next barrier then covers
  // the entries as well, and nothing waits for them by itself.  The eight rows a wave requests are the same for all
  // its lanes.  An empty slot is fetched as token 0 and masked.
  uint32_t g_now[RA];   // byte offset of the token row behind this lane's k-row of the next A request
  const __amdgpu_buffer_rsrc_t rG = make_rsrc(p.gather, GATHER ? L::map_bytes(p) : 0u);
  auto gather_fetch = [&](int row0) -> int {   // entries past the map read as zero; rows past the row count are masked
    return (int)__builtin_amdgcn_raw_buffer_load_b32(rG, (row0 + lane) * 4, 0, 0);
  };
  auto gather_rows = [&](int entry) -> uint64_t {   // returns which of the 64 slots are occupied
    constexpr int RPR = A_NC ? 64 / ACPR : 1;   // k-rows per request
    const uint32_t tok = p.gather_k == 1 ? (uint32_t)entry : __umulhi((uint32_t)entry, p.gather_magic);
    const bool full = entry >= 0 && (int64_t)tok < p.gather_rows;
    const uint32_t off = full ? tok * (uint32_t)(p.lda * 2) : 0u;
#pragma unroll
    for (int j = 0; j < RA; ++j) {
      uint32_t o = (uint32_t)__builtin_amdgcn_readlane((int)off, (wave * RA + j) * RPR);
#pragma unroll
      for (int u = 1; u < RPR; ++u) {
        const uint32_t v = (uint32_t)__builtin_amdgcn_readlane((int)off, (wave * RA + j) * RPR + u);
        o = lane / ACPR == u ? v : o;
      }
      g_now[j] = o;
    }
    return __ballot(full);
  };
  // PIECES: byte offsets of this lane's k-rows in the newest k tile (A's next requests) and the one before it (B's)
  uint32_t ka_off[PIECES ? RA : 1], kb_off[PIECES ? RB : 1], kb_new[PIECES ? RB : 1];
  static_assert(!PIECES || SA == SB + 1, "B's requests are a k tile behind A's");
  auto next_ktile = [&]() -> KTile {
    KTile t{0, 0};                                   // past the end: no rows
    if (EPI != EPI_PART || !PIECES || k_left-- > 0) t = walk.next(DK);
    if constexpr (PIECES) {
#pragma unroll
      for (int j = 0; j < RB; ++j) { kb_off[j] = kb_new[j]; kb_new[j] = (uint32_t)t.row0 * ldb2 + b_ko[j]; }
#pragma unroll
      for (int j = 0; j < RA; ++j) ka_off[j] = (uint32_t)t.row0 * lda2 + a_ko[j];
      {
        while (t.lim > 0 && t.lim < DK) {
          const KTile piece = walk.next(DK - t.lim);
          if (piece.lim == 0) break;
          const uint32_t d = (uint32_t)(piece.row0 - t.lim);
#pragma unroll
          for (int j = 0; j < RA; ++j) ka_off[j] = a_k[j] >= t.lim ? d * lda2 + a_ko[j] : ka_off[j];
#pragma unroll
          for (int j = 0; j < RB; ++j) kb_new[j] = b_k[j] >= t.lim ? d * ldb2 + b_ko[j] : kb_new[j];
          t.lim += piece.lim;
        }
      }
      if (t.lim < DK) {   // missing k rows are fetched from the tile's first one
#pragma unroll
        for (int j = 0; j < RA; ++j) ka_off[j] = a_k[j] < t.lim ? ka_off[j] : (uint32_t)t.row0 * lda2;
#pragma unroll
        for (int j = 0; j < RB; ++j) kb_new[j] = b_k[j] < t.lim ? kb_new[j] : (uint32_t)t.row0 * ldb2;
      }
    }
    return t;
  };
  // One request (1 KiB) of k tile kt into ring slot `slot`.
  auto request_a = [&](const KTile& kt, int slot, int j) {
    const uint32_t in = a_k[j] < kt.lim ? a_ko[j] : 0u;   // missing k rows are fetched from the tile's first one
    const uint32_t add = GATHER ? g_now[j] : PIECES ? ka_off[PIECES ? j : 0] : (uint32_t)kt.row0 * (A_NC ? lda2 : 2u) + in;
    dma16(rA, smem + slot * CF::A_UNIT + (wave * RA + j) * 1024, a_req[j] + add);
  };
  auto request_b = [&](const KTile& kt, int slot, int j) {
    const uint32_t in = b_k[j] < kt.lim ? b_ko[j] : 0u;
    const uint32_t add = PIECES ? kb_off[PIECES ? j : 0] : (B_NC ? (uint32_t)kt.row0 * ldb2 : (uint32_t)kt.row0 * 2u) + in;
    dma16(rB, smem + SA * CF::A_UNIT + slot * CF::B_UNIT + (wave * RB + j) * 1024, b_req[j] + add);
  };
  auto ktile_at = [&](int t) -> KTile { return KTile{t * DK, p.Kdim - t * DK}; };   // row-tiled GEMMs

  // ---- per-lane fragment addresses (bytes); see the layout above ----
  const uint32_t lds0 = (uint32_t)(uintptr_t)(LDS_AS char*)smem;
  uint32_t a_fr[A_NC ? MB : 1], b_fr[B_NC ? NB : 1];
  {
    const int b = lane >> 4, s = lane & 15;
    const int chunk = ((wk * SPT * (KS / 8) + lane / MR) ^ ((lane >> 1) & 7)) * 16;
    const int oct = MR == 32 ? b >> 1 : b, half = MR == 32 ? 16 * (b & 1) : 0;   // k-slow: the 16-lane group's patch
    const int knc = KS * wk * SPT + 8 * oct + (s >> 2);
    if (!A_NC) {
      a_fr[0] = lds0 + (wm * WTM + (lane & (MR - 1))) * 128 + chunk;
    } else {
#pragma unroll
      for (int i = 0; i < (A_NC ? MB : 1); ++i) {
        const int col = wm * WTM + MR * i + half + 4 * (s & 3);
        a_fr[i] = lds0 + knc * (2 * TM) + (((col >> 3) ^ swz_nc(knc, ACPR)) * 16) + ((s & 1) * 8);
      }
    }
    if (!B_NC) {
      b_fr[0] = lds0 + SA * CF::A_UNIT + (wn * WTN + (lane & (MR - 1))) * 128 + chunk;
    } else {
#pragma unroll
      for (int j = 0; j < (B_NC ? NB : 1); ++j) {
        const int col = wn * WTN + MR * j + half + 4 * (s & 3);
        b_fr[j] = lds0 + SA * CF::A_UNIT + knc * (2 * TN) + (((col >> 3) ^ swz_nc(knc, BCPR)) * 16) + ((s & 1) * 8);
      }
    }
  }
  // a row's A fragment is replaced by the next step's once the row has been multiplied; B has two register sets
  Frag fa[MB], fb[2][NB];
  using RD = Reads<KIND, CF>;
  constexpr int BR = RD::BR;
  auto read_op = [&](int slot_a, int slot_b, auto st_tag, auto op_tag) {   // read `op` of step ST
    constexpr int ST = decltype(st_tag)::value, OP = decltype(op_tag)::value, I = RD::of(OP);
    if constexpr (RD::is_b(OP)) {
      const uint32_t so = (uint32_t)slot_b * CF::B_UNIT;
      if constexpr (!B_NC) lds_read_kc<I * MR * 128>(fb[ST & 1][I], (b_fr[0] + so) ^ (2u * KS * ST));
      else lds_read_nc<ST * KS * 2 * TN, 8 * TN>(fb[ST & 1][I], b_fr[B_NC ? I : 0] + so);
    } else {
      const uint32_t so = (uint32_t)slot_a * CF::A_UNIT;
      if constexpr (!A_NC) lds_read_kc<I * MR * 128>(fa[I], (a_fr[0] + so) ^ (2u * KS * ST));
      else lds_read_nc<ST * KS * 2 * TM, 8 * TM>(fa[I], a_fr[A_NC ? I : 0] + so);
    }
  };
  auto frags_ready = [&](int set) {
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
#pragma unroll
    for (int i = 0; i < MB; ++i) ready(fa[i]);
#pragma unroll
    for (int j = 0; j < NB; ++j) ready(fb[set][j]);
  };

  typename AccBlock<MR>::type acc[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int q = 0; q < MR * MR / 64; ++q) acc[i][j][q] = 0.f;

  // Refill set t (issued after the barrier of tile t): tile t+SB of B, then tile t+SA of A.  kb, ka: its tiles.
  constexpr int NREQ = RA + RB;
  // The requests of a set are spread evenly over the MFMAs up to the next barrier: issued together they stall the waves (all
  // behind the barrier, 128 x 128 tiles over 860 k tiles: 604 -> 724 us; two at a time, the merged launch of 256 x 256
  // tiles: 17.1 -> 18.1 ms).
  constexpr int SL_LAST = (MB - BR) * NB + 1, SL = SL_LAST + (SPT - 1) * MB * NB;   // slots: in the last step, in all
  constexpr auto slot_of = [](int r) constexpr { return r * SL / NREQ; };
  constexpr auto before = [](int slot) constexpr {
    int n = 0;
    for (int r = 0; r < NREQ; ++r) n += r * SL / NREQ < slot;
    return n;
  };
  constexpr int N_LAST = before(SL_LAST);                            // requests issued in the last step
  // newer requests than those of tile t+1, at barrier t
  constexpr int IN_FLIGHT = (SA > SB ? RA : 0) + (SB - 2) * (NREQ + (GATHER ? 1 : 0));
  KTile ka{0, 0}, kb{0, 0};
  int g_entry = 0;        // GATHER: slot-map entries of g_next, the tile after ka
  KTile g_next{0, 0};
  uint64_t k_mask[SA];    // TN: which k-rows of tiles t .. t + SA - 1 exist (GATHER: and are occupied)
  int k_lim[SA];          // GATHER: their numbers of rows
  auto mask_of = [&](const KTile& kt, uint64_t full) -> uint64_t {
    return kt.lim >= DK ? full : kt.lim <= 0 ? 0ull : full & ((1ull << kt.lim) - 1ull);
  };
  // prologue: the refills that would have gone before the first tile, and the last-step part of set -1
  {
    KTile pro[SA];
#pragma unroll
    for (int t = 0; t < SA; ++t)
      if (!PIECES) pro[t] = KIND == KIND_TN ? next_ktile() : ktile_at(t);
    int g_pro[SA];
    if (GATHER) {
#pragma unroll
      for (int t = 0; t < SA; ++t) g_pro[t] = gather_fetch(pro[t].row0);
      g_next = next_ktile();
      g_entry = gather_fetch(g_next.row0);
    }
    auto pro_a = [&](int t) {
      const uint64_t full = GATHER ? gather_rows(g_pro[t]) : ~0ull;
      k_mask[t] = mask_of(pro[t], full);
      k_lim[t] = pro[t].lim;
    };
#pragma unroll
    for (int st = -SA; st <= -2; ++st) {
      if (PIECES) pro[st + SA] = next_ktile();
      if (st + SB >= 0) {
#pragma unroll
        for (int j = 0; j < RB; ++j)
          if (pro[st + SB].lim > 0) request_b(pro[st + SB], st + SB, j);
      }
      pro_a(st + SA);
#pragma unroll
      for (int j = 0; j < RA; ++j)
        if (pro[st + SA].lim > 0) request_a(pro[st + SA], st + SA, j);
    }
    if (PIECES) pro[SA - 1] = next_ktile();
    ka = pro[SA - 1];
    kb = pro[SB - 1];
    pro_a(SA - 1);
    unrolled<0, N_LAST>([&](auto r) {
      constexpr int R = decltype(r)::value;
      if constexpr (R < RB) { if (kb.lim > 0) request_b(kb, SB - 1, R); }
      else { if (ka.lim > 0) request_a(ka, SA - 1, R - RB); }
    });
    // this wave's requests for tile 0 have landed
    if (nk >= SA) __builtin_amdgcn_s_waitcnt(vmcnt_imm(IN_FLIGHT + N_LAST));
    else __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
    __builtin_amdgcn_s_barrier();
  }
  using K0 = std::integral_constant<int, 0>;
  unrolled<0, RD::N>([&](auto op) { read_op(0, 0, K0{}, op); });

  auto mfma = [&](int set, int i, int j) {
    if constexpr (MR == 32) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[set][j].v, fa[i].v, acc[i][j], 0, 0, 0);
    else acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[set][j].v, fa[i].v, acc[i][j], 0, 0, 0);
  };
  int sa = 0, sb = 0;                 // ring slots of the current tile
  int wa = SA - 1, wb = SB - 1;       // ring slots that the refill set in progress goes to
  auto issue = [&](auto slot_tag, auto last_tag) {    // the requests of a slot; LAST: the tile may be past the end
    constexpr bool LAST = decltype(last_tag)::value;
    unrolled<0, NREQ>([&](auto r) {
      constexpr int R = decltype(r)::value;
      if constexpr (slot_of(R) == decltype(slot_tag)::value) {
        if constexpr (R < RB) { if (!LAST || kb.lim > 0) request_b(kb, wb, R); }
        else { if (!LAST || ka.lim > 0) request_a(ka, wa, R - RB); }
      }
    });
  };
  // zeroes the k-rows of set `set` (step ST of a tile) that do not exist, in both operands: what was fetched in their
  // place may be an infinity.  (GATHER: an empty slot is a row of zeros in A only, as in the dispatched buffer.)
  auto mask_frags = [&](uint64_t mask_a, uint64_t mask_b, auto st_tag) {
    constexpr int ST = decltype(st_tag)::value;
    auto lanes = [&](uint64_t mask) {
      const uint32_t bits = (uint32_t)(mask >> (KS * (wk * SPT + ST))) >> (8 * (lane / MR));
      u32x4_t m;
      if (KIND != KIND_TN) {   // K % 8 == 0: a lane's 8 values exist together
        const uint32_t all = (bits & 1u) ? ~0u : 0u;
        m = u32x4_t{all, all, all, all};
        return m;
      }
#pragma unroll
      for (int d = 0; d < 4; ++d) m[d] = ((bits >> (2 * d)) & 1u) * 0x0000FFFFu + ((bits >> (2 * d + 1)) & 1u) * 0xFFFF0000u;
      return m;
    };
    const u32x4_t ma = lanes(mask_a), mb = GATHER ? lanes(mask_b) : ma;
#pragma unroll
    for (int i = 0; i < MB; ++i) fa[i].q &= ma;
#pragma unroll
    for (int j = 0; j < NB; ++j) fb[ST & 1][j].q &= mb;
  };
  // one k tile; LAST: one of the last SA tiles, whose refills may be past the end
  auto k_tile = [&](int t, auto last_tag) {
    constexpr bool LAST = decltype(last_tag)::value;
    const int na = sa + 1 == SA ? 0 : sa + 1, nb = sb + 1 == SB ? 0 : sb + 1;   // slots of tile t+1
    const uint64_t mask = KIND == KIND_TN ? k_mask[0] : LAST ? mask_of(ktile_at(t), ~0ull) : ~0ull;
    const uint64_t mask_b = GATHER ? mask_of(KTile{0, k_lim[0]}, ~0ull) : mask;
    unrolled<0, SPT>([&](auto st) {
      constexpr int ST = decltype(st)::value;
      using NEXT = std::integral_constant<int, (ST + 1) % SPT>;
      // row 0 needs its own A fragment and all B fragments; a step with missing k rows waits for everything and masks it
      __builtin_amdgcn_s_waitcnt(lgkmcnt_imm(RD::newer(ST, 0)));
#pragma unroll
      for (int j = 0; j < NB; ++j) ready(fb[ST & 1][j]);
      ready(fa[0]);
      if constexpr (KIND == KIND_TN || LAST) {
        if (__builtin_expect(mask != ~0ull, 0)) {   // (its code stays out of the k loop's way)
          frags_ready(ST & 1);
          mask_frags(mask, mask_b, st);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      unrolled<0, MB>([&](auto i) {
        constexpr int I = decltype(i)::value;
        if constexpr (I > 0) {
          if constexpr (ST < SPT - 1 || I < BR) __builtin_amdgcn_s_waitcnt(lgkmcnt_imm(RD::newer(ST, I)));
          ready(fa[I]);
        }
        unrolled<0, NB>([&](auto j) {
          constexpr int J = decltype(j)::value, AT = I * NB + J;
          __builtin_amdgcn_sched_barrier(0);
          mfma(ST & 1, I, J);
          __builtin_amdgcn_sched_barrier(0);
          if constexpr (ST == SPT - 1 && AT == BR * NB - 1) {
            // this wave's requests for tile t+1 have landed; so have its reads of tile t
            __builtin_amdgcn_s_waitcnt(vmcnt_imm(LAST ? 0 : IN_FLIGHT) & 0xF0FF);
            __builtin_amdgcn_s_barrier();                        // everyone is done with tile t, and tile t+1 is complete
            __builtin_amdgcn_sched_barrier(0);
            wa = sa; wb = sb;
            if (KIND == KIND_TN) {
              const KTile nx = GATHER ? g_next : next_ktile();
              if constexpr (SA > SB) kb = ka; else kb = nx;
              ka = nx;
              uint64_t full = ~0ull;
              if (GATHER) {
                full = gather_rows(g_entry);
                g_next = next_ktile();
                g_entry = gather_fetch(g_next.row0);
              }
#pragma unroll
              for (int u = 0; u + 1 < SA; ++u) { k_mask[u] = k_mask[u + 1]; k_lim[u] = k_lim[u + 1]; }
              k_mask[SA - 1] = mask_of(ka, full);
              k_lim[SA - 1] = ka.lim;
            } else {
              ka = ktile_at(t + SA);
              kb = ktile_at(t + SB);
            }
          }
          unrolled<0, RD::N>([&](auto op) {
            if constexpr (RD::place(ST, decltype(op)::value) == AT) {
              if constexpr (ST < SPT - 1) read_op(sa, sb, NEXT{}, op);
              else read_op(na, nb, NEXT{}, op);
            }
          });
          if constexpr (ST < SPT - 1) issue(std::integral_constant<int, SL_LAST + ST * MB * NB + AT>{}, last_tag);
          else if constexpr (AT >= BR * NB - 1) issue(std::integral_constant<int, AT - BR * NB + 1>{}, last_tag);
          __builtin_amdgcn_sched_barrier(0);
        });
      });
    });
    sa = na; sb = nb;
  };
  const int n_main = nk - SA;    // every refill of these tiles exists
  int t = 0;
  for (; t < n_main; ++t) k_tile(t, std::false_type{});
  for (; t < nk; ++t) k_tile(t, std::true_type{});
  // The last tile (or, without k tiles, the prologue) has read a first step that nobody multiplies: its registers stay
  // taken until the reads have landed, or they would overwrite what the compiler puts there.
  frags_ready(0);
  __builtin_amdgcn_s_waitcnt(0x0070);  // every request is done before LDS is reused
  __syncthreads();

  if constexpr (WK == 2) {   // each of the two wave groups finishes half of the blocks: exchange the other halves
    f32x16_t mine[EMB][ENB];
    float4* xch = reinterpret_cast<float4*>(smem) + (size_t)wave * (EMB * ENB * 4 * 64);
    const float4* oth = reinterpret_cast<const float4*>(smem) + (size_t)(wave ^ (WM * WN)) * (EMB * ENB * 4 * 64);
#pragma unroll
    for (int i = 0; i < EMB; ++i)
#pragma unroll
      for (int j = 0; j < ENB; ++j)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          float own[4], snd[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float lo = acc[i][j][q4 * 4 + e];
            const float hi = ONE ? lo : acc[MB >= 2 ? EMB + i : i][MB >= 2 ? j : (ONE ? 0 : ENB) + j][q4 * 4 + e];
            own[e] = wk ? hi : lo;
            snd[e] = wk ? lo : hi;
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) mine[i][j][q4 * 4 + e] = own[e];
          xch[((i * ENB + j) * 4 + q4) * 64 + lane] = make_float4(snd[0], snd[1], snd[2], snd[3]);
        }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < EMB; ++i)
#pragma unroll
      for (int j = 0; j < ENB; ++j)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const float4 v = oth[((i * ENB + j) * 4 + q4) * 64 + lane];
          mine[i][j][q4 * 4 + 0] += v.x; mine[i][j][q4 * 4 + 1] += v.y;
          mine[i][j][q4 * 4 + 2] += v.z; mine[i][j][q4 * 4 + 3] += v.w;
        }
    __syncthreads();
    if (ONE && wk != 0) return;
    if constexpr (EPI == EPI_PART) {   // straight from the registers: 4 columns of a row per lane and group
      float* dst = p.part + ((int64_t)part * p.G + g) * p.Mdim * p.Ndim;
#pragma unroll
      for (int i = 0; i < EMB; ++i)
#pragma unroll
        for (int j = 0; j < ENB; ++j)
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            const int m = m0 + wm * WTM + 32 * (e_i + i) + (lane & 31), n = e_n + 32 * j + 8 * q4 + 4 * (lane >> 5);
            if (m < p.Mdim && n < p.Ndim)
              *reinterpret_cast<float4*>(dst + (int64_t)m * p.Ndim + n) =
                  make_float4(mine[i][j][q4 * 4], mine[i][j][q4 * 4 + 1], mine[i][j][q4 * 4 + 2], mine[i][j][q4 * 4 + 3]);
          }
      return;
    }
    L::template store<KIND, EPI, 32, EMB, ENB>(p, mine, e_lds, g, m0 + wm * WTM, 32 * e_i, e_n, out_off, lane);
  } else {
    L::template store<KIND, EPI, MR, EMB, ENB>(p, acc, e_lds, g, m0 + wm * WTM, 0, e_n, out_off, lane);
  }
}

using Tile256 = TileCfg<256, 256, 2, 4, 1, 3, 2>;
using Tile192 = TileCfg<192, 256, 2, 4, 1, 3, 2>;
using Tile128 = TileCfg<128, 128, 2, 2, 2, 3, 2>;
using Tile64x128 = TileCfg<64, 128, 1, 4, 2, 3, 3>;
using Tile64 = TileCfg<64, 64, 1, 2, 2, 5, 5>;
using Tile32x64 = TileCfg<32, 64, 1, 2, 2, 6, 6>;

// ------------------------------------------------------------------------------------------
// fp32 kernel: fp64 matrix cores (v_mfma_f64_16x16x4_f64: lane l supplies A[l % 16][l / 16] and B[l / 16][l % 16] and
// receives D[4 r + l / 16][l % 16], r = 0..3), fp64 accumulation.
//
// TM x TN tile, four waves: TM / 16 of them own 16 rows each, with two row waves the other two take the other half of every k
// chunk, and the halves' sums meet in LDS.  k chunks of 32.  Which k a quarter of the lanes feeds in which step is free as
// long as both operands agree: it takes SPL consecutive ones, one a step.  So A needs no LDS: a lane's values are 16-byte pieces
// of its row (weight gradients: single values, 16 lanes to 64 bytes).  B is converted to fp64 once per workgroup on its way into
// LDS ([k][column], pitch TN + 2 doubles: the k rows of a 32-lane read fall into different halves of the banks), in two buffers:
// the next chunk is converted and stored between the current one's products, and the one after it requested.  No fetch
// stands in a branch, so that the compiler can wait for them by count: what does not exist is fetched from somewhere else in the
// tensor and, along k, zeroed.
// Bound by the fp64 matrix rate (77 TFLOP/s measured for the bare instruction) less the vector instructions between, of which
// a conversion costs a tenth of a matrix instruction.  8192 rows x 2048 x 2048, forward and backward call, with both operands staged
// and two barriers per chunk 2.31 and 4.63 ms (59 TFLOP/s) -> 2.06 and 4.07 ms (67); 8 experts of 256 x 512 x 2048 180 and
// 324 -> 158 and 284 us; 8 of 51 x 1024 x 4096 204 and 409 -> 178 and 338; 4 of 62 x 64 x 128 8.5 and 9.9 -> 8.4 and 9.5; but one chunk
// alone is latency and code that is fetched for the first time, 4 of 62 x 32 x 32 6.3 and 8.3 -> 6.6 and 8.5.
// ------------------------------------------------------------------------------------------
typedef double f64x4_t __attribute__((ext_vector_type(4)));
constexpr int FK = 32;   // k chunk
template <int TM, int TN>
constexpr int f32_lds() { return 2 * FK * (TN + 2) * 8; }
template <int KIND, int EPI, int TM, int TN, bool WIDE, typename L>   // WIDE: leading dimensions that 32-bit offsets do not reach
__device__ __forceinline__ void gemm_f32_tile(const typename L::Args& p, double* Bs, int vb) {
  constexpr bool A_NC = KIND == KIND_TN, B_NC = KIND != KIND_NT;   // k is the slow index in memory
  constexpr int RW = TM / 16, KW = 4 / RW, NJ = TN / 16;            // row waves, k halves, blocks of 16 columns
  constexpr int SPL = 8 / KW;                                       // steps of a wave per chunk
  constexpr int PB = TN + 2, BUF = FK * PB, UB = TN * FK / 4 / 256; // 16-byte pieces of B per thread and chunk
  static_assert(RW * KW == 4 && NJ % KW == 0 && (KW == 1 || RW * 64 * (4 * NJ + 1) <= 2 * BUF), "the halves' sums fit in the buffers");
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), rw = wave % RW, kw = wave / RW;
  const int kb = kw * (FK / KW) + SPL * (lane >> 4);                // this lane's first k of a chunk
  typename L::Place at;
  if (!L::template find<KIND, EPI, 4, TM, TN>(p, vb, at)) return;
  const int g = at.g, m0 = at.tm * TM, n0 = at.tn * TN;
  const float* __restrict__ A = reinterpret_cast<const float*>(p.A);
  const float* __restrict__ B = reinterpret_cast<const float*>(p.B) + (KIND == KIND_TN ? 0 : (int64_t)g * p.b_goff + p.b_off);

  // rows (row-tiled GEMMs): of this lane's A values and, lane l, of output row l of the tile
  int a_row = 0, o_row = 0;
  bool o_zero = false;
  if (KIND != KIND_TN) L::template rows_f32<TM>(p, at, m0, m0 + rw * 16 + (lane & 15), m0 + lane, a_row, o_row, o_zero);
  typename L::template Walk<false> walk(p, at, 0);
  const int nk = KIND == KIND_TN ? walk.start(FK, false) : (p.Kdim + FK - 1) / FK;
  auto ktile = [&](int t) -> KTile {      // behind the last one: no k, and row 0
    if (KIND == KIND_TN) return walk.next(FK);
    return t < nk ? KTile{t * FK, p.Kdim - t * FK} : KTile{0, 0};
  };

  // ---- A: this lane's SPL values of a chunk.  Weight gradients: column m of rows kb .. kb + SPL - 1 of the chunk.
  const int m = min(m0 + rw * 16 + (lane & 15), p.Mdim - 1);       // (weight gradients) past the end: any column, not stored
  const float* a_ptr = A_NC ? A + m : A + (int64_t)a_row * p.lda;
  uint32_t a_off[A_NC ? SPL : 1];     // byte offsets from the chunk's first row
#pragma unroll
  for (int s = 0; s < (A_NC ? SPL : 1); ++s) a_off[s] = ((uint32_t)(kb + s) * (uint32_t)p.lda + (uint32_t)m) * 4u;
  constexpr uint32_t ALL = (1u << SPL) - 1u;
  struct Piece {
    float v[SPL];
    uint32_t keep;      // which of them exist
  };
  const __amdgpu_buffer_rsrc_t rG = make_rsrc(p.gather, A_NC && p.gather ? L::map_bytes(p) : 0u);
  const bool gathered = A_NC && p.gather != nullptr;
  struct Slots {
    int v[A_NC ? SPL : 1];
  };
  Slots slots;                      // gathered rows: slot-map entries of the chunk that is fetched next
  auto fetch_map = [&](Slots& d, const KTile& kt) {     // entries behind the map read as zero; rows behind the count are masked
#pragma unroll
    for (int s = 0; s < (A_NC ? SPL : 1); ++s) d.v[s] = (int)__builtin_amdgcn_raw_buffer_load_b32(rG, (int)((uint32_t)(kt.row0 + kb + s) * 4u), 0, 0);
  };
  auto fetch_a = [&](Piece& d, const KTile& kt, const Slots& map) {
    d.keep = (1u << min(max(kt.lim - kb, 0), SPL)) - 1u;
    if (!A_NC) {        // K % 8 == 0: the values of a lane's quarter exist together or (SPL = 8) in halves of 4
#pragma unroll
      for (int q = 0; q < SPL / 4; ++q) {
        const float4 v = *reinterpret_cast<const float4*>(a_ptr + kt.row0 + (kb + 4 * q < kt.lim ? kb + 4 * q : 0));
        d.v[4 * q] = v.x; d.v[4 * q + 1] = v.y; d.v[4 * q + 2] = v.z; d.v[4 * q + 3] = v.w;
      }
    } else if (gathered) {
#pragma unroll
      for (int s = 0; s < SPL; ++s) {
        const int iv = map.v[A_NC ? s : 0];
        const uint32_t tok = p.gather_k == 1 ? (uint32_t)iv : __umulhi((uint32_t)iv, p.gather_magic);
        const bool full = iv >= 0 && (int64_t)tok < p.gather_rows;     // an empty slot is a row of zeros
        if (!full) d.keep &= ~(1u << s);
        d.v[s] = a_ptr[(full && kb + s < kt.lim ? (int64_t)tok : 0) * p.lda];
      }
    } else if (WIDE) {
      const float* q = a_ptr + (int64_t)kt.row0 * p.lda;
#pragma unroll
      for (int s = 0; s < SPL; ++s) d.v[s] = q[(kb + s < kt.lim ? (int64_t)(kb + s) : 0) * p.lda];
    } else {            // through a descriptor that ends with the chunk's last row: rows behind it are zeros
      const __amdgpu_buffer_rsrc_t r = make_rsrc(A + (int64_t)kt.row0 * p.lda, (uint32_t)max(min(kt.lim, FK), 0) * (uint32_t)p.lda * 4u);
#pragma unroll
      for (int s = 0; s < SPL; ++s) d.v[s] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(r, (int)a_off[A_NC ? s : 0], 0, 0));
      d.keep = ALL;
    }
  };
  // ---- B: through LDS.  A column behind the last one is fetched from the tile's first one.
  struct Rows {
    float4 v[UB];
  };
  Rows rb;
  int b_k[UB];
  uint32_t b_at[UB], b_off[UB];      // element of the piece in its buffer; byte offset from where the chunk starts
#pragma unroll
  for (int u = 0; u < UB; ++u) {
    const int i = tid + 256 * u;
    if (B_NC) {
      const int n = (i % (TN / 4)) * 4;
      b_k[u] = i / (TN / 4);
      b_at[u] = (uint32_t)(b_k[u] * PB + n);
      b_off[u] = ((uint32_t)b_k[u] * (uint32_t)p.ldb + (uint32_t)(n0 + n < p.Ndim ? n0 + n : n0)) * 4u;
    } else {
      const int n = i / (FK / 4);
      b_k[u] = (i % (FK / 4)) * 4;
      b_at[u] = (uint32_t)(b_k[u] * PB + n);
      b_off[u] = ((uint32_t)min(n, p.Ndim - 1 - n0) * (uint32_t)p.ldb + (uint32_t)b_k[u]) * 4u;
    }
  }
  auto fetch_b = [&](Rows& d, const KTile& kt) {
    if constexpr (WIDE) {
#pragma unroll
      for (int u = 0; u < UB; ++u) {
        const int i = tid + 256 * u, k = kt.row0 + (b_k[u] < kt.lim ? b_k[u] : 0), n = n0 + (B_NC ? (i % (TN / 4)) * 4 : i / (FK / 4));
        d.v[u] = *reinterpret_cast<const float4*>(B_NC ? B + (int64_t)k * p.ldb + (n < p.Ndim ? n : n0)
                                                       : B + (int64_t)min(n, p.Ndim - 1) * p.ldb + k);
      }
      return;
    }
    const __amdgpu_buffer_rsrc_t r =     // B_NC: ends with the chunk's last row, rows behind it are zeros
        B_NC ? make_rsrc(B + (int64_t)kt.row0 * p.ldb, (uint32_t)max(min(kt.lim, FK), 0) * (uint32_t)p.ldb * 4u)
             : make_rsrc(B + (int64_t)n0 * p.ldb + kt.row0, OOB);
#pragma unroll
    for (int u = 0; u < UB; ++u) {
      const uint4 v = ldb16(r, B_NC || b_k[u] < kt.lim ? b_off[u] : b_off[u] - (uint32_t)b_k[u] * 4u);
      d.v[u] = make_float4(__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w));
    }
  };
  auto stage_b = [&](Rows& src, int buf, int lim) {
    double* d = Bs + buf * BUF;
#pragma unroll
    for (int u = 0; u < UB; ++u) {
      if ((!B_NC || WIDE) && lim < FK) {
        if (b_k[u] >= lim) src.v[u] = make_float4(0.f, 0.f, 0.f, 0.f);
      }
      const double x[4] = {(double)src.v[u].x, (double)src.v[u].y, (double)src.v[u].z, (double)src.v[u].w};
#pragma unroll
      for (int q = 0; q < 4; ++q) d[b_at[u] + (B_NC ? q : q * PB)] = x[q];
    }
  };

  f64x4_t acc[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) acc[j] = f64x4_t{0.0, 0.0, 0.0, 0.0};
  Piece pa[2];
  int lim_b;              // of the chunk in rb
  KTile t2;               // chunk c + 2
  {
    const KTile t0 = ktile(0), t1 = ktile(1);
    t2 = ktile(2);
    Slots s0, s1;
    Rows r0;
    if (gathered) { fetch_map(s0, t0); fetch_map(s1, t1); fetch_map(slots, t2); }
    fetch_b(r0, t0);
    fetch_b(rb, t1);
    fetch_a(pa[0], t0, s0);
    fetch_a(pa[1], t1, s1);
    stage_b(r0, 0, t0.lim);
    lim_b = t1.lim;
  }
  auto zero_missing = [&](Piece& a) {
    if (A_NC ? gathered || WIDE : a.keep != ALL) {
#pragma unroll
      for (int s = 0; s < SPL; ++s) a.v[s] = (a.keep >> s) & 1u ? a.v[s] : 0.f;
    }
  };
  auto products = [&](const Piece& pc, const double* w, int s0, int s1) {
#pragma unroll
    for (int s = s0; s < s1; ++s) {
      const double a = (double)pc.v[s];
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[j] = __builtin_amdgcn_mfma_f64_16x16x4f64(a, w[s * PB + 16 * j], acc[j], 0, 0, 0);
    }
  };
  auto step = [&](int c, auto set_tag) {
    constexpr int SET = decltype(set_tag)::value;
    const double* wb = Bs + kb * PB + (lane & 15);
    __syncthreads();      // chunk c is staged, and the other buffer is consumed
    zero_missing(pa[SET]);
    products(pa[SET], wb + SET * BUF, 0, SPL / 2);
    stage_b(rb, SET ^ 1, lim_b);
    fetch_b(rb, t2);
    lim_b = t2.lim;
    products(pa[SET], wb + SET * BUF, SPL / 2, SPL);
    fetch_a(pa[SET], t2, slots);
    t2 = ktile(c + 3);
    if (gathered) fetch_map(slots, t2);
  };
  int c = 0;
  for (; c + 2 < nk; c += 2) {
    step(c, std::integral_constant<int, 0>{});
    step(c + 1, std::integral_constant<int, 1>{});
  }
  // The last chunk or two, behind which nothing is fetched or staged.  In the loop's steps the last one waited for a chunk that does
  // not exist, and an odd number of chunks had one of zeros multiplied: 4 experts of 62 rows x 64 x 128, forward and backward call, 8.87 and
  // 10.1 us, now 8.4 and 9.4; 8 of 2000 x 96 x 96 26.4 and 60, now 22.3 and 56; 12 of 100 x 200 x 328 23.3 and 36.4, now 21.5 and 34.1.
  const double* w = Bs + kb * PB + (lane & 15);
  auto last = [&]() {
    __syncthreads();
    zero_missing(pa[0]);
    products(pa[0], w, 0, SPL);
  };
  if (c + 2 == nk) {
    last();
    stage_b(rb, 1, lim_b);
    pa[0] = pa[1];
    w += BUF;
    ++c;
  }
  if (c < nk) last();
  if constexpr (KW == 2) {
    __syncthreads();
    // Of two neighbouring blocks of columns the first half finishes one and the second the other: with the second idle here, the
    // other's epilogue, eight values a lane, took 0.4 us more of every launch.
    double* red = Bs + (rw * 64 + lane) * (4 * NJ + 1);   // + 1: lanes on different banks
#pragma unroll
    for (int j = 0; j < NJ; j += 2)
#pragma unroll
      for (int r = 0; r < 4; ++r) red[4 * (j + 1 - kw) + r] = kw == 0 ? acc[j + 1][r] : acc[j][r];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < NJ; j += 2)
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[j / 2][r] = (kw == 0 ? acc[j][r] : acc[j + 1][r]) + red[4 * (j + kw) + r];
  }
  L::template store_f32<KIND, EPI, TM, TN, KW>(p, acc, Bs, g, m0, n0, rw, kw, lane, o_row, o_zero);
}

// ---- host side ----
inline int num_cus() {
  static int n = 0;   // same on every device of a node
  if (n == 0) {
    int dev = 0, v = 0;
    if (hipGetDevice(&dev) == hipSuccess &&
        hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess && v > 0) n = v;
    else n = 256;
  }
  return n;
}

// Tile of a bf16 grouped GEMM, tile_m x tile_n.
struct TilePlan {
  int tile_m, tile_n;
};
// The tiles a row-tiled GEMM may take, and what one costs (microseconds, measured): a k tile of 64 with few and with all
// compute units busy (in a launch of its own; a compute unit then holds one workgroup of the first two, two of the
// others), and everything outside the k loop.  Large tiles move the fewest bytes per flop; small ones fill the chip when
// there are few rows, and their k tile is short when a long reduction is what a launch waits for.
// The prices of the two largest tiles are those of a loop with 32x32x16 MFMAs and requests in bursts; the present one is
// shorter with every compute unit busy, and they have not been measured again.  For dX in the merged backward launch with
// 256 x 256 weight gradients they are an approximation: there a compute unit holds one workgroup whatever its tile (the
// launch reserves the LDS of a 256 x 256 tile), and the weight gradients queue behind dX.
struct TileCost {
  TilePlan tile;
  int per_cu;
  float k_few, k_all, fixed;
};
constexpr TileCost ROW_TILES[] = {{{256, 256}, 1, 0.95f, 1.50f, 10.f}, {{192, 256}, 1, 0.72f, 1.22f, 9.f},
                                  {{128, 128}, 2, 0.50f, 1.05f, 7.f},  {{64, 128}, 2, 0.31f, 0.66f, 6.f},
                                  {{64, 64}, 2, 0.24f, 0.42f, 6.f},    {{32, 64}, 2, 0.20f, 0.30f, 5.f}};

}  // namespace moe
