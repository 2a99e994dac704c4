// Matrix products on the gfx950 matrix cores: C = A W^T with an epilogue (paper Sec. 2.2: the reranker's latency is
// dominated by the matrix multiplications of its transformer blocks).
//
// A [M,K] and W [N,K] row-major (K-contiguous, which is what the MFMA operand registers want: 16 consecutive bytes of k per lane).
// Both bf16 or both IEEE half, fp32 accumulation in v_mfma_f32_16x16x32_{bf16,f16} (gemm_16.hip launches these); or both 8-bit integers with
// a scale for each row, sums in 32-bit integers in v_mfma_i32_16x16x64_i8 (gemm_q8.hip).  That instruction takes the same bytes in the same
// cycles, so tiles, loops and LDS are shared: K counts units of two bytes, a 16-bit value or two codes.
//
// Workgroup tile BM x BN x 64, WM x WN wavefronts, each owning a (BM/WM) x (BN/WN) block of the accumulator.  The
// large-launch shape is 256 x 256 with 2 x 2 wavefronts (one per SIMD, 128 x 128 each,
// 256 accumulator registers in AGPRs); launches with few tiles per compute unit take one of seven smaller tiles
// down to 32 x 32 (see the choice at the launcher).  A and W tiles are staged in LDS (a ring of S stages, 256 x 256: three
// of A and two of W; 16-byte chunks XOR-swizzled by row so that the 16-row operand reads spread over the banks) by direct
// global->LDS loads, which need no staging registers.  Every K loop is generated text (gen_gemm_kloop.py), because its waits count loads
// and fragment reads exactly; rows beyond the matrix are clamped in the load offsets, so edge tiles run the same loop.
//
// Epilogues: plain store (16 bits or fp32), residual add into the fp32 stream, and SwiGLU, where the B tile is
// made of BN/2 gate rows and the BN/2 matching up rows so that a lane holds g and u of one element.
//
// Workgroup ids are remapped so that each XCD (ids are dealt round-robin over the 8 XCDs) owns a
// contiguous range of tiles, walked in groups of 4 or 8 row-tiles, to keep the operand panels in its L2.
#pragma once

#include <mutex>
#include <type_traits>

#include "common.h"
#include "gemm_16_kloop.inc"
#include "gemm_q8_kloop.inc"
#include "gemm_q8.h"

namespace prism {

typedef __attribute__((ext_vector_type(4))) unsigned u32x4_t;
static constexpr int BK = 64;            // K-slice per stage (elements)
static constexpr int kChunks = BK / 8;   // 16-byte chunks per tile row

// LDS serves a 16-byte read of 16 consecutive lanes per cycle out of 64 banks; with 128-byte rows the bank
// half is the row's parity, so the chunk is rotated by bits 1..3 of the row.
__device__ __forceinline__ int swz(int row, int chunk) { return chunk ^ ((row >> 1) & 7); }

#define PRISM_GLOBAL_PTR(p) ((const __attribute__((address_space(1))) void *)(p))
#define PRISM_LDS_PTR(p) ((__attribute__((address_space(3))) void *)(p))

// silu(g) * u in fp32, rounded to 16 bits by its callers.  The division is correctly rounded: a product with the reciprocal
// instruction takes half of this epilogue's arithmetic away (13.8 -> 9.2 thousand cycles of a 256 x 256 tile) and no time where the
// chip is full and at its power limit (24576 x 24576 x 4096: 3350 us, with the division 3337), but is off by
// an ulp more and returns 0 where 1 + e^-g exceeds 2^126, values that bf16 still holds.
__device__ __forceinline__ float silu_mul(float g, float u) { return g / (1.0f + __expf(-g)) * u; }

// Stages of a tile's operands in LDS, and their bytes.  Tiles of 256 columns: S = 2 is three of A and two of W, 3 two and three, 4 three of both
template <int BN, int S> constexpr int a_stages() { return BN == 256 ? (S == 3 ? 2 : 3) : S; }
template <int BN, int S> constexpr int w_stages() { return BN == 256 ? (S == 2 ? 2 : 3) : S; }
template <int BM, int BN, int S> constexpr int stage_bytes() { return (a_stages<BN, S>() * BM + w_stages<BN, S>() * BN) * BK * 2; }

// lda, ldw: bytes from row to row of 8-bit operands (multiples of 16), in front of what the loop does not wait for, so that they arrive in registers with the launch (build.py)
// OT: type of 16-bit operands and outputs; IT: the operands' (OT or int8_t)
template <typename OT, int BM, int BN, int WM, int WN, int EPI, int S, typename IT = OT>
__global__ __launch_bounds__(WM *WN * 64, (stage_bytes<BM, BN, S>() > 81920 ? 1 : 2)) void gemm_16_kernel(
    const IT *__restrict__ A, const IT *__restrict__ W, int M, int N, int K, int nM, int nN, uint32_t lda, uint32_t ldw, void *__restrict__ out_,
    std::conditional_t<std::is_same_v<IT, int8_t>, Q8Operands, QkvEpilogue> qe) {
  constexpr bool kQ8 = std::is_same_v<IT, int8_t>;
  constexpr int NW = WM * WN;
  constexpr bool kHeads = EPI == kEpiQkv;
  constexpr int WMT = BM / WM, WNT = BN / WN;      // wave tile
  constexpr int TM = WMT / 16, TN = WNT / 16;      // 16 x 16 accumulator tiles per wave
  // one direct-to-LDS instruction of a wave moves 64 x 16 B = 8 tile rows
  constexpr int A_ITERS = BM / 8 / NW, B_ITERS = BN / 8 / NW;
  static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0, "tile/waves mismatch");
  static_assert(!kQ8 || !kHeads, "8-bit products have no heads");
  static_assert(EPI != PRISM_EPI_SWIGLU || TN % 2 == 0, "SwiGLU pairs gate and up tiles");
  static_assert(TM * TN * 4 <= 256, "accumulator registers");
  extern __shared__ __align__(16) unsigned char smem[];
  constexpr bool kBig = BN == 256;
  unsigned char *lA = smem;                                          // [stages of A][BM][BK] of two bytes
  unsigned char *lB = lA + a_stages<BN, S>() * BM * BK * 2;       // [stages of W][BN][BK]

  // ---- tile mapping: XCD-contiguous ranges, grouped walk ----
  const int n_tiles = nM * nN;
  int bid = blockIdx.x;
  {
    const int per = (n_tiles + 7) / 8, x = bid % 8, r = bid / 8;
    // XCD x owns logical ids [x*per, ...); ids beyond n_tiles idle
    bid = x * per + r;
    if (r >= per || bid >= n_tiles) return;
  }
  // 256 x 256: an XCD runs 32 tiles at a time, 4 row-tiles x 8 column-tiles of them or 8 x 4 - the same operand bytes - but 4 is
  // 3 % faster at 24576 x 24576 x 4096 (1364 -> 1410 TFLOP/s; 3, 5, 6, 8, 16: 1-4 % slower, on some chips 6 %), and 4 % than 8
  // at 32768 x 4096 x 12288
  constexpr int GM = kBig || EPI == PRISM_EPI_RESIDUAL ? 4 : 8;
  const int group = bid / (GM * nN), first_m = group * GM;
  const int gsz = (nM - first_m) < GM ? (nM - first_m) : GM;
  const int tile_m = first_m + (bid % (GM * nN)) % gsz, tile_n = (bid % (GM * nN)) / gsz;
  const int m0 = tile_m * BM;
  const int F = EPI == PRISM_EPI_SWIGLU ? N / 2 : N;         // output columns
  constexpr int BNO = EPI == PRISM_EPI_SWIGLU ? BN / 2 : BN; // output columns per tile
  const int n0 = tile_n * (EPI == PRISM_EPI_SWIGLU ? BN / 2 : BN);

  // read from a lane, so that what follows from the wave's place stays in scalar registers
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN;

  // ---- global -> LDS staging without registers (global_load_lds_dwordx4).  Instruction j of wave w
  //      fills tile rows (w * ITERS + j) * 8 .. + 8, lane l landing at row l / 8, chunk slot l % 8.
  //      The XOR swizzle is applied on the source side: slot p of row r receives chunk swz(r, p).
  const int lrow = lane >> 3;
  // byte offsets from the tile's first row of A / W, rows beyond the matrix clamped; four loads share one destination register and
  // carry 0, 1, 2, 3 KiB in the instruction, which shifts the source too: taken off here, with 4 KiB in hand (kBias)
  constexpr uint32_t kBias = 4096;
  uint32_t gA[A_ITERS], gB[B_ITERS];
  uint32_t rowA = (uint32_t)K * 2u, rowB = rowA;                     // bytes from row to row
  if constexpr (kQ8) { rowA = lda; rowB = ldw; }
#pragma unroll
  for (int j = 0; j < A_ITERS; ++j) {
    const int row = (wave * A_ITERS + j) * 8 + lrow;
    const int r = m0 + row < M ? row : M - 1 - m0;
    gA[j] = (uint32_t)r * rowA + swz(row, lane & 7) * 16u + kBias - j % 4 * 1024u;
  }
#pragma unroll
  for (int j = 0; j < B_ITERS; ++j) {
    const int row = (wave * B_ITERS + j) * 8 + lrow;
    const int half = EPI == PRISM_EPI_SWIGLU ? row / (BN / 2) : 0, rr = row - half * (BN / 2);   // gate rows, then up rows
    const int r = (n0 + rr < F ? rr : F - 1 - n0) + half * F;
    gB[j] = (uint32_t)r * rowB + swz(row, lane & 7) * 16u + kBias - j % 4 * 1024u;
  }
  // ---- LDS rows this lane reads as MFMA operands: row (A) and first column (B) of its first fragment; it feeds 8 of the
  //      32 k of one of 16 rows to an MFMA
  const int frow = lane & 15, kpart = lane >> 4;
  const int rA0 = wm * WMT + frow, rB0 = wn * (EPI == PRISM_EPI_SWIGLU ? WNT / 2 : WNT) + frow;

  // accumulator tile (i, j) is a[4 t .. 4 t + 3], t = i TN + j: four tiles to an operand of the K loop, which clears them
  f32x16 acc[(TM * TN + 3) / 4];

  const int nk = K / BK;

  // ---- epilogue geometry (see the epilogue): everything it reads or writes goes along the rows, 16 bytes per lane.
  //      Residual epilogue: the old values of a block of 32 rows (16 in the smallest tiles) are requested one block ahead, the first block's
  //      before the K loop where registers are left (tiles below 256; the big tile spills).  The same for what the q/k/v
  //      epilogue reads by row: a small tile's loop is a few microseconds, and each dependent load behind it about one.
  //      (28 layers of the 0.6B shape on 391 rows, with the same in the RMSNorm: 2749 -> 2687 us.)
  constexpr bool kEarly = !kBig;
  constexpr bool kF32Out = EPI == PRISM_EPI_RESIDUAL || EPI == PRISM_EPI_STORE_F32;
  constexpr int ES = kF32Out ? 4 : 2;                               // bytes per output element
  constexpr int OUTW = EPI == PRISM_EPI_SWIGLU ? WNT / 2 : WNT;    // output columns of the wave
  constexpr int RB = OUTW * ES, CPR = RB / 16;                      // bytes / 16-byte chunks per staged row
  constexpr int BR = WMT % 32 ? 16 : 32, RPB = BR / 16;             // rows of a block, of those in a lane
  constexpr int NBLK = WMT / BR;                                    // blocks of the wave
  constexpr int NR = 1024 / RB < BR ? 1024 / RB : BR, NI = BR / NR; // rows per instruction, instructions per block
  // lane -> (row within an instruction, chunk); 16 rows of 16 16-bit columns are less than an instruction moves: half the lanes idle
  const int f_row = lane / CPR % NR, f_chunk = lane % CPR;
  const bool f_on = lane / CPR < NR;
  const bool full_n = n0 + BNO <= F && (kQ8 || (F * ES) % 16 == 0);
  // rows of 8-bit products lie anywhere: memory takes 16 bytes at any multiple of two
  typedef u32x4_t u32x4_any __attribute__((aligned(2)));
  typedef f32x4 f32x4_any __attribute__((aligned(4)));
  using Out16 = std::conditional_t<kQ8, u32x4_any, u32x4_t>;
  using OutF4 = std::conditional_t<kQ8, f32x4_any, f32x4>;
  f32x4 old[2][EPI == PRISM_EPI_RESIDUAL ? NI : 1];
  // An access goes to a wave-uniform address (scalar) plus a lane offset that stays the same: multiplying rows by the pitch per
  // lane and access took a third of the epilogue's vector time.
  int64_t out_row = F;                                              // values from row to row
  if constexpr (kQ8) out_row = qe.ldo;
  const int64_t out_pitch = out_row * ES;                           // bytes
  const unsigned f_off = (unsigned)f_row * (unsigned)out_pitch + (unsigned)f_chunk * 16u;   // < 32 rows: far below 4 GiB
  unsigned char *const out_w = reinterpret_cast<unsigned char *>(out_) + (int64_t)(m0 + wm * WMT) * out_pitch + (int64_t)(n0 + wn * OUTW) * ES;
  const int rows_left = M - m0 - wm * WMT;                          // of the wave's rows inside the matrix
  const int64_t out_step = NR * out_pitch;
  const unsigned char *old_at = out_w;                              // steps along with the loads
  const int cols_left = F - (n0 + wn * OUTW + f_chunk * (16 / ES)); // of the output's columns from the lane's chunk on
  // (whole: every row is inside the matrix, no guard per access; ragged: columns may not be, 8-bit products)
  auto load_old = [&](int i, auto whole, auto ragged) __attribute__((always_inline)) {
    if constexpr (EPI == PRISM_EPI_RESIDUAL) {
#pragma unroll
      for (int rr = 0; rr < NI; ++rr) {
        const int r = i * BR + rr * NR;
        if (ragged && cols_left < 4) {
#pragma unroll
          for (int e = 0; e < 3; ++e)
            if (r + f_row < rows_left && e < cols_left) old[i & 1][rr][e] = *reinterpret_cast<const float *>(old_at + f_off + e * 4);
        } else if (whole || r + f_row < rows_left) old[i & 1][rr] = __builtin_nontemporal_load(reinterpret_cast<const OutF4 *>(old_at + f_off));
        old_at += out_step;
      }
    }
  };

  int row_in[kHeads ? TM : 1];                                // q, k heads: positions; v heads: V^T columns
  auto load_rows = [&]() __attribute__((always_inline)) {
    if constexpr (kHeads) {
      const int32_t *src = ((n0 + wn * WNT) >> 7) < qe.nq + qe.nkv ? qe.pos : qe.vt_col;
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const int row = m0 + wm * WMT + i * 16 + frow;
        row_in[i] = src[row < M ? row : M - 1];
      }
    }
  };
  // 8-bit products: the scales of the lane's rows and columns (gate columns, then up columns), clamped to the matrix, on their way
  // during the loop
  float sa[kQ8 ? TM : 1];
  f32x4 sw[kQ8 ? TN : 1];
  if constexpr (kQ8) {
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int row = m0 + wm * WMT + i * 16 + frow;
      sa[i] = qe.sa[row < M ? row : M - 1];
    }
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const int up = EPI == PRISM_EPI_SWIGLU && j >= TN / 2, c0 = n0 + wn * OUTW + (j - up * (TN / 2)) * 16 + kpart * 4;
      if (n0 + BNO <= F) sw[j] = *reinterpret_cast<const f32x4_any *>(qe.sw + up * F + c0);
      else
        for (int q = 0; q < 4; ++q) sw[j][q] = qe.sw[up * F + (c0 + q < F ? c0 + q : F - 1)];
    }
  }
  if constexpr (kEarly) {
    if constexpr (kHeads) load_rows();
    else if (full_n) load_old(0, std::false_type{}, std::false_type{});
    else if constexpr (kQ8) load_old(0, std::false_type{}, std::true_type{});
  }

  // ---- epilogue.  The W fragment was the instruction's first operand, so the 16 x 16 accumulator tile (i, j) is transposed:
  //      a lane holds ONE row of A, 16 i + lane % 16, and 4 consecutive output columns 16 j + 4 (lane / 16) + q, q = 0..3.
  //      Written straight from that layout, one store instruction touches 32 rows with 16-32 bytes in each, and
  //      the number of cache lines an instruction touches - not the bytes - is what the memory path charges for
  //      (measured: 12-29 us per 256 x 256 tile, a tenth to a fifth of the tile's time).  So every block of rows goes
  //      through LDS, which is free once the K loop is done: lanes write their row's values, then read back 16 bytes
  //      each along the rows, so that an instruction reads or writes whole lines (2-8 complete rows of the wave's
  //      columns).  LDS requests of one wave are served in order, so no barrier is needed between the two phases.
  auto epilogue = [&]() __attribute__((always_inline)) {
  // Accumulator element (i, j, q), fetched from its accumulation register when it is needed: behind the hand-scheduled
  // loop all 256 of them sit in AGPRs, and read as plain values the compiler would copy the whole set into vector
  // registers at once, leaving none for the epilogue's own arithmetic.
  // (The compiler does not look inside these statements, so the wait between a matrix instruction and the first read
  // of its result is spelled out: every accumulator tile passes through an empty statement, which puts all matrix
  // instructions before it, then 32 idle cycles - more than the deepest instruction needs to retire.  All of these are
  // volatile, which keeps them in this order.)
#pragma unroll
  for (int t = 0; t < (TM * TN + 3) / 4; ++t) asm volatile("" : "+a"(acc[t]));
  asm volatile("s_nop 15\n\ts_nop 15");
  auto AC = [&](int i, int j, int q) __attribute__((always_inline)) {
    const int t = i * TN + j;
    if constexpr (kQ8) {
      int n;
      asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(n) : "a"(acc[t / 4][t % 4 * 4 + q]));
      return q8_scaled(n, sa[i], sw[j][q]);
    } else {
      float r;
      asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(r) : "a"(acc[t / 4][t % 4 * 4 + q]));
      return r;
    }
  };
  __syncthreads();              // every wave's operand loads have landed and nobody reads operands any more
  constexpr int SWZ = CPR >= 16 ? 15 : CPR - 1;                     // chunk rotation by row: spreads a column of 16-byte
                                                                    // writes (one per row) over the banks
  // the lane's place again, from the thread index: kept over the loop, one of these ends in scratch memory, and its reload waits for
  // every old value requested before it
  unsigned again = threadIdx.x;
  asm volatile("" : "+v"(again));
  const int e_row = again & 15, e_col = (again & 63) >> 4 << 2;     // row and column in an accumulator tile
  static_assert(NR * RB == 1024 || !kF32Out, "the residual's accesses have no idle lanes");
  static_assert(BR * RB <= stage_bytes<BM, BN, S>() / NW, "staging block must fit the wave's share of LDS");
  unsigned char *stg = smem + wave * (stage_bytes<BM, BN, S>() / NW);
  // values for columns n .. n + 3 (n a multiple of 4, within the wave's columns) of staged row m
  auto put32 = [&](int m, int n, const f32x4 &v) __attribute__((always_inline)) {
    *reinterpret_cast<f32x4 *>(stg + m * RB + (((n >> 2) ^ (m & SWZ)) << 4)) = v;
  };
  auto put16 = [&](int m, int n, const typename Mfma<OT>::vec4 &v) __attribute__((always_inline)) {
    *reinterpret_cast<typename Mfma<OT>::vec4 *>(stg + m * RB + (((n >> 3) ^ (m & SWZ)) << 4) + (n & 4) * 2) = v;
  };
  auto staged = [&](int rr) __attribute__((always_inline)) {
    const int r = rr * NR + f_row;
    return *reinterpret_cast<const uint4 *>(stg + r * RB + ((f_chunk ^ (r & SWZ)) << 4));
  };
  // Flushes the staged block i of the wave's rows to a row-major destination (wave-uniform address of the wave's first row and
  // column, row pitch, the lane's offset).
  auto flush_store = [&](unsigned char *dst, int64_t pitch, unsigned off, int i, auto ragged) __attribute__((always_inline)) {
    dst += (int64_t)i * BR * pitch;
#pragma unroll
    for (int rr = 0; rr < NI; ++rr) {
      const uint4 v = staged(rr);
      if (ragged && cols_left < 16 / ES) {
        const u32x4_t w = __builtin_bit_cast(u32x4_t, v);
        if (f_on && i * BR + rr * NR + f_row < rows_left)
#pragma unroll
          for (int e = 0; e < 16 / ES - 1; ++e)
            if (e < cols_left) {
              if constexpr (ES == 4) *reinterpret_cast<unsigned *>(dst + off + e * 4) = w[e];
              else *reinterpret_cast<unsigned short *>(dst + off + e * 2) = (unsigned short)(w[e / 2] >> e % 2 * 16);
            }
      } else if (f_on && i * BR + rr * NR + f_row < rows_left) __builtin_nontemporal_store(__builtin_bit_cast(u32x4_t, v), reinterpret_cast<Out16 *>(dst + off));
      dst += NR * pitch;
    }
  };

  if constexpr (kHeads) {
    // The wave's 128 columns are one head.  A row's 128 values sit in the 4 lanes with the same lane % 16; the rotate-half
    // partner of column d is d + 64 = the same register of accumulator tile j + 4, so the per-head RMSNorm
    // (two cross-lane adds), the rotation and the single rounding all happen on the accumulators.  What the memory path
    // charges for is cache lines touched per instruction, so the cos/sin pairs come from the TRANSPOSED table (the 16
    // tokens of a load are consecutive positions of a sequence almost always: four lines per load instead of
    // one or two per lane) and the finished q / k rows go through the staging block like the other epilogues' outputs.
    static_assert(WNT == 128, "one head per wavefront");
    typedef typename Mfma<OT>::vec4 vec4;
    const int head = (n0 + wn * WNT) >> 7;                 // wave-uniform
    if constexpr (!kEarly) load_rows();                    // all rows' at once: one memory latency, not one per block
    if (head < qe.nq + qe.nkv) {
      const OT *gain = reinterpret_cast<const OT *>(head < qe.nq ? qe.q_gain : qe.k_gain);
      vec4 ga[4], gb[4];
      if (qe.qk_norm) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          ga[j] = *reinterpret_cast<const vec4 *>(gain + j * 16 + e_col);
          gb[j] = *reinterpret_cast<const vec4 *>(gain + j * 16 + e_col + 64);
        }
      }
      const int64_t pitch = (int64_t)(qe.nq + qe.nkv) * 128 * 2;
      unsigned char *const qk_w = reinterpret_cast<unsigned char *>(qe.QK) + (int64_t)(m0 + wm * WMT) * pitch + (int64_t)head * 128 * 2;
      const unsigned qk_off = (unsigned)f_row * (unsigned)pitch + (unsigned)f_chunk * 16u;
      // (cos, sin) of (pos, d) sits at [d * stride + pos]: a wave-uniform base per column plus one 32-bit lane offset (in bytes, or
      // the compiler cannot rule out a carry and adds 64-bit addresses per lane).
      // The pairs of block i + 1 are requested before block i is worked on, so the tile pays the memory latency once,
      // not once per block.
      unsigned lane_off[TM];
#pragma unroll
      for (int i = 0; i < TM; ++i) lane_off[i] = ((unsigned)(e_col) * (unsigned)qe.rope_stride + (unsigned)row_in[i]) * 8u;
      float2 cs[2][RPB][4][4];
      auto load_cs = [&](int b) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < RPB; ++h)
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const char *col = reinterpret_cast<const char *>(qe.rope_tab_t + (int64_t)(j * 16 + q) * qe.rope_stride);
              cs[b & 1][h][j][q] = *reinterpret_cast<const float2 *>(col + lane_off[b * RPB + h]);
            }
      };
      load_cs(0);
#pragma unroll
      for (int b = 0; b < NBLK; ++b) {
        if (b + 1 < NBLK) load_cs(b + 1);
        float r[RPB];
#pragma unroll
        for (int h = 0; h < RPB; ++h) {
          r[h] = 1.f;
          if (qe.qk_norm) {
            // the finishing kernel's order of the sum of squares: column pairs (d, d + 64), then halving over the bits of d, 32 first
            const int i = b * RPB + h;
            float p[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              auto pair = [&](int j) __attribute__((always_inline)) {
                const float x = AC(i, j, q), y = AC(i, j + 4, q);
                return __builtin_fmaf(x, x, y * y);
              };
              p[q] = sum_xor16(sum_xor32((pair(0) + pair(2)) + (pair(1) + pair(3))));
            }
            r[h] = 1.0f / sqrtf(((p[0] + p[2]) + (p[1] + p[3])) / 128.f + qe.eps);
          }
        }
#pragma unroll
        for (int h = 0; h < RPB; ++h)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            vec4 lo, hi;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const float2 c = cs[b & 1][h][j][q];
              float x = AC(b * RPB + h, j, q), y = AC(b * RPB + h, j + 4, q);
              if (qe.qk_norm) {
                x = x * r[h] * to_f32(ga[j][q]);
                y = y * r[h] * to_f32(gb[j][q]);
              }
              lo[q] = from_f32<OT>(__builtin_fmaf(x, c.x, -(y * c.y)));
              hi[q] = from_f32<OT>(__builtin_fmaf(y, c.x, x * c.y));
            }
            put16(h * 16 + e_row, j * 16 + e_col, lo);
            put16(h * 16 + e_row, j * 16 + e_col + 64, hi);
          }
        flush_store(qk_w, pitch, qk_off, b, std::false_type{});
      }
    } else {
      // v head: rounded to the operand type, stored as half, transposed (16 consecutive tokens of one d are contiguous)
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        if (m0 + wm * WMT + i * 16 + e_row >= M) continue;
        f16 *vt = reinterpret_cast<f16 *>(qe.Vt) + ((int64_t)(head - qe.nq - qe.nkv) * 128 + e_col) * qe.vt_stride + row_in[i];
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            vt[(int64_t)(j * 16 + q) * qe.vt_stride] = from_f32<f16>(to_f32(from_f32<OT>(AC(i, j, q))));
      }
    }
    return;
  }

  if (EPI == PRISM_EPI_RESIDUAL && (kQ8 || full_n)) {
    // read-modify-write of the fp32 stream, whole lines per instruction; the loads of the next block are requested
    // before this block is staged, so the tile pays the memory latency once, not per block
    auto residual = [&](auto whole, auto ragged) __attribute__((always_inline)) {
      if constexpr (!kEarly) load_old(0, whole, ragged);
      int64_t new_at = 0;
      asm volatile("" : "+s"(new_at));       // a chain of its own: 64 addresses shared with the loads would not fit the scalar registers
#pragma unroll
      for (int b = 0; b < NBLK; ++b) {
        if (b + 1 < NBLK) load_old(b + 1, whole, ragged);
#pragma unroll
        for (int h = 0; h < RPB; ++h)
#pragma unroll
          for (int j = 0; j < TN; ++j) {
            f32x4 v;
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = AC(b * RPB + h, j, q);
            put32(h * 16 + e_row, j * 16 + e_col, v);
          }
#pragma unroll
        for (int rr = 0; rr < NI; ++rr) {
          const int r = b * BR + rr * NR;
          const uint4 u = staged(rr);
          f32x4 v = old[b & 1][rr];
          v[0] += __uint_as_float(u.x); v[1] += __uint_as_float(u.y); v[2] += __uint_as_float(u.z); v[3] += __uint_as_float(u.w);
          if (ragged && cols_left < 4) {
#pragma unroll
            for (int e = 0; e < 3; ++e)
              if (r + f_row < rows_left && e < cols_left) *reinterpret_cast<float *>(out_w + new_at + f_off + e * 4) = v[e];
          } else if (whole || r + f_row < rows_left) __builtin_nontemporal_store(v, reinterpret_cast<OutF4 *>(out_w + new_at + f_off));
          new_at += out_step;
        }
      }
    };
    if (kQ8 && !full_n) { if constexpr (kQ8) residual(std::false_type{}, std::true_type{}); }
    else if (rows_left >= WMT) residual(std::true_type{}, std::false_type{});
    else residual(std::false_type{}, std::false_type{});
    return;
  }
  auto store = [&](auto ragged) __attribute__((always_inline)) {
#pragma unroll
    for (int b = 0; b < NBLK; ++b) {
#pragma unroll
      for (int h = 0; h < RPB; ++h)
#pragma unroll
        for (int j = 0; j < OUTW / 16; ++j) {
          const int i = b * RPB + h, row = h * 16 + e_row, col = j * 16 + e_col;
          if constexpr (EPI == PRISM_EPI_STORE_F32) {
            f32x4 v;
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = AC(i, j, q);
            put32(row, col, v);
          } else if constexpr (kQ8) {
            f32x4 v;
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = EPI == PRISM_EPI_SWIGLU ? q8_silu_mul(AC(i, j, q), AC(i, j + TN / 2, q)) : AC(i, j, q);
            put16(row, col, q8_round4<OT>(v));
          } else {
            typename Mfma<OT>::vec4 v;
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = from_f32<OT>(EPI == PRISM_EPI_SWIGLU ? silu_mul(AC(i, j, q), AC(i, j + TN / 2, q)) : AC(i, j, q));
            put16(row, col, v);
          }
        }
      flush_store(out_w, out_pitch, f_off, b, ragged);
    }
  };
  if (full_n) {
    store(std::false_type{});
    return;
  }
  if constexpr (kQ8) {
    store(std::true_type{});
    return;
  }

  // ---- ragged last column tile (N not a multiple of the tile, or rows not 16-byte aligned): element by element
  if constexpr (!kHeads && !kQ8) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < OUTW / 16; ++j)
        for (int q = 0; q < 4; ++q) {
          const int row = m0 + wm * WMT + i * 16 + e_row, col = n0 + wn * OUTW + j * 16 + e_col + q;
          if (row >= M || col >= F) continue;
          if (EPI == PRISM_EPI_SWIGLU) {
            reinterpret_cast<OT *>(out_)[row * out_row + col] = from_f32<OT>(silu_mul(AC(i, j, q), AC(i, j + TN / 2, q)));
          } else if (EPI == PRISM_EPI_RESIDUAL) {
            reinterpret_cast<float *>(out_)[row * out_row + col] += AC(i, j, q);
          } else if (EPI == PRISM_EPI_STORE_F32) {
            reinterpret_cast<float *>(out_)[row * out_row + col] = AC(i, j, q);
          } else {
            reinterpret_cast<OT *>(out_)[row * out_row + col] = from_f32<OT>(AC(i, j, q));
          }
        }
  }
  };

  const unsigned ldsA = (unsigned)(uintptr_t)PRISM_LDS_PTR(lA), ldsB = (unsigned)(uintptr_t)PRISM_LDS_PTR(lB);
  const unsigned aA0 = ldsA + (unsigned)(rA0 * BK + swz(rA0, kpart) * 8) * 2u;
  const unsigned aB0 = ldsB + (unsigned)(rB0 * BK + swz(rB0, kpart) * 8) * 2u;
  // wave w's load instruction j fills tile rows (w * ITERS + j) * 8 .. + 8 of an operand (1 KiB of LDS)
  const unsigned ldsA_w = __builtin_amdgcn_readfirstlane(ldsA + (unsigned)wave * A_ITERS * 8 * BK * 2);
  const unsigned ldsB_w = __builtin_amdgcn_readfirstlane(ldsB + (unsigned)wave * B_ITERS * 8 * BK * 2);
  uint64_t baseA = (uint64_t)(uintptr_t)A + (uint64_t)m0 * rowA - kBias, baseB = (uint64_t)(uintptr_t)W + (uint64_t)n0 * rowB - kBias;
  int to_end = nk, back = 0;                                         // slices to the row's end from where the loop begins; its step there
  if constexpr (kQ8) {
    const unsigned first = (unsigned)tile_n * qe.turn % (unsigned)nk;
    baseA += first * 128u;
    baseB += first * 128u;
    to_end = nk - (int)first;
    back = 128 - nk * 128;
  }
  // the upper half of the wave's columns: SwiGLU's are the up rows, half a tile further (the swizzle repeats every 16 rows)
  const unsigned aB1 = aB0 + (unsigned)((EPI == PRISM_EPI_SWIGLU ? BN / 2 : WNT / 2) * BK) * 2u;
#define PRISM_ACC1 "={a[0:15]}"(acc[0])
#define PRISM_ACC2 PRISM_ACC1, "={a[16:31]}"(acc[1])
#define PRISM_ACC4 PRISM_ACC2, "={a[32:47]}"(acc[2]), "={a[48:63]}"(acc[3])
#define PRISM_ACC8 PRISM_ACC4, "={a[64:79]}"(acc[4]), "={a[80:95]}"(acc[5]), "={a[96:111]}"(acc[6]), "={a[112:127]}"(acc[7])
#define PRISM_ACC10 PRISM_ACC8, "={a[128:143]}"(acc[8]), "={a[144:159]}"(acc[9])
#define PRISM_ACC12 PRISM_ACC10, "={a[160:175]}"(acc[10]), "={a[176:191]}"(acc[11])
#define PRISM_ACC14 PRISM_ACC12, "={a[192:207]}"(acc[12]), "={a[208:223]}"(acc[13])
#define PRISM_ACC16                                                                                                               \
  PRISM_ACC4, "={a[64:79]}"(acc[4]), "={a[80:95]}"(acc[5]), "={a[96:111]}"(acc[6]), "={a[112:127]}"(acc[7]),                        \
      "={a[128:143]}"(acc[8]), "={a[144:159]}"(acc[9]), "={a[160:175]}"(acc[10]), "={a[176:191]}"(acc[11]), "={a[192:207]}"(acc[12]), \
      "={a[208:223]}"(acc[13]), "={a[224:239]}"(acc[14]), "={a[240:255]}"(acc[15])
  // (offsets of loads that a tile does not have are never named by its loop)
#define PRISM_AB(j) [ga##j] "v"(gA[j < A_ITERS ? j : 0]), [gb##j] "v"(gB[j < B_ITERS ? j : 0])
#define PRISM_RUN_TY(LOOP, CLOBBERS, ...)                                                                                       \
  asm volatile(LOOP : __VA_ARGS__                                                                                              \
               : [aa] "v"(aA0), [ab] "v"(aB0), [ab2] "v"(aB1), PRISM_AB(0), PRISM_AB(1), PRISM_AB(2), PRISM_AB(3), PRISM_AB(4), \
                 PRISM_AB(5), PRISM_AB(6), PRISM_AB(7), [la] "s"(ldsA_w), [lb] "s"(ldsB_w), [pa] "s"(baseA), [pb] "s"(baseB),   \
                 [nk] "s"(nk), [bk] "s"(back), [wr] "s"(to_end)                                                                \
               : CLOBBERS)
#define PRISM_RUN_Q8(NAME, LIKE, ...) PRISM_RUN_TY(PRISM_KLOOP_Q8_##NAME, PRISM_KLOOP_Q8_CLOBBERS_##LIKE, __VA_ARGS__)
#define PRISM_RUN_16(NAME, ...)                                                                                                 \
  do {                                                                                                                         \
    if constexpr (Mfma<OT>::kIsF16) PRISM_RUN_TY(PRISM_KLOOP_##NAME("f16"), PRISM_KLOOP_CLOBBERS_##NAME, __VA_ARGS__);          \
    else PRISM_RUN_TY(PRISM_KLOOP_##NAME("bf16"), PRISM_KLOOP_CLOBBERS_##NAME, __VA_ARGS__);                                    \
  } while (0)
#define PRISM_RUN(NAME, ...)                                                                                                    \
  do {                                                                                                                         \
    if constexpr (kQ8) PRISM_RUN_Q8(NAME, NAME, __VA_ARGS__);                                                                   \
    else PRISM_RUN_16(NAME, __VA_ARGS__);                                                                                       \
  } while (0)
  if constexpr (BM == 256) PRISM_RUN(256, PRISM_ACC16);
  else if constexpr (kBig && BM == 224) PRISM_RUN_Q8(224, 256, PRISM_ACC14);
  else if constexpr (kBig && BM == 192) PRISM_RUN_Q8(192, 256, PRISM_ACC12);
  else if constexpr (kBig && BM == 160) PRISM_RUN_Q8(160, 256, PRISM_ACC10);
  else if constexpr (kBig) PRISM_RUN_Q8(128, 256, PRISM_ACC8);
  else if constexpr (kHeads && BM == 64 && S == 6) PRISM_RUN_16(64x128_6_HEAD, PRISM_ACC2);
  else if constexpr (kHeads && BM == 64) PRISM_RUN_16(64x128_3_HEAD, PRISM_ACC2);
  else if constexpr (kHeads && S == 5) PRISM_RUN_16(128x128_5_HEAD, PRISM_ACC4);
  else if constexpr (kHeads && S == 3) PRISM_RUN_16(128x128_3_HEAD, PRISM_ACC4);
  else if constexpr (kHeads) PRISM_RUN_16(128x128_2_HEAD, PRISM_ACC4);
  else if constexpr (BM == 32 && BN == 32) PRISM_RUN(32x32_9, PRISM_ACC1);
  else if constexpr (BM == 64 && BN == 32) PRISM_RUN(64x32_7, PRISM_ACC1);
  else if constexpr (BM == 32 && BN == 64) PRISM_RUN(32x64_4, PRISM_ACC2);
  else if constexpr (BM == 64 && BN == 64) PRISM_RUN(64x64_5, PRISM_ACC1);
  else if constexpr (BM == 128 && BN == 64 && S == 6) PRISM_RUN(128x64_6, PRISM_ACC2);
  else if constexpr (BM == 128 && BN == 64) PRISM_RUN(128x64_3, PRISM_ACC2);
  else if constexpr (S == 5) PRISM_RUN(128x128_5, PRISM_ACC4);
  else if constexpr (S == 4) PRISM_RUN_16(128x128_4, PRISM_ACC4);
  else PRISM_RUN(128x128_2, PRISM_ACC4);
#undef PRISM_RUN
#undef PRISM_RUN_16
#undef PRISM_RUN_Q8
#undef PRISM_RUN_TY
#undef PRISM_AB
  epilogue();
}

static constexpr int kDevices = 64;      // of a process

// One launch of a tile over M rows.  K: units of two bytes that the loop reads; lda, ldw: of 8-bit operands
template <typename OT, int BM, int BN, int WM, int WN, int EPI, int S, typename IT, typename Extra>
static int launch_tile(const IT *A, const IT *W, void *out, int M, int N, int K, hipStream_t s, const Extra &extra, uint32_t lda = 0, uint32_t ldw = 0) {
  constexpr size_t lds = stage_bytes<BM, BN, S>();
  auto kern = gemm_16_kernel<OT, BM, BN, WM, WN, EPI, S, IT>;
  // the attribute is per function and device: set once for each, also when several contexts launch from different threads
  static std::once_flag attr_once[kDevices];
  static hipError_t attr_rc[kDevices];
  int device = 0;
  PRISM_HIP(hipGetDevice(&device));
  PRISM_REQUIRE(device < kDevices, PRISM_EUNSUPPORTED, "gemm: device %d", device);
  std::call_once(attr_once[device], [&] {
    attr_rc[device] = hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  });
  PRISM_HIP(attr_rc[device]);
  const int ncols = EPI == PRISM_EPI_SWIGLU ? N / 2 : N, bn_out = EPI == PRISM_EPI_SWIGLU ? BN / 2 : BN;
  const int nM = cdiv(M, BM), nN = cdiv(ncols, bn_out);
  const int grid = cdiv((int64_t)nM * nN, 8) * 8;
  kern<<<grid, WM * WN * 64, lds, s>>>(A, W, M, N, K, nM, nN, lda, ldw, out, extra);
  PRISM_HIP(hipGetLastError());
  return PRISM_OK;
}

}  // namespace prism
