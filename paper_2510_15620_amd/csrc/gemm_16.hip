// 16-bit-operand layer contractions on the gfx950 matrix cores (paper Sec. 2.2: the reranker's latency is
// dominated by the matrix multiplications of its transformer blocks): C = A W^T, A [M,K] and W [N,K] row-major, both bf16 or both
// IEEE half.  The kernel is gemm_tile.h's; here stands which tile a launch uses.
#include <algorithm>

#include "gemm_tile.h"

namespace prism {

bool gemm_16_supported(int epilogue, int N, int K) {
  if (K <= 0 || K % BK != 0 || N <= 0) return false;
  if (epilogue == PRISM_EPI_SWIGLU && N % 2 != 0) return false;
  return epilogue >= PRISM_EPI_STORE && epilogue <= PRISM_EPI_STORE_F32;
}

template <typename OT, int BM, int BN, int WM, int WN, int EPI, int S>
static int launch_cfg(const OT *A, const OT *W, void *out, int M, int N, int K, hipStream_t s,
                      const QkvEpilogue &qe = QkvEpilogue{}) {
  return launch_tile<OT, BM, BN, WM, WN, EPI, S>(A, W, out, M, N, K, s, qe);
}

// ---- which tile a launch uses -----------------------------------------------------------------------------------------
// Rows are independent, columns are independent, and every tile size gives an element the same bits (one accumulator, K in
// order), so the choice is made on time alone.  A launch deals its tiles over 256 compute units; n = tiles per unit, rounded
// up.  A tile's time is its K slices plus a fixed part (dispatch, first slice, epilogue), and a slice's time depends on how
// many tiles share the unit: alone it is a chain of latencies, together the matrix pipes and LDS.  The constants were fit to loops
// on 32x32x16 MFMAs with operands that stay in the caches (256 x 256: to those of today); with weights from memory and the loops of
// today they are off by 11-23 % (root mean square) per tile, 256 x 256 by 30 % where the chip is not full, but what counts is the pick: on
// 265 launches (N 1024-24576, K 1024-12288, 1 to 20000 rows, three epilogues) it is on average 0.6 % above the best tile and ring.  The
// costs are of the shallow rings (deep_ring, below, only says which ring the picked tile runs on), so the worst picks stand beside a 128 x 64
// tile on its deeper one: 150 x 6144 x 2560 stored 21.7 us on 32 x 64, 16.8 there, 150 x 6144 x 4096 28.4 and 23.1; next 64 x 19456 x 2560 with
// SwiGLU, 35.1 on 64 x 64 and 30.4 on 128 x 128.  Examples, us with weights from memory, 32x32x16 loops -> now: 100 x 4096 x 12288
// 38.8 -> 38.7 (64 x 32), 391 x 1024 x 3072 10.2 -> 10.0 (64 x 32), 33 x 2560 x 9728 19.3 -> 18.5 (32 x 32), 777 x 6144 x 1024 with SwiGLU
// 19.7 -> 19.1 (128 x 128), 3699 x 1024 x 3072 34.0 -> 32.8 (128 x 128, four stages).
// (256 x 256: on chips of different speed a slice takes 1.34-1.7 us, the fixed part 11 us with SwiGLU and 17 with a residual or a
// head; 1024 x 24576 x 4096 with SwiGLU 233 us on 128 x 128 tiles, 203 on these; 1536 x 6144 x 4096 with heads 103 and 90.)
struct TileCost {
  int bm, bn, occ;              // tile, workgroups that share a compute unit
  float alone, shared, fixed;   // us per 64-deep slice: one workgroup on the unit; per workgroup when occ of them share it; us per tile
};
enum { kTile256, kTile128, kTile128Deep, kTile128x64, kTile64, kTile32x64, kTile64x32, kTile32, kTileKinds };
static constexpr TileCost kTileCost[kTileKinds] = {
    {256, 256, 1, 1.45f, 1.45f, 9.2f}, {128, 128, 2, 0.72f, 0.50f, 4.5f}, {128, 128, 1, 0.52f, 0.52f, 3.4f}, {128, 64, 2, 0.34f, 0.36f, 2.3f},
    {64, 64, 2, 0.204f, 0.204f, 2.1f}, {32, 64, 3, 0.176f, 0.149f, 2.4f}, {64, 32, 1, 0.128f, 0.128f, 2.3f}, {32, 32, 2, 0.106f, 0.083f, 2.6f}};
// The fused q/k/v projection: tiles whose waves own whole heads (the same: off by 9-18 %, 256 x 256 by 25 %; the pick is the best tile and
// ring of 33 of 34 launches of 1 to 12000 rows, 2 % off on one).  Its epilogue is longer: two dependent loads (position, rotation)
// and the per-head arithmetic.  391 x 4096 x 1024: 11 us, where the projection to fp32 and its two finishing kernels took 48;
// 777 x 6144 x 4096: 62.
enum { kHead256, kHead128, kHead128Deep, kHead64, kHeadKinds };
static constexpr TileCost kHeadCost[kHeadKinds] = {
    {256, 256, 1, 1.40f, 1.40f, 17.f}, {128, 128, 2, 0.70f, 0.55f, 5.5f}, {128, 128, 1, 0.52f, 0.52f, 5.0f}, {64, 128, 2, 0.29f, 0.37f, 5.0f}};

static double tile_cost(const TileCost &t, int64_t M, int64_t ncols, int K, bool glu) {
  const int bn = glu ? t.bn / 2 : t.bn;
  const int64_t tiles = (M + t.bm - 1) / t.bm * ((ncols + bn - 1) / bn), n = (tiles + 255) / 256;
  const int64_t full = n / t.occ, rest = n % t.occ;
  const double slice = full * std::max(t.alone, t.shared * t.occ) + (rest ? std::max(t.alone, t.shared * rest) : 0.f);
  return (K / BK) * slice + (double)((n + t.occ - 1) / t.occ) * t.fixed;
}

// What a launch of M rows runs: rows_big rows (whole 256-row tiles, possibly none) on tile kind 0, the rest on kind `kind`.
struct TilePlan { int rows_big, kind; };
static TilePlan plan_tiles(const TileCost *costs, int kinds, int M, int ncols, int K, bool glu) {
  auto best = [&](int rows, double *cost) {
    int at = 0;
    *cost = tile_cost(costs[0], rows, ncols, K, glu);
    for (int k = 1; k < kinds; ++k) {
      if (glu && costs[k].bn == 32) continue;              // SwiGLU pairs a gate and an up tile in a wave
      const double c = tile_cost(costs[k], rows, ncols, K, glu);
      if (c < *cost) { *cost = c; at = k; }
    }
    return at;
  };
  double whole, rest;
  TilePlan p{0, best(M, &whole)};
  // The last round of big tiles may fill only a few compute units at a whole tile's price: then the row tiles that fill
  // whole rounds go to the big tile and the remaining rows to a second launch with whatever suits them.
  const int nN = cdiv(ncols, glu ? 128 : 256), nM = cdiv(M, 256);
  const int rows_big = (int)std::min<int64_t>(nM, ((int64_t)nM * nN / 256) * 256 / nN) * 256;
  if (rows_big > 0 && rows_big < M) {
    const int kind = best(M - rows_big, &rest);
    if (kind != 0 && tile_cost(costs[0], rows_big, ncols, K, glu) + rest < 0.98 * whole) p = {rows_big, kind};
  }
  return p;
}

// Tiles of 128 rows, and of the heads' 64 x 128, have a second ring of slices that takes a whole compute unit's LDS: two more
// slices in flight (128 x 64 and 64 x 128: 6 stages for 3, 128 x 128: 5 for 4 or 3).  It pays where no unit has a second tile to
// run beside the first (over 256 tiles of 128 x 64: up to 25 % slower) and the loop is long enough for its longer start.  us, weights from
// memory, 128 x 64: 391 x 4096 x 12288 78.7 -> 63.6, 391 x 2560 x 9728 59.5 -> 46.6, 1154 x 1024 x 3072 21.0 -> 17.6, with SwiGLU 200 x
// 6144 x 1024 9.7 -> 9.1; of the 59 launches that the rule takes 4-26 % faster or level, where a residual add of K = 1024, which it leaves out, lost up to
// 14 % (2000 x 1024 x 1024 9.1 -> 10.4).  128 x 128: 1154 x 2560 x 9728 76.1 -> 69.0, 900 x 4096 x 12288 103 -> 93; K = 1024 lost 2-27 %
// (777 x 4096 x 1024 11.8 -> 14.7).  64 x 128 of the heads: 391 x 4096 x 1024 11.4 -> 10.8, 200 x 6144 x 4096 31.1 -> 27.1, 64 x 6144 x 2560 26.6 -> 26.9 (the
// worst).  The gain is that of a last row tile with few rows inside the matrix, whose unit loads less.  Where it is more than half full, 128 x 128
// is level on a long K (SwiGLU 100 x 24576 x 4096 48.1 -> 48.2, 128 x 24576 x 4096 50.3 -> 50.8, residual 1500 x 2560 x 4096 39.7 -> 39.4) and loses up to 6 % on a
// shorter one: residual 3699 x 1024 x 3072 32.8 -> 34.1, 2000 x 1024 x 3072 27.5 -> 29.1, SwiGLU 256 x 16384 x 2048 25.2 -> 26.3, 100 x 19456 x 2560 32.3 -> 32.9, heads
// 896 x 4096 x 2048 23.3 -> 23.5, where SwiGLU of 391 x 8192 x 2048 takes 21.9 -> 21.0 and heads of 777 x 4096 x 2048 21.1 -> 20.1.  128 x 64 with SwiGLU,
// 200 x 8192 x 1024 10.0 -> 9.6, 256 x 8192 x 1024 10.5 -> 10.7, 256 x 5504 x 2048 17.0 -> 16.6.  On weights that the caches hold, which a layer's are not behind
// the layers before it: 128 x 64, 391 x 2560 x 4096 20.9 -> 19.7, but 391 x 4096 x 1024 stored 7.1 -> 7.6; 128 x 128, 777 x 4096 x 4096 31.2 -> 31.9.
// 128 x 128 on all units: from K = 3072 on (916 x 4096 x 3072 of heads 30.8 -> 30.7, x 4096 38.5 -> 36.3, but x 2048 22.7 -> 25.5, residual 956 x 4096 x 2048 23.9
// -> 24.5, SwiGLU 148 x 16384 x 2048 22.5 -> 23.9; 224 tiles, 788 x 4096 x 2048 of heads 22.1 -> 21.6, residual 21.9 -> 21.4).  Four contexts that call at once share units no worse: six short
// candidates, eight layers of the 0.6B shape 205 us a call with these rings, 206 without.
static constexpr int kNever = 1 << 30;
struct DeepRing {
  int slices, last_rows, full_slices;      // K from `slices` on where the last row tile has up to last_rows rows, else from full_slices on
  int chip_slices;                         // more than 224 tiles: from here on
};
static bool deep_ring(const TileCost &t, bool glu, const DeepRing &r, int64_t M, int64_t ncols, int K) {
  const int bn = glu ? t.bn / 2 : t.bn;
  const int64_t tiles = (M + t.bm - 1) / t.bm * ((ncols + bn - 1) / bn), last = (M - 1) % t.bm + 1;
  return tiles <= 256 && K / BK >= (last <= r.last_rows ? r.slices : r.full_slices) && (tiles <= 224 || K / BK >= r.chip_slices);
}
static bool deep_tile(int kind, int epi, int M, int ncols, int K) {
  const bool glu = epi == PRISM_EPI_SWIGLU;
  if (kind == kTile128Deep) return deep_ring(kTileCost[kind], glu, DeepRing{32, 64, kNever, 48}, M, ncols, K);
  if (kind == kTile128x64)
    return deep_ring(kTileCost[kind], glu, glu ? DeepRing{16, 96, 32, 0} : epi == PRISM_EPI_RESIDUAL ? DeepRing{32, 128, 32, 0} : DeepRing{16, 128, 16, 0}, M, ncols, K);
  return false;
}
static bool deep_head(int kind, int M, int ncols, int K) {
  if (kind == kHead128Deep) return deep_ring(kHeadCost[kind], false, DeepRing{32, 96, kNever, 48}, M, ncols, K);
  return kind == kHead64 && deep_ring(kHeadCost[kind], false, DeepRing{16, 64, 16, 0}, M, ncols, K);
}

template <typename OT, int EPI>
static int launch_kind(int kind, const OT *A, const OT *W, void *out, int M, int N, int K, hipStream_t s) {
  if (deep_tile(kind, EPI, M, EPI == PRISM_EPI_SWIGLU ? N / 2 : N, K)) {
    if (kind == kTile128Deep) return launch_cfg<OT, 128, 128, 2, 2, EPI, 5>(A, W, out, M, N, K, s);
    return launch_cfg<OT, 128, 64, 4, 1, EPI, 6>(A, W, out, M, N, K, s);
  }
  switch (kind) {
    case kTile256: return launch_cfg<OT, 256, 256, 2, 2, EPI, 2>(A, W, out, M, N, K, s);
    case kTile128: return launch_cfg<OT, 128, 128, 2, 2, EPI, 2>(A, W, out, M, N, K, s);
    case kTile128Deep: return launch_cfg<OT, 128, 128, 2, 2, EPI, 4>(A, W, out, M, N, K, s);
    case kTile128x64: return launch_cfg<OT, 128, 64, 4, 1, EPI, 3>(A, W, out, M, N, K, s);
    case kTile64: return launch_cfg<OT, 64, 64, 2, 2, EPI, 5>(A, W, out, M, N, K, s);
    case kTile32x64: return launch_cfg<OT, 32, 64, 1, 1, EPI, 4>(A, W, out, M, N, K, s);
    default: break;
  }
  if constexpr (EPI != PRISM_EPI_SWIGLU) {
    if (kind == kTile64x32) return launch_cfg<OT, 64, 32, 2, 1, EPI, 7>(A, W, out, M, N, K, s);
    return launch_cfg<OT, 32, 32, 2, 2, EPI, 9>(A, W, out, M, N, K, s);
  }
  return PRISM_EUNSUPPORTED;
}

template <typename OT, int EPI>
static int launch_epi(const OT *A, const OT *W, void *out, int M, int N, int K, hipStream_t s) {
  constexpr bool kGlu = EPI == PRISM_EPI_SWIGLU;
  constexpr size_t out_elem = EPI == PRISM_EPI_RESIDUAL || EPI == PRISM_EPI_STORE_F32 ? 4 : 2;
  const int ncols = kGlu ? N / 2 : N;
  const TilePlan p = plan_tiles(kTileCost, kTileKinds, M, ncols, K, kGlu);
  if (p.rows_big > 0) PRISM_TRY((launch_kind<OT, EPI>(kTile256, A, W, out, p.rows_big, N, K, s)));
  return launch_kind<OT, EPI>(p.kind, A + (size_t)p.rows_big * K, W, reinterpret_cast<char *>(out) + (size_t)p.rows_big * ncols * out_elem,
                              M - p.rows_big, N, K, s);
}

template <typename OT>
static int launch_typed(int epilogue, const OT *A, const OT *W, void *out, int M, int N, int K, hipStream_t s) {
  switch (epilogue) {
    case PRISM_EPI_STORE: return launch_epi<OT, PRISM_EPI_STORE>(A, W, out, M, N, K, s);
    case PRISM_EPI_RESIDUAL: return launch_epi<OT, PRISM_EPI_RESIDUAL>(A, W, out, M, N, K, s);
    case PRISM_EPI_STORE_F32: return launch_epi<OT, PRISM_EPI_STORE_F32>(A, W, out, M, N, K, s);
    default: return launch_epi<OT, PRISM_EPI_SWIGLU>(A, W, out, M, N, K, s);
  }
}

// The kernel addresses its operands with 32-bit byte offsets.  W has to fit that; A (and the output rows with it) is
// cut into row panels that do: rows of a GEMM are independent, so the panels are separate launches.
static int rows_per_launch(int K) {
  const int64_t rows = (((int64_t)1 << 32) - 1) / ((int64_t)K * 2);
  return (int)std::max<int64_t>(256, rows / 256 * 256);
}

int launch_gemm_16(int dtype, int epilogue, const void *A, const void *W, void *out, int M, int N, int K, hipStream_t s) {
  PRISM_REQUIRE(A && W && out && M >= 0 && is16(dtype), PRISM_EINVAL, "gemm: bad arguments");
  PRISM_REQUIRE(gemm_16_supported(epilogue, N, K), PRISM_EUNSUPPORTED,
                "gemm: N = %d, K = %d, epilogue %d not supported (K must be a multiple of %d)", N, K, epilogue, BK);
  PRISM_REQUIRE((int64_t)N * K * 2 < ((int64_t)1 << 32) && (int64_t)256 * K * 2 < ((int64_t)1 << 32), PRISM_EUNSUPPORTED,
                "gemm: a weight operand of %d x %d 16-bit elements exceeds 4 GiB", N, K);
  const int step = rows_per_launch(K);
  const int out_cols = epilogue == PRISM_EPI_SWIGLU ? N / 2 : N;
  const size_t out_elem = epilogue == PRISM_EPI_RESIDUAL || epilogue == PRISM_EPI_STORE_F32 ? 4 : 2;
  for (int m0 = 0; m0 < M; m0 += step) {
    const int rows = std::min(step, M - m0);
    const char *a = reinterpret_cast<const char *>(A) + (size_t)m0 * K * 2;
    char *o = reinterpret_cast<char *>(out) + (size_t)m0 * out_cols * out_elem;
    if (dtype == PRISM_DTYPE_BF16) PRISM_TRY(launch_typed<bf16>(epilogue, (const bf16 *)a, (const bf16 *)W, o, rows, N, K, s));
    else PRISM_TRY(launch_typed<f16>(epilogue, (const f16 *)a, (const f16 *)W, o, rows, N, K, s));
  }
  return PRISM_OK;
}

bool gemm_16_qkv_large(int M, int nq, int nkv) {
  return (nq + 2 * nkv) % 2 == 0 && (int64_t)cdiv(M, 256) * ((nq + 2 * nkv) / 2) >= 256;
}

bool gemm_16_qkv_supported(int nq, int nkv, int hd, int K) {
  return hd == 128 && nq > 0 && nkv > 0 && K > 0 && K % BK == 0;          // one head per wavefront
}

template <typename OT>
static int launch_head(int kind, const QkvEpilogue &e, const OT *A, const OT *W, int M, int N, int K, hipStream_t s) {
  if (deep_head(kind, M, N, K)) {
    if (kind == kHead128Deep) return launch_cfg<OT, 128, 128, 4, 1, kEpiQkv, 5>(A, W, e.QK, M, N, K, s, e);
    return launch_cfg<OT, 64, 128, 4, 1, kEpiQkv, 6>(A, W, e.QK, M, N, K, s, e);
  }
  switch (kind) {
    case kHead256: return launch_cfg<OT, 256, 256, 2, 2, kEpiQkv, 2>(A, W, e.QK, M, N, K, s, e);
    case kHead128: return launch_cfg<OT, 128, 128, 4, 1, kEpiQkv, 2>(A, W, e.QK, M, N, K, s, e);
    case kHead128Deep: return launch_cfg<OT, 128, 128, 4, 1, kEpiQkv, 3>(A, W, e.QK, M, N, K, s, e);
    default: return launch_cfg<OT, 64, 128, 4, 1, kEpiQkv, 3>(A, W, e.QK, M, N, K, s, e);
  }
}

template <typename OT>
static int launch_qkv_typed(const QkvEpilogue &e, const OT *A, const OT *W, int M, int N, int K, hipStream_t s) {
  const int step = rows_per_launch(K);
  // an odd number of heads leaves half a 256-wide tile outside the matrix, and that tile's epilogue has no column guard
  const bool wide = (e.nq + 2 * e.nkv) % 2 == 0;
  auto rows_on = [&](int kind, int m0, int rows) {             // every per-row array moves with the rows
    QkvEpilogue p = e;
    p.pos += m0;
    p.vt_col += m0;
    p.QK = reinterpret_cast<char *>(e.QK) + (size_t)m0 * (e.nq + e.nkv) * 128 * 2;
    return launch_head(kind, p, A + (size_t)m0 * K, W, rows, N, K, s);
  };
  for (int m0 = 0; m0 < M; m0 += step) {
    const int rows = std::min(step, M - m0);
    TilePlan p = plan_tiles(kHeadCost, kHeadKinds, rows, N, K, false);
    if (!wide && (p.rows_big > 0 || p.kind == kHead256)) p = {0, kHead128};
    if (p.rows_big > 0) PRISM_TRY(rows_on(kHead256, m0, p.rows_big));
    PRISM_TRY(rows_on(p.kind, m0 + p.rows_big, rows - p.rows_big));
  }
  return PRISM_OK;
}

int launch_gemm_16_qkv(int dtype, const void *Xn, const void *Wqkv, int M, int K, int hd, const QkvEpilogue &e, hipStream_t s) {
  PRISM_REQUIRE(Xn && Wqkv && M >= 0 && is16(dtype) && e.pos && e.vt_col && e.rope_tab_t && e.rope_stride > 0 && e.QK && e.Vt, PRISM_EINVAL,
                "qkv gemm: bad arguments");
  PRISM_REQUIRE(!e.qk_norm || (e.q_gain && e.k_gain), PRISM_EINVAL, "qkv gemm: gains missing");
  PRISM_REQUIRE(gemm_16_qkv_supported(e.nq, e.nkv, hd, K), PRISM_EUNSUPPORTED, "qkv gemm: shape not supported by the fused epilogue");
  const int N = (e.nq + 2 * e.nkv) * 128;
  PRISM_REQUIRE((int64_t)N * K * 2 < ((int64_t)1 << 32) && (int64_t)256 * K * 2 < ((int64_t)1 << 32), PRISM_EUNSUPPORTED,
                "qkv gemm: the weight operand exceeds 4 GiB");
  // one order of every sum, the finishing kernel's, so this gives the bits of prism_op_gemm + prism_op_qkv_finish at every size
  return dtype == PRISM_DTYPE_BF16 ? launch_qkv_typed(e, (const bf16 *)Xn, (const bf16 *)Wqkv, M, N, K, s)
                                   : launch_qkv_typed(e, (const f16 *)Xn, (const f16 *)Wqkv, M, N, K, s);
}

}  // namespace prism
