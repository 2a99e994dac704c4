// Attention of a step's tokens over a paged K/V cache on the gfx950 matrix cores (16-bit types).
//
// A work item (paged.h) is up to 128 query rows of one (sequence, KV head) and a run of 64-key tiles.  A row is a (token, query
// head) pair, the G heads of a token side by side: whatever G is, a tile of K and V is read once for all of them, and a single token
// still gives the matrix cores G rows.  Row r of a block sees key k iff k <= p, k > p - window and k's page exists, p = position of
// its token.  As in attn_16.hip everything is computed transposed, S^T = K Q^T and O^T += V^T P^T, so that a lane owns one row and
// the accumulators of S^T are the second contraction's operand as they are.  K and V lie in the cache as they are projected, a row
// per key; V^T's fragments come out of LDS by the transposing read (ds_read_b64_tr_b16), so that appending a token is a row's store.
// P is rounded to the type of V, which the matrix cores ask for, and the denominators sum the rounded weights: 11 bits in half, as in
// attn_16.hip, 8 in bf16, whose values half cannot hold.  Items of up to 32 rows, which wait for memory, take a bf16 weight as two numbers, the
// second product with V costing nothing (100 sequences 315 us, 8.95 to 9.3 for three short ones); of more rows one, for there it would cost a fifth
// (us: 32 heads of 128 with a cap 596 and 756, two chunks of 300 to 500 tokens 100 and 123, 60 passages 153 and 180).
//
// Two ways of dividing an item between its workgroup's four waves:
//   more than 32 rows (chunks; matrix and vector work by turns, half of the cycles each): 32 rows per wave, tiles of 64 keys shared
//     through two LDS stages.  6900 tokens over up to 9700 each, 32 query heads over 8 of 128, half: 910 to 990 us, 860 to 930 TFLOP/s;
//   up to 32 rows (single tokens; HBM-bound): every wave takes all rows and its own 32 keys of every 128, through LDS of its own,
//     without a barrier until the four partial results meet.  A token of 100 sequences over up to 8000 each: 1.76 GB in 315 us,
//     5.6 TB/s; of one over 150 000: 0.61 GB in 115 us, 7 of them for joining.
// Keys of a sequence that were split over several items meet in paged_join_kernel.
#include <type_traits>

#include "paged.h"

namespace prism {

#define PRISM_GLOBAL_PTR(p) ((const __attribute__((address_space(1))) void *)(p))
#define PRISM_LDS_PTR(p) ((__attribute__((address_space(3))) void *)(p))

typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4;

template <typename T> struct Paged16;
template <> struct Paged16<bf16> {
  static constexpr bool kTwoParts = true;                      // weights of items of few rows: two numbers
  static constexpr float kLift = 0.f;
  static constexpr unsigned kExp = 0x7F80u;
  typedef bf16x2 vec2;
  static __device__ __forceinline__ float sum2(vec2 p, float c) { const vec2 one = {(bf16)1.0f, (bf16)1.0f}; return __builtin_amdgcn_fdot2_f32_bf16(p, one, c, false); }
  static __device__ __forceinline__ f32x4 mma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Paged16<f16> {
  static constexpr bool kTwoParts = false;
  static constexpr float kLift = 12.f;                         // weights are held times 2^12 (most 1): their small ones stay normal numbers
  static constexpr unsigned kExp = 0x7C00u;
  typedef __attribute__((ext_vector_type(2))) _Float16 vec2;
  static __device__ __forceinline__ float sum2(vec2 p, float c) { const vec2 one = {(f16)1.0f, (f16)1.0f}; return __builtin_amdgcn_fdot2(p, one, c, false); }
  static __device__ __forceinline__ f32x4 mma16(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};

// Which 16-byte chunk of a row stands where in LDS (chunk c of row r at slot c ^ swizzle).  K: the 16 rows that one pass of a read
// touches spread over all banks.  V: a transposing read takes 32 bytes of four rows per 16 lanes; the rows of one pass, four
// consecutive keys and 64 bytes (wide items) or eight and 32 bytes (narrow), spread over all banks.
template <int HD> __device__ __forceinline__ constexpr int swizzle_k(int r) { return HD == 128 ? r & 15 : (r >> 1) & 7; }
template <int HD> __device__ __forceinline__ constexpr int swizzle_v(int r) {
  return HD == 128 ? ((r & 3) << 2) | ((r & 4) >> 1) : ((r & 2) << 1) | ((r & 4) >> 1);
}

template <typename OT> __device__ __forceinline__ s16x4 read_transposed(const OT *p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)p);
}
// Reads whose results are waited for inside, for the loop that keeps loads to other places of LDS under way: in front of reads of its
// own the compiler waits for all of them.
__device__ __forceinline__ uint32_t lds_address(const void *p) { return (uint32_t)(uintptr_t)PRISM_LDS_PTR(p); }
template <typename V8> __device__ __forceinline__ void read_rows(V8 (&r)[4], const uint32_t (&p)[4]) {
  asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %5\n\tds_read_b128 %2, %6\n\tds_read_b128 %3, %7\n\ts_waitcnt lgkmcnt(0)"
               : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]) : "v"(p[0]), "v"(p[1]), "v"(p[2]), "v"(p[3]) : "memory");
}
template <typename V8> __device__ __forceinline__ void read_rows(V8 (&r)[8], const uint32_t (&p)[8]) {
  asm volatile("ds_read_b128 %0, %8\n\tds_read_b128 %1, %9\n\tds_read_b128 %2, %10\n\tds_read_b128 %3, %11\n\t"
               "ds_read_b128 %4, %12\n\tds_read_b128 %5, %13\n\tds_read_b128 %6, %14\n\tds_read_b128 %7, %15\n\ts_waitcnt lgkmcnt(0)"
               : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7])
               : "v"(p[0]), "v"(p[1]), "v"(p[2]), "v"(p[3]), "v"(p[4]), "v"(p[5]), "v"(p[6]), "v"(p[7]) : "memory");
}
__device__ __forceinline__ void read_transposed(s16x4 (&r)[8], const uint32_t (&p)[8]) {
  asm volatile("ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %9\n\tds_read_b64_tr_b16 %2, %10\n\tds_read_b64_tr_b16 %3, %11\n\t"
               "ds_read_b64_tr_b16 %4, %12\n\tds_read_b64_tr_b16 %5, %13\n\tds_read_b64_tr_b16 %6, %14\n\tds_read_b64_tr_b16 %7, %15\n\t"
               "s_waitcnt lgkmcnt(0)"
               : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7])
               : "v"(p[0]), "v"(p[1]), "v"(p[2]), "v"(p[3]), "v"(p[4]), "v"(p[5]), "v"(p[6]), "v"(p[7]) : "memory");
}
template <typename V8> __device__ __forceinline__ V8 join_halves(s16x4 a, s16x4 b) {
  union { s16x4 h[2]; V8 v; } u;
  u.h[0] = a;
  u.h[1] = b;
  return u.v;
}

// A V^T fragment of a tile in which some rows do not see some keys.  A weight of zero times a value that is not finite would reach the
// sum, so: values of keys that no row sees (`keep` has their bits clear) become zero; `worst` collects the largest magnitude bits.
__device__ __forceinline__ u32x4 clean_fragment(u32x4 v, u32x4 keep, u16x2 &worst) {
  v &= keep;
#pragma unroll
  for (int w = 0; w < 4; ++w) worst = __builtin_elementwise_max(worst, __builtin_bit_cast(u16x2, v[w] & 0x7FFF7FFFu));
  return v;
}
template <typename OT> __device__ __forceinline__ bool not_finite(u16x2 worst) { return worst[0] >= Paged16<OT>::kExp || worst[1] >= Paged16<OT>::kExp; }
// Of keys that some rows see and others do not, the finite values go through the matrix cores, and the others where they are seen, at the end
template <typename OT> __device__ __forceinline__ u32x4 finite_only(u32x4 v) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if ((v[w] & Paged16<OT>::kExp) == Paged16<OT>::kExp) v[w] &= 0xFFFF0000u;
    if ((v[w] >> 16 & Paged16<OT>::kExp) == Paged16<OT>::kExp) v[w] &= 0xFFFFu;
  }
  return v;
}

// Scores with a cap, slopes or both, in units of log 2: (cap tanh(u) - slope (p - k)) log2(e), u = s scale / cap.
//   caps up to kExactCap: with tanh(u) = 1 - 2 / (1 + e^2u) a score is -2 cap / (1 + 2^(in s)) + (slope k + rest), off by 2^-22 of the cap, at most
//     2^-16, no more than what the weights lose to their own rounding;
//   larger caps: that would be as large as the scores themselves.  Where |u| <= 1/2, (in s) (tanh(u) / u) + (slope k + rest) with a polynomial of
//     u^2, off by 2^-23 of the score; beyond, tanh as above, 2^-22 of a cap that the score is no longer small against.
// The factors hold scale and log2(e), k counts from the tile's first key of the lane and rest has slope, the row's position and the first form's cap.
struct Modifier {
  static constexpr float kLog2e = 1.4426950408889634f, kExactCap = 64.f;
  float in, small, cap, slope, rest;                          // small: from s to u
  bool capped, large;
  __device__ __forceinline__ Modifier(float scale, float softcap, float slope_, int away) {
    capped = softcap > 0.f;
    large = softcap > kExactCap;
    small = capped ? scale / softcap : 0.f;
    in = capped && !large ? scale * (2.0f * kLog2e) / softcap : scale * kLog2e;
    cap = softcap * kLog2e;
    slope = slope_ * kLog2e;
    rest = (capped && !large ? cap : 0.f) - slope * (float)away;
  }
  // tanh(u) / u for u^2 = z <= 1/4: of the polynomials of degree 4 that are 1 at 0 the one whose largest relative error is smallest (2^-26)
  static __device__ __forceinline__ float ratio(float z) {
    return __builtin_fmaf(__builtin_fmaf(__builtin_fmaf(__builtin_fmaf(0.017241491f, z, -0.0530454926f), z, 0.13325879f), z, -0.333331436f), z, 1.0f);
  }
  // Scores s[i] of the keys key(i), i < N.  One branch around all of them: with one around each none of the exponentials and
  // reciprocals overlap (32 heads of 128, a cap, 7000 tokens over 2000 to 4000 more: 752 and 631 us).  With the polynomial for caps of 50 too
  // they take 622 instead of 599, and where scores reach the cap 881
  template <int N, typename S, typename Key> __device__ __forceinline__ void operator()(S &s, Key key) const {
    if (large) {
      float most = 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i) most = fmaxf(most, fabsf(s[i]));
      if (__builtin_amdgcn_ballot_w64(most * small > 0.5f) == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float u = s[i] * small;
          s[i] = __builtin_fmaf(s[i] * in, ratio(u * u), bias(key(i)));
        }
      } else {                                                // each by its size: small ones beside one that reaches minus the cap have all the weight
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float u = s[i] * small;
          const float far = __builtin_fmaf(-2.0f * cap, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(u * (2.0f * kLog2e))), cap);
          s[i] = (fabsf(u) <= 0.5f ? s[i] * in * ratio(u * u) : far) + bias(key(i));
        }
      }
    } else if (capped) {
#pragma unroll
      for (int i = 0; i < N; ++i) s[i] = __builtin_fmaf(-2.0f * cap, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(s[i] * in)), bias(key(i)));
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) s[i] = __builtin_fmaf(s[i], in, bias(key(i)));
    }
  }
  __device__ __forceinline__ float bias(int key) const { return __builtin_fmaf(slope, (float)key, rest); }
};

// Exponents are s c - mb, an instruction a score, with mb the maximum's product.  Beyond kFar mb's rounding shows in the weights (2^-8 there, and
// from 2^27 on they would leave half's range), so the maximum is subtracted from the scores first.
static constexpr float kFar = 65536.f;

// Two workgroups on a compute unit where the registers of three do not hold all (MOD, HD 64, chunks of 14 heads over a window of 1000:
// 55 us, with three and 18 values kept in memory 64)
template <typename OT, int HD, bool MOD>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(HD == 128 || MOD ? 2 : 3, HD == 128 || MOD ? 2 : 3)))
void attention_paged_16_kernel(const PagedAttn a) {
  typedef typename Mfma<OT>::vec8 vec8;
  typedef typename Mfma<OT>::vec4 vec4;
  typedef Paged16<OT> P16;
  constexpr int CH = HD / 8;                                  // 16-byte chunks of a row
  constexpr int RI = 64 / CH;                                 // rows that a wave's load instruction moves
  constexpr int NI = 16 / RI;                                 // instructions for 16 rows
  // groups of 16 keys whose V^T fragments are read ahead of the softmax; two next to modified scores do not fit into the registers
  constexpr int VK = MOD ? 1 : 2;
  // Four objects, so that the compiler knows which reads a load in flight cannot touch.  Wide: stages 0 and 1 of K and of V, 64 rows
  // each.  Narrow: 16 rows of each for every wave, keys 0-15 and 16-31 of its step.  Aligned so that flipping bits within a row is flipping them in the address.
  __shared__ __align__(1024) OT lK0[64 * HD], lK1[64 * HD], lV0[64 * HD], lV1[64 * HD];

  const int nkv = a.shape.n_kv_heads, G = a.shape.n_q_heads / nkv;
  const int kvh = blockIdx.x % nkv, item = blockIdx.x / nkv;
  PlanItem it;
  if (!load_item(a, item, it)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rows = it.n_tok * G, window = a.shape.window;
  const int cap_keys = a.shape.max_pages << a.page_shift;
  const int last = it.pos0 + it.n_tok - 1;                    // the block's last position
  const int limit = last + 1 < cap_keys ? last + 1 : cap_keys;   // keys that some row of it may see end here
  const int32_t *const table = a.table + (int64_t)it.seq * a.shape.max_pages;
  const OT *const Kh = (const OT *)a.K + ((int64_t)kvh * HD << a.page_shift);
  const OT *const Vh = (const OT *)a.V + ((int64_t)kvh * HD << a.page_shift);
  const float c_exp = a.unit;                                 // scores times c_exp: in units of log 2

  // Table entry of the 16 keys from k0 on (a multiple of 16; behind the last key, that key's), and the page that it gives, none: -1.
  // Apart, because waiting for a scalar load is waiting for all LDS reads under way: entries are asked for a step before they are used
  auto entry_of = [&](int k0) __attribute__((always_inline)) { return load_const(table + ((k0 < limit ? k0 : limit - 1) >> a.page_shift)); };
  auto page_from = [&](int entry, int k0) __attribute__((always_inline)) { return k0 < limit && (unsigned)entry < (unsigned)a.shape.n_pages ? entry : -1; };
  auto page_of = [&](int k0) __attribute__((always_inline)) { return page_from(entry_of(k0), k0); };
  // values in front of those keys' rows; keys without a page read the first one, under the mask
  auto rows_at = [&](int page, int k0) __attribute__((always_inline)) {
    return (int64_t)(page < 0 ? 0 : page) * a.page_stride + (int64_t)(k0 & ((1 << a.page_shift) - 1)) * HD;
  };
  // This lane's chunk of a load instruction of RI rows: row lane / CH, slot lane % CH; the swizzle is applied to the source
  uint32_t oK[NI], oV[NI];
#pragma unroll
  for (int j = 0; j < NI; ++j) {
    const int r = j * RI + lane / CH, c = lane % CH;
    oK[j] = (lane / CH * HD + (c ^ swizzle_k<HD>(r)) * 8) * 2;   // bytes, from the instruction's first row
    oV[j] = (lane / CH * HD + (c ^ swizzle_v<HD>(r)) * 8) * 2;
  }
  // 16 rows: an instruction's 1 KiB lies as far from the first one's in memory as in LDS, so the offset of both is an immediate
  auto load16 = [&](const OT *src, const uint32_t (&o)[NI], OT *dst) __attribute__((always_inline)) {
    const char *const s = reinterpret_cast<const char *>(src);
    __builtin_amdgcn_global_load_lds(PRISM_GLOBAL_PTR(s + o[0]), PRISM_LDS_PTR(dst), 16, 0, 0);
    __builtin_amdgcn_global_load_lds(PRISM_GLOBAL_PTR(s + o[1]), PRISM_LDS_PTR(dst), 16, 1024, 0);
    if constexpr (NI == 4) {
      __builtin_amdgcn_global_load_lds(PRISM_GLOBAL_PTR(s + o[2]), PRISM_LDS_PTR(dst), 16, 2 * 1024, 0);
      __builtin_amdgcn_global_load_lds(PRISM_GLOBAL_PTR(s + o[3]), PRISM_LDS_PTR(dst), 16, 3 * 1024, 0);
    }
  };

  if (rows <= 32) {
    // ------------------------------------------------------------------------------------------------ narrow
    const int g = lane >> 4, c = lane & 15;
    OT *const k0p = lK0 + wave * 16 * HD, *const k1p = lK1 + wave * 16 * HD, *const v0p = lV0 + wave * 16 * HD, *const v1p = lV1 + wave * 16 * HD;
    const int n_steps = (limit + 31) >> 5;
    const int s_end = it.tile1 * 2 < n_steps ? it.tile1 * 2 : n_steps;
    // reads: K row c, chunk 4 kk + g; V^T of dimensions 16 t + c, keys 4 g .. 4 g + 3 of 16
    const int rdK = c * HD + ((g ^ (swizzle_k<HD>(c) & 3)) | (swizzle_k<HD>(c) & ~3)) * 8;      // kk flips the bits from 4 on
    const int vr = 4 * g + (c >> 2);
    const int rdV = vr * HD + (((c & 3) >> 1) ^ swizzle_v<HD>(vr)) * 8 + (c & 1) * 4;          // t flips the bits from 2 on
    const uint32_t at_k0 = lds_address(k0p + rdK), at_k1 = lds_address(k1p + rdK), at_v0 = lds_address(v0p + rdV), at_v1 = lds_address(v1p + rdV);
    auto narrow = [&](auto rb_tag) __attribute__((always_inline)) {
      constexpr int RB = decltype(rb_tag)::value;            // blocks of 16 rows
      vec8 qf[RB][HD / 32];
      int pos[RB];
      float slope[RB], m_run[RB], l_run[RB];
      f32x4 o[RB][HD / 16];
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        const int r = b * 16 + c < rows ? b * 16 + c : rows - 1, t = r / G, h = kvh * G + r - t * G;
        pos[b] = it.pos0 + t;
        slope[b] = MOD && a.slopes ? a.slopes[h] : 0.f;
        const OT *q = (const OT *)a.Q + (int64_t)(it.row0 + t) * a.q_stride + (int64_t)h * HD + g * 8;
#pragma unroll
        for (int kk = 0; kk < HD / 32; ++kk) qf[b][kk] = *reinterpret_cast<const vec8 *>(q + kk * 32);
        m_run[b] = -INFINITY;
        l_run[b] = 0.f;
#pragma unroll
        for (int t16 = 0; t16 < HD / 16; ++t16) o[b][t16] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
      // some row sees a key of the 32 from k0 on that another does not, or some of them do not exist
      auto mixed = [&](int k0) __attribute__((always_inline)) {
        return k0 + 31 > it.pos0 || k0 + 31 >= limit || (window > 0 && k0 <= last - window);
      };
      bool odd = false;                                      // values that are not finite were taken out of such a step
      int st = it.tile0 * 2 + wave;
      if (st < s_end) {
        int pg0 = page_of(st * 32), pg1 = page_of(st * 32 + 16);   // pages of the step's two groups of 16 keys
        load16(Kh + rows_at(pg0, st * 32), oK, k0p);
        load16(Kh + rows_at(pg1, st * 32 + 16), oK, k1p);
        load16(Vh + rows_at(pg0, st * 32), oV, v0p);
        load16(Vh + rows_at(pg1, st * 32 + 16), oV, v1p);
        int nx0 = entry_of(st * 32 + 128), nx1 = entry_of(st * 32 + 144);    // of the next step's
        wait_loads<4 * NI>();                                  // the queries are here: nothing in the loop waits for them
        for (; st < s_end; st += 4) {
          const int k0 = st * 32, kg = k0 + 4 * g;             // key 16 kb + e of this lane: kg + 16 kb + e
          const bool more = st + 4 < s_end;
          f32x4 s[RB][2];
          // no barrier here: this wave's own loads.  K's have landed when only V's 2 NI, which were issued behind them, are under way
          vec8 kf[HD / 16];                                  // fragment 2 kk + kb
          uint32_t at[HD / 16];
#pragma unroll
          for (int f = 0; f < HD / 16; ++f) at[f] = ((f & 1) ? at_k1 : at_k0) ^ ((f >> 1) * 64);
          wait_loads<2 * NI>();
          read_rows(kf, at);
          const int cur0 = pg0, cur1 = pg1;
          if (more) {                                        // K's LDS is free: the next step's keys may come
            pg0 = page_from(nx0, k0 + 128);
            pg1 = page_from(nx1, k0 + 144);
            load16(Kh + rows_at(pg0, k0 + 128), oK, k0p);
            load16(Kh + rows_at(pg1, k0 + 144), oK, k1p);
            nx0 = entry_of(k0 + 256);
            nx1 = entry_of(k0 + 272);
          }
#pragma unroll
          for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
              s[b][kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int kk = 0; kk < HD / 32; ++kk) s[b][kb] = P16::mma16(kf[2 * kk + kb], qf[b][kk], s[b][kb]);
            }
          const bool masked = cur0 < 0 || cur1 < 0 || mixed(k0);
          vec8 pf[RB], rest[P16::kTwoParts ? RB : 1];           // weights, and what their rounding left
#pragma unroll
          for (int b = 0; b < RB; ++b) {
            if (MOD) {
              const Modifier modified(a.scale, a.softcap, slope[b], pos[b] - kg);
              float x[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) x[i] = s[b][i >> 2][i & 3];
              modified.template operator()<8>(x, [](int i) { return (i >> 2) * 16 + (i & 3); });
#pragma unroll
              for (int i = 0; i < 8; ++i) s[b][i >> 2][i & 3] = x[i];
            }
            if (masked) {
              const int lo = (window > 0 ? pos[b] - window + 1 : 0) - kg, hi = (pos[b] < limit - 1 ? pos[b] : limit - 1) - kg;
#pragma unroll
              for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const int key = kb * 16 + e;                 // from kg on
                  if (!(key >= lo && key <= hi && (kb ? cur1 : cur0) >= 0)) s[b][kb][e] = -INFINITY;
                }
            }
            float mx = fmaxf(fmaxf(fmaxf(s[b][0][0], s[b][0][1]), fmaxf(s[b][0][2], s[b][0][3])),
                             fmaxf(fmaxf(s[b][1][0], s[b][1][1]), fmaxf(s[b][1][2], s[b][1][3])));
            mx = max_xor32(max_xor16(mx));
            const float m_new = fmaxf(m_run[b], mx);
            const float ref = m_new == -INFINITY ? 0.f : m_new;   // no key yet: weights exp(-inf) = 0
            const float alpha = __builtin_amdgcn_exp2f((m_run[b] - ref) * c_exp);
            float mb = ref * c_exp - P16::kLift;
            if (__builtin_amdgcn_ballot_w64(!(fabsf(mb) < kFar)) != 0) {
              mb = -P16::kLift;
#pragma unroll
              for (int kb = 0; kb < 2; ++kb) s[b][kb] -= ref;
            }
            m_run[b] = m_new;
            float psum = 0.f;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
              for (int e = 0; e < 4; e += 2) {
                const float p0 = __builtin_amdgcn_exp2f(s[b][kb][e] * c_exp - mb), p1 = __builtin_amdgcn_exp2f(s[b][kb][e + 1] * c_exp - mb);
                const typename P16::vec2 ph = {(OT)p0, (OT)p1};
                psum = P16::sum2(ph, psum);
                pf[b][kb * 4 + e] = ph[0];
                pf[b][kb * 4 + e + 1] = ph[1];
                if constexpr (P16::kTwoParts) {
                  const typename P16::vec2 pr = {(OT)(p0 - to_f32(ph[0])), (OT)(p1 - to_f32(ph[1]))};
                  psum = P16::sum2(pr, psum);
                  rest[b][kb * 4 + e] = pr[0];
                  rest[b][kb * 4 + e + 1] = pr[1];
                }
              }
            l_run[b] = l_run[b] * alpha + psum;
            // the running maxima usually settle after a few steps; opaque, or the compiler makes it an unconditional multiply again
            unsigned long long moved = __builtin_amdgcn_ballot_w64(alpha != 1.0f);
            asm volatile("" : "+s"(moved));
            if (moved != 0) {
#pragma unroll
              for (int t = 0; t < HD / 16; ++t) o[b][t] *= alpha;
            }
          }
          vec8 vf[HD / 16];
          if (more) wait_loads<2 * NI>();                    // V's have landed when only the next K's are under way
          else wait_loads<0>();
#pragma unroll
          for (int t = 0; t < HD / 16; t += 4) {
            s16x4 half8[8];
            uint32_t at_v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) at_v[u] = ((u & 1) ? at_v1 : at_v0) ^ ((t + (u >> 1)) * 32);
            read_transposed(half8, at_v);
#pragma unroll
            for (int u = 0; u < 4; ++u) vf[t + u] = join_halves<vec8>(half8[2 * u], half8[2 * u + 1]);
          }
          if (more) {
            load16(Vh + rows_at(pg0, k0 + 128), oV, v0p);
            load16(Vh + rows_at(pg1, k0 + 144), oV, v1p);
          }
          if (masked) {
            u32x4 keep;
#pragma unroll
            for (int w = 0; w < 4; ++w) {                      // halves 2 w and 2 w + 1: keys 16 (w / 2) + 4 g + 2 (w % 2) and the next
              const int key = (w >> 1) * 16 + (w & 1) * 2;
              const bool page = ((w >> 1) ? cur1 : cur0) >= 0;
              keep[w] = (page && key < limit - kg ? 0xFFFFu : 0u) | (page && key + 1 < limit - kg ? 0xFFFF0000u : 0u);
            }
            u16x2 worst = {0, 0};
#pragma unroll
            for (int t = 0; t < HD / 16; ++t) vf[t] = __builtin_bit_cast(vec8, clean_fragment(__builtin_bit_cast(u32x4, vf[t]), keep, worst));
            if (__builtin_amdgcn_ballot_w64(not_finite<OT>(worst)) != 0) {
              odd = true;
#pragma unroll
              for (int t = 0; t < HD / 16; ++t) vf[t] = __builtin_bit_cast(vec8, finite_only<OT>(__builtin_bit_cast(u32x4, vf[t])));
            }
          }
#pragma unroll
          for (int t = 0; t < HD / 16; ++t)
#pragma unroll
            for (int b = 0; b < RB; ++b) {
              o[b][t] = P16::mma16(vf[t], pf[b], o[b][t]);
              if constexpr (P16::kTwoParts) o[b][t] = P16::mma16(vf[t], rest[b], o[b][t]);
            }
        }
      }
      // ---- the four waves' results meet: values in lK0 / lK1 (two waves each), maxima and sums in lV0, a sum's sign says `odd`; 16 rows at a time
      float *const mine = reinterpret_cast<float *>(wave < 2 ? lK0 : lK1) + (wave & 1) * 16 * HD;
      float2 *const ml = reinterpret_cast<float2 *>(lV0);
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        __syncthreads();
#pragma unroll
        for (int t = 0; t < HD / 16; ++t) *reinterpret_cast<f32x4 *>(mine + c * HD + ((t * 4 + g) ^ c) * 4) = o[b][t];
        const float l = sum_xor32(sum_xor16(l_run[b]));
        if (g == 0) ml[wave * 16 + c] = make_float2(m_run[b], odd ? -l : l);
        __syncthreads();
        const int r = tid / CH, d = tid % CH;                // row of the 16, eight of its dimensions
        const int row = b * 16 + r;
        if (r < 16 && row < rows) {
          float m = -INFINITY;
#pragma unroll
          for (int w = 0; w < 4; ++w) m = fmaxf(m, ml[w * 16 + r].x);
          const float ref = m == -INFINITY ? 0.f : m;
          unsigned signs = 0;
          float sum = 0.f, v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const float2 x = ml[w * 16 + r];
            const float f = __builtin_amdgcn_exp2f((x.x - ref) * c_exp);
            const float *src = reinterpret_cast<const float *>(w < 2 ? lK0 : lK1) + (w & 1) * 16 * HD + r * HD;
            sum += f * fabsf(x.y);
            signs |= __float_as_uint(x.y);
            if (x.x != -INFINITY) {                          // a wave without keys has nothing (and its zero weight is none)
#pragma unroll
              for (int q = 0; q < 2; ++q) {
                const f32x4 y = *reinterpret_cast<const f32x4 *>(src + ((d * 2 + q) ^ r) * 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[q * 4 + e] += f * y[e];
              }
            }
          }
          const int t = row / G, h = kvh * G + row - t * G;
          float most = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) most = worst_of(v[e], most);
          if (__builtin_amdgcn_ballot_w64(((signs >> 31 != 0) | (most != most)) & (sum == sum)) != 0) {
            float y[8] = {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
            settle<OT, HD>(a, table, Vh + d * 8, it.tile0 * 64, it.tile1 * 64 < limit ? it.tile1 * 64 : limit,
                           window > 0 ? it.pos0 + t - window + 1 : 0, it.pos0 + t, signs >> 31, y);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = y[e];
          }
          if (it.part0 < 0) {
            const float inv = sum == 0.f ? 0.f : 1.0f / sum;
            vec8 y;
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = round_to<OT>(v[e] * inv);
            *reinterpret_cast<vec8 *>((OT *)a.out + (int64_t)(it.row0 + t) * a.out_stride + (int64_t)h * HD + d * 8) = y;
          } else {
            const int64_t at = (int64_t)(it.part0 + row) * nkv + kvh;
#pragma unroll
            for (int q = 0; q < 2; ++q) *reinterpret_cast<f32x4 *>(a.part_O + at * HD + d * 8 + q * 4) = f32x4{v[q * 4], v[q * 4 + 1], v[q * 4 + 2], v[q * 4 + 3]};
            if (d == 0) a.part_ml[at] = make_float2(m, sum);
          }
        }
      }
    };
    if (rows <= 16) narrow(std::integral_constant<int, 1>{});
    else narrow(std::integral_constant<int, 2>{});
    return;
  }

  // -------------------------------------------------------------------------------------------------- wide
  const int half = lane >> 5, c = lane & 31;
  const int r_first = wave * 32;
  const int r = r_first + c < rows ? r_first + c : rows - 1, tok = r / G, head = kvh * G + r - tok * G;
  const int pos = it.pos0 + tok;
  const bool active = r_first < rows;
  const int r_last = r_first + 31 < rows ? r_first + 31 : rows - 1;
  const int w_first = it.pos0 + r_first / G, w_last = it.pos0 + r_last / G;       // positions of the wave's first and last row
  const float slope = MOD && a.slopes ? a.slopes[head] : 0.f;
  vec8 qf[HD / 16];
  {
    const OT *q = (const OT *)a.Q + (int64_t)(it.row0 + tok) * a.q_stride + (int64_t)head * HD + half * 8;
#pragma unroll
    for (int kk = 0; kk < HD / 16; ++kk) qf[kk] = *reinterpret_cast<const vec8 *>(q + kk * 16);
  }
  f32x16 o[HD / 32];
#pragma unroll
  for (int t = 0; t < HD / 32; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[t][e] = 0.f;
  // What the exponents are taken from: a row's largest score, but an old one until a new one is 2^3 times its weight.  With 32 rows some
  // maximum moves in many tiles, and every move is a multiplication of all accumulators; weights of up to 2^3 cost nothing (half holds
  // them times 2^12, so up to 2^15).  us with every new maximum taken and with this: chunks of 16 heads of 64 250, 238; of 32 heads of 128
  // with a cap 636, 617, without 951, 949
  const float slack = fminf(3.0f / c_exp, 1e30f);
  float m_run = -INFINITY, m_move = -INFINITY, mb = -P16::kLift, l_run = 0.f;      // a score above m_move moves m_run; mb: what exponents lose

  // a wave stages the tile's keys 16 wave .. 16 wave + 15; all four groups' pages say which keys exist
  struct Entries { int e[4]; };
  struct Pages { int own; unsigned there; };
  auto entries_of = [&](int kt) __attribute__((always_inline)) {
    Entries n;
#pragma unroll
    for (int q = 0; q < 4; ++q) n.e[q] = entry_of(kt * 64 + q * 16);
    return n;
  };
  auto pages_from = [&](const Entries &n, int kt) __attribute__((always_inline)) {
    Pages p = {-1, 0};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int page = page_from(n.e[q], kt * 64 + q * 16);
      p.there |= page >= 0 ? 1u << q : 0u;
      p.own = q == wave ? page : p.own;
    }
    return p;
  };
  auto stage = [&](int kt, int page, auto buf_tag) __attribute__((always_inline)) {
    constexpr int BUF = decltype(buf_tag)::value;
    const int k0 = kt * 64 + wave * 16;
    load16(Kh + rows_at(page, k0), oK, (BUF ? lK1 : lK0) + wave * 16 * HD);
    load16(Vh + rows_at(page, k0), oV, (BUF ? lV1 : lV0) + wave * 16 * HD);
  };
  const int rdK = c * HD + ((half ^ (swizzle_k<HD>(c) & 1)) | (swizzle_k<HD>(c) & ~1)) * 8;                // kk flips the bits from 2 on
  // V^T of dimensions 32 t + c, keys 16 ks + 4 half .. + 3 (and + 8): lane i of 16 reads row i / 4, dimensions 16 ((lane / 16) % 2) + 4 (i % 4)
  const int vr = 4 * half + ((lane & 15) >> 2), vc = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
  const int rdV = vr * HD + (vc ^ swizzle_v<HD>(vr)) * 8 + (lane & 1) * 4;                                 // t flips the bits from 4 on

  // of the 64 keys from k0 on: some row of the wave may see some; some row of the wave sees a key that another does not, or some keys do
  // not exist; the same for any two rows of the block
  auto touched = [&](int k0) __attribute__((always_inline)) { return active && k0 <= w_last && (window == 0 || k0 + 63 > w_first - window); };
  auto mixed = [&](int k0, int first, int last) __attribute__((always_inline)) {
    return k0 + 63 > first || k0 + 63 >= limit || (window > 0 && k0 <= last - window);
  };
  // A tile in which some rows of the block do not see some keys: a weight of zero times a value that is not finite would reach the sum.
  // So before the others read it, a wave clears what it staged of keys that nobody sees, and of the other keys what is not finite; rows
  // that see those values get them at the end (`odd`).
  bool odd = false;
  auto clean = [&](int kt, int page, auto buf_tag) __attribute__((always_inline)) {
    OT *const v = (decltype(buf_tag)::value ? lV1 : lV0) + wave * 16 * HD + lane * 8;
    wait_loads<0>();
    u16x2 worst = {0, 0};
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const unsigned there = page >= 0 && kt * 64 + wave * 16 + j * RI + lane / CH < limit ? ~0u : 0u;
      const u32x4 x = clean_fragment(*reinterpret_cast<const u32x4 *>(v + j * RI * HD), u32x4{there, there, there, there}, worst);
      *reinterpret_cast<u32x4 *>(v + j * RI * HD) = finite_only<OT>(x);
    }
    odd = odd || __builtin_amdgcn_ballot_w64(not_finite<OT>(worst)) != 0;
  };
  const int kt_end = it.tile1;
  Pages cur = {-1, 0};
  Entries ahead = entries_of(it.tile0);                       // of the next tile that is not under way
  if (it.tile0 < kt_end) {
    cur = pages_from(ahead, it.tile0);
    stage(it.tile0, cur.own, std::integral_constant<int, 0>{});
    ahead = entries_of(it.tile0 + 1);
    if (cur.there != 15u || mixed(it.tile0 * 64, it.pos0, last)) clean(it.tile0, cur.own, std::integral_constant<int, 0>{});
  }
  __syncthreads();                                            // also waits for this wave's own loads

  auto step = [&](int kt, auto cur_tag) __attribute__((always_inline)) {
    constexpr int CUR = decltype(cur_tag)::value;
    const OT *const lK = CUR ? lK1 : lK0;
    const OT *const lV = CUR ? lV1 : lV0;
    const Pages next = pages_from(ahead, kt + 1);
    if (kt + 1 < kt_end) stage(kt + 1, next.own, std::integral_constant<int, CUR ^ 1>{});
    ahead = entries_of(kt + 2);
    const int k0 = kt * 64, kh = k0 + 4 * half;
    if (touched(k0)) {
      int atK = rdK, atV = rdV;                               // opaque: the 16 addresses of either stage are one instruction each to make,
      asm volatile("" : "+v"(atK), "+v"(atV));                // and registers that spill if they are kept over the loop
      f32x16 s[2];
      vec8 kf[2][HD / 16];
      wait_lds();                                             // of the scalar loads: with one under way, no LDS read can be waited for alone
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int kk = 0; kk < HD / 16; ++kk) kf[kb][kk] = *reinterpret_cast<const vec8 *>(&lK[(atK ^ (kk * 16)) + kb * 32 * HD]);
      __builtin_amdgcn_sched_barrier(0);                      // all under way before the first is waited for
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int e = 0; e < 16; ++e) s[kb][e] = 0.f;
        if (kb == 1) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int kk = 0; kk < HD / 16; ++kk) s[kb] = Mfma<OT>::mma(kf[kb][kk], qf[kk], s[kb]);
      }
      vec8 vf[VK][HD / 32];
      auto read_v = [&](int t, int ks) __attribute__((always_inline)) {
        return join_halves<vec8>(read_transposed(&lV[(atV ^ (t * 32)) + ks * 16 * HD]), read_transposed(&lV[(atV ^ (t * 32)) + (ks * 16 + 8) * HD]));
      };
#pragma unroll
      for (int ks = 0; ks < VK; ++ks)
#pragma unroll
        for (int t = 0; t < HD / 32; ++t) vf[ks][t] = read_v(t, ks);
      // key kb * 32 + (e / 4) * 8 + e % 4 from kh on
      if (MOD) {
        const Modifier modified(a.scale, a.softcap, slope, pos - kh);
        float x[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) x[i] = s[i >> 4][i & 15];
        modified.template operator()<32>(x, [](int i) { return (i >> 2) * 8 + (i & 3); });
#pragma unroll
        for (int i = 0; i < 32; ++i) s[i >> 4][i & 15] = x[i];
      }
      if (cur.there != 15u || mixed(k0, w_first, w_last)) {
        const int lo = (window > 0 ? pos - window + 1 : 0) - kh, hi = (pos < limit - 1 ? pos : limit - 1) - kh;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int key = kb * 32 + (e >> 2) * 8 + (e & 3);
            if (!(key >= lo && key <= hi && (cur.there >> (kb * 2 + (e >> 3)) & 1))) s[kb][e] = -INFINITY;
          }
      }
      float mxk[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e) mxk[kb] = fmaxf(mxk[kb], s[kb][e]);
      __builtin_amdgcn_sched_barrier(0);
      const float mx = max_xor32(fmaxf(mxk[0], mxk[1]));
      if (__builtin_amdgcn_ballot_w64(mx > m_move) != 0) {
        const float m_new = mx > m_move ? fmaxf(mx, m_run) : m_run;
        const float ref = m_new == -INFINITY ? 0.f : m_new;   // no key yet: weights exp(-inf) = 0
        const float alpha = __builtin_amdgcn_exp2f((m_run - ref) * c_exp);
        m_run = m_new;
        m_move = m_new + slack;
        mb = ref * c_exp - P16::kLift;
        l_run *= alpha;
#pragma unroll
        for (int t = 0; t < HD / 32; ++t)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[t][e] *= alpha;
        if (__builtin_amdgcn_ballot_w64(!(fabsf(mb) < kFar)) != 0) {
          mb = -P16::kLift;
          m_move = -INFINITY;                                 // here again in the next tile, and in all that have a key
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[kb][e] -= ref;
        }
      }
      float psum = 0.f;
      vec8 pf[4];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
          typename P16::vec2 ph;
          ph[0] = (OT)__builtin_amdgcn_exp2f(s[kb][e] * c_exp - mb);
          ph[1] = (OT)__builtin_amdgcn_exp2f(s[kb][e + 1] * c_exp - mb);
          psum = P16::sum2(ph, psum);
          pf[kb * 2 + (e >> 3)][e & 7] = ph[0];
          pf[kb * 2 + (e >> 3)][(e & 7) + 1] = ph[1];
        }
      l_run += psum;
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
#pragma unroll
        for (int t = 0; t < HD / 32; ++t) {
          const vec8 v = ks < VK ? vf[ks < VK ? ks : 0][t] : read_v(t, ks);
          o[t] = Mfma<OT>::mma(v, pf[ks], o[t]);
        }
      }
    }
    cur = next;
    if (kt + 1 < kt_end && (cur.there != 15u || mixed(k0 + 64, it.pos0, last))) clean(kt + 1, cur.own, std::integral_constant<int, CUR ^ 1>{});
    __syncthreads();                                          // the next tile has landed and everyone is done with this one
  };
  for (int kt = it.tile0; kt < kt_end; kt += 2) {
    step(kt, std::integral_constant<int, 0>{});
    if (kt + 1 < kt_end) step(kt + 1, std::integral_constant<int, 1>{});
  }

  // any wave's clearing concerns all rows
  int *const odd_waves = reinterpret_cast<int *>(lK0);
  if (lane == 0) odd_waves[wave] = odd;
  __syncthreads();
  odd = odd_waves[0] | odd_waves[1] | odd_waves[2] | odd_waves[3];
  const float l_tot = sum_xor32(l_run);
  if (!active) return;
  // lane holds d = 32 t + 8 (e / 4) + 4 half + e % 4 of its row
  float most = 0.f;
#pragma unroll
  for (int t = 0; t < HD / 32; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) most = worst_of(o[t][e], most);
  OT *const mine = (wave < 2 ? lV0 : lV1) + (wave & 1) * 32 * HD;          // LDS of the wave's own
  if (odd || __builtin_amdgcn_ballot_w64(most != most && l_tot == l_tot) != 0) {
    // half of the sums at a time through LDS, a lane's own four side by side, so that a loop can take them: unrolled over the registers, this would
    // be more code than the rest of the kernel
    f32x4 *const sums = reinterpret_cast<f32x4 *>(mine) + lane;
#pragma unroll
    for (int t0 = 0; t0 < HD / 32; t0 += HD / 64) {
#pragma unroll
      for (int i = 0; i < HD / 16; ++i)
        sums[i * 64] = f32x4{o[t0 + i / 4][i % 4 * 4], o[t0 + i / 4][i % 4 * 4 + 1], o[t0 + i / 4][i % 4 * 4 + 2], o[t0 + i / 4][i % 4 * 4 + 3]};
#pragma unroll 1
      for (int i = 0; i < HD / 16; ++i) {
        const f32x4 x = sums[i * 64];
        float y[4] = {x[0], x[1], x[2], x[3]};
        if (!odd && __builtin_amdgcn_ballot_w64(y[0] != y[0] || y[1] != y[1] || y[2] != y[2] || y[3] != y[3]) == 0) continue;
        settle<OT, HD>(a, table, Vh + t0 * 32 + i * 8 + half * 4, it.tile0 * 64, it.tile1 * 64 < limit ? it.tile1 * 64 : limit,
                       window > 0 ? pos - window + 1 : 0, pos, odd, y);
        sums[i * 64] = f32x4{y[0], y[1], y[2], y[3]};
      }
#pragma unroll
      for (int i = 0; i < HD / 16; ++i) {
        const f32x4 x = sums[i * 64];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[t0 + i / 4][i % 4 * 4 + e] = x[e];
      }
    }
  }
  if (it.part0 < 0) {
    const float inv = l_tot == 0.f ? 0.f : 1.0f / l_tot;
    // through that LDS, so that a store is whole rows: stored from the accumulators, eight bytes of 32 rows at a time, 60
    // passages of 100 to 500 tokens take 165 us instead of 153
#pragma unroll
    for (int t = 0; t < HD / 32; ++t)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        vec4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = round_to<OT>(o[t][q * 4 + e] * inv);
        *reinterpret_cast<vec4 *>(mine + c * HD + ((t * 4 + q) ^ swizzle_k<HD>(c)) * 8 + half * 4) = v;
      }
    // (LDS serves a wave in order; the fences keep the compiler to it, the barrier, no instruction, makes the lanes meet)
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    const int64_t to = (int64_t)(it.row0 + tok) * a.out_stride + (int64_t)head * HD;
#pragma unroll
    for (int j = 0; j < 32 / RI; ++j) {
      const int row = j * RI + lane / CH, d = lane % CH;
      const int64_t row_to = (int64_t)(uint32_t)__shfl((int)(to & 0xFFFFFFFF), row, 64) | (int64_t)__shfl((int)(to >> 32), row, 64) << 32;
      const vec8 v = *reinterpret_cast<const vec8 *>(mine + row * HD + (d ^ swizzle_k<HD>(row)) * 8);
      if (r_first + row < rows) *reinterpret_cast<vec8 *>((OT *)a.out + row_to + d * 8) = v;
    }
  } else if (r_first + c < rows) {
    const int64_t at = (int64_t)(it.part0 + r_first + c) * nkv + kvh;
    float *op = a.part_O + at * HD + half * 4;
#pragma unroll
    for (int t = 0; t < HD / 32; ++t)
#pragma unroll
      for (int q = 0; q < 4; ++q) *reinterpret_cast<f32x4 *>(op + t * 32 + q * 8) = f32x4{o[t][q * 4], o[t][q * 4 + 1], o[t][q * 4 + 2], o[t][q * 4 + 3]};
    if (half == 0) a.part_ml[at] = make_float2(m_run, l_tot);
  }
}

// Rows whose keys were split: out = sum_j w_j O_j / sum_j w_j l_j with w_j = 2^(unit (m_j - m)), HD / 4 lanes per row.  A row's parts are dealt to
// 1, 2, 4 or 8 such groups of lanes, which meet in LDS, and a group requests eight parts together.  Bound by launch and memory latency: 3 to
// 7 us.  In a launch of its own because the other way, the workgroup that writes a block's last part joins it, needs fences that write back
// and drop the L2 caches (100 single tokens 313 us and 600), or accesses that pass them (one long sequence 117 and 136).
template <typename OT, int HD>
__global__ __launch_bounds__(2 * HD) void paged_join_kernel(const PagedAttn a) {
  constexpr int L = HD / 4, N = 8, U = 8;                     // lanes of a row, groups of lanes, parts of a group under way together
  struct alignas(4 * sizeof(OT)) Out { OT v[4]; };
  __shared__ __align__(16) float lO[N][HD];
  __shared__ float2 lml[N];
  const int nkv = a.shape.n_kv_heads, G = a.shape.n_q_heads / nkv;
  if (a.plan->magic != kPlanMagic || !same_shape(a.plan->shape, a.shape)) return;
  const int n = a.plan->n_joins * nkv;
  for (int i = blockIdx.x; i < n; i += gridDim.x) {
    const int kvh = i % nkv;
    const PlanJoin jn = a.joins[i / nkv];
    const int group = threadIdx.x / L, d = (threadIdx.x % L) * 4;
    const int deal = jn.n_parts > 4 * U ? 8 : jn.n_parts > 2 * U ? 4 : jn.n_parts > U ? 2 : 1, own = group % deal, rows = jn.n_tok * G, at_once = N / deal;
    for (int r0 = blockIdx.y * at_once; r0 < rows; r0 += gridDim.y * at_once) {
      const int r = r0 + group / deal < rows ? r0 + group / deal : rows - 1;
      float m = -INFINITY, sum = 0.f;
      f32x4 v = {0.f, 0.f, 0.f, 0.f};
      for (int j0 = own; j0 < jn.n_parts; j0 += U * deal) {
        float2 x[U];
        f32x4 y[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int j = j0 + u * deal;
          const int64_t at = (int64_t)(jn.part0 + (j < jn.n_parts ? j : own) * jn.step + r) * nkv + kvh;
          x[u] = a.part_ml[at];
          y[u] = *reinterpret_cast<const f32x4 *>(a.part_O + at * HD + d);
          if (j >= jn.n_parts) x[u] = make_float2(-INFINITY, 0.f);
        }
        float mx = m;
#pragma unroll
        for (int u = 0; u < U; ++u) mx = fmaxf(mx, x[u].x);
        const float ref = mx == -INFINITY ? 0.f : mx;
        const float f0 = __builtin_amdgcn_exp2f((m - ref) * a.unit);
        m = mx;
        sum *= f0;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = weighed(f0, v[e]);
#pragma unroll
        for (int u = 0; u < U; ++u) {                           // (a part without keys has zeros, one in the place of none weighs nothing)
          const float f = __builtin_amdgcn_exp2f((x[u].x - ref) * a.unit);
          sum += f * x[u].y;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] += weighed(f, y[u][e]);
        }
      }
      *reinterpret_cast<f32x4 *>(&lO[group][d]) = v;
      if (d == 0) lml[group] = make_float2(m, sum);
      __syncthreads();
      if (group < at_once && r0 + group < rows) {               // this group's lanes: row r0 + group
        const int first = group * deal, row = r0 + group;
        float mx = -INFINITY;
        for (int j = 0; j < deal; ++j) mx = fmaxf(mx, lml[first + j].x);
        const float ref = mx == -INFINITY ? 0.f : mx;
        float total = 0.f;
        f32x4 w = {0.f, 0.f, 0.f, 0.f};
        for (int j = 0; j < deal; ++j) {
          const float2 x = lml[first + j];
          const float f = __builtin_amdgcn_exp2f((x.x - ref) * a.unit);
          const f32x4 y = *reinterpret_cast<const f32x4 *>(&lO[first + j][d]);
          total += f * x.y;
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] += weighed(f, y[e]);
        }
        const int t = row / G, h = kvh * G + row - t * G;
        Out o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o.v[e] = round_to<OT>(total == 0.f ? 0.f : w[e] / total);
        *reinterpret_cast<Out *>((OT *)a.out + (int64_t)(jn.row0 + t) * a.out_stride + (int64_t)h * HD + d) = o;
      }
      __syncthreads();
    }
  }
}

template <typename OT, int HD>
static int launch_join(const PagedAttn &a, hipStream_t s) {
  if (!plan_may_cut(a.shape)) return PRISM_OK;               // single tokens of 20 sequences over up to 250 keys 5.8 us, with the launch 7.3
  const int64_t joins = plan_joins(a.shape) * a.shape.n_kv_heads;     // there may be far fewer
  // few joins: they have few rows and many parts, and the rows go to workgroups of their own
  paged_join_kernel<OT, HD><<<dim3(joins < 8192 ? joins : 8192, joins < 512 ? 4 : 1), 2 * HD, 0, s>>>(a);
  PRISM_HIP(hipGetLastError());
  return PRISM_OK;
}

template <typename OT, int HD>
static int launch_16(const PagedAttn &a, hipStream_t s) {
  const int grid = (int)(plan_items(a.shape) * a.shape.n_kv_heads);
  if (a.softcap > 0.f || a.slopes) attention_paged_16_kernel<OT, HD, true><<<grid, 256, 0, s>>>(a);
  else attention_paged_16_kernel<OT, HD, false><<<grid, 256, 0, s>>>(a);
  PRISM_HIP(hipGetLastError());
  return launch_join<OT, HD>(a, s);
}

static size_t part_ml_at(const prism_page_shape &s, int hd) {
  return (size_t)plan_part_rows(s) * s.n_kv_heads * hd * sizeof(float);
}

}  // namespace prism

using namespace prism;

extern "C" int64_t prism_attention_paged_workspace(const prism_page_shape *shape, int32_t head_dim) {
  if (check_page_shape(shape, "attention_paged_workspace") != PRISM_OK) return -1;
  if (head_dim <= 0 || head_dim > 128) {
    set_error("attention_paged_workspace: head_dim %d", head_dim);
    return -1;
  }
  return (int64_t)(part_ml_at(*shape, head_dim) + (size_t)plan_part_rows(*shape) * shape->n_kv_heads * sizeof(float2)) + 16;
}

extern "C" int prism_op_attention_paged(const prism_page_shape *shape, const prism_kv_cache *cache, const void *plan, const int32_t *table,
                                        const void *Q, int64_t q_stride, float scale, float softcap, const float *slopes, void *out,
                                        int64_t out_stride, void *workspace, int64_t workspace_bytes, void *stream) {
  PRISM_TRY(check_page_shape(shape, "attention_paged"));
  PRISM_TRY(check_kv_cache(cache, "attention_paged"));
  PRISM_REQUIRE(shape->n_kv_heads == cache->n_kv_heads && shape->page_size == cache->page_size && shape->n_pages == cache->n_pages, PRISM_EINVAL,
                "attention_paged: the plan's pages are not the cache's");
  // (the factors that the kernels make of them, with log2(e) in them, have to be numbers too)
  PRISM_REQUIRE(scale >= 0.f && softcap >= 0.f && scale < 1e37f && softcap < 1e37f &&
                (softcap == 0.f || (scale > 0.f ? scale : 1.0f) / softcap < 1e37f), PRISM_EINVAL, "attention_paged: scale %g, softcap %g", scale, softcap);
  if (shape->n_tokens == 0 || shape->n_seqs == 0) return PRISM_OK;
  PRISM_REQUIRE(plan && table && Q && out && workspace, PRISM_EINVAL, "attention_paged: bad arguments");
  const int hd = cache->head_dim;
  PRISM_REQUIRE(workspace_bytes >= prism_attention_paged_workspace(shape, hd), PRISM_EINVAL, "attention_paged: workspace of %lld bytes, %lld needed",
                (long long)workspace_bytes, (long long)prism_attention_paged_workspace(shape, hd));
  const int64_t row = (int64_t)shape->n_q_heads * hd, vec = 16 / (int64_t)dtype_size(cache->dtype);
  PRISM_REQUIRE(q_stride >= row && out_stride >= row && q_stride % vec == 0 && out_stride % vec == 0 &&
                ((uintptr_t)plan | (uintptr_t)Q | (uintptr_t)out | (uintptr_t)workspace) % 16 == 0, PRISM_EINVAL,
                "attention_paged: rows shorter than their heads, or not 16-byte aligned");
  // (a launch has fewer than 2^32 threads along its first axis)
  PRISM_REQUIRE(plan_items(*shape) * shape->n_kv_heads < (int64_t)1 << 24, PRISM_EUNSUPPORTED, "attention_paged: too many work items (%lld over %d KV heads)",
                (long long)plan_items(*shape), shape->n_kv_heads);
  PagedAttn a;
  a.shape = *shape;
  a.plan = (const PlanHeader *)plan;
  a.items = (const PlanItem *)((const char *)plan + plan_items_at(*shape));
  a.joins = (const PlanJoin *)((const char *)plan + plan_joins_at(*shape));
  a.table = table; a.Q = Q; a.K = cache->K; a.V = cache->V; a.out = out; a.slopes = slopes;
  a.part_O = (float *)workspace;
  a.part_ml = (float2 *)((char *)workspace + part_ml_at(*shape, hd));
  a.q_stride = q_stride; a.out_stride = out_stride; a.page_stride = cache->page_stride;
  a.scale = scale > 0.f ? scale : 1.0f / sqrtf((float)hd);
  a.softcap = softcap;
  const float log2e = 1.4426950408889634f;                    // the 16-bit kernels keep plain scores unscaled, all others are in units of log 2
  a.unit = cache->dtype == PRISM_DTYPE_FP32 || softcap > 0.f || slopes ? 1.0f : a.scale * log2e;
  a.page_shift = __builtin_ctz(cache->page_size);
  hipStream_t s = (hipStream_t)stream;
  if (cache->dtype == PRISM_DTYPE_FP32) {
    PRISM_TRY(launch_attention_paged_fp32(a, hd, s));
    return hd == 32 ? launch_join<float, 32>(a, s) : hd == 64 ? launch_join<float, 64>(a, s) : launch_join<float, 128>(a, s);
  }
  if (cache->dtype == PRISM_DTYPE_BF16) return hd == 64 ? launch_16<bf16, 64>(a, s) : launch_16<bf16, 128>(a, s);
  return hd == 64 ? launch_16<f16, 64>(a, s) : launch_16<f16, 128>(a, s);
}
