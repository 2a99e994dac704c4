// The fp32 form of the attention over a paged cache, on v_mfma_f32_16x16x4_f32.  Work items, rows and masks as in attn_paged.hip;
// arithmetic and operand layout as in attn_fp32.hip: both products transposed, so that a lane owns one row (lane % 16) and the
// accumulators of S^T are the next contraction's operand.
//
// A workgroup of four waves takes 32 rows of an item.  Every wave has all of them, as two blocks of 16 that share a group of 16 keys in
// registers, and every fourth group; the four meet in LDS.  What bounds it: the products keep the matrix pipes busy
// for 17 us of the 54 that 40 ragged chunks over up to 900 keys take, 4 heads of 64; the rest is the softmax's instructions (some 120 to 32
// products of 16 rows and keys) and compute units with a long chunk more than others.  With 16 rows per wave instead of 32 it was 76
// to 70; head size 128, where two blocks spill, 164 to 285.  Weights are powers of 2 of scores in units of log 2: the factor's rounding
// is 2^-25 of a score, as much as the score's own, and expf's range steps and exact splitting cost 9 us.
#include <type_traits>

#include "paged.h"

namespace prism {

// (head size 128: two blocks of rows would not fit the registers)
constexpr int fp32_rows(int nb) { return nb <= 4 ? 32 : 16; }

template <int NB, bool MOD>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(NB <= 4 ? 3 : 2)))
void attention_paged_fp32_kernel(const PagedAttn a) {
  constexpr int HD = 16 * NB;
  constexpr int W = 4, kRows = fp32_rows(NB);                 // waves; rows of a workgroup
  constexpr int CH = HD / 4, RI = 64 / CH, NI = 16 / RI;      // 16-byte chunks of a row; rows of a load instruction, instructions for 16 rows
  __shared__ __align__(16) float lO[W][16][HD];               // a wave's 16 keys, at the end its results
  __shared__ float2 lml[W][16];                               // maxima and sums; a sum's sign says `found`
  const int nkv = a.shape.n_kv_heads, G = a.shape.n_q_heads / nkv;
  const int kvh = blockIdx.x % nkv, item = blockIdx.x / nkv;
  PlanItem it;
  if (!load_item(a, item, it)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
  const int rows = it.n_tok * G, row_begin = blockIdx.y * kRows, window = a.shape.window, cap_keys = a.shape.max_pages << a.page_shift;
  const int last = it.pos0 + it.n_tok - 1, limit = last + 1 < cap_keys ? last + 1 : cap_keys;
  const int32_t *const table = a.table + (int64_t)it.seq * a.shape.max_pages;
  const float *const Kh = (const float *)a.K + ((int64_t)kvh * HD << a.page_shift), *const Vh = (const float *)a.V + ((int64_t)kvh * HD << a.page_shift);
  // table entry of the 16 keys from k0 on (behind the last key, that key's), and the page that it gives, none: -1
  auto entry_of = [&](int k0) __attribute__((always_inline)) { return load_const(table + ((k0 < limit ? k0 : limit - 1) >> a.page_shift)); };
  auto page_from = [&](int entry, int k0) __attribute__((always_inline)) { return k0 < limit && (unsigned)entry < (unsigned)a.shape.n_pages ? entry : -1; };
  // K goes through LDS of the wave's own: a lane's operand is four dimensions of key lane % 16, and fetched as that, every lane of a load
  // would be in a line of its own.  Chunk c of row r stands at slot c ^ swizzle(r), so that the 16 rows of a read spread over all banks.
  auto swizzle = [](int r) { return HD == 32 ? (r >> 1) & 7 : r & 15; };
  float *const lK = &lO[wave][0][0];
  const uint32_t oK = (lane / CH * HD + ((lane % CH) ^ swizzle(lane / CH)) * 4) * 4;    // bytes; instruction j: its bits flipped
  auto load_k = [&](const float *src) __attribute__((always_inline)) {
    const char *const s = reinterpret_cast<const char *>(src);
    constexpr uint32_t kFlip = HD == 32 ? 64 : RI * 16;
    auto one = [&](auto j) __attribute__((always_inline)) {
      constexpr int J = decltype(j)::value, kBase = J / 4 * 4096, kOffset = J % 4 * 1024;
      static_assert(kOffset < 4096, "the immediate offset has 12 bits and a sign, and a larger one wraps without a word");
      if constexpr (J < NI)
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(s + kBase + (oK ^ (J * kFlip))),
                                         (__attribute__((address_space(3))) void *)(lK + kBase / 4), 16, kOffset, 0);
    };
    one(std::integral_constant<int, 0>{}); one(std::integral_constant<int, 1>{}); one(std::integral_constant<int, 2>{}); one(std::integral_constant<int, 3>{});
    one(std::integral_constant<int, 4>{}); one(std::integral_constant<int, 5>{}); one(std::integral_constant<int, 6>{}); one(std::integral_constant<int, 7>{});
  };
  struct Values { float v[4][NB]; };                          // s: key 4 g + s, dimensions NB c ..
  auto load_v = [&](const float *src, Values &t) __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const float *vp = src + (4 * g + s) * HD + NB * c;
      if constexpr (NB == 2) {
        const float2 v = *reinterpret_cast<const float2 *>(vp);
        t.v[s][0] = v.x; t.v[s][1] = v.y;
      } else {
#pragma unroll
        for (int j = 0; j < NB; j += 4) {
          const f32x4 v = *reinterpret_cast<const f32x4 *>(vp + j);
          t.v[s][j] = v[0]; t.v[s][j + 1] = v[1]; t.v[s][j + 2] = v[2]; t.v[s][j + 3] = v[3];
        }
      }
    }
  };
  auto rows_at = [&](int page, int k0) __attribute__((always_inline)) {
    return (int64_t)(page < 0 ? 0 : page) * a.page_stride + (int64_t)(k0 & ((1 << a.page_shift) - 1)) * HD;
  };
  if (row_begin >= rows) return;
  const int n_groups = (limit + 15) >> 4, g_end = it.tile1 * 4 < n_groups ? it.tile1 * 4 : n_groups;
  const int g_first = it.tile0 * 4 + wave;
  constexpr int RB = kRows / 16;
  const bool both = RB > 1 && row_begin + 16 < rows;
  int pos[RB], b_first[RB], b_last[RB];                       // b_first, b_last: positions of a block's first and last row
  float slope[RB], m_run[RB], l_run[RB];
  bool found = false;                                         // values that are not finite were kept from the products
  f32x4 qf[RB][NB], o[RB][NB];
#pragma unroll
  for (int i = 0; i < RB; ++i) {
    const int r0 = row_begin + i * 16 < rows ? row_begin + i * 16 : rows - 1, r_last = r0 + 15 < rows ? r0 + 15 : rows - 1;
    const int r = r0 + c < rows ? r0 + c : rows - 1, tok = r / G, head = kvh * G + r - tok * G;
    pos[i] = it.pos0 + tok;
    b_first[i] = it.pos0 + r0 / G;
    b_last[i] = it.pos0 + r_last / G;
    slope[i] = MOD && a.slopes ? a.slopes[head] : 0.f;
    m_run[i] = -INFINITY;
    l_run[i] = 0.f;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      qf[i][b] = *reinterpret_cast<const f32x4 *>((const float *)a.Q + (int64_t)(it.row0 + tok) * a.q_stride + (int64_t)head * HD + 16 * b + 4 * g);
      o[i][b] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
  constexpr float kLog2e = 1.4426950408889634f;
  const float scale2 = a.scale * kLog2e;
  wait_loads<0>();                                            // the queries are here: nothing in the loop waits for them
  auto work = [&](auto block, int grp, int page, const f32x4 (&k)[NB], const Values &t) __attribute__((always_inline)) {
    constexpr int I = decltype(block)::value;
    const int k0 = grp * 16;
    if (k0 > b_last[I] || (window > 0 && k0 + 15 <= b_first[I] - window)) return;   // no row of the block sees a key of it
    f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int b = 0; b < NB; b += 2)
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[b][s], qf[I][b][s], s0, 0, 0, 0);
        s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[b + 1][s], qf[I][b + 1][s], s1, 0, 0, 0);
      }
    // scores in units of log 2
    const bool masked = page < 0 || k0 + 15 > b_first[I] || k0 + 15 >= limit || (window > 0 && k0 <= b_last[I] - window);
    float p[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) p[s] = s0[s] + s1[s];
    if (MOD) {
      if (a.softcap > 0.f) {
#pragma unroll
        for (int s = 0; s < 4; ++s) p[s] = a.softcap * tanhf(p[s] * a.scale / a.softcap);
      } else {
#pragma unroll
        for (int s = 0; s < 4; ++s) p[s] *= a.scale;
      }
#pragma unroll
      for (int s = 0; s < 4; ++s) p[s] = (p[s] - slope[I] * (float)(pos[I] - (k0 + 4 * g + s))) * kLog2e;
    } else {
#pragma unroll
      for (int s = 0; s < 4; ++s) p[s] *= scale2;
    }
    bool see[4] = {true, true, true, true}, odd = false;
    float v[4][NB];
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int b = 0; b < NB; ++b) v[s][b] = t.v[s][b];
    if (masked) {
      const int lo = window > 0 ? pos[I] - window + 1 : 0, hi = pos[I] < limit - 1 ? pos[I] : limit - 1;
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const int key = k0 + 4 * g + s;
        see[s] = page >= 0 && key >= lo && key <= hi;
        if (!see[s]) p[s] = -INFINITY;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          // a weight of zero times a value that is not finite would reach the sum: values of keys that no row sees become zero
          if (page < 0 || key >= limit) v[s][b] = 0.f;
          odd = odd || !(fabsf(v[s][b]) < INFINITY);
        }
      }
    }
    const float mx = max_xor32(max_xor16(fmaxf(fmaxf(p[0], p[1]), fmaxf(p[2], p[3]))));
    // exponents are taken from an old maximum until a new one is 2^3 times its weight: as it moves the accumulators have to be multiplied
    if (__builtin_amdgcn_ballot_w64(mx > m_run[I] + 3.0f) != 0) {
      const float m_new = mx > m_run[I] + 3.0f ? mx : m_run[I];
      const float alpha = __builtin_amdgcn_exp2f(m_run[I] - (m_new == -INFINITY ? 0.f : m_new));
      m_run[I] = m_new;
      l_run[I] *= alpha;
#pragma unroll
      for (int b = 0; b < NB; ++b) o[I][b] *= alpha;
    }
    const float ref = m_run[I] == -INFINITY ? 0.f : m_run[I];  // no key yet: weights exp(-inf) = 0
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      p[s] = __builtin_amdgcn_exp2f(p[s] - ref);
      l_run[I] += p[s];
    }
    if (masked && __builtin_amdgcn_ballot_w64(odd) != 0) {
      found = true;                                           // rows that see those of keys that others do not see get them at the end
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int b = 0; b < NB; ++b) v[s][b] = fabsf(v[s][b]) < INFINITY ? v[s][b] : 0.f;
    }
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int b = 0; b < NB; ++b) o[I][b] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[s][b], p[s], o[I][b], 0, 0, 0);
  };
  // A group's K is in LDS and its V in registers when its turn comes.  Its K goes to registers at once, and the next group's K and V are
  // requested ahead of its work, K into the LDS that is free now; a group's page is looked up a group ahead of that.
  Values cur, next;
  int grp = g_first, page = -1, ahead = -1;   // ahead: the next group's table entry
  if (grp < g_end) {
    page = page_from(entry_of(grp * 16), grp * 16);
    load_k(Kh + rows_at(page, grp * 16));
    load_v(Vh + rows_at(page, grp * 16), cur);
    ahead = entry_of((grp + W) * 16);
  }
  auto step = [&](const Values &own, Values &other) __attribute__((always_inline)) {
    f32x4 k[NB];
    wait_loads<0>();
#pragma unroll
    for (int b = 0; b < NB; ++b) k[b] = *reinterpret_cast<const f32x4 *>(lK + c * HD + ((4 * b + g) ^ swizzle(c)) * 4);
    const int next_grp = grp + W, page_own = page;
    page = page_from(ahead, next_grp * 16);
    if (next_grp < g_end) load_v(Vh + rows_at(page, next_grp * 16), other);
    wait_lds();
    if (next_grp < g_end) load_k(Kh + rows_at(page, next_grp * 16));
    ahead = entry_of((next_grp + W) * 16);
    __builtin_amdgcn_sched_barrier(0);
    work(std::integral_constant<int, 0>{}, grp, page_own, k, own);
    if (both) work(std::integral_constant<int, RB - 1>{}, grp, page_own, k, own);
    grp = next_grp;
  };
  while (grp < g_end) {
    step(cur, next);
    if (grp < g_end) step(next, cur);
  }
#pragma unroll
  for (int i = 0; i < RB; ++i) {
    if (row_begin + i * 16 >= rows) break;
    const float l_tot = sum_xor32(sum_xor16(l_run[i]));
    // o[b][e] is dimension NB (4 g + e) + b of row c; this wave's keys have been read
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      f32x4 y;
#pragma unroll
      for (int q = 0; q < 4; ++q) y[q] = o[i][(4 * j + q) % NB][(4 * j + q) / NB];
      *reinterpret_cast<f32x4 *>(&lO[wave][c][((NB * g + j) ^ swizzle(c)) * 4]) = y;
    }
    if (g == 0) lml[wave][c] = make_float2(m_run[i], found ? -l_tot : l_tot);
    __syncthreads();
    for (int e = threadIdx.x; e < 16 * HD / 4; e += 64 * W) {
      const int r16 = e / (HD / 4), d = e % (HD / 4) * 4, row = row_begin + i * 16 + r16;
      if (row >= rows) continue;
      float m = -INFINITY, sum = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) m = fmaxf(m, lml[w][r16].x);
      const float ref = m == -INFINITY ? 0.f : m;
      unsigned signs = 0;
      f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float2 x = lml[w][r16];
        const float f = __builtin_amdgcn_exp2f(x.x - ref);
        const f32x4 z = *reinterpret_cast<const f32x4 *>(&lO[w][r16][(d / 4 ^ swizzle(r16)) * 4]);
        sum += f * fabsf(x.y);
        signs |= __float_as_uint(x.y);
#pragma unroll
        for (int q = 0; q < 4; ++q) y[q] += f * z[q];
      }
      const int t = row / G, h = kvh * G + row - t * G;
      float most = 0.f;
#pragma unroll
      for (int q = 0; q < 4; ++q) most = worst_of(y[q], most);
      if (__builtin_amdgcn_ballot_w64(((signs >> 31 != 0) | (most != most)) & (sum == sum)) != 0) {
        float w[4] = {y[0], y[1], y[2], y[3]};
        settle<float, HD>(a, table, Vh + d, it.tile0 * 64, it.tile1 * 64 < limit ? it.tile1 * 64 : limit, window > 0 ? it.pos0 + t - window + 1 : 0,
                          it.pos0 + t, signs >> 31, w);
        y = f32x4{w[0], w[1], w[2], w[3]};
      }
      if (it.part0 < 0) {
#pragma unroll
        for (int q = 0; q < 4; ++q) y[q] = sum == 0.f ? 0.f : y[q] / sum;
        *reinterpret_cast<f32x4 *>((float *)a.out + (int64_t)(it.row0 + t) * a.out_stride + (int64_t)h * HD + d) = y;
      } else {
        const int64_t at = (int64_t)(it.part0 + row) * nkv + kvh;
        *reinterpret_cast<f32x4 *>(a.part_O + at * HD + d) = y;
        if (d == 0) a.part_ml[at] = make_float2(m, sum);
      }
    }
    __syncthreads();                                          // the next block's results may come
  }
}

int launch_attention_paged_fp32(const PagedAttn &a, int hd, hipStream_t s) {
  const int grid = (int)(plan_items(a.shape) * a.shape.n_kv_heads);
  const bool mod = a.softcap > 0.f || a.slopes;
  auto run = [&](auto nb) {
    constexpr int NB = decltype(nb)::value;
    if (mod) attention_paged_fp32_kernel<NB, true><<<dim3(grid, kPlanRows / fp32_rows(NB)), 256, 0, s>>>(a);
    else attention_paged_fp32_kernel<NB, false><<<dim3(grid, kPlanRows / fp32_rows(NB)), 256, 0, s>>>(a);
  };
  if (hd == 32) run(std::integral_constant<int, 2>{});
  else if (hd == 64) run(std::integral_constant<int, 4>{});
  else run(std::integral_constant<int, 8>{});
  PRISM_HIP(hipGetLastError());
  return PRISM_OK;
}

}  // namespace prism
