// The fp32 form of the attention over a paged cache, on v_mfma_f32_16x16x4_f32.  Work items, rows and masks as in attn_paged.hip;
// arithmetic and operand layout as in attn_fp32.hip: both products transposed, so that a lane owns one row (lane % 16) and the
// accumulators of S^T are the next contraction's operand; operands straight from memory, one group of 16 keys ahead.
//
// A wave takes 16 rows.  Items of more than 32 rows: a wave per 16 rows, each over all keys, in two workgroups (the matrix work of an
// item is 16 times that of the 16-bit types, and a step of short chunks has few items).  Items of up to 32 rows: one workgroup whose
// waves take the same rows and every fourth group of keys, and meet in LDS.
#include <type_traits>

#include "paged.h"

namespace prism {

template <int NB, bool MOD>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(NB <= 4 ? 3 : 2)))
void attention_paged_fp32_kernel(const PagedAttn a) {
  constexpr int HD = 16 * NB;
  __shared__ __align__(16) float lO[4][16][HD];
  __shared__ float2 lml[4][16];
  const int nkv = a.shape.n_kv_heads, G = a.shape.n_q_heads / nkv;
  const int kvh = blockIdx.x % nkv, item = blockIdx.x / nkv;
  const PlanItem it = load_const(a.items + item);
  const PlanHeader plan = load_const(a.plan);
  if (plan.magic != kPlanMagic || !same_shape(plan.shape, a.shape) || item >= plan.n_items) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
  const int rows = it.n_tok * G, row_begin = blockIdx.y * 64, window = a.shape.window, cap_keys = a.shape.max_pages << a.page_shift;
  const int last = it.pos0 + it.n_tok - 1, limit = last + 1 < cap_keys ? last + 1 : cap_keys;
  const int32_t *const table = a.table + (int64_t)it.seq * a.shape.max_pages;
  const float *const Kh = (const float *)a.K + ((int64_t)kvh * HD << a.page_shift), *const Vh = (const float *)a.V + ((int64_t)kvh * HD << a.page_shift);
  auto page_of = [&](int k0) __attribute__((always_inline)) {
    if (k0 >= limit) return -1;
    const int p = load_const(table + (k0 >> a.page_shift));
    return (unsigned)p < (unsigned)a.shape.n_pages ? p : -1;
  };
  struct Tile { f32x4 k[NB]; float v[4][NB]; int page; };
  auto fetch = [&](int k0, Tile &t) __attribute__((always_inline)) {
    t.page = page_of(k0);
    const int64_t at = (int64_t)(t.page < 0 ? 0 : t.page) * a.page_stride + (int64_t)(k0 & ((1 << a.page_shift) - 1)) * HD;
    const float *kp = Kh + at + c * HD + 4 * g;
#pragma unroll
    for (int b = 0; b < NB; ++b) t.k[b] = *reinterpret_cast<const f32x4 *>(kp + 16 * b);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const float *vp = Vh + at + (4 * g + s) * HD + NB * c;
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
  const bool shared = rows <= 32;
  if (row_begin >= rows) return;
  const int n_groups = (limit + 15) >> 4, g_end = it.tile1 * 4 < n_groups ? it.tile1 * 4 : n_groups;
  const int g_first = it.tile0 * 4 + (shared ? wave : 0), g_step = shared ? 4 : 1;
  const int blocks = ((rows < row_begin + 64 ? rows : row_begin + 64) + 15) / 16;
  for (int rb = shared ? 0 : row_begin / 16 + wave; rb < blocks; rb += shared ? 1 : 4) {
    const int r = rb * 16 + c < rows ? rb * 16 + c : rows - 1, tok = r / G, head = kvh * G + r - tok * G, pos = it.pos0 + tok;
    const int r_last = rb * 16 + 15 < rows ? rb * 16 + 15 : rows - 1;
    const int b_first = it.pos0 + rb * 16 / G, b_last = it.pos0 + r_last / G;    // positions of the block's first and last row
    const float slope = MOD && a.slopes ? a.slopes[head] : 0.f;
    f32x4 qf[NB], o[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      qf[b] = *reinterpret_cast<const f32x4 *>((const float *)a.Q + (int64_t)(it.row0 + tok) * a.q_stride + (int64_t)head * HD + 16 * b + 4 * g);
      o[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    float m_run = -INFINITY, l_run = 0.f;
    auto work = [&](int grp, const Tile &t) __attribute__((always_inline)) {
      const int k0 = grp * 16;
      if (k0 > b_last || (window > 0 && k0 + 15 <= b_first - window)) return;   // no row of the block sees a key of it
      f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int b = 0; b < NB; b += 2)
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(t.k[b][s], qf[b][s], s0, 0, 0, 0);
          s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(t.k[b + 1][s], qf[b + 1][s], s1, 0, 0, 0);
        }
      const bool masked = t.page < 0 || k0 + 15 > b_first || k0 + 15 >= limit || (window > 0 && k0 <= b_last - window);
      const int lo = window > 0 ? pos - window + 1 : 0, hi = pos < limit - 1 ? pos : limit - 1;
      float p[4], mx = -INFINITY;
      bool see[4];
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const int key = k0 + 4 * g + s;
        p[s] = (s0[s] + s1[s]) * a.scale;
        if (MOD) {
          if (a.softcap > 0.f) p[s] = a.softcap * tanhf(p[s] / a.softcap);
          p[s] -= slope * (float)(pos - key);
        }
        see[s] = !masked || (t.page >= 0 && key >= lo && key <= hi);
        if (!see[s]) p[s] = -INFINITY;
        mx = fmaxf(mx, p[s]);
      }
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const float m_new = fmaxf(m_run, mx), ref = m_new == -INFINITY ? 0.f : m_new;   // no key yet: weights exp(-inf) = 0
      const float alpha = expf(m_run - ref);
      m_run = m_new;
      float sum = 0.f;
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        p[s] = expf(p[s] - ref);
        sum += p[s];
      }
      l_run = l_run * alpha + sum;
#pragma unroll
      for (int b = 0; b < NB; ++b) o[b] *= alpha;
      float v[4][NB];
      bool odd = false;
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          v[s][b] = t.v[s][b];
          // a weight of zero times a value that is not finite would reach the sum: values of keys that no row sees become zero
          if (masked && (t.page < 0 || k0 + 4 * g + s >= limit)) v[s][b] = 0.f;
          odd = odd || !(fabsf(v[s][b]) < INFINITY);
        }
      if (masked && __builtin_amdgcn_ballot_w64(odd) != 0) {
        // those of keys that some rows see and others do not go to the rows that see them by indicators
#pragma unroll 1
        for (int kind = 0; kind < 3; ++kind) {
          const float add = kind == 0 ? INFINITY : kind == 1 ? -INFINITY : NAN;
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            f32x4 n = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < 4; ++s) {
              const float x = v[s][b];
              const bool is = kind == 2 ? x != x : x == add;
              n = __builtin_amdgcn_mfma_f32_16x16x4f32(is ? 1.0f : 0.0f, see[s] ? 1.0f : 0.0f, n, 0, 0, 0);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) o[b][e] += n[e] > 0.f ? add : 0.f;
          }
        }
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
          for (int b = 0; b < NB; ++b) v[s][b] = fabsf(v[s][b]) < INFINITY ? v[s][b] : 0.f;
      }
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int b = 0; b < NB; ++b) o[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[s][b], p[s], o[b], 0, 0, 0);
    };
    // two groups' registers in turn; the scheduling barriers keep a group's loads in front of the work on the group before
    Tile cur, next;
    int grp = g_first;
    if (grp < g_end) fetch(grp * 16, cur);
    for (; grp < g_end; grp += 2 * g_step) {
      const bool two = grp + g_step < g_end;
      if (two) fetch((grp + g_step) * 16, next);
      __builtin_amdgcn_sched_barrier(0);
      work(grp, cur);
      if (grp + 2 * g_step < g_end) fetch((grp + 2 * g_step) * 16, cur);
      __builtin_amdgcn_sched_barrier(0);
      if (two) work(grp + g_step, next);
    }
    l_run += __shfl_xor(l_run, 16);
    l_run += __shfl_xor(l_run, 32);
    if (shared) {
      // o[b][e] is dimension NB (4 g + e) + b of row c
      __syncthreads();
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        f32x4 y;
#pragma unroll
        for (int q = 0; q < 4; ++q) y[q] = o[(4 * j + q) % NB][(4 * j + q) / NB];
        *reinterpret_cast<f32x4 *>(&lO[wave][c][NB * 4 * g + 4 * j]) = y;
      }
      if (g == 0) lml[wave][c] = make_float2(m_run, l_run);
      __syncthreads();
      for (int e = threadIdx.x; e < 16 * HD / 4; e += 256) {
        const int rr = e / (HD / 4), d = e % (HD / 4) * 4, row = rb * 16 + rr;
        if (row >= rows) continue;
        float m = -INFINITY, sum = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) m = fmaxf(m, lml[w][rr].x);
        const float ref = m == -INFINITY ? 0.f : m;
        f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float2 x = lml[w][rr];
          if (x.x == -INFINITY) continue;                    // a wave without keys has nothing
          const float f = expf(x.x - ref);
          const f32x4 z = *reinterpret_cast<const f32x4 *>(&lO[w][rr][d]);
          sum += f * x.y;
#pragma unroll
          for (int q = 0; q < 4; ++q) y[q] += f * z[q];
        }
        const int t = row / G, h = kvh * G + row - t * G;
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
      continue;
    }
    if (rb * 16 + c >= rows) continue;
    const int64_t at = (int64_t)(it.part0 + rb * 16 + c) * nkv + kvh;
    float *op = it.part0 < 0 ? (float *)a.out + (int64_t)(it.row0 + tok) * a.out_stride + (int64_t)head * HD : a.part_O + at * HD;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      f32x4 y;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        y[q] = o[(4 * j + q) % NB][(4 * j + q) / NB];
        if (it.part0 < 0) y[q] = l_run == 0.f ? 0.f : y[q] / l_run;
      }
      *reinterpret_cast<f32x4 *>(op + NB * 4 * g + 4 * j) = y;
    }
    if (it.part0 >= 0 && g == 0) a.part_ml[at] = make_float2(m_run, l_run);
  }
}

int launch_attention_paged_fp32(const PagedAttn &a, int hd, hipStream_t s) {
  const int grid = (int)(plan_items(a.shape) * a.shape.n_kv_heads);
  const bool mod = a.softcap > 0.f || a.slopes;
  auto run = [&](auto nb) {
    constexpr int NB = decltype(nb)::value;
    if (mod) attention_paged_fp32_kernel<NB, true><<<dim3(grid, kPlanRows / 64), 256, 0, s>>>(a);
    else attention_paged_fp32_kernel<NB, false><<<dim3(grid, kPlanRows / 64), 256, 0, s>>>(a);
  };
  if (hd == 32) run(std::integral_constant<int, 2>{});
  else if (hd == 64) run(std::integral_constant<int, 4>{});
  else run(std::integral_constant<int, 8>{});
  PRISM_HIP(hipGetLastError());
  return PRISM_OK;
}

}  // namespace prism
