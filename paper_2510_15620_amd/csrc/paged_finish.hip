// Finishing of the q/k/v projection for a paged cache: per-head RMSNorm (optional) and rotate-half RoPE on q and k, one rounding, q to
// its rows and k and v to their pages.
//
// A workgroup takes four tokens.  Their 4 hd / 2 rotations are evaluated in fp64 once, while the first values are on their way, and
// meet in LDS.  HD / 8 lanes hold a head of a token, four values of each rotation half per lane, so a lane owns whole pairs, a
// head's sum of squares is a butterfly over those lanes and every access is 16 or 8 bytes of a run of 2 HD or 4 HD bytes.
// HBM-bound: each value is read and written once.  37 000 tokens of 32 + 8 heads of 128, fp32 to half: 1.37 GB in 260 us, 5.2 TB/s; 7 tokens
// 3.4 us.
#include <type_traits>

#include "paged.h"

namespace prism {

struct FinishArgs {
  const void *QKV, *q_gain, *k_gain;
  const int32_t *pos, *slot;
  void *Q, *K, *V;
  int64_t qkv_stride, q_stride, page_stride;
  int n_tok, nq, nkv, page_shift, heads_of_group, qk_norm;
  int64_t n_slots;
  float eps;
  double log2_base;
};

template <typename TI, typename TO, int HD>
__global__ __launch_bounds__(256) void qkv_finish_paged_kernel(const FinishArgs a) {
  constexpr int L = HD / 8, kStep = 256 / L / 4, kHeads = 4, HALF = HD / 2;    // lanes of a head; heads of a step; steps in flight
  struct alignas(4 * sizeof(TI)) In { TI v[4]; };
  struct alignas(4 * sizeof(TO)) Out { TO v[4]; };
  __shared__ float2 rot[4][HALF];
  const int t0 = blockIdx.x * 4, heads = a.nq + 2 * a.nkv;
  const int group = threadIdx.x / L, i = (threadIdx.x % L) * 4, tk = group & 3;
  const int t = t0 + tk < a.n_tok ? t0 + tk : a.n_tok - 1;
  const int h_begin = blockIdx.y * a.heads_of_group, h_end = h_begin + a.heads_of_group < heads ? h_begin + a.heads_of_group : heads;
  const TI *x = (const TI *)a.QKV + (int64_t)t * a.qkv_stride + i;
  In lo[kHeads], hi[kHeads];
  auto fetch = [&](int h0) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < kHeads; ++u) {
      const int h = h0 + kStep * u;
      if (h < h_end) {
        lo[u] = *reinterpret_cast<const In *>(x + h * HD);
        hi[u] = *reinterpret_cast<const In *>(x + h * HD + HALF);
      }
    }
  };
  const int h_first = h_begin + (group >> 2);
  fetch(h_first);
  const int slot = a.slot[t];
  if (h_begin < a.nq + a.nkv) {
    for (int e = threadIdx.x; e < 4 * HALF; e += 256) {
      const int rt = t0 + e / HALF;
      rot[e / HALF][e % HALF] = rotation(a.pos[rt < a.n_tok ? rt : a.n_tok - 1], e % HALF, HALF, a.log2_base);
    }
  }
  __syncthreads();
  const bool real = t0 + tk < a.n_tok, kept = real && (uint32_t)slot < (uint64_t)a.n_slots;
  const int64_t page = (int64_t)(slot >> a.page_shift) * a.page_stride;
  const int off = slot & ((1 << a.page_shift) - 1);
  TO *q_out = (TO *)a.Q + (int64_t)t * a.q_stride + i;
  float2 cs[4];
  Out gq[2], gk[2];
  if (h_begin < a.nq + a.nkv) {
#pragma unroll
    for (int e = 0; e < 4; ++e) cs[e] = rot[tk][i + e];
    if (a.qk_norm) {
      gq[0] = *reinterpret_cast<const Out *>((const TO *)a.q_gain + i);
      gq[1] = *reinterpret_cast<const Out *>((const TO *)a.q_gain + i + HALF);
      gk[0] = *reinterpret_cast<const Out *>((const TO *)a.k_gain + i);
      gk[1] = *reinterpret_cast<const Out *>((const TO *)a.k_gain + i + HALF);
    }
  }
  for (int h0 = h_first; h0 < h_end; h0 += kStep * kHeads) {
    if (h0 != h_first) fetch(h0);
#pragma unroll
    for (int u = 0; u < kHeads; ++u) {
      const int h = h0 + kStep * u;
      if (h >= h_end) break;
      float p[4], q[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) { p[e] = to_f32(lo[u].v[e]); q[e] = to_f32(hi[u].v[e]); }
      Out o0, o1;
      if (h < a.nq + a.nkv) {
        if (a.qk_norm) {
          float ss = 0.f;
#pragma unroll
          for (int e = 0; e < 4; ++e) ss += p[e] * p[e] + q[e] * q[e];
#pragma unroll
          for (int m = L / 2; m > 0; m >>= 1) ss += __shfl_xor(ss, m, 64);
          const float r = 1.0f / sqrtf(ss / (float)HD + a.eps);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            p[e] = p[e] * r * to_f32(h < a.nq ? gq[0].v[e] : gk[0].v[e]);
            q[e] = q[e] * r * to_f32(h < a.nq ? gq[1].v[e] : gk[1].v[e]);
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          o0.v[e] = round_to<TO>(__builtin_fmaf(p[e], cs[e].x, -(q[e] * cs[e].y)));
          o1.v[e] = round_to<TO>(__builtin_fmaf(q[e], cs[e].x, p[e] * cs[e].y));
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) { o0.v[e] = round_to<TO>(p[e]); o1.v[e] = round_to<TO>(q[e]); }
      }
      TO *o;
      if (h < a.nq) {
        if (!real) continue;
        o = q_out + (int64_t)h * HD;
      } else {
        if (!kept) continue;
        const int kh = h < a.nq + a.nkv ? h - a.nq : h - a.nq - a.nkv;
        o = (TO *)(h < a.nq + a.nkv ? a.K : a.V) + page + (((int64_t)kh << a.page_shift) + off) * HD + i;
      }
      *reinterpret_cast<Out *>(o) = o0;
      *reinterpret_cast<Out *>(o + HALF) = o1;
    }
  }
}

template <typename TI, typename TO>
static void launch_typed(const FinishArgs &a, int hd, dim3 grid, hipStream_t s) {
  if (hd == 32) qkv_finish_paged_kernel<TI, TO, 32><<<grid, 256, 0, s>>>(a);
  else if (hd == 64) qkv_finish_paged_kernel<TI, TO, 64><<<grid, 256, 0, s>>>(a);
  else qkv_finish_paged_kernel<TI, TO, 128><<<grid, 256, 0, s>>>(a);
}

int check_kv_cache(const prism_kv_cache *c, const char *who) {
  PRISM_REQUIRE(c && c->K && c->V, PRISM_EINVAL, "%s: no cache", who);
  PRISM_REQUIRE(c->dtype == PRISM_DTYPE_FP32 || is16(c->dtype), PRISM_EINVAL, "%s: unknown dtype %d", who, c->dtype);
  PRISM_REQUIRE(c->n_kv_heads > 0 && c->n_kv_heads <= 256 && c->n_pages > 0, PRISM_EINVAL, "%s: %d KV heads, %d pages", who, c->n_kv_heads, c->n_pages);
  PRISM_REQUIRE(c->head_dim == 64 || c->head_dim == 128 || (c->head_dim == 32 && c->dtype == PRISM_DTYPE_FP32), PRISM_EUNSUPPORTED,
                "%s: head_dim %d (64 and 128, in fp32 also 32)", who, c->head_dim);
  PRISM_REQUIRE(c->page_size >= 16 && c->page_size <= 256 && (c->page_size & (c->page_size - 1)) == 0, PRISM_EUNSUPPORTED,
                "%s: pages of %d tokens (16, 32, 64, 128 or 256)", who, c->page_size);
  PRISM_REQUIRE((int64_t)c->n_pages * c->page_size <= INT32_MAX, PRISM_EINVAL, "%s: %d pages of %d tokens", who, c->n_pages, c->page_size);
  const int64_t page = (int64_t)c->n_kv_heads * c->page_size * c->head_dim;
  PRISM_REQUIRE(c->page_stride >= page && c->page_stride <= INT64_MAX / 8 / c->n_pages && c->page_stride * (int64_t)dtype_size(c->dtype) % 16 == 0 &&
                ((uintptr_t)c->K | (uintptr_t)c->V) % 16 == 0, PRISM_EINVAL,
                "%s: pages have to be 16-byte aligned and %lld values apart at least", who, (long long)page);
  return PRISM_OK;
}

}  // namespace prism

using namespace prism;

extern "C" int prism_op_qkv_finish_paged(const prism_kv_cache *cache, int32_t qkv_dtype, const void *QKV, int64_t qkv_stride, int32_t T,
                                         const int32_t *pos, const int32_t *slot, int32_t nq, const void *q_gain, const void *k_gain,
                                         float eps, float rope_base, int32_t qk_norm, void *Q, int64_t q_stride, void *stream) {
  PRISM_TRY(check_kv_cache(cache, "qkv_finish_paged"));
  const int hd = cache->head_dim, nkv = cache->n_kv_heads;
  PRISM_REQUIRE(T >= 0 && T <= PRISM_MAX_STEP && nq > 0 && nq <= 65536 && nq % nkv == 0 && rope_base > 0, PRISM_EINVAL, "qkv_finish_paged: bad arguments");
  PRISM_REQUIRE(qkv_dtype == PRISM_DTYPE_FP32 || qkv_dtype == cache->dtype, PRISM_EINVAL,
                "qkv_finish_paged: the projection is fp32 or has the cache's type");
  if (T == 0) return PRISM_OK;
  PRISM_REQUIRE(QKV && pos && slot && Q && (!qk_norm || (q_gain && k_gain)), PRISM_EINVAL, "qkv_finish_paged: bad arguments");
  const size_t in4 = 4 * dtype_size(qkv_dtype), out4 = 4 * dtype_size(cache->dtype);
  PRISM_REQUIRE(qkv_stride >= (int64_t)(nq + 2 * nkv) * hd && q_stride >= (int64_t)nq * hd && qkv_stride % 4 == 0 && q_stride % 4 == 0 &&
                (uintptr_t)QKV % in4 == 0 && ((uintptr_t)Q | (qk_norm ? (uintptr_t)q_gain | (uintptr_t)k_gain : 0)) % out4 == 0, PRISM_EINVAL,
                "qkv_finish_paged: rows shorter than their heads, or not aligned to four values");
  FinishArgs a;
  a.QKV = QKV; a.q_gain = q_gain; a.k_gain = k_gain; a.pos = pos; a.slot = slot; a.Q = Q; a.K = cache->K; a.V = cache->V;
  a.qkv_stride = qkv_stride; a.q_stride = q_stride; a.page_stride = cache->page_stride;
  a.n_tok = T; a.nq = nq; a.nkv = nkv; a.page_shift = __builtin_ctz(cache->page_size); a.qk_norm = qk_norm;
  a.n_slots = (int64_t)cache->n_pages * cache->page_size;
  a.eps = eps; a.log2_base = log2((double)rope_base);
  // Few tokens: their heads go to several workgroups, each of which evaluates the rotations again, so that the launch reaches the compute
  // units and keeps enough bytes under way.  Up to 1024 workgroups: us at 256, 1024 and 4096 (32 + 8 heads of 128), 250 tokens 4.7, 4.6, 4.6;
  // 1000 8.7, 8.8, 10.1; 2100 far into a context 16.3, 14.7, 15.2; 8000 in half 38.1, 38.0, 44.5
  const int heads = nq + 2 * nkv, step = 256 / (hd / 8) / 4, groups = cdiv(T, 4);
  int split = 1;
  while (groups * split < 1024 && cdiv(heads, split) > step) split *= 2;
  a.heads_of_group = cdiv(cdiv(heads, split), step) * step;
  const dim3 grid(groups, cdiv(heads, a.heads_of_group));
  hipStream_t s = (hipStream_t)stream;
  if (cache->dtype == PRISM_DTYPE_FP32) launch_typed<float, float>(a, hd, grid, s);
  else if (cache->dtype == PRISM_DTYPE_BF16) {
    if (qkv_dtype == PRISM_DTYPE_FP32) launch_typed<float, bf16>(a, hd, grid, s);
    else launch_typed<bf16, bf16>(a, hd, grid, s);
  } else {
    if (qkv_dtype == PRISM_DTYPE_FP32) launch_typed<float, f16>(a, hd, grid, s);
    else launch_typed<f16, f16>(a, hd, grid, s);
  }
  PRISM_HIP(hipGetLastError());
  return PRISM_OK;
}
