// Shared declarations of the operators on a paged K/V cache (paged_plan.hip, paged_finish.hip, attn_paged.hip, attn_paged_fp32.hip).
#pragma once

#include "common.h"

namespace prism {

// A plan is one device buffer: header, one record per sequence, work items of the attention, blocks whose keys were split.
//
// A block is up to 128 query rows of one (sequence, KV head): whole tokens, the G query heads of the KV head side by side, so that
// every head grouping fills the matrix cores' rows and K/V are read once for all of them.  An item is a block and a run of 64-key
// tiles.  A sequence's blocks are all cut into the same number of runs, by its longest block's tiles.  What a cut costs is the
// partial results, written and read again in fp32: little for a sequence of up to kPlanNarrow rows, which is cut into runs of the
// step's tiles over plan_goal (two items for each of the 512 workgroups that the chip holds); as much as four tiles for a block of
// 128 rows, so those are cut into runs of twice that, and only where they have half as many again.  So per KV head
//   items <= plan_goal + blocks,   items of cut blocks < 2 plan_goal, their rows < 128 plan_goal,
// which is what bounds a launch's grid and the room for partial results without the host knowing a length.
// Sequences of more than kPlanNarrow rows come first in the list: their items take longest, and the others fill what is left at the end
// (30 single tokens over up to 4000 keys and a chunk of 500 behind them, 32 query heads over 8: 52 us, in the sequences' order 65).
static const int kPlanRows = 128;        // query rows of a block
static const int kPlanTile = 64;         // keys of a tile
static const int kPlanItems = 1024;      // items wanted over all KV heads: twice the two workgroups that each of 256 compute units holds
// tiles of an item at least, where that leaves fewer items than wanted (us for chunks of 40 passages in fp32, 4 heads of 64, with 4, 8
// for blocks of many rows: 57, 62; in 16 bits equal)
static const int kPlanMinTiles = 4;
static const int kPlanNarrow = 32;       // rows of a sequence whose keys are cut freely
static const int kJoinRows = 8;          // query rows whose parts one workgroup joins
static const int kPlanMagic = 0x70616765;
static const int kGroupMax = kPlanRows;  // query heads per KV head

struct PlanHeader {
  int32_t magic;
  prism_page_shape shape;
  int32_t n_items, n_joins, n_free;       // n_free: free pages before the step
  int32_t pad[4];
};
static_assert(sizeof(PlanHeader) == 64, "one cache-line half");
// page0: rank of its first new page; item0: its first item where those of all sequences follow each other, and item0 + shift in the list,
// where the sequences of many rows come first
struct PlanSeq { int32_t row0, rows, cached, has, page0, n_parts, item0, shift, part0, join0, pad[2]; };
struct PlanItem { int32_t seq, row0, n_tok, pos0, tile0, tile1, part0, pad; };        // part0: first partial row, -1: the block is whole
struct PlanJoin { int32_t row0, n_tok, part0, n_parts, step, pad[3]; };                 // part j of its rows: from part0 + j * step on

// tokens of a join and of a block, which holds whole joins
__host__ __device__ inline int plan_join_tokens(const prism_page_shape &s) {
  const int g = s.n_q_heads / s.n_kv_heads;
  return g < kJoinRows ? kJoinRows / g : 1;
}
__host__ __device__ inline int plan_block_tokens(const prism_page_shape &s) {
  const int t = plan_join_tokens(s);
  return kPlanRows / (s.n_q_heads / s.n_kv_heads) / t * t;
}
__host__ __device__ inline int plan_goal(const prism_page_shape &s) { return (kPlanItems + s.n_kv_heads - 1) / s.n_kv_heads; }
// half of it, but one at least: items of the wide blocks are as long as 1 / plan_wide_goal of all tiles, which is 2 / plan_goal or more
__host__ __device__ inline int plan_wide_goal(const prism_page_shape &s) { return plan_goal(s) > 1 ? plan_goal(s) / 2 : 1; }
__host__ __device__ inline int64_t plan_blocks(const prism_page_shape &s) { return s.n_tokens / plan_block_tokens(s) + s.n_seqs; }
__host__ __device__ inline int64_t plan_items(const prism_page_shape &s) { return plan_blocks(s) + plan_goal(s); }
__host__ __device__ inline int64_t plan_joins(const prism_page_shape &s) {
  const int t = plan_join_tokens(s);
  const int64_t by_tokens = s.n_tokens / t + s.n_seqs, by_blocks = (int64_t)plan_goal(s) * (plan_block_tokens(s) / t);
  return by_tokens < by_blocks ? by_tokens : by_blocks;    // fewer than goal blocks are cut
}
// tiles that a block's window can touch, and those of the longest sequence: where they are too few for a cut, there is nothing to join
__host__ __device__ inline int64_t plan_window_tiles(const prism_page_shape &s) {
  return ((int64_t)s.window + plan_block_tokens(s) + kPlanTile - 2) / kPlanTile + 1;
}
inline bool plan_may_cut(const prism_page_shape &s) {
  return ((int64_t)s.max_pages * s.page_size + kPlanTile - 1) / kPlanTile > kPlanMinTiles && (s.window == 0 || plan_window_tiles(s) > kPlanMinTiles);
}
// Partial rows of a KV head.  Of the tiles, w in wide blocks and n in narrow ones, w + n = 1: fewer than 2 n goal parts of up to
// kPlanNarrow rows and w goal of up to kPlanRows, so goal kPlanRows at most; and every row is in goal + 1 parts at most.
__host__ __device__ inline int64_t plan_part_rows(const prism_page_shape &s) {
  const int64_t by_parts = (int64_t)plan_goal(s) * kPlanRows;
  const int64_t by_rows = (int64_t)s.n_tokens * (s.n_q_heads / s.n_kv_heads) * (plan_goal(s) + 1);
  return by_parts < by_rows ? by_parts : by_rows;
}
__host__ __device__ inline size_t plan_items_at(const prism_page_shape &s) { return sizeof(PlanHeader) + (size_t)s.n_seqs * sizeof(PlanSeq); }
__host__ __device__ inline size_t plan_joins_at(const prism_page_shape &s) { return plan_items_at(s) + (size_t)plan_items(s) * sizeof(PlanItem); }
__host__ __device__ inline size_t plan_bytes(const prism_page_shape &s) { return plan_joins_at(s) + (size_t)plan_joins(s) * sizeof(PlanJoin); }

// without branches: on the device every one would be a wait of its own
__host__ __device__ inline bool same_shape(const prism_page_shape &a, const prism_page_shape &b) {
  return (a.n_seqs == b.n_seqs) & (a.n_tokens == b.n_tokens) & (a.n_q_heads == b.n_q_heads) & (a.n_kv_heads == b.n_kv_heads) &
         (a.page_size == b.page_size) & (a.n_pages == b.n_pages) & (a.max_pages == b.max_pages) & (a.window == b.window);
}
int check_page_shape(const prism_page_shape *s, const char *who);
int check_kv_cache(const prism_kv_cache *c, const char *who);

// 16-bit results of these operators: as from_f32, but NaN stays NaN
template <typename T> __device__ __forceinline__ T round_to(float v) { return from_f32<T>(v); }
template <> __device__ __forceinline__ f16 round_to<f16>(float v) { return v == v ? from_f32<f16>(v) : (f16)v; }

// max of v over lanes l, l ^ 16 / l, l ^ 32
__device__ __forceinline__ float max_xor32(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float max_xor16(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// A value that nothing writes while the kernel runs, at an address that is the same for the whole wave: by the scalar unit, so that
// waiting for it is not waiting for the loads of K and V that are under way
template <typename T> __device__ __forceinline__ T load_const(const T *p) {
  typedef const __attribute__((address_space(4))) uint32_t *Words;
  union { T v; uint32_t w[sizeof(T) / 4]; } u;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(T) / 4); ++i) u.w[i] = ((Words)(uintptr_t)p)[i];
  return u.v;
}

// Until at most N of this wave's memory accesses are under way.  They end in their order; others among them only make it wait longer.
// By the builtin, so that the compiler knows which loads are done and does not wait for them again, with newer ones under way
template <int N> __device__ __forceinline__ void wait_loads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | 7 << 4 | 15 << 8 | (N >> 4) << 14);      // vector loads; others: no wait
  asm volatile("" ::: "memory");
}
// Until this wave's LDS reads have returned, so that what they read may be written again
__device__ __forceinline__ void wait_lds() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(15 | 7 << 4 | 3 << 14);
  asm volatile("" ::: "memory");
}

// What an attention launch reads and writes.  Partial results of part row i and KV head h: values at O[(i * n_kv + h) * hd], running
// maximum and sum of weights at ml[i * n_kv + h].  unit: from a difference of the maxima to the exponent of 2 that its weight has.
struct PagedAttn {
  prism_page_shape shape;
  const PlanHeader *plan;
  const PlanItem *items;
  const PlanJoin *joins;
  const int32_t *table;
  const void *Q, *K, *V;
  void *out;
  const float *slopes;
  float *part_O;
  float2 *part_ml;
  int64_t q_stride, out_stride, page_stride;
  float scale, softcap, unit;
  int page_shift;
};
// Item `item` of the plan into `it`; false: there is none, or the plan was made for another shape.  The header and the item, which lies
// within the list's room whatever it holds, are asked for together: left to itself the compiler asks for one field after the other
__device__ __forceinline__ bool load_item(const PagedAttn &a, int item, PlanItem &it) {
  it = load_const(a.items + item);
  const PlanHeader h = load_const(a.plan);
  asm volatile("" : : "s"(it.seq), "s"(it.row0), "s"(it.n_tok), "s"(it.pos0), "s"(it.tile0), "s"(it.tile1), "s"(it.part0), "s"(h.magic),
               "s"(h.shape.n_seqs), "s"(h.shape.n_tokens), "s"(h.shape.n_q_heads), "s"(h.shape.n_kv_heads), "s"(h.shape.page_size),
               "s"(h.shape.n_pages), "s"(h.shape.max_pages), "s"(h.shape.window), "s"(h.n_items));
  return (h.magic == kPlanMagic) & same_shape(h.shape, a.shape) & (item < h.n_items);
}
// max(|x|, most), NaN if one of them is
__device__ __forceinline__ float worst_of(float x, float most) { return __builtin_elementwise_maximum(__builtin_fabsf(x), most); }
// y: a row's sums of weights and values in N dimensions, V the place of its KV head in the pool from these on, keys k_begin .. k_end - 1 (k_begin a
// multiple of 16), of which it sees first .. pos.  A seen value that is not finite is the result, whatever its weight: in the products the weight may
// underflow, at once or later with the maximum, and zero times the value is NaN.  So where a sum is NaN, or such values were kept from rows that do
// not see them (`all`), what is not finite is looked up again here and its sum taken instead, if there is any.  That is V read once more, until all
// that is open is known to be NaN (in bf16 also where an infinity meets a weight's two parts): a token of 100 sequences over up to 8000 keys each,
// with an infinity in every one, 1.4 ms instead of 0.32; with a NaN among the first keys no more than without.
template <typename T, int HD, int N>
__device__ __forceinline__ void settle(const PagedAttn &a, const int32_t *table, const T *V, int k_begin, int k_end, int first, int pos, bool all, float (&y)[N]) {
  constexpr int U = 8;                                        // rows under way together
  struct alignas(N * sizeof(T)) Row { T v[N]; };
  float sum[N];
#pragma unroll
  for (int e = 0; e < N; ++e) sum[e] = 0.f;
  for (int k0 = k_begin; k0 < k_end; k0 += U) {
    const int page = load_const(table + (k0 >> a.page_shift));
    if ((unsigned)page >= (unsigned)a.shape.n_pages) continue;
    const T *v = V + (int64_t)page * a.page_stride + (int64_t)(k0 & ((1 << a.page_shift) - 1)) * HD;
    Row x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = *reinterpret_cast<const Row *>(v + u * HD);     // (of the same page, behind the last key too)
    bool open = false;
#pragma unroll
    for (int e = 0; e < N; ++e) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float f = to_f32(x[u].v[e]);
        const int key = k0 + u;
        sum[e] += key >= first && key <= pos && key < k_end && !(fabsf(f) < INFINITY) ? f : 0.f;
      }
      open = open || ((all || y[e] != y[e]) && sum[e] == sum[e]);
    }
    if (__builtin_amdgcn_ballot_w64(open) == 0) break;
  }
#pragma unroll
  for (int e = 0; e < N; ++e) y[e] = (all || y[e] != y[e]) && sum[e] != 0.f ? sum[e] : y[e];
}
// Weight times a partial result, which stands whatever the weight where it is not finite
__device__ __forceinline__ float weighed(float f, float y) { return fabsf(y) < INFINITY ? f * y : y; }

int launch_attention_paged_fp32(const PagedAttn &a, int hd, hipStream_t s);

}  // namespace prism
