// A step's layout in a paged K/V cache, made on the device from the sequences' lengths: row offsets, positions, cache slots, new
// pages from a free list, and the work list of the attention that reads the cache (paged.h has its bounds).
//
// Everything is a sum over the sequences in front: rows, new pages, items.  One workgroup takes those sums (page_plan_kernel: up to
// four sequences per thread, three scans); what they say about each row and item is then independent work, found by a binary
// search.  Steps of up to kPlanAlone rows are finished by the same workgroup, larger ones by a second launch of many.
// Bound by launch and memory latency: a step's bytes are nothing.
#include "paged.h"

namespace prism {

static const int kPlanThreads = 1024;
static const int kPlanAlone = 4096;      // rows that the summing workgroup lays out itself

struct PlanArgs {
  prism_page_shape s;
  const int32_t *cached, *fresh;
  int32_t *table;
  const int32_t *free_pages, *n_free;
  int32_t free_cap;
  int32_t *n_free_left, *cu, *pos, *slot, *status;
  char *plan;
};

// inclusive sums over the workgroup's threads of three values at once; total: the last thread's
struct Sums { int64_t a, b, c; };
__device__ __forceinline__ Sums block_scan(Sums v, Sums *lds, Sums &total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t a = __shfl_up(v.a, o, 64), b = __shfl_up(v.b, o, 64), c = __shfl_up(v.c, o, 64);
    if (lane >= o) { v.a += a; v.b += b; v.c += c; }
  }
  if (lane == 63) lds[wave] = v;
  __syncthreads();
  Sums before = {0, 0, 0};
  total = {0, 0, 0};
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    const Sums t = lds[w];
    if (w < wave) { before.a += t.a; before.b += t.b; before.c += t.c; }
    total.a += t.a; total.b += t.b; total.c += t.c;
  }
  __syncthreads();
  return {v.a + before.a, v.b + before.b, v.c + before.c};
}

// the last i in [0, n) with first[i] <= x; first[0] = 0
__device__ __forceinline__ int last_at_or_before(const int32_t *first, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

// Rows and items that thread `me` of `all` lays out; row0 and item0: the sequences' first ones, in LDS.
__device__ void lay_out(const PlanArgs &a, const int32_t *row0, const int32_t *item0, int64_t me, int64_t all) {
  const prism_page_shape &s = a.s;
  const PlanHeader *h = reinterpret_cast<const PlanHeader *>(a.plan);
  const PlanSeq *seqs = reinterpret_cast<const PlanSeq *>(a.plan + sizeof(PlanHeader));
  PlanItem *items = reinterpret_cast<PlanItem *>(a.plan + plan_items_at(s));
  PlanJoin *joins = reinterpret_cast<PlanJoin *>(a.plan + plan_joins_at(s));
  const int total = row0[s.n_seqs];
  const int n_free = h->pad[0];
  for (int64_t r = me; r < s.n_tokens; r += all) {
    int pos = 0, slot = -1;
    if (r < total) {
      const int q = last_at_or_before(row0, s.n_seqs, (int)r);
      const PlanSeq sq = seqs[q];
      pos = sq.cached + (int)r - sq.row0;
      const int idx = pos / s.page_size, off = pos % s.page_size;
      if (idx < s.max_pages) {
        int32_t *entry = a.table + (int64_t)q * s.max_pages + idx;
        int page;
        if (idx >= sq.has) {                                 // a new page, whose first position is a row of this step
          const int rank = sq.page0 + idx - sq.has;
          page = rank < n_free ? a.free_pages[n_free - 1 - rank] : -1;
          if (off == 0) *entry = page;
        } else {
          page = *entry;
        }
        if ((uint32_t)page < (uint32_t)s.n_pages) slot = page * s.page_size + off;
      }
    }
    a.pos[r] = pos;
    a.slot[r] = slot;
  }
  const int G = s.n_q_heads / s.n_kv_heads, bt = plan_block_tokens(s), jt = plan_join_tokens(s);
  const int64_t cap = (int64_t)s.max_pages * s.page_size;
  for (int64_t i = me; i < h->n_items; i += all) {
    const int q = last_at_or_before(item0, s.n_seqs, (int)i);
    const PlanSeq sq = seqs[q];
    const int local = (int)i - sq.item0, n_blocks = (sq.rows + bt - 1) / bt;
    const int b = n_blocks - 1 - local / sq.n_parts, j = local % sq.n_parts;    // the last block, which has most keys, first
    const int n_tok = sq.rows - b * bt < bt ? sq.rows - b * bt : bt, p0 = sq.cached + b * bt;
    const int64_t end = (int64_t)p0 + n_tok < cap ? p0 + n_tok : cap;
    const int lo = s.window > 0 && p0 >= s.window ? (p0 - s.window + 1) / kPlanTile : 0;
    const int hi = (int)((end + kPlanTile - 1) / kPlanTile), n = hi > lo ? hi - lo : 0;
    PlanItem it;
    it.seq = q;
    it.row0 = sq.row0 + b * bt;
    it.n_tok = n_tok;
    it.pos0 = p0;
    it.tile0 = lo + (int)((int64_t)n * j / sq.n_parts);
    it.tile1 = lo + (int)((int64_t)n * (j + 1) / sq.n_parts);
    it.part0 = -1;
    it.pad = 0;
    if (sq.n_parts > 1) {
      const int first = sq.part0 + b * sq.n_parts * bt * G;
      it.part0 = first + j * n_tok * G;
      if (j == 0)
        for (int e = 0, t = 0; t < n_tok; ++e, t += jt)
          joins[sq.join0 + b * (bt / jt) + e] = {it.row0 + t, n_tok - t < jt ? n_tok - t : jt, first + t * G, sq.n_parts, n_tok * G, {0, 0, 0}};
    }
    items[i] = it;
  }
}

__global__ __launch_bounds__(kPlanThreads) void page_plan_kernel(const PlanArgs a) {
  __shared__ Sums scan[kPlanThreads / 64];
  __shared__ int32_t row0[PRISM_MAX_CANDS + 1], item0[PRISM_MAX_CANDS];
  constexpr int kPer = PRISM_MAX_CANDS / kPlanThreads;
  const prism_page_shape &s = a.s;
  const int per = (s.n_seqs + kPlanThreads - 1) / kPlanThreads, first = threadIdx.x * per;
  const int bt = plan_block_tokens(s), jt = plan_join_tokens(s), G = s.n_q_heads / s.n_kv_heads;
  const int64_t cap = (int64_t)s.max_pages * s.page_size;
  PlanHeader *h = reinterpret_cast<PlanHeader *>(a.plan);
  PlanSeq *seqs = reinterpret_cast<PlanSeq *>(a.plan + sizeof(PlanHeader));

  int n_free = *a.n_free;
  n_free = n_free < 0 ? 0 : n_free > a.free_cap ? a.free_cap : n_free;
  int cached[kPer], rows[kPer], tiles[kPer];
  Sums total, mine = {0, 0, 0};
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const bool in = k < per && first + k < s.n_seqs;
    const int c = in ? a.cached[first + k] : 0, f = in ? a.fresh[first + k] : 0;
    cached[k] = c < 0 ? 0 : c > (1 << 29) ? 1 << 29 : c;
    rows[k] = f < 0 ? 0 : f > s.n_tokens ? s.n_tokens : f;   // the sums stay far below 2^63
    mine.a += rows[k];
  }
  int64_t at = block_scan(mine, scan, total).a - mine.a;
  const int64_t asked = total.a;
  // rows behind the last of T are left out; pages, blocks and tiles of what is left
  int64_t r0[kPer], blocks_tiles = 0;
  int has[kPer], fresh_pages[kPer], n_blocks[kPer];
  mine = {0, 0, 0};
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    r0[k] = at < s.n_tokens ? at : s.n_tokens;
    at += rows[k];
    rows[k] = (int)((at < s.n_tokens ? at : s.n_tokens) - r0[k]);
    const int64_t end = (int64_t)cached[k] + rows[k];
    const int64_t hp = ((int64_t)cached[k] + s.page_size - 1) / s.page_size, np = (end + s.page_size - 1) / s.page_size;
    has[k] = (int)(hp < s.max_pages ? hp : s.max_pages);
    fresh_pages[k] = rows[k] > 0 ? (int)(np < s.max_pages ? np : s.max_pages) - has[k] : 0;
    n_blocks[k] = (rows[k] + bt - 1) / bt;
    int64_t t = ((end < cap ? end : cap) + kPlanTile - 1) / kPlanTile;
    if (s.window > 0) {                                      // tiles that a block's window can touch
      const int64_t w = ((int64_t)s.window + bt - 1 + kPlanTile - 1) / kPlanTile + 1;
      t = t < w ? t : w;
    }
    tiles[k] = (int)t;
    blocks_tiles += t * n_blocks[k];
    mine.a += fresh_pages[k];
  }
  mine.b = blocks_tiles;
  Sums run = block_scan(mine, scan, total);
  int64_t page = run.a - mine.a;
  const int64_t pages = total.a;
  const int64_t goal = plan_goal(s);
  int64_t per_item = (total.b + goal - 1) / goal;
  if (per_item < kPlanMinTiles) per_item = kPlanMinTiles;
  int n_parts[kPer];
  mine = {0, 0, 0};
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    n_parts[k] = (int)((tiles[k] + per_item - 1) / per_item);
    if (n_parts[k] < 1) n_parts[k] = 1;
    mine.a += (int64_t)n_blocks[k] * n_parts[k];
    if (n_parts[k] > 1) {
      mine.b += (int64_t)rows[k] * G * n_parts[k];
      mine.c += (rows[k] + jt - 1) / jt;
    }
  }
  run = block_scan(mine, scan, total);
  int64_t item = run.a - mine.a, part = run.b - mine.b, join = run.c - mine.c;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int q = first + k;
    if (k >= per || q >= s.n_seqs) continue;
    PlanSeq o;
    o.row0 = (int)r0[k];
    o.rows = rows[k];
    o.cached = cached[k];
    o.has = has[k];
    o.page0 = (int)(page < n_free ? page : n_free);          // ranks from n_free on have no page, however many there are
    o.n_parts = n_parts[k];
    o.item0 = (int)item;
    o.part0 = (int)part;
    o.join0 = (int)join;
    o.pad[0] = o.pad[1] = o.pad[2] = 0;
    seqs[q] = o;
    row0[q] = o.row0;
    item0[q] = o.item0;
    a.cu[q] = o.row0;
    page += fresh_pages[k];
    item += (int64_t)n_blocks[k] * n_parts[k];
    if (n_parts[k] > 1) {
      part += (int64_t)rows[k] * G * n_parts[k];
      join += (rows[k] + jt - 1) / jt;
    }
  }
  if (threadIdx.x == 0) {
    const int64_t done = asked < s.n_tokens ? asked : s.n_tokens, taken = pages < n_free ? pages : n_free;
    row0[s.n_seqs] = a.cu[s.n_seqs] = (int)done;
    *a.n_free_left = (int)(n_free - taken);
    if (a.status) {
      const int64_t most = INT32_MAX;
      a.status[0] = (int)done;
      a.status[1] = (int)taken;
      a.status[2] = (int)(pages - taken < most ? pages - taken : most);
      a.status[3] = (int)(asked - done < most ? asked - done : most);
    }
    PlanHeader o;
    o.magic = kPlanMagic;
    o.shape = s;
    o.n_items = (int)total.a;
    o.n_joins = (int)total.c;
    o.pad[0] = n_free;                                       // the caller's count may be overwritten before the rows are laid out
    for (int k = 1; k < 5; ++k) o.pad[k] = 0;
    *h = o;
  }
  if (s.n_tokens > kPlanAlone) return;
  __syncthreads();
  lay_out(a, row0, item0, threadIdx.x, kPlanThreads);
}

__global__ __launch_bounds__(256) void page_rows_kernel(const PlanArgs a) {
  __shared__ int32_t row0[PRISM_MAX_CANDS + 1], item0[PRISM_MAX_CANDS];
  const PlanSeq *seqs = reinterpret_cast<const PlanSeq *>(a.plan + sizeof(PlanHeader));
  for (int i = threadIdx.x; i < a.s.n_seqs; i += 256) {
    row0[i] = seqs[i].row0;
    item0[i] = seqs[i].item0;
  }
  if (threadIdx.x == 0) row0[a.s.n_seqs] = a.cu[a.s.n_seqs];
  __syncthreads();
  lay_out(a, row0, item0, (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256);
}

int check_page_shape(const prism_page_shape *s, const char *who) {
  PRISM_REQUIRE(s, PRISM_EINVAL, "%s: no shape", who);
  PRISM_REQUIRE(s->n_seqs >= 0 && s->n_seqs <= PRISM_MAX_CANDS && s->n_tokens >= 0 && s->n_tokens <= PRISM_MAX_STEP, PRISM_EINVAL,
                "%s: %d sequences (up to %d), %d tokens (up to %d)", who, s->n_seqs, PRISM_MAX_CANDS, s->n_tokens, PRISM_MAX_STEP);
  PRISM_REQUIRE(s->n_q_heads > 0 && s->n_kv_heads > 0 && s->n_q_heads % s->n_kv_heads == 0, PRISM_EINVAL, "%s: %d query heads over %d KV heads",
                who, s->n_q_heads, s->n_kv_heads);
  PRISM_REQUIRE(s->n_kv_heads <= 256 && s->n_q_heads / s->n_kv_heads <= kGroupMax, PRISM_EUNSUPPORTED, "%s: %d query heads over %d KV heads", who,
                s->n_q_heads, s->n_kv_heads);
  PRISM_REQUIRE(s->page_size >= 16 && s->page_size <= 256 && (s->page_size & (s->page_size - 1)) == 0, PRISM_EUNSUPPORTED,
                "%s: pages of %d tokens (16, 32, 64, 128 or 256)", who, s->page_size);
  PRISM_REQUIRE(s->n_pages > 0 && (int64_t)s->n_pages * s->page_size <= INT32_MAX && s->max_pages > 0 &&
                (int64_t)s->max_pages * s->page_size <= 1 << 29 && s->window >= 0, PRISM_EINVAL, "%s: %d pages, %d of a sequence, window %d", who,
                s->n_pages, s->max_pages, s->window);
  return PRISM_OK;
}

}  // namespace prism

using namespace prism;

extern "C" int64_t prism_page_plan_bytes(const prism_page_shape *shape) {
  return check_page_shape(shape, "page_plan_bytes") == PRISM_OK ? (int64_t)plan_bytes(*shape) : -1;
}

extern "C" int prism_op_page_plan(const prism_page_shape *shape, const int32_t *cached, const int32_t *fresh, int32_t *table,
                                  const int32_t *free_pages, int32_t free_cap, const int32_t *n_free, int32_t *n_free_left, int32_t *cu,
                                  int32_t *pos, int32_t *slot, int32_t *status, void *plan, void *stream) {
  PRISM_TRY(check_page_shape(shape, "page_plan"));
  PRISM_REQUIRE(n_free && n_free_left && cu && plan && free_cap >= 0 && (free_pages || free_cap == 0), PRISM_EINVAL, "page_plan: bad arguments");
  PRISM_REQUIRE(shape->n_seqs == 0 || (cached && fresh && table), PRISM_EINVAL, "page_plan: bad arguments");
  PRISM_REQUIRE(shape->n_tokens == 0 || (pos && slot), PRISM_EINVAL, "page_plan: bad arguments");
  PRISM_REQUIRE((uintptr_t)plan % 16 == 0, PRISM_EINVAL, "page_plan: the plan must be 16-byte aligned");
  PlanArgs a = {*shape, cached, fresh, table, free_pages, n_free, free_cap, n_free_left, cu, pos, slot, status, (char *)plan};
  hipStream_t s = (hipStream_t)stream;
  page_plan_kernel<<<1, kPlanThreads, 0, s>>>(a);
  PRISM_HIP(hipGetLastError());
  if (shape->n_tokens > kPlanAlone) {
    const int grid = cdiv(shape->n_tokens, 512);
    page_rows_kernel<<<grid < 1024 ? grid : 1024, 256, 0, s>>>(a);
    PRISM_HIP(hipGetLastError());
  }
  return PRISM_OK;
}
