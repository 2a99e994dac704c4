// A step's layout in a paged K/V cache, made on the device from the sequences' lengths: row offsets, positions, cache slots, new
// pages from a free list, and the work list of the attention that reads the cache (paged.h has its bounds).
//
// Everything is a sum over the sequences in front: rows, new pages, items.  One workgroup takes those sums (page_plan_kernel: up to
// four sequences per thread, three scans); what they say about each row and item is then independent work, found by a binary
// search.  Steps of up to kPlanAlone rows are finished by the same workgroup, larger ones by a second launch of many.
// Bound by launch and memory latency and by the chain of the sums, a step's bytes being nothing: 24 sequences of a token each 6.1 us, 500
// of 332 tokens in the mean 11.5 us in two launches.  So there is no division but by shift and multiplication, every wave's load of a
// value is asked for once, and 64 bits only where a sum needs them.
#include "paged.h"

namespace prism {

static const int kPlanAlone = 4096;      // rows that the summing workgroup lays out itself, of up to kPlanInLds sequences
static const int kPlanInLds = 1024;

// x / d for x up to 2^20 and d up to 128: the product's error, x (2^32 / d rounded up - 2^32 / d), stays below 2^32 / d
struct Divisor {
  uint32_t d, m;
  __device__ __forceinline__ int operator()(int x) const { return d == 1 ? x : (int)__umulhi((uint32_t)x, m); }
};
static Divisor divisor(int d) { return {(uint32_t)d, (uint32_t)((((uint64_t)1 << 32) + d - 1) / d)}; }

struct PlanArgs {
  prism_page_shape s;
  const int32_t *cached, *fresh;
  int32_t *table;
  const int32_t *free_pages, *n_free;
  int32_t *n_free_left, *cu, *pos, *slot, *status;
  PlanHeader *head;
  PlanSeq *seqs;
  PlanItem *items;
  PlanJoin *joins;
  Divisor block, join;                    // by the tokens of a block and of a join
  int free_cap, page_shift, G, goal, wide_goal, window_tiles;
};

// Sums that stop at 2^31 - 1: of terms that are not negative, in any grouping the same
__device__ __forceinline__ int add_capped(int a, int b) { return __builtin_elementwise_add_sat(a, b); }

// Sum over this lane and those in front of it: within rows of 16 lanes, then each row's last one to the rows behind it.  By moves between
// lanes within the vector unit: a step through LDS's crossbar takes some ten times as long, and every sum here is waited for
template <int CTRL, int ROWS> __device__ __forceinline__ int add_from(int x) {
  return add_capped(x, __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xF, false));
}
__device__ __forceinline__ int wave_scan(int x) {
  x = add_from<0x111, 0xF>(x);                               // from 1, 2, 4 and 8 lanes in front
  x = add_from<0x112, 0xF>(x);
  x = add_from<0x114, 0xF>(x);
  x = add_from<0x118, 0xF>(x);
  x = add_from<0x142, 0xA>(x);                               // lanes 15 and 47 to the row behind them
  return add_from<0x143, 0xC>(x);                            // lane 31 to the upper half
}
// sums over the workgroup's threads in front of this one, of N values at once; total: over all of them
template <int N> struct Sums { int v[N]; };
template <int WAVES, int N>
__device__ __forceinline__ Sums<N> block_scan(Sums<N> s, int32_t (&lds)[4][WAVES], Sums<N> &total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Sums<N> out;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int x = wave_scan(s.v[i]);
    if (lane == 63) lds[i][wave] = x;
    out.v[i] = __builtin_amdgcn_update_dpp(0, x, 0x138, 0xF, 0xF, false);      // of the lane in front
    total.v[i] = 0;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      if (w == wave) out.v[i] = add_capped(out.v[i], total.v[i]);
      total.v[i] = add_capped(total.v[i], lds[i][w]);
    }
  __syncthreads();
  return out;
}

// the last i in [0, n) with first[i] <= x; first[0] = 0
__device__ __forceinline__ int last_at_or_before(const int32_t *first, int n, int x) {
  int lo = 0;
  for (int step = 1 << (31 - __builtin_clz(n)); step > 0; step >>= 1)
    if (lo + step < n && first[lo + step] <= x) lo += step;
  return lo;
}

// Rows and items that thread `me` of `all` lays out; row0, item0 and seqs of the n sequences, of which total rows and n_items are.
__device__ __forceinline__ void lay_out(const PlanArgs &a, const int32_t *row0, const int32_t *item0, const PlanSeq *seqs, int total, int n_items,
                                        int n_free, int me, int all) {
  const prism_page_shape &s = a.s;
  for (int r = me; r < s.n_tokens; r += all) {
    int pos = 0, slot = -1;
    if (r < total) {
      const int q = last_at_or_before(row0, s.n_seqs, r);
      const PlanSeq sq = seqs[q];
      pos = sq.cached + r - sq.row0;
      const int idx = pos >> a.page_shift, off = pos & ((1 << a.page_shift) - 1);
      if (idx < s.max_pages) {
        int32_t *entry = a.table + (int64_t)q * s.max_pages + idx;
        int page;
        if (idx >= sq.has) {                                 // a new page, whose first position is a row of this step
          const int rank = add_capped(sq.page0, idx - sq.has);
          page = rank < n_free ? a.free_pages[n_free - 1 - rank] : -1;
          if (off == 0) *entry = page;
        } else {
          page = *entry;
        }
        if ((uint32_t)page < (uint32_t)s.n_pages) slot = (page << a.page_shift) + off;
      }
    }
    a.pos[r] = pos;
    a.slot[r] = slot;
  }
  const int bt = a.block.d, jt = a.join.d, cap = s.max_pages << a.page_shift;
  for (int i = me; i < n_items; i += all) {
    const int q = last_at_or_before(item0, s.n_seqs, i);
    const PlanSeq sq = seqs[q];
    const int local = i - sq.item0, n_blocks = a.block(sq.rows + bt - 1);
    const int nth = sq.n_parts == 1 ? local : local / sq.n_parts, j = local - nth * sq.n_parts;
    const int b = n_blocks - 1 - nth;                        // the last block, which has most keys, first
    const int n_tok = sq.rows - b * bt < bt ? sq.rows - b * bt : bt, p0 = sq.cached + b * bt;
    const int end = p0 + n_tok < cap ? p0 + n_tok : cap;
    const int lo = s.window > 0 && p0 >= s.window ? (p0 - s.window + 1) / kPlanTile : 0;
    const int hi = (end + kPlanTile - 1) / kPlanTile, n = hi > lo ? hi - lo : 0;
    PlanItem it;
    it.seq = q;
    it.row0 = sq.row0 + b * bt;
    it.n_tok = n_tok;
    it.pos0 = p0;
    it.part0 = -1;
    it.pad = 0;
    if (sq.n_parts > 1) {
      // n = each * parts + more: the first `more` parts get one tile more
      const int each = n / sq.n_parts, more = n - each * sq.n_parts, first = sq.part0 + b * sq.n_parts * bt * a.G;
      it.tile0 = lo + j * each + (j < more ? j : more);
      it.tile1 = it.tile0 + each + (j < more ? 1 : 0);
      it.part0 = first + j * n_tok * a.G;
      if (j == 0)
        for (int e = 0, t = 0; t < n_tok; ++e, t += jt)
          a.joins[sq.join0 + b * a.join(bt) + e] = {it.row0 + t, n_tok - t < jt ? n_tok - t : jt, first + t * a.G, sq.n_parts, n_tok * a.G, {0, 0, 0}};
    } else {
      it.tile0 = lo;
      it.tile1 = lo + n;
    }
    a.items[i + sq.shift] = it;
  }
}

// THREADS threads take the sums of up to PER * THREADS sequences
template <int THREADS, int PER>
__global__ __launch_bounds__(THREADS) void page_plan_kernel(const PlanArgs a) {
  constexpr bool kRecords = THREADS * PER <= kPlanInLds;     // the sequences' records in LDS too, for laying rows out
  __shared__ __align__(16) int32_t scan[4][THREADS / 64];
  __shared__ int32_t row0[kRecords ? THREADS * PER : 1], item0[kRecords ? THREADS * PER : 1];
  __shared__ PlanSeq records[kRecords ? THREADS * PER : 1];
  const prism_page_shape &s = a.s;
  const int first = threadIdx.x * PER, bt = a.block.d, jt = a.join.d, psize = 1 << a.page_shift, cap = s.max_pages << a.page_shift;

  const int window_tiles = a.window_tiles;
  int n_free = *a.n_free;
  n_free = n_free < 0 ? 0 : n_free > a.free_cap ? a.free_cap : n_free;
  int cached[PER], rows[PER], tiles[PER], has[PER], fresh_pages[PER], n_blocks[PER], n_parts[PER], r0[PER];
  Sums<1> sum = {0}, run, total;
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const bool in = first + k < s.n_seqs;
    const int c = in ? a.cached[first + k] : 0, f = in ? a.fresh[first + k] : 0;
    cached[k] = c < 0 ? 0 : c > (1 << 29) ? 1 << 29 : c;
    rows[k] = f < 0 ? 0 : f;
    sum.v[0] = add_capped(sum.v[0], rows[k]);
  }
  run = block_scan<THREADS / 64>(sum, scan, total);
  const int asked = total.v[0], done = asked < s.n_tokens ? asked : s.n_tokens;
  // rows behind the last of T are left out; pages, blocks and tiles of what is left
  int at = run.v[0];
  int64_t block_tiles = 0;                                    // of up to four sequences: below 2^46
  Sums<4> part = {{0, 0, 0, 0}}, parts;                       // new pages; the tiles, 16 bits at a time
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    r0[k] = at < s.n_tokens ? at : s.n_tokens;
    at = add_capped(at, rows[k]);
    rows[k] = (at < s.n_tokens ? at : s.n_tokens) - r0[k];
    const int end = cached[k] + rows[k];                     // below 2^30
    const int hp = (cached[k] + psize - 1) >> a.page_shift, np = (end + psize - 1) >> a.page_shift;
    has[k] = hp < s.max_pages ? hp : s.max_pages;
    fresh_pages[k] = rows[k] > 0 ? (np < s.max_pages ? np : s.max_pages) - has[k] : 0;
    n_blocks[k] = a.block(rows[k] + bt - 1);
    int t = ((end < cap ? end : cap) + kPlanTile - 1) / kPlanTile;
    t = t < window_tiles ? t : window_tiles;
    tiles[k] = t;
    block_tiles += (int64_t)t * n_blocks[k];
    part.v[0] = add_capped(part.v[0], fresh_pages[k]);
  }
#pragma unroll
  for (int i = 0; i < 3; ++i) part.v[1 + i] = (int)(block_tiles >> (16 * i)) & 0xFFFF;
  int page = block_scan<THREADS / 64>(part, scan, parts).v[0];
  const int pages = parts.v[0];
  const int64_t all_tiles = parts.v[1] + ((int64_t)parts.v[2] << 16) + ((int64_t)parts.v[3] << 32);
  // Tiles of an item, rounded up, so at least the quotient (exact below 2^53): what bounds the number of items
  auto share = [&](int goal, int least) {
    const double x = ceil((double)all_tiles / goal);
    return x < least ? least : x > 1 << 30 ? 1 << 30 : (int)x;
  };
  const int narrow = share(a.goal, kPlanMinTiles), wide = share(a.wide_goal, kPlanMinTiles);
  enum { kItems, kWide, kRows, kJoins };                     // items, those of them with many rows, partial rows, joins
  Sums<4> mine = {{0, 0, 0, 0}}, all;
  auto add = [&](Sums<4> &x, int k) {
    const int items = n_blocks[k] * n_parts[k];
    x.v[kItems] += items;
    if (rows[k] * a.G > kPlanNarrow) x.v[kWide] += items;
    if (n_parts[k] > 1) {
      x.v[kRows] += rows[k] * a.G * n_parts[k];
      x.v[kJoins] += a.join(rows[k] + jt - 1);
    }
  };
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const bool one = rows[k] * a.G <= kPlanNarrow;
    const int per_item = one ? narrow : wide;
    n_parts[k] = (one ? tiles[k] > narrow : tiles[k] > wide + wide / 2) ? (tiles[k] + per_item - 1) / per_item : 1;
    add(mine, k);
  }
  Sums<4> front = block_scan<THREADS / 64>(mine, scan, all);
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int q = first + k;
    if (q >= s.n_seqs) break;
    const int shift = rows[k] * a.G > kPlanNarrow ? front.v[kWide] - front.v[kItems] : all.v[kWide] - front.v[kWide];
    const PlanSeq o = {r0[k], rows[k], cached[k], has[k], page, n_parts[k], front.v[kItems], shift, front.v[kRows], front.v[kJoins], {0, 0}};
    a.seqs[q] = o;
    if (kRecords) {
      row0[q] = o.row0;
      item0[q] = o.item0;
      records[q] = o;
    }
    a.cu[q] = o.row0;
    page = add_capped(page, fresh_pages[k]);
    add(front, k);
  }
  if (threadIdx.x == 0) {
    const int taken = pages < n_free ? pages : n_free;
    a.cu[s.n_seqs] = done;
    *a.n_free_left = n_free - taken;
    if (a.status) {
      a.status[0] = done;
      a.status[1] = taken;
      a.status[2] = pages - taken;
      a.status[3] = asked - done;
    }
    PlanHeader o;
    o.magic = kPlanMagic;
    o.shape = s;
    o.n_items = all.v[kItems];
    o.n_joins = all.v[kJoins];
    o.n_free = n_free;                                       // the caller's count may be overwritten before the rows are laid out
    for (int k = 0; k < 4; ++k) o.pad[k] = 0;
    *a.head = o;
  }
  if (!kRecords || s.n_tokens > kPlanAlone) return;
  __syncthreads();
  lay_out(a, row0, item0, records, done, all.v[kItems], n_free, threadIdx.x, THREADS);
}

__global__ __launch_bounds__(256) void page_rows_kernel(const PlanArgs a) {
  __shared__ int32_t row0[PRISM_MAX_CANDS], item0[PRISM_MAX_CANDS];
  for (int i = threadIdx.x; i < a.s.n_seqs; i += 256) {
    row0[i] = a.seqs[i].row0;
    item0[i] = a.seqs[i].item0;
  }
  const int total = a.cu[a.s.n_seqs], n_items = a.head->n_items, n_free = a.head->n_free;
  __syncthreads();
  lay_out(a, row0, item0, a.seqs, total, n_items, n_free, (int)(blockIdx.x * 256 + threadIdx.x), (int)(gridDim.x * 256));
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
  PlanArgs a;
  a.s = *shape;
  a.cached = cached; a.fresh = fresh; a.table = table; a.free_pages = free_pages; a.n_free = n_free;
  a.n_free_left = n_free_left; a.cu = cu; a.pos = pos; a.slot = slot; a.status = status;
  a.head = (PlanHeader *)plan;
  a.seqs = (PlanSeq *)((char *)plan + sizeof(PlanHeader));
  a.items = (PlanItem *)((char *)plan + plan_items_at(*shape));
  a.joins = (PlanJoin *)((char *)plan + plan_joins_at(*shape));
  a.block = divisor(plan_block_tokens(*shape));
  a.join = divisor(plan_join_tokens(*shape));
  a.free_cap = free_cap;
  a.page_shift = __builtin_ctz(shape->page_size);
  a.G = shape->n_q_heads / shape->n_kv_heads;
  a.goal = plan_goal(*shape);
  a.wide_goal = plan_wide_goal(*shape);
  a.window_tiles = shape->window > 0 ? (int)plan_window_tiles(*shape) : INT32_MAX;
  hipStream_t s = (hipStream_t)stream;
  // Every barrier waits for all waves, so few of them where they only sum: us with four waves and with sixteen, 4 sequences 7.6, 10.2, 60
  // 9.0, 11.5, 500 11.5, 13.6, 900 13.9, 15.1; more than that 20.7, 18.2 (1500).  Where the workgroup lays the rows out too, sixteen from 1024 rows on
  const bool alone = shape->n_tokens <= kPlanAlone;
  if (shape->n_seqs <= 256 && (shape->n_tokens <= 1024 || !alone)) page_plan_kernel<256, 1><<<1, 256, 0, s>>>(a);
  else if (shape->n_seqs <= 512 && !alone) page_plan_kernel<256, 2><<<1, 256, 0, s>>>(a);
  else if (shape->n_seqs <= kPlanInLds && !alone) page_plan_kernel<256, 4><<<1, 256, 0, s>>>(a);
  else if (shape->n_seqs <= kPlanInLds) page_plan_kernel<1024, 1><<<1, 1024, 0, s>>>(a);
  else page_plan_kernel<1024, PRISM_MAX_CANDS / 1024><<<1, 1024, 0, s>>>(a);
  PRISM_HIP(hipGetLastError());
  if (shape->n_tokens > (shape->n_seqs > kPlanInLds ? 0 : kPlanAlone)) {
    const int grid = cdiv(shape->n_tokens, 512);
    page_rows_kernel<<<grid < 1024 ? grid : 1024, 256, 0, s>>>(a);
    PRISM_HIP(hipGetLastError());
  }
  return PRISM_OK;
}
