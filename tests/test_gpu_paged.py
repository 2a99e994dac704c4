"""The operators on a paged K/V cache (page plan, finishing with append, attention) against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2510_15620_amd import binding as B
from tests import paged_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


# ------------------------------------------------------------------------------------------------------------ page plan

def _run_plan(cached, fresh, table, free, n_free, T, page, n_pages, nq=8, nkv=2, window=0):
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)  # noqa: E731
    plan = B.PagePlan(len(cached), T, nq, nkv, page, n_pages, table.shape[1], window=window)
    d_table, left = dev(table), torch.full((1,), -7, dtype=torch.int32, device=DEV)
    cu, pos, slot, status = (torch.full((n,), -77, dtype=torch.int32, device=DEV) for n in (len(cached) + 1, T, T, 4))
    B.op_page_plan(plan, dev(cached), dev(fresh), d_table, dev(free), dev([n_free]), left, cu, pos, slot, status)
    torch.cuda.synchronize()
    return plan, [x.cpu().numpy() for x in (cu, pos, slot, d_table, left, status)]


def _check_plan(cached, fresh, table, free, n_free, T, page, n_pages, nq=8, nkv=2, window=0):
    plan, got = _run_plan(cached, fresh, table, free, n_free, T, page, n_pages, nq, nkv, window)
    want = R.plan(cached, fresh, table, free, n_free, T, page, n_pages)
    for g, w, name in zip(got, want, ("cu", "pos", "slot", "table", "left", "status")):
        assert np.array_equal(g.reshape(-1), np.array(w, np.int64).reshape(-1)), name
    _check_work(plan, want[0], np.maximum(cached, 0), page, table.shape[1], nq // nkv, nkv, window)


def _check_work(plan, cu, cached, page, width, G, nkv, window):
    """The work list: every row's blocks once, their runs of tiles cover what a row may see, partial rows and joins stay in their bounds."""
    raw = plan.buffer.cpu().numpy().view(np.int32)
    n_items, n_joins = int(raw[9]), int(raw[10])
    n = plan.n_seqs
    goal, jt = -(-1024 // nkv), max(1, 8 // G)
    bt = 128 // G // jt * jt
    items_at = 16 + 12 * n
    most = plan.n_tokens // bt + n + goal
    assert n_items <= most
    items = raw[items_at: items_at + 8 * n_items].reshape(-1, 8)
    joins = raw[items_at + 8 * most:][: 8 * n_joins].reshape(-1, 8)
    room = min(goal * 128, plan.n_tokens * G * (goal + 1))
    many = [(cu[seq + 1] - cu[seq]) * G > 32 for seq in items[:, 0].tolist()]
    assert many == sorted(many, reverse=True), "sequences of many rows come first"
    seen, parts = {}, {}
    for seq, row0, n_tok, pos0, t0, t1, part, _ in items.tolist():
        assert 0 <= seq < n and 1 <= n_tok <= bt and cu[seq] <= row0 and row0 + n_tok <= cu[seq + 1] and (row0 - cu[seq]) % bt == 0
        assert pos0 == cached[seq] + row0 - cu[seq] and t0 <= t1
        seen.setdefault((seq, row0, n_tok), []).append((t0, t1))
        if part >= 0:
            assert part + n_tok * G <= room
            parts.setdefault(row0, []).append((part, n_tok * G))
    covered = np.zeros(cu[-1], np.int64)
    for (seq, row0, n_tok), runs in seen.items():
        covered[row0: row0 + n_tok] += 1
        runs.sort()
        assert all(a[1] == b[0] for a, b in zip(runs, runs[1:]))
        p0 = cached[seq] + row0 - cu[seq]
        end = min(p0 + n_tok, width * page)
        lo = max(0, p0 - window + 1) // 64 if window else 0
        assert runs[0][0] <= lo and runs[-1][1] >= -(-end // 64) or lo * 64 >= end
        assert (len(runs) > 1) == (row0 in parts)
    assert (covered == 1).all()
    used = sorted(x for v in parts.values() for x in v)
    assert all(a[0] + a[1] <= b[0] for a, b in zip(used, used[1:]))
    joined = np.zeros(cu[-1], np.int64)
    for row0, n_tok, part, n_parts, step, *_ in joins.tolist():
        joined[row0: row0 + n_tok] += 1
        first = max(r for r in parts if r <= row0)
        p = sorted(parts[first])
        assert n_parts == len(p) and n_tok <= jt and step == p[0][1]
        assert all(part + j * step == p[j][0] + (row0 - first) * G for j in range(n_parts))
    for row0, p in parts.items():
        assert (joined[row0: row0 + p[0][1] // G] == 1).all()
    assert joined.sum() == sum(p[0][1] // G for p in parts.values())


def _lengths(r, n, c_hi, f_hi):
    c, f = r.integers(0, c_hi + 1, n), r.integers(0, f_hi + 1, n)
    c[r.random(n) < 0.2] = 0
    f[r.random(n) < 0.2] = 0
    return c.astype(np.int32), f.astype(np.int32)


@pytest.mark.parametrize("n,c_hi,f_hi,page,pad,nq,nkv,window", [
    (1, 0, 1, 16, 0, 8, 2, 0), (3, 40, 20, 16, 5, 8, 8, 0), (70, 900, 3, 32, 0, 32, 8, 0), (300, 200, 40, 64, 100, 14, 2, 100),
    (1500, 60, 9, 256, 3, 3, 1, 17), (256, 500, 90, 16, 0, 32, 8, 0), (257, 500, 90, 16, 7, 14, 2, 64), (513, 70, 40, 64, 0, 8, 1, 0), (1024, 50, 30, 16, 2, 8, 2, 0),
    (4096, 33, 2, 16, 0, 32, 8, 0), (2, 9000, 6000, 128, 1, 71, 1, 0), (40, 100, 400, 16, 0, 6, 2, 64)])
def test_plan_of_ragged_steps(n, c_hi, f_hi, page, pad, nq, nkv, window):
    r = np.random.default_rng(n + page)
    c, f = _lengths(r, n, c_hi, f_hi)
    has, need = -(-c // page), -(-(c + f) // page)
    n_pages = int(need.sum()) + 3
    order = r.permutation(n_pages).astype(np.int32)
    table = np.full((n, int(need.max()) + 1), -5, np.int32)
    at = 0
    for s in range(n):
        table[s, : has[s]] = order[at: at + has[s]]
        at += has[s]
    _check_plan(c, f, table, order[at:], len(order) - at, int(f.sum()) + pad, page, n_pages, nq, nkv, window)


def test_plan_where_pages_or_rows_run_out():
    c, f = np.array([5, 0, 100, 17], np.int32), np.array([40, 33, 0, 50], np.int32)
    table = np.full((4, 8), -1, np.int32)
    table[0, 0], table[2, :7], table[3, :2] = 3, np.arange(4, 11), (11, 12)
    free = np.array([20, 21, 22, 23], np.int32)
    for n_free in (0, 1, 3, 4, 9, -2):
        _check_plan(c, f, table, free, n_free, 130, 16, 30)
        _check_plan(c, f, table, free, n_free, 60, 16, 30)           # rows behind the 60th are left out


def test_plan_of_bad_entries_and_lengths():
    """A page outside the pool gives no slot, lengths below zero count as none, positions behind the table's end have no page."""
    c, f = np.array([5, -3, 250, 1000], np.int32), np.array([4, 20, 30, 7], np.int32)
    table = np.full((4, 16), 7, np.int32)
    table[0, 0] = 99
    _check_plan(c, f, table, np.array([1, 2, 500, 3], np.int32), 4, 61, 16, 40)
    _check_plan(c, np.array([-1, 0, -9, 0], np.int32), table, np.array([1], np.int32), 1, 3, 16, 40)


def test_plan_of_no_sequences():
    _, got = _run_plan(np.zeros(0), np.zeros(0), np.zeros((0, 2)), np.array([4, 5]), 2, 5, 16, 8)
    cu, pos, slot, _, left, status = got
    assert cu.tolist() == [0] and not pos.any() and (slot == -1).all() and left[0] == 2 and status.tolist() == [0, 0, 0, 0]


def test_plan_again_gives_the_same_pages_and_counts_in_place():
    s = R.Step([30, 0, 7], [5, 40, 1], 16, 8, 2, 64, F16)
    first = {k: v.clone() for k, v in s.make_plan().items()}
    table = s.d_table.clone()
    left = s.device([len(s.free)])
    B.op_page_plan(s.plan, s.device(s.cached), s.device(s.fresh), s.d_table, s.device(s.free), left, left, s.d["cu"], s.d["pos"], s.d["slot"])
    assert torch.equal(table, s.d_table) and torch.equal(left, first["left"]) and all(torch.equal(first[k], s.d[k]) for k in ("cu", "pos", "slot"))


# ------------------------------------------------------------------------------------------------------------ finishing

def _finish_case(dtype, qkv_dtype, nq, nkv, hd, page, T, norm, far, seed=1, stride=0, interleaved=False, scale=2.0):
    g = torch.Generator().manual_seed(seed)
    n_pages = T // page + 4
    width = (nq + 2 * nkv) * hd
    big = (torch.randn(T, width + stride, generator=g) * scale).to(qkv_dtype).to(DEV)
    QKV = big[:, :width]
    pos = torch.randint(0, far, (T,), generator=g, dtype=torch.int32)
    slot = torch.randperm(n_pages * page, generator=g)[:T].to(torch.int32)
    if T > 5:
        slot[1], slot[3], slot[5] = -1, n_pages * page, 2 ** 31 - 1
    pool = torch.randn(n_pages, 2, nkv, page, hd, generator=g).to(dtype).to(DEV)
    K, V = (pool[:, 0], pool[:, 1]) if interleaved else (pool[:, 0].contiguous(), pool[:, 1].contiguous())
    gains = [(1 + 0.2 * torch.randn(hd, generator=g)).to(dtype) if norm else None for _ in range(2)]
    Q = torch.full((T + 2, nq * hd + stride), 7.0, dtype=dtype, device=DEV)
    want = R.finish(QKV.double().cpu(), pos, slot, K.double().cpu(), V.double().cpu(), *[x if x is None else x.double() for x in gains], 1e-6, 1e6, nq, nkv, hd)
    cache = B.KVCache(K, V)
    B.op_qkv_finish_paged(QKV, pos.to(DEV), slot.to(DEV), cache, *[x if x is None else x.to(DEV) for x in gains], 1e-6, 1e6, norm, Q[:T, : nq * hd])
    torch.cuda.synchronize()
    assert (Q[T:] == 7).all() and (Q[:, nq * hd:] == 7).all()
    # One rounding of the result; before it, in fp32: hd + 6 roundings in the norm's factor (half of them reach the root), two in its
    # application, three in the rotation, the cosine's and the sine's own: at most 2^-24 (hd / 2 + 12) of a + b, the pair's magnitudes
    u = R.HALF_STEP[dtype]
    for got, ref, name in zip((Q[:T, : nq * hd], K, V), want, "QKV"):
        half = ref.reshape(-1, hd)
        pair = (half.abs()[:, : hd // 2] + half.abs()[:, hd // 2:]).repeat(1, 2)
        room = (u * 1.01 * half.abs() + 2.0 ** -24 * (hd / 2 + 12) * 1.5 * pair + (2.0 ** -25 if dtype == F16 else 0)).reshape(ref.shape)
        if dtype == F16:
            ref = ref.clamp(-65504, 65504)
        R.close(got, ref, room)


@pytest.mark.parametrize("dtype,qkv_dtype", [(F32, F32), (BF16, F32), (BF16, BF16), (F16, F32), (F16, F16)])
@pytest.mark.parametrize("nq,nkv,hd,page,T,norm,far", [
    (16, 8, 128, 16, 1, True, 50), (4, 2, 64, 32, 7, True, 3000), (14, 2, 64, 64, 33, False, 200000), (32, 8, 128, 256, 130, True, 2000000),
    (3, 3, 128, 128, 1025, True, 9000), (5, 1, 64, 16, 2050, True, 100)])
def test_finish(dtype, qkv_dtype, nq, nkv, hd, page, T, norm, far):
    _finish_case(dtype, qkv_dtype, nq, nkv, hd, page, T, norm, far)


def test_finish_with_strides_interleaved_pages_and_small_heads():
    _finish_case(F16, F32, 8, 2, 128, 32, 77, True, 500, stride=12, interleaved=True)
    _finish_case(BF16, BF16, 8, 2, 64, 16, 41, False, 500, stride=4, interleaved=True)
    _finish_case(F32, F32, 6, 3, 32, 16, 50, True, 500, stride=8, interleaved=True)


def test_finish_saturates_half_and_keeps_nan():
    _finish_case(F16, F32, 2, 1, 64, 16, 3, False, 5, scale=1e5)
    QKV = torch.zeros(2, 4 * 64, dtype=F32, device=DEV)
    QKV[0, 5], QKV[1, 200] = float("nan"), float("nan")
    K, V = torch.zeros(1, 1, 16, 64, dtype=F16, device=DEV), torch.zeros(1, 1, 16, 64, dtype=F16, device=DEV)
    Q = torch.zeros(2, 2 * 64, dtype=F16, device=DEV)
    ints = lambda *a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
    B.op_qkv_finish_paged(QKV, ints(0, 1), ints(4, 5), B.KVCache(K, V), None, None, 1e-6, 1e6, False, Q)
    assert torch.isnan(Q).nonzero().tolist() == [[0, 5], [0, 37]]
    assert torch.isnan(V).nonzero().tolist() == [[0, 0, 5, 8]] and not torch.isnan(K).any()


# ------------------------------------------------------------------------------------------------------------ attention

LAYOUTS = [(F16, 16, 8, 128), (BF16, 32, 8, 128), (F16, 14, 2, 64), (BF16, 8, 1, 64), (F16, 3, 3, 128), (BF16, 71, 1, 128), (F16, 40, 2, 128),
           (F32, 4, 2, 64), (F32, 6, 3, 32), (F32, 10, 2, 128), (F32, 33, 1, 64)]


@pytest.mark.parametrize("dtype,nq,nkv,hd", LAYOUTS)
@pytest.mark.parametrize("cached,fresh,page", [
    ([0], [1], 16), ([0, 15, 16, 62, 63, 64, 65, 127], [1] * 8, 16), ([0, 31, 100, 0, 500], [2, 1, 3, 0, 1], 32),
    ([0, 10, 64, 130, 0], [63, 64, 65, 100, 0], 64), ([700, 0], [33, 200], 128), ([300, 5], [9, 70], 256)])
def test_attention(dtype, nq, nkv, hd, cached, fresh, page):
    """Lengths around the tiles' and pages' ends, single tokens, empty sequences, every head grouping; stale cache memory is NaN."""
    s = R.Step(cached, fresh, page, nq, nkv, hd, dtype, seed=nq + page, pad=3, stale=float("nan"))
    s.make_plan()
    s.check()


@pytest.mark.parametrize("dtype,nq,nkv,hd", [(F16, 16, 8, 128), (BF16, 8, 2, 128), (F16, 7, 1, 64), (F32, 4, 2, 64)])
@pytest.mark.parametrize("cached,fresh", [([20011], [1]), ([9000, 30, 4000], [1, 1, 5]), ([6000], [40]), ([5000, 0], [3, 300])])
def test_attention_over_split_keys(dtype, nq, nkv, hd, cached, fresh):
    s = R.Step(cached, fresh, 64, nq, nkv, hd, dtype, seed=7, pad=1, stale=float("inf"))
    s.make_plan()
    assert int(s.plan.buffer[: 64].view(torch.int32)[10]) > 0, "no keys were split"
    s.check()


@pytest.mark.parametrize("dtype,nq,nkv,hd", [(F16, 8, 8, 128), (BF16, 4, 1, 64), (F32, 2, 2, 64)])
@pytest.mark.parametrize("cached,fresh,width,window", [([255, 200, 100, 0], [1, 1, 40, 256], 16, 0), ([256, 200], [1, 72], 17, 0), ([9000, 255, 50], [1, 1, 90], None, 65),
                                                       ([9000, 255, 50], [1, 1, 90], None, 66), ([9000, 700], [1, 200], None, 200)])
def test_attention_around_the_fewest_tiles_that_are_cut(dtype, nq, nkv, hd, cached, fresh, width, window):
    """Caches and windows of four tiles are never cut, and their results are written without a joining launch; of five they may be."""
    s = R.Step(cached, fresh, 16, nq, nkv, hd, dtype, seed=11, window=window, width=width, stale=float("nan"))
    s.make_plan()
    tiles = min(s.table.shape[1] * 16 / 64, (window + 128 // (nq // nkv) + 62) // 64 + 1 if window else 1e9)
    assert tiles > 4 or int(s.plan.buffer[:64].view(torch.int32)[10]) == 0
    s.check()


@pytest.mark.parametrize("dtype,nq,nkv,hd", [(F16, 16, 8, 128), (BF16, 14, 2, 64), (F32, 6, 2, 64)])
@pytest.mark.parametrize("window,softcap,with_slopes,scale", [(1, 0.0, False, 0.0), (50, 0.0, False, 0.0), (64, 5.0, False, 0.3), (0, 30.0, True, 0.0),
                                                              (200, 0.0, True, 0.0), (5000, 2.0, True, 1.0)])
def test_attention_with_window_cap_and_slopes(dtype, nq, nkv, hd, window, softcap, with_slopes, scale):
    s = R.Step([0, 63, 300, 2000, 7000], [70, 1, 130, 1, 20], 16, nq, nkv, hd, dtype, seed=3, window=window, stale=float("nan"))
    s.make_plan()
    slopes = torch.exp2(-8.0 * torch.arange(1, nq + 1) / nq).to(DEV) if with_slopes else None
    s.check(scale, softcap, slopes)


@pytest.mark.parametrize("dtype,hd", [(F16, 128), (BF16, 64), (F32, 64)])
def test_attention_where_pages_are_missing(dtype, hd):
    """Entries outside the pool are keys that nobody sees; rows without any key give zeros; tokens behind the table's end see what it has."""
    s = R.Step([100, 40, 0, 3000, 90], [1, 30, 16, 2, 60], 16, 8, 2, hd, dtype, seed=5, stale=float("nan"))
    s.make_plan()
    bad = s.full_table.copy()
    bad[0, 2], bad[0, 6], bad[1, :] = -1, 2 ** 31 - 1, s.n_pages
    bad[2, 0], bad[3, 5:150], bad[4, 0] = -9, -1, -2 ** 31
    s.d_table = s.device(bad)
    s.check(table=bad)
    narrow = R.Step([100, 40], [1, 60], 16, 8, 2, hd, dtype, seed=5, width=4, spare=40)
    narrow.make_plan()
    narrow.check()


@pytest.mark.parametrize("dtype,hd", [(F16, 128), (BF16, 64), (F32, 64)])
@pytest.mark.parametrize("fresh", [[5], [90]])
def test_attention_keeps_what_is_not_seen_out(dtype, hd, fresh):
    """Values and keys that are not finite: rows in front of them are untouched, rows behind them get exactly their share."""
    s = R.Step([70], fresh, 16, 8, 2, hd, dtype, seed=9, stale=float("nan"))
    where = lambda p: (int(s.full_table[0, p // 16]), p % 16)  # noqa: E731
    for p, what, d in ((72, float("inf"), 3), (73, float("nan"), 9), (74, -float("inf"), 3), (74, float("inf"), 40)):
        pg, off = where(p)
        s.V[pg, 1, off, d] = what
    pg, off = where(73)
    s.K[pg, 0, off, 2] = float("nan")
    s.make_plan()
    out = s.attend()
    ref, room = R.attend(s.Q, s.K, s.V, s.full_table, s.cached, s.cu, s.nq, s.nkv, s.hd, dtype=dtype)
    if dtype == F16:                                             # half results saturate
        ref = torch.where(torch.isinf(ref), torch.sign(ref) * 65504.0, ref)
    R.close(out, ref, room)
    assert torch.isfinite(out[:2]).all()


@pytest.mark.parametrize("dtype,nq,hd", [(F16, 8, 128), (BF16, 14, 64), (F32, 8, 64)])
@pytest.mark.parametrize("fresh,window", [(1, 40), (3, 40), (8, 100), (60, 40), (150, 130)])
def test_attention_window_drops_values_that_are_not_finite(dtype, nq, hd, fresh, window):
    """Cached values and keys that are not finite, some behind the window of every token, some of a few, some of none."""
    s = R.Step([200], [fresh], 16, nq, 2, hd, dtype, seed=fresh, window=window, stale=float("nan"))
    first = 200 - window + 1                                     # the first position that the first token sees
    for p, what, d in ((first - 70, float("nan"), 1), (first - 1, float("inf"), 2), (first, -float("inf"), 3), (first + 2, float("nan"), 4),
                       (first + 5, float("inf"), 3), (199 + fresh // 2, float("inf"), 5)):
        s.V[int(s.full_table[0, p // 16]), 0, p % 16, d] = what
    s.K[int(s.full_table[0, (first - 1) // 16]), 1, (first - 1) % 16, 0] = float("inf")
    s.make_plan()
    out = s.attend()
    ref, room = R.attend(s.Q, s.K, s.V, s.full_table, s.cached, s.cu, nq, 2, hd, window=window, dtype=dtype)
    if dtype == F16:
        ref = torch.where(torch.isinf(ref), torch.sign(ref) * 65504.0, ref)
    R.close(out, ref, room)


@pytest.mark.parametrize("dtype,nq,nkv,hd", [(F16, 128, 1, 128), (BF16, 256, 256, 64), (F16, 33, 1, 64), (F32, 96, 1, 32)])
def test_attention_of_the_widest_head_groups(dtype, nq, nkv, hd):
    s = R.Step([0, 70, 300], [3, 1, 20], 32, nq, nkv, hd, dtype, seed=nq, stale=float("nan"))
    s.make_plan()
    s.check()


def test_attention_with_strided_rows_in_place_and_interleaved_pages():
    s = R.Step([100, 3], [40, 2], 32, 8, 2, 128, F16, seed=11, interleaved=True)
    s.make_plan()
    want = s.check()
    wide = torch.full((s.T, 8 * 128 + 2 * 128), 3.0, dtype=F16, device=DEV)
    wide[:, : 1024] = s.Q
    ws = B.attention_paged_workspace(s.plan, s.cache)
    B.op_attention_paged(s.plan, wide[:, :1024], s.cache, s.d_table, wide[:, :1024], ws)
    assert torch.equal(wide[:, :1024], want) and (wide[:, 1024:] == 3).all()


def test_attention_of_a_plan_of_another_shape_writes_nothing():
    s = R.Step([100, 3], [40, 2], 32, 8, 2, 128, F16, seed=11)
    s.make_plan()
    right, s.plan.buffer = s.plan.buffer, torch.zeros_like(s.plan.buffer)
    assert (s.attend() == 7).all()
    other = R.Step([100, 3], [40, 2], 32, 8, 2, 128, F16, seed=11, window=5)
    other.make_plan()
    s.plan.buffer = other.plan.buffer
    assert (s.attend() == 7).all()
    s.plan.buffer = right
    s.check()


def test_long_cache_beyond_32_bit_offsets():
    """Pages whose values lie more than 2^32 values into the pool."""
    n_pages, page, nkv, hd = 70000, 128, 4, 128                     # 4.6e9 values
    K = torch.zeros(n_pages, nkv, page, hd, dtype=F16, device=DEV)
    V = torch.zeros(n_pages, nkv, page, hd, dtype=F16, device=DEV)
    g = torch.Generator().manual_seed(2)
    ids = np.array([n_pages - 1, 0, n_pages - 2], np.int32)
    small = [torch.randn(3, nkv, page, hd, generator=g).to(F16) for _ in range(2)]
    for t, x in zip((K, V), small):
        t[torch.from_numpy(ids).long().to(DEV)] = x.to(DEV)
    fresh = 3
    cached = 3 * page - fresh
    plan = B.PagePlan(1, fresh, 8, nkv, page, n_pages, 3)
    ints = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
    table, cu, pos, slot, left = ints([ids.tolist()]), ints([0, 0]), ints([0] * fresh), ints([0] * fresh), ints([0])
    B.op_page_plan(plan, ints([cached]), ints([fresh]), table, ints([0]), ints([0]), left, cu, pos, slot)
    assert slot.tolist() == [(n_pages - 2) * page + page - fresh + i for i in range(fresh)]
    cache = B.KVCache(K, V)
    QKV = torch.randn(fresh, (8 + 2 * nkv) * hd, generator=g).to(F16).to(DEV)
    Q, out = torch.zeros(fresh, 8 * hd, dtype=F16, device=DEV), torch.zeros(fresh, 8 * hd, dtype=F16, device=DEV)
    B.op_qkv_finish_paged(QKV, pos, slot, cache, None, None, 1e-6, 1e6, False, Q)
    assert torch.equal(V[n_pages - 2, :, page - fresh:].transpose(0, 1).reshape(fresh, -1), QKV[:, (8 + nkv) * hd:])
    B.op_attention_paged(plan, Q, cache, table, out, B.attention_paged_workspace(plan, cache))
    near = [t[torch.from_numpy(ids).long().to(DEV)] for t in (K, V)]
    ref, room = R.attend(Q, *near, np.array([[0, 1, 2]]), [cached], [0, fresh], 8, nkv, hd, dtype=F16)
    R.close(out, ref, room)


# ------------------------------------------------------------------------------------------------------------ together

@pytest.mark.parametrize("dtype,nq,nkv,hd", [(F16, 8, 2, 128), (BF16, 14, 2, 64), (F32, 4, 2, 64)])
def test_reading_a_document_in_chunks_is_reading_it_whole(dtype, nq, nkv, hd):
    """Two sequences read in steps of uneven chunks, pages taken from one free list as they go: every step's results are those of the
    definition on everything read so far, in the caches' own rounded keys and values."""
    page, n_pages, width = 16, 60, 30
    g = torch.Generator().manual_seed(4)
    K, V = (torch.full((n_pages, nkv, page, hd), float("nan"), dtype=dtype, device=DEV) for _ in range(2))
    cache = B.KVCache(K, V)
    ints = lambda a: torch.as_tensor(np.asarray(a, np.int32)).to(DEV)  # noqa: E731
    table, free, n_free = ints(np.full((2, width), -1)), ints(np.random.default_rng(1).permutation(n_pages)), ints([n_pages])
    gains = [(1 + 0.1 * torch.randn(hd, generator=g)).to(dtype).to(DEV) for _ in range(2)]
    cached = np.zeros(2, np.int32)
    for fresh in ([130, 1], [1, 1], [0, 47], [3, 200], [1, 0], [100, 5]):
        T = sum(fresh)
        plan = B.PagePlan(2, T, nq, nkv, page, n_pages, width)
        cu, pos, slot, status = ints([0] * 3), ints([0] * T), ints([0] * T), ints([0] * 4)
        B.op_page_plan(plan, ints(cached), ints(fresh), table, free, n_free, n_free, cu, pos, slot, status)
        QKV = torch.randn(T, (nq + 2 * nkv) * hd, generator=g).to(DEV)
        Q, out = (torch.empty(T, nq * hd, dtype=dtype, device=DEV) for _ in range(2))
        before = K.double().cpu(), V.double().cpu()
        B.op_qkv_finish_paged(QKV, pos, slot, cache, *gains, 1e-6, 1e6, True, Q)
        B.op_attention_paged(plan, Q, cache, table, out, B.attention_paged_workspace(plan, cache))
        assert status.tolist()[:1] == [T] and status.tolist()[2:] == [0, 0]
        wq, wk, wv = R.finish(QKV.double().cpu(), pos.cpu(), slot.cpu(), *before, *[x.double().cpu() for x in gains], 1e-6, 1e6, nq, nkv, hd)
        for got, want in ((Q, wq), (K, wk), (V, wv)):
            R.close(got, want, want.abs() * R.HALF_STEP[dtype] * 1.01 + 2.0 ** -24 * (hd / 2 + 12) * 3 * want.abs().nan_to_num(0.0).max())
        ref, room = R.attend(Q, K, V, table.cpu().numpy(), cached, cu.cpu().numpy(), nq, nkv, hd, dtype=dtype)
        R.close(out, ref, room)
        cached = cached + np.array(fresh, np.int32)


def test_a_captured_step_replays_on_new_lengths():
    """Plan, finishing and attention of one step in a graph: replayed on other lengths, lists and values, with eager work between the
    replays, each replay gives the bits of the same calls made eagerly."""
    nq, nkv, hd, page, n_pages, width, n, T = 8, 2, 128, 16, 400, 100, 5, 150
    ints = lambda a: torch.as_tensor(np.asarray(a, np.int32)).to(DEV)  # noqa: E731
    g = torch.Generator().manual_seed(8)
    pool = [torch.randn(n_pages, nkv, page, hd, generator=g).to(F16).to(DEV) for _ in range(2)]
    order = np.random.default_rng(3).permutation(n_pages)

    def state():
        s = {"K": pool[0].clone(), "V": pool[1].clone(), "cached": ints([0] * n), "fresh": ints([0] * n), "table": ints(np.zeros((n, width))),
             "free": ints([0] * n_pages), "n_free": ints([0]), "cu": ints([0] * (n + 1)), "pos": ints([0] * T), "slot": ints([0] * T),
             "QKV": torch.zeros(T, (nq + 2 * nkv) * hd, device=DEV), "Q": torch.zeros(T, nq * hd, dtype=F16, device=DEV),
             "out": torch.zeros(T, nq * hd, dtype=F16, device=DEV)}
        s["cache"], s["plan"] = B.KVCache(s["K"], s["V"]), B.PagePlan(n, T, nq, nkv, page, n_pages, width)
        s["ws"] = B.attention_paged_workspace(s["plan"], s["cache"])
        return s

    def calls(s):
        B.op_page_plan(s["plan"], s["cached"], s["fresh"], s["table"], s["free"], s["n_free"], s["n_free"], s["cu"], s["pos"], s["slot"])
        B.op_qkv_finish_paged(s["QKV"], s["pos"], s["slot"], s["cache"], None, None, 1e-6, 1e6, False, s["Q"])
        B.op_attention_paged(s["plan"], s["Q"], s["cache"], s["table"], s["out"], s["ws"])

    def load(s, k):
        r = np.random.default_rng(100 + k)
        c = r.integers(0, 1000, n)
        f = r.multinomial(T - int(r.integers(0, 40)), np.ones(n) / n) if k % 2 else np.array([1, 1, 0, 1, 1])
        table, at = np.full((n, width), -1), 0
        for i in range(n):
            m = -(-int(c[i]) // page)
            table[i, :m] = order[at: at + m]
            at += m
        free = np.zeros(n_pages)
        free[: n_pages - at] = order[at:]
        for key, v in (("cached", c), ("fresh", f), ("table", table), ("free", free), ("n_free", [n_pages - at])):
            s[key].copy_(ints(v))
        s["QKV"].copy_(torch.randn(T, (nq + 2 * nkv) * hd, generator=torch.Generator().manual_seed(k)))
        s["K"].copy_(pool[0])
        s["V"].copy_(pool[1])
        s["out"].fill_(5.0)
        s["Q"].fill_(5.0)

    graphed, eager = state(), state()
    load(graphed, 0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls(graphed)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(graphed)
    for k in range(1, 6):
        load(graphed, k)
        load(eager, k)
        graph.replay()
        calls(eager)
        torch.cuda.synchronize()
        for name in ("table", "n_free", "cu", "pos", "slot", "Q", "K", "V", "out"):
            assert torch.equal(graphed[name], eager[name]), (k, name)


@pytest.mark.parametrize("dtype,nq,hd", [(F16, 8, 128), (BF16, 14, 64), (F32, 8, 64)])
@pytest.mark.parametrize("fresh", [1, 3, 90])
@pytest.mark.parametrize("factor,rising", [(0.05, True), (30.0, False), (30.0, True), (3000.0, True)])
def test_attention_of_small_and_large_scores_that_rise(dtype, nq, hd, fresh, factor, rising):
    """Scores whose maxima stay close together, or rise from key to key by little or by much: what the exponents are taken from moves late,
    once, or in every tile."""
    s = R.Step([1500], [fresh], 64, nq, 2, hd, dtype, seed=5, stale=float("nan"))
    s.make_plan()
    up = torch.linspace(0.2, 1.0, 1500 + fresh).to(DEV) if rising else torch.ones(1500 + fresh, device=DEV)
    pages = s.d_table[0].long()[torch.arange(1500 + fresh, device=DEV) // 64]
    key = s.Q[0, :hd].float().abs() + 0.1
    s.K[pages, :, torch.arange(1500 + fresh, device=DEV) % 64] = (up[:, None, None] * key).to(dtype).expand(-1, 2, -1)
    s.Q.copy_((s.Q.float().abs() + 0.1).to(dtype))
    s.check(factor / hd, 0.0, None)


@pytest.mark.parametrize("dtype,nq,hd", [(F16, 8, 128), (BF16, 14, 64), (F32, 8, 64)])
@pytest.mark.parametrize("fresh", [1, 3, 90])
@pytest.mark.parametrize("power", [6, 12, 20, 24])
def test_attention_of_far_scores(dtype, nq, hd, fresh, power):
    """Scores far from zero and from each other: the keys with the largest share all the weight equally."""
    n = 700 + fresh
    s = R.Step([700], [fresh], 64, nq, 2, hd, dtype, seed=6, stale=float("nan"))
    s.make_plan()
    pages, at = s.d_table[0].long()[torch.arange(n, device=DEV) // 64], torch.arange(n, device=DEV) % 64
    size = 2.0 ** (min(power, 14) if dtype is F16 else power)
    k = torch.zeros(n, hd, device=DEV)
    k[:, 0] = torch.arange(n, device=DEV) % 3 * size                          # 0, 1 and 2 times: every third key has the largest score
    s.K[pages, :, at] = k.to(dtype)[:, None].expand(-1, 2, -1)
    s.Q.zero_()
    s.Q[:, ::hd] = 2.0 ** (min(power, 15) if dtype is F16 else power)
    out = s.attend()
    top = torch.arange(n, device=DEV) % 3 == 2
    for h in range(nq):
        v = s.V[pages, h // (nq // 2), at].double()
        for i in range(fresh):
            seen = top & (torch.arange(n, device=DEV) <= 700 + i)
            want = v[seen].mean(0)
            step = 2 * R.HALF_STEP[dtype] * want.abs() + n * 2.0 ** -24 * v.abs().max()     # its rounding, and the sums'
            assert ((out[i, h * hd:(h + 1) * hd].double() - want).abs() <= step).all()


@pytest.mark.parametrize("dtype,nq,hd", [(F16, 8, 128), (BF16, 14, 64), (F32, 8, 64)])
@pytest.mark.parametrize("cached,fresh,window", [([500], [90], 0), ([500], [90], 100), ([3, 500], [70, 3], 0), ([9000], [40], 0)])
def test_attention_of_far_rows_beside_near_ones(dtype, nq, hd, cached, fresh, window):
    """One head of a group has scores of some 2^17, the others of a few; eight keys of a page have twice the others'."""
    s = R.Step(cached, fresh, 16, nq, 2, hd, dtype, seed=8, window=window, stale=float("nan"))
    s.make_plan()
    s.Q[:, :hd] *= 4096.0
    s.K[:, :, : 8] *= 2.0
    s.check()


def test_same_inputs_same_bits():
    s = R.Step([9000, 30, 500], [1, 1, 70], 16, 8, 2, 128, BF16, seed=2)
    s.make_plan()
    first = s.attend()
    for _ in range(3):
        assert torch.equal(first, s.attend())


def test_plan_of_the_largest_step():
    """As many sequences and rows as a step may have."""
    r = np.random.default_rng(1)
    f = r.integers(0, 512, 4096)
    f[7] += 1048576 - f.sum()
    c = r.integers(0, 40, 4096)
    has, need = -(-c // 64), -(-(c + f) // 64)
    table = np.full((4096, int(need.max())), -1, np.int32)
    order, at = r.permutation(int(need.sum())).astype(np.int32), 0
    for s in range(4096):
        table[s, : has[s]] = order[at: at + has[s]]
        at += has[s]
    _check_plan(c.astype(np.int32), f.astype(np.int32), table, order[at:], len(order) - at, 1048576, 64, len(order), 32, 8)


def test_refusals_of_tensors():
    """Types, shapes, strides and devices that do not fit are refused before anything is launched."""
    s = R.Step([20], [3], 16, 4, 2, 64, F16)
    out = s.make_plan()
    ints = lambda n: torch.zeros(n, dtype=torch.int32, device=DEV)  # noqa: E731
    good = [s.device(s.cached), s.device(s.fresh), s.d_table, s.device(s.free), s.device([len(s.free)]), out["left"], out["cu"], out["pos"], out["slot"]]
    for i, bad in ((0, ints(1).long()), (1, ints(0)), (2, s.d_table.cpu()), (2, ints(0)), (4, ints(0)), (6, ints(1)), (7, ints(2)), (8, ints(6)[::2]), (5, ints(1).float())):
        with pytest.raises(B.PrismError) as e:
            B.op_page_plan(s.plan, *good[:i], bad, *good[i + 1:])
        assert e.value.code == B.EINVAL
    QKV, Q, g = torch.zeros(3, 8 * 64, device=DEV), torch.zeros(3, 4 * 64, dtype=F16, device=DEV), torch.ones(64, dtype=F16, device=DEV)
    finish = lambda QKV=QKV, pos=out["pos"], slot=out["slot"], cache=s.cache, a=g, b=g, Q=Q: B.op_qkv_finish_paged(QKV, pos, slot, cache, a, b, 1e-6, 1e6, True, Q)  # noqa: E731
    finish()
    for bad in (dict(QKV=QKV.bfloat16()), dict(QKV=QKV[:, :500]), dict(QKV=QKV.T), dict(QKV=QKV[:2]), dict(QKV=QKV.cpu()), dict(pos=ints(2)), dict(slot=ints(3).long()),
                dict(a=None), dict(b=g.float()), dict(a=g[:32]), dict(Q=Q.float()), dict(Q=torch.zeros(3, 250, dtype=F16, device=DEV)), dict(QKV=QKV.view(-1))):
        with pytest.raises(B.PrismError) as e:
            finish(**bad)
        assert e.value.code == B.EINVAL, bad
    ws = B.attention_paged_workspace(s.plan, s.cache)
    attend = lambda Q=s.Q, table=s.d_table, o=Q, ws=ws, **more: B.op_attention_paged(s.plan, Q, s.cache, table, o, ws, **more)  # noqa: E731
    attend()
    for bad in (dict(Q=s.Q.bfloat16()), dict(Q=s.Q[:2]), dict(Q=s.Q[:, :128]), dict(o=Q.cpu()), dict(o=Q.T), dict(table=s.d_table.long()), dict(table=ints(1)), dict(ws=ws[:16]),
                dict(ws=ws[1:]), dict(ws=ws.cpu()), dict(slopes=torch.zeros(3, device=DEV)), dict(slopes=torch.zeros(4, dtype=F16, device=DEV)), dict(scale=-1.0), dict(softcap=-2.0)):
        with pytest.raises(B.PrismError) as e:
            attend(**bad)
        assert e.value.code == B.EINVAL, bad
    for K, V in ((torch.zeros(2, 2, 16, 64, device=DEV), torch.zeros(2, 2, 16, 64, dtype=F16, device=DEV)), (torch.zeros(2, 2, 16, 64).half(), torch.zeros(2, 2, 16, 64).half()),
                 (torch.zeros(2, 2, 64, 16, device=DEV).transpose(2, 3), torch.zeros(2, 2, 16, 64, device=DEV)), (torch.zeros(2, 2, 16, 64, device=DEV),) * 1 + (torch.zeros(3, 2, 16, 64, device=DEV),),
                 (torch.zeros(2, 2, 16, 64, dtype=torch.float64, device=DEV),) * 2, (torch.zeros(2, 16, 64, device=DEV),) * 2):
        with pytest.raises(B.PrismError):
            B.KVCache(K, V)
    for bad in (dict(n_seqs=-1), dict(page_size=24), dict(n_q_heads=5), dict(max_pages=0)):
        v = dict(n_seqs=1, n_tokens=3, n_q_heads=4, n_kv_heads=2, page_size=16, n_pages=4, max_pages=2)
        v.update(bad)
        with pytest.raises(B.PrismError):
            B.PagePlan(**v)
    torch.cuda.synchronize()
