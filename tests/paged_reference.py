"""The operators on a paged cache in 64 bits, written out from their definitions, and how far a kernel's result may be from them."""
import math

import numpy as np
import torch

from paper_2510_15620_amd import binding as B

DEV = "cuda"
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def plan(cached, fresh, table, free, n_free, T, page, n_pages):
    """-> cu, pos, slot, table, n_free_left, status (python and numpy integers)."""
    table = np.array(table, np.int64).reshape(len(cached), -1)
    width = table.shape[1]
    n_free = min(max(int(n_free), 0), len(free))
    left, missing, row, cu, asked = n_free, 0, 0, [0], 0
    pos, slot = np.zeros(T, np.int64), np.full(T, -1, np.int64)
    for s, (c, f) in enumerate(zip(cached, fresh)):
        c, f = max(int(c), 0), max(int(f), 0)
        asked += f
        f = min(f, T - row)
        for idx in range(-(-c // page), min(width, -(-(c + f) // page)) if f else 0):
            if left > 0:
                left -= 1
                table[s, idx] = free[left]
            else:
                table[s, idx] = -1
                missing += 1
        for i in range(f):
            p = c + i
            pos[row + i] = p
            if p // page < width and 0 <= table[s, p // page] < n_pages:
                slot[row + i] = table[s, p // page] * page + p % page
        row += f
        cu.append(row)
    return cu, pos, slot, table, left, [row, n_free - left, missing, asked - row]


def finish(QKV, pos, slot, K, V, q_gain, k_gain, eps, base, nq, nkv, hd):
    """QKV [T, (nq + 2 nkv) * hd]; K, V [pages, nkv, page, hd]; gains None: no norm.  All float64 in and out."""
    x = QKV.reshape(len(pos), nq + 2 * nkv, hd)
    K, V, half, page = K.clone(), V.clone(), hd // 2, K.shape[2]
    out = []
    for h in range(nq + nkv):
        y, gain = x[:, h], q_gain if h < nq else k_gain
        if gain is not None:
            y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * gain
        theta = torch.tensor([base ** (-2.0 * i / hd) for i in range(half)], dtype=torch.float64)
        angle = pos.double()[:, None] * theta
        a, b = y[:, :half], y[:, half:]
        out.append(torch.cat([a * torch.cos(angle) - b * torch.sin(angle), b * torch.cos(angle) + a * torch.sin(angle)], -1))
    for t, s in enumerate(slot.tolist()):
        if 0 <= s < K.shape[0] * page:
            for h in range(nkv):
                K[s // page, h, s % page], V[s // page, h, s % page] = out[nq + h][t], x[t, nq + nkv + h]
    return torch.stack(out[:nq], 1).reshape(len(pos), nq * hd), K, V


def attend(Q, K, V, table, cached, cu, nq, nkv, hd, scale=0.0, cap=0.0, window=0, slopes=None, dtype=torch.float32):
    """Results [rows of the sequences, nq * hd] in float64 and how far a kernel's result may be from each (float64, same shape).

    The bound: a score's fp32 sum of hd products is off by (hd + 2) 2^-24 of the sum of their magnitudes, its further steps (scale, cap,
    slope, subtraction of the maximum, exponential) by 2^-20 of the magnitudes that they handle, cap included; a weight is then off by
    that much relatively, for 16-bit types also by half a step of its own rounding (e), and the sums over n keys by n 2^-24.  Numerator
    and denominator share the weights, so the result is off by e times the spread of V, at most 2 max |V|, and its own half step."""
    T, G, page = int(cu[-1]), nq // nkv, K.shape[2]
    out, room = torch.zeros(T, nq, hd, dtype=torch.float64), torch.zeros(T, nq, 1, dtype=torch.float64)
    u = HALF_STEP[dtype]
    K, V, Q = K.double().cpu(), V.double().cpu(), Q.double().cpu().reshape(-1, nq, hd)
    scale = scale or 1.0 / math.sqrt(hd)
    for s in range(len(cached)):
        r0, r1, c = int(cu[s]), int(cu[s + 1]), max(int(cached[s]), 0)
        if r0 == r1:
            continue
        n = min(c + r1 - r0, table.shape[1] * page)
        key = torch.arange(n)
        pages = torch.as_tensor(np.asarray(table[s]), dtype=torch.int64)[key // page]
        there = (pages >= 0) & (pages < K.shape[0])
        pages = torch.where(there, pages, 0)
        p = torch.arange(c, c + r1 - r0)[:, None]
        see = there & (key <= p)
        if window:
            see = see & (key > p - window)
        for h in range(nkv):
            k, v = K[pages, h, key % page], V[pages, h, key % page]
            any_row = see.any(0)
            k, v = torch.where(any_row[:, None], k, 0.0), torch.where(any_row[:, None], v, 0.0)
            q = Q[r0:r1, h * G:(h + 1) * G].transpose(0, 1)                       # [G, rows, hd]
            x = q @ k.T * scale
            err = (hd + 2) * 2.0 ** -24 * ((q.abs() @ k.abs().T) * abs(scale)).nan_to_num(0.0, 0.0, 0.0).amax((-2, -1), keepdim=True)
            size = x.abs().nan_to_num(0.0, 0.0, 0.0).amax((-2, -1), keepdim=True) + cap
            if cap:
                x = cap * torch.tanh(x / cap)
            if slopes is not None:
                bias = slopes.double().cpu()[h * G:(h + 1) * G, None, None] * (p - key)
                x, size = x - bias, size + bias.abs().amax((-2, -1), keepdim=True)
            x = torch.where(see, x, -math.inf)
            top = x.amax(-1, keepdim=True)
            w = torch.exp(x - torch.where(torch.isinf(top) & (top < 0), 0.0, top))
            total = w.sum(-1, keepdim=True)
            if not torch.isfinite(v).all():                                       # 0 times what a row does not see is nothing
                o = torch.stack([torch.stack([(w[g, i, see[i]][:, None] * v[see[i]]).sum(0) for i in range(r1 - r0)]) for g in range(G)])
            else:
                o = w @ v
            o = torch.where(total == 0, torch.zeros((), dtype=torch.float64), o / total)
            e = err + size * 2.0 ** -20 + n * 2.0 ** -24 + (u if dtype != torch.float32 else 2.0 ** -22)
            big = v.abs().nan_to_num(0.0, 0.0, 0.0).max()
            out[r0:r1, h * G:(h + 1) * G] = o.transpose(0, 1)
            room[r0:r1, h * G:(h + 1) * G] = (2 * e * big * 1.05).expand(G, r1 - r0, 1).transpose(0, 1)
    room = room + u * 1.01 * out.abs().nan_to_num(0.0, 0.0, 0.0) + (2.0 ** -25 if dtype == torch.float16 else 0.0)   # half's subnormal step
    return out.reshape(T, nq * hd), room.expand(T, nq, hd).reshape(T, nq * hd)


def close(got, ref, room):
    """Where the definition's result is not finite, the kernel's is the same; elsewhere it is within `room`."""
    got, ref = got.double().cpu().reshape(-1), ref.reshape(-1)
    fine = torch.isfinite(ref)
    assert torch.equal(torch.isnan(got[~fine]), torch.isnan(ref[~fine]))
    inf = torch.isinf(ref)
    assert torch.equal(torch.sign(got[inf]), torch.sign(ref[inf]))
    off = (got[fine] - ref[fine]).abs() - room.reshape(-1)[fine]
    assert not torch.isnan(off).any(), "NaN where the result is finite"
    assert off.numel() == 0 or off.max() <= 0, f"off by {(got[fine] - ref[fine]).abs().max():.3g}, {off.max():.3g} more than it may be"


class Step:
    """A step on a cache of its own: shuffled pages, filled with `stale` wherever no token of the step's sequences is."""

    def __init__(self, cached, fresh, page, nq, nkv, hd, dtype, seed=0, pad=0, window=0, stale=0.0, spare=3, width=None, interleaved=False):
        r = np.random.default_rng(seed)
        g = torch.Generator().manual_seed(seed)
        self.cached, self.fresh = np.asarray(cached, np.int32), np.asarray(fresh, np.int32)
        self.page, self.nq, self.nkv, self.hd, self.dtype, self.window = page, nq, nkv, hd, dtype, window
        total = self.cached + self.fresh
        need = -(-total // page)
        self.n_pages = int(need.sum()) + spare
        order = r.permutation(self.n_pages)
        self.table = np.full((len(total), width or max(1, int(need.max(initial=1)))), -1, np.int32)
        at = 0
        for s, n in enumerate(np.minimum(-(-self.cached // page), self.table.shape[1])):
            self.table[s, :n] = order[at: at + n]
            at += n
        self.free = order[at:].astype(np.int32)
        self.T = int(self.fresh.sum()) + pad
        self.cu, self.pos, self.slot, self.full_table, self.left, self.status = plan(
            self.cached, self.fresh, self.table, self.free, len(self.free), self.T, page, self.n_pages)
        shape = (self.n_pages, nkv, page, hd)
        both = torch.full((2, *shape), stale, dtype=torch.float32)
        for s in range(len(total)):
            for i, pg in enumerate(self.full_table[s]):
                n = min(page, int(total[s]) - i * page)
                if 0 <= pg < self.n_pages and n > 0:
                    both[:, pg, :, :n] = torch.randn(2, nkv, n, hd, generator=g)
        if interleaved:
            pool = both.transpose(0, 1).contiguous().to(dtype).to(DEV)
            self.K, self.V = pool[:, 0], pool[:, 1]
        else:
            self.K, self.V = both.to(dtype).to(DEV)
        self.Q = torch.randn(self.T, nq * hd, generator=g).to(dtype).to(DEV)

    def device(self, a):
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)

    def make_plan(self):
        self.cache = B.KVCache(self.K, self.V)
        self.plan = B.PagePlan(len(self.cached), self.T, self.nq, self.nkv, self.page, self.n_pages, self.table.shape[1], window=self.window)
        self.d_table = self.device(self.table)
        out = {k: torch.full((n,), -77, dtype=torch.int32, device=DEV)
               for k, n in (("left", 1), ("cu", len(self.cached) + 1), ("pos", self.T), ("slot", self.T), ("status", 4))}
        B.op_page_plan(self.plan, self.device(self.cached), self.device(self.fresh), self.d_table, self.device(self.free),
                       self.device([len(self.free)]), out["left"], out["cu"], out["pos"], out["slot"], out["status"])
        self.d = out
        return out

    def attend(self, scale=0.0, softcap=0.0, slopes=None, fill=7.0):
        self.workspace = B.attention_paged_workspace(self.plan, self.cache)
        out = torch.full((self.T, self.nq * self.hd), fill, dtype=self.dtype, device=DEV)
        B.op_attention_paged(self.plan, self.Q, self.cache, self.d_table, out, self.workspace, scale, softcap, slopes)
        torch.cuda.synchronize()
        return out

    def check(self, scale=0.0, softcap=0.0, slopes=None, table=None):
        out = self.attend(scale, softcap, slopes)
        ref, room = attend(self.Q, self.K, self.V, self.full_table if table is None else table, self.cached, self.cu, self.nq, self.nkv, self.hd,
                           scale, softcap, self.window, slopes, self.dtype)
        close(out[: self.cu[-1]], ref, room)
        assert (out[self.cu[-1]:] == 7.0).all(), "rows behind the last sequence were written"
        return out
