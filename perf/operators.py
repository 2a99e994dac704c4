"""Operators on a paged key/value cache, as cases with stated inputs, plain forms and exact results.

Three kinds of work, one operator each: `plan` (positions, cache slots and block tables of a step from the sequences' lengths),
`finish` (per-head norm and rotation of a projection, keys and values appended to their pages) and `attend` (attention of the step's
tokens over the cache).  Lengths are a function of the case; values, the order of the pages and the free list of the seed.

The cache holds pages [kv head][slot][head_dim] for keys and the same for values; sequence s finds the keys of positions
i * page .. (i + 1) * page - 1 in page table[s][i].  Of every sequence `cached` tokens are in the cache before the step, which
brings `fresh` more.
"""
import math
import zlib

import numpy as np
import torch

own = False

TORCH = {"f16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
EPS, BASE = 1e-6, 1e6


def listed():
    return [
        # a step of a small serving batch: 24 sequences, one new token each
        {"name": "plan_step", "kind": "plan", "q_heads": 16, "kv_heads": 8, "page": 16, "seqs": 24, "ones": 24, "fresh_lo": 1,
         "fresh_hi": 1, "ctx_lo": 0, "ctx_hi": 3000, "pad": 0},
        # a pool of 500 documents read for the first time, ragged lengths, rows padded to a round number
        {"name": "plan_pool", "kind": "plan", "q_heads": 32, "kv_heads": 8, "page": 64, "seqs": 500, "ones": 0, "fresh_lo": 32,
         "fresh_hi": 640, "ctx_lo": 0, "ctx_hi": 100, "pad": 37},
        # the smallest append: 7 tokens of the 0.6B head layout, latency
        {"name": "finish_step", "kind": "finish", "dtype": "f16", "input": "fp32", "q_heads": 16, "kv_heads": 8, "head_dim": 128,
         "page": 16, "norm": True, "seqs": 7, "ones": 7, "fresh_lo": 1, "fresh_hi": 1, "ctx_lo": 50, "ctx_hi": 1200},
        # a chunk of the 8B head layout at positions far into a long context, a 16-bit projection
        {"name": "finish_chunk_far", "kind": "finish", "dtype": "bf16", "input": "bf16", "q_heads": 32, "kv_heads": 8, "head_dim": 128,
         "page": 64, "norm": True, "seqs": 3, "ones": 0, "fresh_lo": 500, "fresh_hi": 900, "ctx_lo": 60000, "ctx_hi": 120000},
        # a whole pool's first pass, 8B head layout, fp32 projection
        {"name": "finish_pool", "kind": "finish", "dtype": "f16", "input": "fp32", "q_heads": 32, "kv_heads": 8, "head_dim": 128,
         "page": 32, "norm": True, "seqs": 60, "ones": 0, "fresh_lo": 256, "fresh_hi": 992, "ctx_lo": 0, "ctx_hi": 64},
        # single tokens of three short sequences, 0.6B head layout: the smallest call, latency
        {"name": "attend_few", "kind": "attend", "dtype": "f16", "q_heads": 16, "kv_heads": 8, "head_dim": 128, "page": 16,
         "seqs": 3, "ones": 3, "fresh_lo": 1, "fresh_hi": 1, "ctx_lo": 100, "ctx_hi": 900, "window": 0, "cap": 0.0, "slopes": False},
        # single tokens of an ordinary serving batch, 8B head layout: bandwidth
        {"name": "attend_batch", "kind": "attend", "dtype": "bf16", "q_heads": 32, "kv_heads": 8, "head_dim": 128, "page": 16,
         "seqs": 100, "ones": 100, "fresh_lo": 1, "fresh_hi": 1, "ctx_lo": 300, "ctx_hi": 8000, "window": 0, "cap": 0.0, "slopes": False},
        # one token of one very long sequence: the key axis has to be split
        {"name": "attend_long", "kind": "attend", "dtype": "f16", "q_heads": 32, "kv_heads": 8, "head_dim": 128, "page": 64,
         "seqs": 1, "ones": 1, "fresh_lo": 1, "fresh_hi": 1, "ctx_lo": 150001, "ctx_hi": 150001, "window": 0, "cap": 0.0, "slopes": False},
        # chunks of long documents over what was read of them before: matrix work
        {"name": "attend_chunks", "kind": "attend", "dtype": "f16", "q_heads": 32, "kv_heads": 8, "head_dim": 128, "page": 64,
         "seqs": 4, "ones": 0, "fresh_lo": 1500, "fresh_hi": 2048, "ctx_lo": 2000, "ctx_hi": 12000, "window": 0, "cap": 0.0, "slopes": False},
        # one document's chunk beside 30 sequences that go on token by token
        {"name": "attend_mixed", "kind": "attend", "dtype": "bf16", "q_heads": 32, "kv_heads": 8, "head_dim": 128, "page": 32,
         "seqs": 31, "ones": 30, "fresh_lo": 500, "fresh_hi": 500, "ctx_lo": 200, "ctx_hi": 4000, "window": 0, "cap": 0.0, "slopes": False},
        # capped scores and distance slopes under a sliding window, 7 query heads per KV head of 64
        {"name": "attend_window", "kind": "attend", "dtype": "bf16", "q_heads": 14, "kv_heads": 2, "head_dim": 64, "page": 16,
         "seqs": 9, "ones": 0, "fresh_lo": 130, "fresh_hi": 700, "ctx_lo": 0, "ctx_hi": 3000, "window": 1000, "cap": 30.0, "slopes": True},
        # fp32 mode, the tiny configuration's heads, chunks of ordinary passages
        {"name": "attend_fp32", "kind": "attend", "dtype": "fp32", "q_heads": 4, "kv_heads": 2, "head_dim": 64, "page": 16,
         "seqs": 40, "ones": 5, "fresh_lo": 16, "fresh_hi": 300, "ctx_lo": 0, "ctx_hi": 600, "window": 0, "cap": 0.0, "slopes": False},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["plan", "finish", "attend", "attend", "attend"])
    kv = rng.choice([1, 2, 3, 8])
    case = {"kind": kind, "q_heads": kv * rng.choice([1, 2, 4, 4, 7, 8] if kv < 8 else [1, 2, 4]), "kv_heads": kv,
            "page": rng.choice([16, 32, 64, 128, 256])}
    if kind == "plan":
        n = _log_int(rng, 1, 2000)
        hi = _log_int(rng, 1, 150000 // n)
        return {**case, "seqs": n, "ones": rng.randint(0, n), "fresh_lo": rng.randint(0, 1) * hi // 2, "fresh_hi": hi, "ctx_lo": 0,
                "ctx_hi": _log_int(rng, 1, 20000), "pad": rng.randint(0, 50)}
    case["dtype"] = rng.choice(["f16", "bf16", "fp32"])
    case["head_dim"] = rng.choice([64, 128, 128])
    if kind == "finish":
        n = _log_int(rng, 1, 200)
        hi = _log_int(rng, 1, 30000 // n)
        return {**case, "input": rng.choice(["fp32", case["dtype"]]), "norm": rng.random() < 0.8, "seqs": n, "ones": rng.randint(0, n),
                "fresh_lo": max(1, hi // 3), "fresh_hi": hi, "ctx_lo": 0, "ctx_hi": _log_int(rng, 1, 120000 // n)}
    n = _log_int(rng, 1, 100)
    ones = rng.choice([0, n // 2, n])
    hi = 1 if ones == n else _log_int(rng, 2, 2048 if n <= 4 else max(8, 4000 // n))
    ctx = _log_int(rng, 16, min(150000, 400000 // n) if hi == 1 else min(8000, 4000000 // (hi * n) + 16))
    if case["dtype"] == "fp32":
        ctx = min(ctx, 4000)
    return {**case, "seqs": n, "ones": ones, "fresh_lo": max(1, hi // 3), "fresh_hi": hi, "ctx_lo": ctx // 5, "ctx_hi": ctx,
            "window": rng.choice([0, 0, _log_int(rng, 16, 4096)]), "cap": rng.choice([0.0, 0.0, 20.0]), "slopes": rng.random() < 0.3}


def _lengths(case):
    """Tokens cached and fresh per sequence; the first `ones` sequences bring one token."""
    key = ",".join("%s=%s" % (k, case[k]) for k in ("seqs", "ones", "fresh_lo", "fresh_hi", "ctx_lo", "ctx_hi", "page"))
    r = np.random.RandomState(zlib.crc32(key.encode()))
    cached = r.randint(case["ctx_lo"], case["ctx_hi"] + 1, case["seqs"])
    fresh = r.randint(case["fresh_lo"], case["fresh_hi"] + 1, case["seqs"])
    fresh[: case["ones"]] = 1
    return cached.astype(np.int32), fresh.astype(np.int32)


def _pages(case, cached, fresh, seed):
    """Page tables before the step and in it, in a shuffled order of the pool's pages, and the free list before the step, from whose
    end the step's new pages come in order of sequence, then position."""
    P = case["page"]
    has, need = -(-cached // P), -(-(cached + fresh) // P)
    order = np.random.RandomState(seed % (1 << 32)).permutation(int(need.sum()) + 5).astype(np.int32)
    before = np.full((len(cached), int(need.max()) + 1), -1, np.int32)

    def entries(lo, hi):
        seq = np.repeat(np.arange(len(cached)), hi - lo)
        return seq, np.arange(len(seq)) - np.concatenate([[0], np.cumsum(hi - lo)])[seq] + lo[seq]

    old, new = entries(0 * has, has), entries(has, need)
    before[old] = order[: len(old[0])]
    free, within = order[len(old[0]):], before.copy()
    within[new] = free[::-1][: len(new[0])]
    return before, within, free


def prepare(case, seed):
    cached, fresh = _lengths(case)
    kind, P, nq, nkv = case["kind"], case["page"], case["q_heads"], case["kv_heads"]
    before, table, free = _pages(case, cached, fresh, seed)
    n_pages = int((table >= 0).sum()) + 5
    T = int(fresh.sum()) + case.get("pad", 0)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to("cuda")  # noqa: E731
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case, "cached": dev(cached), "fresh": dev(fresh), "table": dev(before if kind == "plan" else table), "T": T, "n_pages": n_pages,
         "free": dev(free), "n_free": dev(np.array([len(free)], np.int32))}
    empty = lambda *shape, dtype=torch.int32: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    if kind == "plan":
        s.update(left=empty(1), cu=empty(len(fresh) + 1), pos=empty(T), slot=empty(T), status=empty(4))
    else:
        dt, hd = TORCH[case["dtype"]], case["head_dim"]
        randn = lambda *shape: torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)  # noqa: E731
        s["K"], s["V"] = (randn(n_pages, nkv, P, hd).to(dt) for _ in range(2))
        if kind == "finish":
            of_seq = np.repeat(np.arange(len(fresh)), fresh)
            pos = cached[of_seq] + np.arange(len(of_seq)) - np.concatenate([[0], np.cumsum(fresh)])[of_seq]
            s.update(pos=dev(pos.astype(np.int32)), slot=dev((table[of_seq, pos // P] * P + pos % P).astype(np.int32)),
                     QKV=(randn(T, (nq + 2 * nkv) * hd) * 1.5).to(TORCH[case["input"]]), Q=empty(T, nq * hd, dtype=dt),
                     q_gain=(1 + 0.1 * randn(hd)).to(dt), k_gain=(1 + 0.1 * randn(hd)).to(dt))
        else:
            s.update(Q=randn(T, nq * hd).to(dt), out=empty(T, nq * hd, dtype=dt),
                     slopes=torch.exp2(-8.0 * torch.arange(1, nq + 1, device="cuda") / nq) if case["slopes"] else None)
    if own:
        # the handles that a serving program keeps: the plan of the step (one for all layers), the cache's description, a workspace
        from paper_2510_15620_amd import binding as B
        if kind != "finish":
            s["plan"] = B.PagePlan(len(fresh), T, nq, nkv, P, n_pages, table.shape[1], window=case.get("window", 0))
        if kind != "plan":
            s["cache"] = B.KVCache(s["K"], s["V"])
        if kind == "attend":
            B.op_page_plan(s["plan"], s["cached"], s["fresh"], s["table"], s["free"], s["n_free"], empty(1), empty(len(fresh) + 1), empty(T),
                           empty(T))
            s["workspace"] = B.attention_paged_workspace(s["plan"], s["cache"])
    return s


def _plan(s):
    """Rows by sequence, positions, slots, and the table with the step's new pages."""
    P = s["case"]["page"]
    cached, fresh, table, T = s["cached"].long(), s["fresh"].long(), s["table"].clone(), s["T"]
    dev = cached.device
    cu = torch.cat([torch.zeros(1, dtype=torch.long, device=dev), torch.cumsum(fresh, 0)])
    has, need = (cached + P - 1) // P, (cached + fresh + P - 1) // P
    new = torch.cumsum(need - has, 0) - (need - has)                         # new pages of the sequences in front
    col = torch.arange(table.shape[1], device=dev)[None]
    rank = new[:, None] + col - has[:, None]
    fill = (col >= has[:, None]) & (col < need[:, None])
    top = s["n_free"].long() - 1
    table = torch.where(fill, s["free"][(top - rank).clamp(0, s["free"].numel() - 1)], table)
    row = torch.arange(T, device=dev)
    seq = (torch.searchsorted(cu, row, right=True) - 1).clamp(max=len(fresh) - 1)
    real = row < cu[-1]
    pos = torch.where(real, cached[seq] + row - cu[seq], 0)
    slot = torch.where(real, table[seq, pos // P].long() * P + pos % P, -1)
    taken = (need - has).sum()
    status = torch.stack([cu[-1], taken, torch.zeros_like(taken), torch.zeros_like(taken)])
    return [x.to(torch.int32) for x in (cu, pos, slot, table, s["n_free"] - taken, status)]


def _finish(s):
    """Per-head norm and rotation in 32 bits (the angles in 64), one rounding; keys and values to their slots."""
    c = s["case"]
    nq, nkv, hd, P, dt = c["q_heads"], c["kv_heads"], c["head_dim"], c["page"], TORCH[c["dtype"]]
    x = s["QKV"].view(s["T"], nq + 2 * nkv, hd).float()
    qk = x[:, : nq + nkv]
    if c["norm"]:
        gain = torch.cat([s["q_gain"].float().expand(nq, hd), s["k_gain"].float().expand(nkv, hd)])
        qk = qk / torch.sqrt((qk * qk).mean(-1, keepdim=True) + EPS) * gain
    half = hd // 2
    angle = s["pos"].double()[:, None] * torch.pow(torch.tensor(BASE, dtype=torch.float64, device="cuda"), -torch.arange(half, device="cuda").double() / half)
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    a, b = qk[..., :half], qk[..., half:]
    qk = torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(dt)
    page, off = s["slot"].long() // P, s["slot"].long() % P
    s["K"][page, :, off] = qk[:, nq:]
    s["V"][page, :, off] = x[:, nq + nkv:].to(dt)
    return [qk[:, :nq].reshape(s["T"], nq * hd), s["K"], s["V"]]


def _attend(s):
    """Softmax attention in 32 bits over the gathered pages, all sequences padded to the longest."""
    c = s["case"]
    nq, nkv, hd, P = c["q_heads"], c["kv_heads"], c["head_dim"], c["page"]
    G, cached, fresh, table = nq // nkv, s["cached"].long(), s["fresh"].long(), s["table"]
    n, longest = len(fresh), s["case"]["fresh_hi"]
    cu = torch.cumsum(fresh, 0) - fresh
    i = torch.arange(longest, device="cuda")
    rows = torch.where(i[None] < fresh[:, None], cu[:, None] + i, 0)
    pages = table.long().clamp(min=0)
    k, v = (s[x][pages].transpose(2, 3).reshape(n, -1, nkv, hd).permute(0, 2, 1, 3).float() for x in ("K", "V"))
    key = torch.arange(k.shape[2], device="cuda")
    p = cached[:, None] + i
    away = p[:, :, None] - key
    seen = (away >= 0) & (table >= 0).repeat_interleave(P, 1)[:, None]
    if c["window"]:
        seen = seen & (away < c["window"])
    q = s["Q"][rows].view(n, longest, nkv, G, hd).permute(0, 2, 3, 1, 4).reshape(n, nkv, G * longest, hd).float()
    score = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(hd)).view(n, nkv, G, longest, -1)
    if c["cap"]:
        score = torch.tanh(score.div_(c["cap"])).mul_(c["cap"])
    if c["slopes"]:
        score = score - s["slopes"].view(nkv, G, 1, 1) * away[:, None, None]
    score = score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    w = score.sub_(top).exp_()
    total = w.sum(-1, keepdim=True)
    o = torch.matmul(w.view(n, nkv, G * longest, -1), v.contiguous()).view(n, nkv, G, longest, hd) / total.clamp(min=torch.finfo(torch.float32).tiny)
    o = o.permute(0, 3, 1, 2, 4).reshape(n, longest, nq * hd)
    s["out"][:] = o[i[None] < fresh[:, None]].to(s["out"].dtype)
    return [s["out"]]


def run(s):
    c = s["case"]
    if not own:
        return {"plan": _plan, "finish": _finish, "attend": _attend}[c["kind"]](s)
    from paper_2510_15620_amd import binding as B
    if c["kind"] == "plan":
        B.op_page_plan(s["plan"], s["cached"], s["fresh"], s["table"], s["free"], s["n_free"], s["left"], s["cu"], s["pos"], s["slot"], s["status"])
        return [s["cu"], s["pos"], s["slot"], s["table"], s["left"], s["status"]]
    if c["kind"] == "finish":
        B.op_qkv_finish_paged(s["QKV"], s["pos"], s["slot"], s["cache"], s["q_gain"], s["k_gain"], EPS, BASE, c["norm"], s["Q"])
        return [s["Q"], s["K"], s["V"]]
    B.op_attention_paged(s["plan"], s["Q"], s["cache"], s["table"], s["out"], s["workspace"], softcap=c["cap"], slopes=s["slopes"])
    return [s["out"]]


def _visible(case, cached, fresh):
    """Keys that the step's tokens see, per sequence: the union's size and the number of (token, key) pairs."""
    w = case["window"] or 1 << 40
    union, pairs = 0, 0
    for c, f in zip(cached.tolist(), fresh.tolist()):
        p = np.arange(c, c + f, dtype=np.int64)
        union += c + f - max(0, c - w + 1)
        pairs += int(np.minimum(p + 1, w).sum())
    return union, pairs


def work(case):
    cached, fresh = _lengths(case)
    T, nq, nkv, P = int(fresh.sum()), case["q_heads"], case["kv_heads"], case["page"]
    if case["kind"] == "plan":
        new = int((-(-(cached + fresh) // P) + cached // -P).sum())
        return {"bytes": 8 * len(fresh) + 4 * (len(fresh) + 1) + 8 * (T + case["pad"]) + 8 * new, "flops": T}
    hd, size = case["head_dim"], 4 if case["dtype"] == "fp32" else 2
    if case["kind"] == "finish":
        values = T * (nq + 2 * nkv) * hd
        return {"bytes": values * (size + (4 if case["input"] == "fp32" else 2)) + 8 * T, "flops": 8 * values}
    union, pairs = _visible(case, cached, fresh)
    return {"bytes": size * hd * (2 * nkv * union + 2 * nq * T), "flops": 4 * nq * hd * pairs}


def _exact_plan(s):
    P, T = s["case"]["page"], s["T"]
    cached, fresh, table, free = (s[k].cpu().numpy().astype(np.int64) for k in ("cached", "fresh", "table", "free"))
    left, row, cu = int(s["n_free"].item()), 0, [0]
    start = left
    pos, slot = np.zeros(T, np.int64), np.full(T, -1, np.int64)
    for i, (c, f) in enumerate(zip(cached.tolist(), fresh.tolist())):
        for page in range(-(-c // P), -(-(c + f) // P)):
            left -= 1
            table[i, page] = free[left]
        p = np.arange(c, c + f)
        pos[row: row + f], slot[row: row + f] = p, table[i, p // P] * P + p % P
        row += f
        cu.append(row)
    return [np.array(x, np.int32) for x in (cu, pos, slot, table, [left], [row, start - left, 0, 0])]


def _exact_finish(s):
    c = s["case"]
    nq, nkv, hd, P = c["q_heads"], c["kv_heads"], c["head_dim"], c["page"]
    heads = s["QKV"].double().view(-1, nq + 2 * nkv, hd)
    freq = torch.exp(torch.arange(hd // 2, device="cuda", dtype=torch.float64) * (-2.0 * math.log(BASE) / hd))
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["pos"].double()[:, None] * freq)
    out = []
    for first, count, gain in ((0, nq, s["q_gain"]), (nq, nkv, s["k_gain"])):
        x = heads[:, first: first + count]
        if c["norm"]:
            x = x * torch.rsqrt(x.square().sum(-1, keepdim=True) / hd + EPS) * gain.double()
        z = torch.complex(x[..., : hd // 2].contiguous(), x[..., hd // 2:].contiguous()) * turn[:, None]
        out.append(torch.cat([z.real, z.imag], -1))
    K, V = (s[x].double().transpose(1, 2).reshape(-1, nkv, hd) for x in ("K", "V"))
    K[s["slot"].long()], V[s["slot"].long()] = out[1], heads[:, nq + nkv:]
    pages = lambda x: x.view(s["n_pages"], P, nkv, hd).transpose(1, 2).contiguous()  # noqa: E731
    return [out[0].reshape(-1, nq * hd), pages(K), pages(V)]


def _exact_attend(s):
    c = s["case"]
    nq, nkv, hd, P = c["q_heads"], c["kv_heads"], c["head_dim"], c["page"]
    G, out, row = nq // nkv, torch.zeros(s["T"], nq, hd, dtype=torch.float64, device="cuda"), 0
    for i, (old, f) in enumerate(zip(s["cached"].tolist(), s["fresh"].tolist())):
        L = old + f
        ids = s["table"][i, : -(-L // P)].long()
        K, V = (s[x][ids].double().transpose(1, 2).reshape(-1, nkv, hd)[:L] for x in ("K", "V"))
        for r in range(0, f, 256):
            p = torch.arange(old + r, old + min(f, r + 256), device="cuda", dtype=torch.float64)
            gap = p[:, None] - torch.arange(L, device="cuda", dtype=torch.float64)
            hidden = gap < 0
            if c["window"]:
                hidden |= gap >= c["window"]
            q = s["Q"][row + r: row + r + len(p)].double().view(-1, nq, hd)
            for h in range(nq):
                x = q[:, h] @ K[:, h // G].T.contiguous() / math.sqrt(hd)
                if c["cap"]:
                    x = c["cap"] * torch.tanh(x / c["cap"])
                if c["slopes"]:
                    x = x - float(s["slopes"][h]) * gap
                out[row + r: row + r + len(p), h] = torch.softmax(x.masked_fill(hidden, -math.inf), -1) @ V[:, h // G].contiguous()
        row += f
    return [out.view(s["T"], nq * hd)]


def exact(case, seed):
    s = prepare(case, seed)
    return {"plan": _exact_plan, "finish": _exact_finish, "attend": _exact_attend}[case["kind"]](s)
