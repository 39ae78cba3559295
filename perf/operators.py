"""Timed cases of the attention operators over a paged key/value cache.

``op`` names the call:

map      block tables and slot maps of one serving step, from request lengths
write    keys and values of new tokens into the pages of the cache
paged    attention of new tokens (one or a chunk per request) over the paged cache
prompt   attention over whole packed prompts, encoders' full attention included
step     one layer's share of a decode step: map, write, plan and paged attention

Request lengths are those of the image-and-text workload c1: prompts lognormal
(6.0, 0.5), outputs lognormal (5.0, 0.6), at most 32767 tokens, four of five
requests with 1 to 4 images of 256 to 1024 patches; batches are its batch knobs 16,
64 and 256.  Head layouts are generic: 32 query heads on 8 or 32 key/value heads of
128, encoders with 16 heads of 64.
"""
import math
import random

import numpy as np
import torch

own = False

_DT = dict(bf16=torch.bfloat16, fp16=torch.float16)
_LONGEST = 32767


def listed():
    return [
        # page bookkeeping of a decode step at the middle batch knob: latency of one call
        dict(name="map_decode_64", op="map", kind="decode", n=64, page=16, mix=1, short=False),
        # page bookkeeping for 256 whole prompts (about 4 x 10^5 tokens) arriving at once
        dict(name="map_prompt_256", op="map", kind="image", n=256, page=16, mix=2, short=False),
        # the new token of each of 256 running requests into the cache
        dict(name="write_decode_256", op="write", kind="decode", n=256, kv_heads=8, dim=128, dtype="bf16",
             page=16, mix=3),
        # 32 whole prompts into the cache, pages of 64
        dict(name="write_prompt_32", op="write", kind="image", n=32, kv_heads=8, dim=128, dtype="fp16",
             page=64, mix=4),
        # one layer of a decode step of 16 requests through all four calls
        dict(name="step_decode_16", op="step", kind="decode", n=16, heads=32, kv_heads=8, dim=128, dtype="bf16",
             page=16, mix=5),
        # decode of one request at the longest context, a key/value head per query head
        dict(name="paged_decode_1_long", op="paged", kind="fixed", n=1, ctx=32766, new=1, heads=32, kv_heads=32,
             dim=128, dtype="fp16", page=64, mix=6),
        # decode of a full batch: the memory-bound bulk of serving
        dict(name="paged_decode_256", op="paged", kind="decode", n=256, heads=32, kv_heads=8, dim=128, dtype="bf16",
             page=16, mix=7),
        # chunks of 1000 new tokens over long cached contexts
        dict(name="paged_chunk_long", op="paged", kind="fixed", n=2, ctx=24001, new=1000, heads=32, kv_heads=8,
             dim=128, dtype="bf16", page=16, mix=8),
        # a step that mixes running requests, whole prompts and waiting requests
        dict(name="paged_mixed_64", op="paged", kind="mixed", n=64, heads=32, kv_heads=8, dim=128, dtype="bf16",
             page=32, mix=9),
        # full attention of an image encoder: 16 images of 256 to 1024 patches
        dict(name="prompt_encoder_16", op="prompt", kind="patches", n=16, heads=16, kv_heads=16, dim=64,
             dtype="fp16", causal=False, mix=10),
        # causal attention of 16 packed text-and-image prompts
        dict(name="prompt_causal_16", op="prompt", kind="image", n=16, heads=32, kv_heads=8, dim=128, dtype="bf16",
             causal=True, mix=11),
        # causal attention of one prompt of the longest length
        dict(name="prompt_causal_long", op="prompt", kind="fixed", n=1, ctx=0, new=32767, heads=32, kv_heads=8,
             dim=128, dtype="bf16", causal=True, mix=12),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["map", "write", "paged", "paged", "paged", "prompt", "prompt", "prompt", "step"])
    c = dict(op=op, mix=rng.randint(100, 10 ** 6))
    page = rng.choice([16, 32, 64, 128])
    if op != "map":
        c.update(dtype=rng.choice(["bf16", "fp16"]))
    if op in ("paged", "prompt", "step"):
        dim = rng.choice([64, 64, 80, 96, 128, 128, 128])
        kv = rng.choice([1, 2, 4, 8, 16])
        group = rng.choice([1, 1, 2, 3, 4, 7, 8, 16])
        while kv * group > 64:
            group = rng.choice([1, 2, 4])
        c.update(heads=kv * group, kv_heads=kv, dim=dim)
    if op == "map":
        c.update(kind=rng.choice(["decode", "text", "image", "mixed"]), n=_log(rng, 1, 4000), page=page,
                 short=rng.random() < 0.25)
        if c["kind"] != "decode":
            c["n"] = min(c["n"], 500)
    elif op == "write":
        c.update(kind=rng.choice(["decode", "text", "image", "mixed"]), kv_heads=rng.choice([1, 2, 4, 8, 32]),
                 dim=rng.choice([64, 80, 128]), page=page, n=_log(rng, 1, 256))
        if c["kind"] != "decode":
            c["n"] = min(c["n"], 32)
    elif op == "step":
        c.update(kind="decode", n=_log(rng, 1, 64), page=page)
    elif op == "paged":
        kind = rng.choice(["decode", "decode", "fixed", "fixed", "mixed"])
        c.update(kind=kind, page=page)
        if kind == "fixed":
            c.update(n=rng.randint(1, 3), ctx=_log(rng, 1, 30000), new=rng.choice([1, 2, 5, _log(rng, 3, 1000)]))
        else:
            c.update(n=_log(rng, 1, 256 if c["kv_heads"] <= 8 else 64))
    else:
        kind = rng.choice(["patches", "text", "image", "fixed", "cross"])
        causal = kind in ("text", "image", "fixed") and rng.random() < 0.8
        c.update(kind=kind, causal=causal, n=_log(rng, 1, 16))
        if kind == "fixed":
            c.update(n=1, ctx=0, new=_log(rng, 1, 12000))
    return c


# ------------------------------------------------------------------ lengths
def _prompt(rng, images):
    n = max(1, min(_LONGEST, round(math.exp(rng.gauss(6.0, 0.5)))))
    if images and rng.random() < 0.8:
        n += sum(rng.randint(256, 1024) for _ in range(rng.randint(1, 4)))
    return min(n, _LONGEST)


def _out(rng):
    return max(1, min(_LONGEST, round(math.exp(rng.gauss(5.0, 0.6)))))


def lengths(case):
    """(tokens already cached, new tokens) of each request: plain lists."""
    rng, n, kind = random.Random(case["mix"]), case["n"], case["kind"]
    if kind == "decode":
        return [_prompt(rng, True) + rng.randint(0, _out(rng)) for _ in range(n)], [1] * n
    if kind in ("text", "image"):
        return [0] * n, [_prompt(rng, kind == "image") for _ in range(n)]
    if kind == "patches":
        return [0] * n, [rng.randint(256, 1024) for _ in range(n)]
    if kind == "fixed":
        return [case["ctx"]] * n, [case["new"]] * n
    ctx, new = [], []
    for i in range(n):  # mixed: whole prompts among running requests, some of them waiting
        if i % 16 == 5:
            ctx.append(0)
            new.append(_prompt(rng, True))
        else:
            ctx.append(_prompt(rng, True) + rng.randint(0, _out(rng)))
            new.append(0 if i % 16 == 9 else 1)
    return ctx, new


def _cross(case):
    """Query and key lengths of the cross-attention cases, some without keys."""
    rng = random.Random(case["mix"])
    q = [rng.randint(1, 1024) for _ in range(case["n"])]
    return q, [0 if rng.random() < 0.1 else _prompt(rng, False) for _ in range(case["n"])]


def _starts(lens):
    return [0] + np.cumsum(lens, dtype=np.int64).tolist()


# ------------------------------------------------------------------ inputs
def _randn(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _pages(ctx, new, page, gen, slack=0.25):
    """A cache's page bookkeeping before the step: pages in random order, the pages of the
    cached tokens in each request's table row, and the free list."""
    used = [-(-c // page) for c in ctx]
    most = max(1, max(-(-(c + m) // page) for c, m in zip(ctx, new)))
    fresh = sum(-(-(c + m) // page) - u for c, m, u in zip(ctx, new, used))
    n_pages = sum(used) + fresh + max(4, int(slack * (sum(used) + fresh)))
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((len(ctx), most), -1, dtype=torch.int32, device="cuda")
    rows = torch.repeat_interleave(torch.arange(len(ctx), device="cuda"), torch.tensor(used, device="cuda"))
    first = torch.tensor(_starts(used)[:-1], device="cuda")
    cols = torch.arange(len(rows), device="cuda") - first[rows]
    table[rows, cols] = order[:len(rows)]
    return n_pages, fresh, table, order[len(rows):].contiguous()


def _cache(gen, n_pages, case):
    shape = (n_pages, case["kv_heads"], case["page"], case["dim"])
    k = torch.empty(shape, dtype=_DT[case["dtype"]], device="cuda")
    v = torch.empty_like(k)
    for c in (k, v):
        for i in range(0, n_pages, 4096):
            c[i:i + 4096] = _randn(gen, c[i:i + 4096].shape, c.dtype)
    return k, v


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]
    s = dict(case=case, op=op)
    if op == "prompt":
        dt, D = _DT[case["dtype"]], case["dim"]
        ql, kl = _cross(case) if case["kind"] == "cross" else (lengths(case)[1],) * 2
        s.update(q_len=ql, k_len=kl, q_start=_i32(_starts(ql)), k_start=_i32(_starts(kl)),
                 q=_randn(gen, (sum(ql), case["heads"], D), dt), k=_randn(gen, (sum(kl), case["kv_heads"], D), dt),
                 v=_randn(gen, (sum(kl), case["kv_heads"], D), dt))
        return s
    ctx, new = lengths(case)
    n_pages, fresh, table, free = _pages(ctx, new, case["page"], gen)
    n_tok = sum(new)
    s.update(ctx=ctx, new=new, n_tok=n_tok, table=table, page=case["page"], n_pages=n_pages)
    if op in ("map", "step"):
        if case.get("short"):
            free = free[:fresh // 2].contiguous()
        s.update(ctx_len=_i32(ctx), new_len=_i32(new), free=free, head=_i32([0]))
    if op == "map":
        return s
    s["k_cache"], s["v_cache"] = _cache(gen, n_pages, case)
    dt, D = _DT[case["dtype"]], case["dim"]
    if op in ("write", "step"):
        s["k"] = _randn(gen, (n_tok, case["kv_heads"], D), dt)
        s["v"] = _randn(gen, (n_tok, case["kv_heads"], D), dt)
    if op in ("paged", "step"):
        s["q"] = _randn(gen, (n_tok, case["heads"], D), dt)
    if op in ("write", "paged"):
        # what the step's bookkeeping has left: every table row filled, slots of the new tokens
        m = _map_plain(_i32(ctx), _i32(new), table, case["page"], free, _i32([0]), n_tok)
        s["table"], s["q_start"], s["kv_len"], s["slots"] = m[0], m[1], m[2], m[3]
    if op == "paged" and own:
        from paper_2512_14098_amd import cf
        s["plan"] = cf.cf_attn_plan(s["q_start"], s["kv_len"], n_tok, max(new), case["heads"], case["kv_heads"], D)
    return s


# ------------------------------------------------------------------ plain forms
def _map_plain(ctx_len, new_len, table, page, free, head, n_tok):
    ctx, new = ctx_len.long(), new_len.long()
    n, most = table.shape
    q_start = torch.zeros(n + 1, dtype=torch.int64, device=table.device)
    q_start[1:] = torch.cumsum(new, 0)
    kv = ctx + new
    have, want = (ctx + page - 1) // page, (kv + page - 1) // page
    too_long = kv > most * page
    need = torch.where(too_long, torch.zeros_like(kv), want - have)
    last = torch.cumsum(need, 0) + head.long()
    no_page = ~too_long & (need > 0) & (last > free.numel())
    no_page = no_page | (~too_long & (torch.cumsum(no_page.long(), 0) > 0) & (need > 0))
    status = too_long.int() + 2 * no_page.int()
    ok = status == 0
    col = torch.arange(most, device=table.device)
    src = (last - need)[:, None] + col[None, :] - have[:, None]
    fill = ok[:, None] & (col[None, :] >= have[:, None]) & (col[None, :] < want[:, None])
    if free.numel():
        out = torch.where(fill, free[torch.clamp(src, 0, free.numel() - 1)], table)
    else:
        out = table.clone()
    tok = torch.arange(n_tok, device=table.device)
    req = torch.clamp(torch.searchsorted(q_start[1:].contiguous(), tok, right=True), max=n - 1)
    pos = ctx[req] + tok - q_start[req]
    at = torch.clamp(pos, max=most * page - 1)
    slot = out[req, at // page].long() * page + at % page
    slots = torch.where(ok[req], slot, torch.full_like(slot, -1))
    taken = torch.where(ok, need, torch.zeros_like(need)).sum()
    return (out, q_start.int(), torch.where(ok, kv, torch.zeros_like(kv)).int(), slots, pos.int(),
            (head.long() + taken).int(), status)


def _write_plain(k, v, k_cache, v_cache, slots, page):
    p, o = slots // page, slots % page
    k_cache[p, :, o] = k
    v_cache[p, :, o] = v


def _attend(q, k, v, first, scale):
    """One request: q [n][H][D] at positions first.. (None: full attention), k and v [m][Hkv][D]."""
    n, H, D = q.shape
    m, Hkv, _ = k.shape
    if m == 0:
        return torch.zeros_like(q, dtype=torch.float32)
    G = H // Hkv
    kf = k.float().permute(1, 2, 0).contiguous()  # [Hkv][D][m]
    vf = v.float().permute(1, 0, 2).contiguous()  # [Hkv][m][D]
    out = torch.empty((n, H, D), dtype=torch.float32, device=q.device)
    step = max(1, min(n, int(1.5e9) // max(1, H * m)))
    for a in range(0, n, step):
        b = min(n, a + step)
        lim = m if first is None else min(m, first + b)
        qs = q[a:b].float().reshape(b - a, Hkv, G, D).permute(1, 2, 0, 3).reshape(Hkv, G * (b - a), D).contiguous()
        x = torch.matmul(qs, kf[:, :, :lim].contiguous()) * scale
        if first is not None:
            x = x.reshape(Hkv, G, b - a, lim)
            row = torch.arange(a, b, device=q.device)[:, None] + first
            hide = torch.arange(lim, device=q.device)[None, :] > row
            x = x.masked_fill(hide, float("-inf")).reshape(Hkv, G * (b - a), lim)
        x = torch.exp(x - x.amax(-1, keepdim=True))
        o = torch.matmul(x, vf[:, :lim]) / x.sum(-1, keepdim=True)
        out[a:b] = o.reshape(Hkv, G, b - a, D).permute(2, 0, 1, 3).reshape(b - a, H, D)
    return out


def _decode_plain(q, k_cache, v_cache, table, kv_len, scale):
    """Every request has one new token: padded to the longest context, some requests at a time."""
    n, H, D = q.shape
    _, Hkv, page, _ = k_cache.shape
    G, most = H // Hkv, table.shape[1]
    out = torch.empty((n, H, D), dtype=torch.float32, device=q.device)
    step = max(1, min(n, int(1e9) // (most * page * Hkv * D)))
    for a in range(0, n, step):
        t = torch.clamp(table[a:a + step], min=0).long()
        b = t.shape[0]
        kf = k_cache[t].float().permute(0, 2, 4, 1, 3).reshape(b * Hkv, D, most * page)
        vf = v_cache[t].float().permute(0, 2, 1, 3, 4).reshape(b * Hkv, most * page, D)
        x = torch.matmul(q[a:a + b].float().reshape(b * Hkv, G, D), kf) * scale
        hide = torch.arange(most * page, device=q.device)[None, :] >= kv_len[a:a + b, None]
        x = x.reshape(b, H, most * page).masked_fill(hide[:, None, :], float("-inf"))
        x = torch.exp(x - x.amax(-1, keepdim=True)).reshape(b * Hkv, G, most * page)
        o = torch.matmul(x, vf) / x.sum(-1, keepdim=True)
        out[a:a + b] = o.reshape(b, H, D)
    return out


def _paged_plain(s, q, k_cache, v_cache, table, kv_len):
    scale = q.shape[2] ** -0.5
    if max(s["new"]) == 1 and min(s["new"]) == 1:
        return _decode_plain(q, k_cache, v_cache, table, kv_len, scale).to(q.dtype)
    out = torch.zeros(q.shape, dtype=torch.float32, device=q.device)
    at, page = 0, k_cache.shape[2]
    for i, (c, m) in enumerate(zip(s["ctx"], s["new"])):
        if m == 0:
            continue
        t = table[i, :-(-(c + m) // page)].long()
        k = k_cache[t].permute(0, 2, 1, 3).reshape(-1, k_cache.shape[1], q.shape[2])[:c + m]
        v = v_cache[t].permute(0, 2, 1, 3).reshape(-1, k_cache.shape[1], q.shape[2])[:c + m]
        out[at:at + m] = _attend(q[at:at + m], k, v, c, scale)
        at += m
    return out.to(q.dtype)


def _prompt_plain(s):
    q, k, v = s["q"], s["k"], s["v"]
    out = torch.empty(q.shape, dtype=torch.float32, device=q.device)
    a = b = 0
    for n, m in zip(s["q_len"], s["k_len"]):
        out[a:a + n] = _attend(q[a:a + n], k[b:b + m], v[b:b + m], 0 if s["case"]["causal"] else None,
                               q.shape[2] ** -0.5)
        a, b = a + n, b + m
    return out.to(q.dtype)


_MAP_OUT = ("table", "q_start", "kv_len", "slots", "pos", "head", "status")


def run(s):
    op = s["op"]
    if own:
        from paper_2512_14098_amd import cf
        if op == "map":
            m = cf.cf_kv_map(s["ctx_len"], s["new_len"], s["table"], s["page"], s["free"], s["head"], s["n_tok"])
            return dict(zip(_MAP_OUT, (s["table"],) + tuple(m)))
        if op == "write":
            cf.cf_kv_write(s["k"], s["v"], s["k_cache"], s["v_cache"], s["slots"])
            return dict(k_cache=s["k_cache"], v_cache=s["v_cache"])
        if op == "paged":
            return cf.cf_attn_paged(s["plan"], s["q"], s["k_cache"], s["v_cache"], s["table"])
        if op == "prompt":
            return cf.cf_attn_prompt(s["q"], s["k"], s["v"], s["q_start"], s["k_start"], causal=s["case"]["causal"])
        q_start, kv_len, slots, pos, head, status = cf.cf_kv_map(
            s["ctx_len"], s["new_len"], s["table"], s["page"], s["free"], s["head"], s["n_tok"])
        cf.cf_kv_write(s["k"], s["v"], s["k_cache"], s["v_cache"], slots)
        c = s["case"]
        plan = cf.cf_attn_plan(q_start, kv_len, s["n_tok"], 1, c["heads"], c["kv_heads"], c["dim"])
        out = cf.cf_attn_paged(plan, s["q"], s["k_cache"], s["v_cache"], s["table"])
        return dict(out=out, k_cache=s["k_cache"], v_cache=s["v_cache"], table=s["table"], head=head)
    if op == "map":
        return dict(zip(_MAP_OUT, _map_plain(s["ctx_len"], s["new_len"], s["table"], s["page"], s["free"], s["head"],
                                             s["n_tok"])))
    if op == "write":
        _write_plain(s["k"], s["v"], s["k_cache"], s["v_cache"], s["slots"], s["page"])
        return dict(k_cache=s["k_cache"], v_cache=s["v_cache"])
    if op == "paged":
        return _paged_plain(s, s["q"], s["k_cache"], s["v_cache"], s["table"], s["kv_len"])
    if op == "prompt":
        return _prompt_plain(s)
    table, _, kv_len, slots, _, head, _ = _map_plain(s["ctx_len"], s["new_len"], s["table"], s["page"], s["free"],
                                                     s["head"], s["n_tok"])
    _write_plain(s["k"], s["v"], s["k_cache"], s["v_cache"], slots, s["page"])
    out = _paged_plain(s, s["q"], s["k_cache"], s["v_cache"], table, kv_len)
    return dict(out=out, k_cache=s["k_cache"], v_cache=s["v_cache"], table=table, head=head)


# ------------------------------------------------------------------ work
def _pairs(ctx, new):
    """(query, visible key) pairs of causal attention."""
    return sum(m * c + m * (m + 1) // 2 for c, m in zip(ctx, new))


def work(case):
    op = case["op"]
    if op == "prompt":
        ql, kl = _cross(case) if case["kind"] == "cross" else (lengths(case)[1],) * 2
        pairs = _pairs([0] * len(ql), ql) if case["causal"] else sum(a * b for a, b in zip(ql, kl))
        io = 2 * case["dim"] * (2 * sum(ql) * case["heads"] + 2 * sum(kl) * case["kv_heads"])
        return dict(bytes=io, flops=4 * pairs * case["heads"] * case["dim"])
    ctx, new = lengths(case)
    n, n_tok, page = case["n"], sum(new), case["page"]
    fresh = sum(-(-(c + m) // page) - -(-c // page) for c, m in zip(ctx, new))
    # lengths in, starts, lengths and status out; a new page's id read and written; the page
    # id that an old partial page's slots need; slot and position of each new token
    map_bytes = n * 20 + fresh * 8 + 4 * sum(1 for c, m in zip(ctx, new) if m and c % page) + n_tok * 12
    if op == "map":
        return dict(bytes=map_bytes, flops=0)
    row = 2 * case["kv_heads"] * case["dim"] * 2  # K and V of one token
    write_bytes = n_tok * (2 * row + 8)
    if op == "write":
        return dict(bytes=write_bytes, flops=0)
    kv = sum(c + m for c, m in zip(ctx, new) if m)
    io = kv * row + 2 * n_tok * case["heads"] * case["dim"] * 2
    flops = 4 * _pairs(ctx, new) * case["heads"] * case["dim"]
    if op == "paged":
        return dict(bytes=io, flops=flops)
    return dict(bytes=io + map_bytes + write_bytes, flops=flops)


# ------------------------------------------------------------------ definitions in 64 bits
def _exact_map(ctx, new, table, page, free, n_tok):
    table, free = table.copy(), free.tolist()
    q_start, kv_len, status, slots, pos = [0], [], [], [], []
    head, blocked = 0, False
    for i, (c, m) in enumerate(zip(ctx, new)):
        st, first, last = 0, -(-c // page), -(-(c + m) // page)
        if c + m > table.shape[1] * page:
            st = 1
        elif last > first and (blocked or head + last - first > len(free)):
            st, blocked = 2, True
        else:
            for j in range(first, last):
                table[i, j] = free[head]
                head += 1
        for t in range(c, c + m):
            slots.append(int(table[i, t // page]) * page + t % page if st == 0 else -1)
            pos.append(t)
        q_start.append(q_start[-1] + m)
        kv_len.append(c + m if st == 0 else 0)
        status.append(st)
    return table, q_start, kv_len, slots, pos, [head], status


def _exact_attend(q, k, v, first):
    """One request in 64 bits, a head at a time."""
    n, H, D = q.shape
    m, Hkv, _ = k.shape
    out = torch.zeros((n, H, D), dtype=torch.float64, device=q.device)
    if m == 0:
        return out
    key = torch.arange(m, device=q.device)
    rows = max(1, int(2.5e8) // m)
    for h in range(H):
        kh, vh = k[:, h * Hkv // H].double(), v[:, h * Hkv // H].double()
        for a in range(0, n, rows):
            x = (q[a:a + rows, h].double() @ kh.t().contiguous()) / math.sqrt(D)
            if first is not None:
                seen = key[None] <= first + a + torch.arange(x.shape[0], device=q.device)[:, None]
                x = torch.where(seen, x, torch.full_like(x, -math.inf))
            out[a:a + rows, h] = torch.softmax(x, 1) @ vh
    return out


def exact(case, seed):
    w = work(case)
    if w["flops"] > 2e13:
        return None
    s = prepare(case, seed)
    op = case["op"]
    if op == "prompt":
        out, a, b = [], 0, 0
        for n, m in zip(s["q_len"], s["k_len"]):
            out.append(_exact_attend(s["q"][a:a + n], s["k"][b:b + m], s["v"][b:b + m], 0 if case["causal"] else None))
            a, b = a + n, b + m
        return torch.cat(out)
    if op in ("map", "step"):
        m = _exact_map(s["ctx"], s["new"], s["table"].cpu().numpy(), s["page"], s["free"].cpu().numpy(), s["n_tok"])
        m = [torch.as_tensor(np.asarray(x)).cuda() for x in m]
        if op == "map":
            return dict(zip(_MAP_OUT, m))
        table, slots, head = m[0], m[3], m[5]
    else:
        table, slots, head = s["table"], s["slots"], None
    if op in ("write", "step"):
        page = s["page"]
        for src, dst in (("k", "k_cache"), ("v", "v_cache")):
            rows = s[dst].permute(0, 2, 1, 3).reshape(s["n_pages"] * page, *s[src].shape[1:]).clone()
            rows[slots.long()] = s[src]
            s[dst] = rows.reshape(s["n_pages"], page, *s[src].shape[1:]).permute(0, 2, 1, 3).contiguous()
        if op == "write":
            return dict(k_cache=s["k_cache"].double(), v_cache=s["v_cache"].double())
    out, at, page = [], 0, s["page"]
    for i, (c, m) in enumerate(zip(s["ctx"], s["new"])):
        idx = torch.arange(c + m, device="cuda")
        p = table[i].long()[idx // page]
        if m:
            out.append(_exact_attend(s["q"][at:at + m], s["k_cache"][p, :, idx % page], s["v_cache"][p, :, idx % page],
                                     c))
        at += m
    out = torch.cat(out) if out else torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    if op == "paged":
        return out
    return dict(out=out, k_cache=s["k_cache"].double(), v_cache=s["v_cache"].double(), table=table, head=head)
