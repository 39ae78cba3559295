"""Attention over the paged cache and its bookkeeping against plain 64-bit forms."""
import numpy as np
import pytest

from tests import attn_ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module")
def cf():
    from paper_2512_14098_amd import cf as _cf
    return _cf


def _say(*a):
    print(*a, flush=True)


def _i32(x):
    return torch.as_tensor(np.asarray(x, np.int32)).cuda()


# ------------------------------------------------------------------ block tables and slots
def _check_map(cf, ctx, new, table, page, free, head, n_tok):
    want = attn_ref.kv_map(ctx, new, table, page, free, head, n_tok)
    t = _i32(table)
    got = cf.cf_kv_map(_i32(ctx), _i32(new), t, page, _i32(free), _i32([head]), n_tok)
    torch.cuda.synchronize()
    got = dict(zip(("q_start", "kv_len", "slots", "pos", "head", "status"), got), table=t)
    for name, w in want.items():
        assert np.array_equal(got[name].cpu().numpy(), np.asarray(w)), name


def _map_inputs(rng, n, page, most, ctx, new, spare):
    used = [max(-(-int(c) // page), 0) for c in ctx]
    need = sum(-(-int(c + m) // page) - u for c, m, u in zip(ctx, new, used))
    order = rng.permutation(sum(used) + max(need, 0) + 50)
    table = np.full((n, most), -7, np.int64)
    at = 0
    for i, u in enumerate(used):
        u = min(u, most)
        table[i, :u] = order[at:at + u]
        at += u
    return table, order[at:at + max(need + spare, 0)]


@pytest.mark.parametrize("n,page,longest,spare", [(1, 16, 40, 3), (3, 32, 100, 0), (64, 16, 300, 7), (255, 64, 90, 1),
                                                  (256, 128, 700, 2), (257, 16, 50, -20), (1000, 16, 20, 4),
                                                  (3000, 256, 9, 5), (40, 16, 3000, -400)])
def test_map_against_sequential_rules(cf, n, page, longest, spare):
    _say("map", n, page, longest, spare)
    rng = np.random.default_rng(n + page)
    ctx = rng.integers(0, longest + 1, n)
    new = np.where(rng.random(n) < 0.3, 0, rng.integers(0, longest + 1, n))
    if n > 2:
        ctx[rng.integers(0, n)], ctx[rng.integers(0, n)] = 0, page * 2
    most = -(-int((ctx + new).max()) // page) + 1
    table, free = _map_inputs(rng, n, page, most, ctx, new, spare)
    _check_map(cf, ctx, new, table, page, free, 0, int(new.sum()))


@pytest.mark.parametrize("n_tok", [0, 1, 90, 2500, 2600])
def test_map_refuses_requests_on_the_device(cf, n_tok):
    """Negative lengths, rows too short for a request, token arrays too short, an empty free list."""
    _say("map refusals", n_tok)
    rng = np.random.default_rng(n_tok)
    n, page = 50, 16
    ctx, new = rng.integers(0, 60, n), rng.integers(0, 60, n)
    ctx[3], new[5], new[9], ctx[11] = -4, -1, 2000, 2 ** 31 - 1
    table = rng.integers(0, 1000, (n, 6))
    for free, head in ((np.arange(1000, 1200), 5), (np.zeros(0, np.int64), 0), (np.arange(20), 20), (np.arange(60), -3)):
        _check_map(cf, ctx, new, table, page, free, head, n_tok)


def test_map_on_a_stream_and_in_a_graph(cf):
    """The step captured once and replayed on lengths that grow, the head carried on the device."""
    n, page, most = 20, 16, 8
    rng = np.random.default_rng(0)
    ctx = rng.integers(0, 40, n)
    new = np.ones(n, np.int64)
    table, free = _map_inputs(rng, n, page, most, ctx, new * 60, 0)
    t, f, c, w, h = _i32(table), _i32(free), _i32(ctx), _i32(new), _i32([0])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        first = cf.cf_kv_map(c, w, t, page, f, h, n)  # warm-up on a copy of nothing: redone below
    torch.cuda.current_stream().wait_stream(s)
    t.copy_(_i32(table))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = cf.cf_kv_map(c, w, t, page, f, h, n)
        h.copy_(out[4])
        c.add_(w)
    want_table, head = table, 0
    for step in range(5):
        g.replay()
        torch.cuda.synchronize()
        want = attn_ref.kv_map(ctx + step, new, want_table, page, free, head, n)
        want_table, head = want["table"], want["head"][0]
        for k, name in enumerate(("q_start", "kv_len", "slots", "pos", "head", "status")):
            assert np.array_equal(out[k].cpu().numpy(), np.asarray(want[name])), (step, name)
        assert np.array_equal(t.cpu().numpy(), want_table)
    assert first[5].sum().item() == 0


# ------------------------------------------------------------------ writes
@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("n,heads,dim,page", [(1, 1, 8, 16), (7, 3, 72, 32), (300, 8, 128, 16), (65, 2, 256, 256)])
def test_write(cf, kind, n, heads, dim, page):
    _say("write", kind, n, heads, dim, page)
    n_pages = -(-n // page) + 3
    g = torch.Generator(device="cuda").manual_seed(n)
    kc = torch.randn((n_pages, heads, page, dim), generator=g, device="cuda").to(DT[kind])
    vc = torch.randn((n_pages, heads, page, dim), generator=g, device="cuda").to(DT[kind])
    # keys and values are slices of a fused projection: strided rows
    qkv = torch.randn((n, 3 * heads, dim), generator=g, device="cuda").to(DT[kind])
    k, v = qkv[:, heads:2 * heads], qkv[:, 2 * heads:]
    slots = torch.randperm(n_pages * page, generator=g, device="cuda")[:n].clone()
    if n > 3:
        slots[0], slots[2] = -1, n_pages * page
    wk, wv = kc.clone(), vc.clone()
    for t, s in enumerate(slots.tolist()):
        if 0 <= s < n_pages * page:
            wk[s // page, :, s % page] = k[t]
            wv[s // page, :, s % page] = v[t]
    cf.cf_kv_write(k, v, kc, vc, slots)
    assert torch.equal(kc, wk) and torch.equal(vc, wv)
    # rows that are not 16-byte aligned or not packed are copied by the binding
    odd = torch.randn((n, heads, dim + 3), generator=g, device="cuda").to(DT[kind])[:, :, 3:]
    cf.cf_kv_write(odd, v, kc, vc, slots)
    for t, s in enumerate(slots.tolist()):
        if 0 <= s < n_pages * page:
            assert torch.equal(kc[s // page, :, s % page], odd[t])


# ------------------------------------------------------------------ paged attention
def _paged_case(kind, ctx, new, heads, kv_heads, dim, page, seed=0, poison=float("nan")):
    """Random caches whose every element outside the requests' tokens is ``poison``."""
    rng = np.random.default_rng(seed)
    n = len(ctx)
    kv = [c + m for c, m in zip(ctx, new)]
    most = max(1, max(-(-x // page) for x in kv))
    used = sum(-(-x // page) for x in kv)
    n_pages = used + 5
    order = rng.permutation(n_pages)
    table = np.full((n, most), -1, np.int64)
    kc = torch.full((n_pages, kv_heads, page, dim), poison, dtype=DT[kind])
    vc = torch.full((n_pages, kv_heads, page, dim), poison, dtype=DT[kind])
    ks, vs, at = [], [], 0
    for i, x in enumerate(kv):
        k = torch.from_numpy(rng.standard_normal((x, kv_heads, dim)).astype(np.float32)).to(DT[kind])
        v = torch.from_numpy(rng.standard_normal((x, kv_heads, dim)).astype(np.float32)).to(DT[kind])
        for p in range(-(-x // page)):
            table[i, p] = order[at]
            a, b = p * page, min((p + 1) * page, x)
            kc[order[at], :, :b - a] = k[a:b].transpose(0, 1)
            vc[order[at], :, :b - a] = v[a:b].transpose(0, 1)
            at += 1
        ks.append(k)
        vs.append(v)
    q = torch.from_numpy((1.5 * rng.standard_normal((sum(new), heads, dim))).astype(np.float32)).to(DT[kind])
    return dict(q=q, kc=kc, vc=vc, table=table, ks=ks, vs=vs, kv=kv,
                q_start=np.concatenate([[0], np.cumsum(new)]))


def _compare(got, lse, want):
    out, wl, tol, ltol = want
    got, lse = got.double().cpu().numpy(), lse.double().cpu().numpy()
    bad = ~(np.abs(got - out) <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3].tolist(), float(np.abs(got - out).max()))
    empty = np.isneginf(wl)
    assert np.array_equal(np.isneginf(lse), empty) and np.all(got[empty] == 0)
    assert np.all(np.abs(lse[~empty] - wl[~empty]) <= ltol[~empty])


def _want_paged(c, ctx, new, scale, kind):
    parts, at = [], 0
    for i, (x, m) in enumerate(zip(ctx, new)):
        q = c["q"][at:at + m].float().numpy()
        parts.append(attn_ref.attend(q, c["ks"][i].float().numpy(), c["vs"][i].float().numpy(),
                                     [x + j + 1 for j in range(m)], scale, kind))
        at += m
    return [np.concatenate(p) for p in zip(*parts)]


def _run_paged(cf, c, new, heads, kv_heads, dim, max_new=None, scale=None, kv_len=None):
    n_tok = int(sum(new))
    plan = cf.cf_attn_plan(_i32(c["q_start"]), _i32(c["kv"] if kv_len is None else kv_len), n_tok,
                           max(new) if max_new is None else max_new, heads, kv_heads, dim)
    return cf.cf_attn_paged(plan, c["q"].cuda(), c["kc"].cuda(), c["vc"].cuda(), _i32(c["table"]), scale=scale, lse=True)


LENS = {
    "one": ([0], [1]),
    "edges": ([0, 14, 15, 16, 30, 31, 32, 62, 63, 64, 255, 256], [1] * 12),
    "waiting": ([3, 40, 0, 77], [1, 0, 0, 1]),
    "several": ([0, 7, 100, 31], [2, 5, 3, 4]),
    "long": ([5000, 3], [1, 1]),
    "chunks": ([0, 1, 70, 33], [65, 17, 40, 128]),
    "mixed": ([200, 0, 64, 9], [1, 90, 0, 2]),
}


@pytest.mark.parametrize("lens", sorted(LENS))
@pytest.mark.parametrize("kind,heads,kv_heads,dim,page", [
    ("bf16", 4, 1, 128, 16), ("fp16", 4, 2, 64, 32), ("bf16", 3, 3, 80, 64), ("fp16", 7, 1, 96, 16),
    ("bf16", 2, 2, 8, 128), ("fp16", 6, 2, 136, 16), ("bf16", 4, 2, 256, 256), ("fp16", 20, 1, 40, 16),
    ("bf16", 8, 1, 104, 64)])
def test_paged(cf, kind, heads, kv_heads, dim, page, lens):
    _say("paged", kind, heads, kv_heads, dim, page, lens)
    ctx, new = LENS[lens]
    c = _paged_case(kind, ctx, new, heads, kv_heads, dim, page)
    want = _want_paged(c, ctx, new, dim ** -0.5, kind)
    for max_new in (None, sum(new)):
        _compare(*_run_paged(cf, c, new, heads, kv_heads, dim, max_new), want)


@pytest.mark.parametrize("new", [1, 5, 70])
def test_split_contexts(cf, new):
    """One request, two key/value heads: the plan splits the context; joined parts are right,
    and the same on every call."""
    _say("split", new)
    c = _paged_case("bf16", [9000], [new], 4, 2, 64, 16)
    want = _want_paged(c, [9000], [new], 0.125, "bf16")
    a = _run_paged(cf, c, [new], 4, 2, 64)
    b = _run_paged(cf, c, [new], 4, 2, 64)
    _compare(*a, want)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("poison", [float("inf"), float("-inf"), 65504.0])
def test_masked_places_hold_anything(cf, poison):
    for ctx, new in (([17, 40], [1, 3]), ([5, 0], [60, 130])):
        c = _paged_case("fp16", ctx, new, 4, 2, 64, 32, poison=poison)
        _compare(*_run_paged(cf, c, new, 4, 2, 64), _want_paged(c, ctx, new, 0.125, "fp16"))


@pytest.mark.parametrize("kind,dim", [("bf16", 128), ("fp16", 64), ("bf16", 72)])
@pytest.mark.parametrize("ctx,new,at", [([60], [4], [62]), ([100], [90], [130, 150]), ([0], [200], [70, 199]),
                                        ([6000], [3], [6001]), ([6000], [40], [6003, 6039])])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_special_values_reach_only_the_rows_that_see_them(cf, kind, dim, ctx, new, at, value):
    """An infinity or NaN among a later token's keys or values leaves earlier rows alone."""
    _say("specials", kind, dim, ctx, new, at, value)
    heads, kv_heads, page = 4, 2, 16
    c = _paged_case(kind, ctx, new, heads, kv_heads, dim, page)
    clean = _want_paged(c, ctx, new, dim ** -0.5, kind)
    for p in at:
        c["vc"][c["table"][0, p // page], 1, p % page, 5] = value
        c["kc"][c["table"][0, p // page], 0, p % page, 3] = float("nan")
    got, lse = _run_paged(cf, c, new, heads, kv_heads, dim)
    got, lse = got.double().cpu().numpy(), lse.double().cpu().numpy()
    out, wl, tol, ltol = clean
    sees = np.array([ctx[0] + j >= min(at) for j in range(new[0])])
    # key/value head 1 (heads 2, 3): only element 5 of the rows that see the value
    hit = np.zeros(got.shape, bool)
    hit[sees, 2:, 5] = True
    hit[sees, :2, :] = True  # key/value head 0: a NaN score spoils the whole row
    assert np.all(~np.isfinite(got[hit]))
    assert np.all(np.abs(got - out)[~hit] <= tol[~hit])
    if value == float("inf"):
        assert np.all(got[sees, 2:, 5] == np.inf)
    assert np.all(np.abs(lse - wl)[:, 2:] <= ltol[:, 2:])


def test_rows_that_see_nothing(cf):
    """kv_len 0 (a refused request) and fewer keys than new tokens: zero rows, lse -inf."""
    for heads in (2, 8):
        ctx, new = [20, 33, 0], [2, 30, 40]
        c = _paged_case("bf16", ctx, new, heads, 2, 64, 16)
        kv = [0, 10, 40]  # request 1: 10 keys, so its first 20 new tokens see none
        got = _run_paged(cf, c, new, heads, 2, 64, kv_len=kv)
        parts, at = [], 0
        for i, m in enumerate(new):
            parts.append(attn_ref.attend(c["q"][at:at + m].float().numpy(), c["ks"][i].float().numpy(),
                                         c["vs"][i].float().numpy(), [kv[i] - m + j + 1 for j in range(m)], 0.125,
                                         "bf16"))
            at += m
        _compare(*got, [np.concatenate(p) for p in zip(*parts)])


def test_pages_outside_the_cache_read_as_zeros(cf):
    ctx, new = [100, 100], [1, 40]
    c = _paged_case("fp16", ctx, new, 4, 2, 64, 16)
    for i, bad in ((0, -5), (1, 10 ** 6)):
        c["table"][i, 2] = bad
        c["ks"][i][32:48] = 0
        c["vs"][i][32:48] = 0
    _compare(*_run_paged(cf, c, new, 4, 2, 64), _want_paged(c, ctx, new, 0.125, "fp16"))


def test_lengths_are_not_trusted(cf):
    """Starts that do not ascend and lengths past the table row stay inside the arrays, and
    requests whose lengths are right stay right."""
    ctx, new = [50, 20, 70], [3, 1, 30]
    c = _paged_case("bf16", ctx, new, 4, 2, 64, 16)
    want = _want_paged(c, ctx, new, 0.125, "bf16")
    c["q_start"] = np.array([0, 3, 4, 5000])
    kv = [53, 2 ** 31 - 1, 100]
    out, _ = _run_paged(cf, c, new, 4, 2, 64, kv_len=kv)
    ok = np.r_[0:3, 4:34]
    assert np.all(np.abs(out.double().cpu().numpy() - want[0])[ok] <= want[2][ok])
    c["q_start"] = np.array([34, 3, -9, 34])
    _run_paged(cf, c, new, 4, 2, 64, kv_len=[-1, 7, 9])
    torch.cuda.synchronize()


def test_strides_scale_and_stream(cf):
    """Queries out of a fused projection, another scale, work on a stream that is not the default."""
    ctx, new = [30, 5, 300], [1, 4, 50]
    c = _paged_case("bf16", ctx, new, 4, 2, 80, 16)
    want = _want_paged(c, ctx, new, 0.3, "bf16")
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        fused = torch.zeros((sum(new), 8, 80), dtype=torch.bfloat16, device="cuda")
        fused[:, 3:7] = c["q"].cuda()
        plan = cf.cf_attn_plan(_i32(c["q_start"]), _i32(c["kv"]), sum(new), 50, 4, 2, 80)
        got = cf.cf_attn_paged(plan, fused[:, 3:7], c["kc"].cuda(), c["vc"].cuda(), _i32(c["table"]), scale=0.3, lse=True)
    s.synchronize()
    _compare(*got, want)


def test_offsets_past_32_bits(cf):
    """A cache of more than 2^32 elements, the request's pages at its far end."""
    heads, dim, page = 4, 128, 64
    n_pages = (1 << 32) // (heads * dim * page) + 40
    _say("cache of", n_pages, "pages")
    c = _paged_case("bf16", [500], [20], heads, heads, dim, page)
    kc = torch.empty((n_pages, heads, page, dim), dtype=torch.bfloat16, device="cuda")
    vc = torch.empty_like(kc)
    small = c["kc"].shape[0]
    kc[-small:], vc[-small:] = c["kc"].cuda(), c["vc"].cuda()
    c["table"] = np.where(c["table"] >= 0, c["table"] + n_pages - small, -1)
    c["kc"], c["vc"] = kc, vc
    _compare(*_run_paged(cf, c, [20], heads, heads, dim), _want_paged(c, [500], [20], dim ** -0.5, "bf16"))
    # and the write of a token there
    k = torch.randn((1, heads, dim), device="cuda").to(torch.bfloat16)
    slot = n_pages * page - 1
    cf.cf_kv_write(k, -k, kc, vc, torch.tensor([slot], device="cuda"))
    assert torch.equal(kc[-1, :, -1], k[0]) and torch.equal(vc[-1, :, -1], -k[0])


def test_decode_step_in_a_graph(cf):
    """map, write, plan and attention captured once and replayed as the requests grow."""
    heads, kv_heads, dim, page, n = 4, 2, 64, 16, 6
    ctx = [0, 15, 16, 40, 100, 31]
    c = _paged_case("bf16", ctx, [0] * n, heads, kv_heads, dim, page, poison=0.0)
    steps, most = 5, 12
    n_pages = 80
    kc = torch.zeros((n_pages, kv_heads, page, dim), dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    kc[:c["kc"].shape[0]], vc[:c["vc"].shape[0]] = c["kc"].cuda(), c["vc"].cuda()
    table = np.full((n, most), -1, np.int64)
    table[:, :c["table"].shape[1]] = c["table"]
    free = np.setdiff1d(np.arange(n_pages), table[table >= 0])
    t, f, cl, nl, h = _i32(table), _i32(free), _i32(ctx), _i32([1] * n), _i32([0])
    g0 = torch.Generator(device="cuda").manual_seed(1)
    qkv = [torch.randn((n, heads + 2 * kv_heads, dim), generator=g0, device="cuda").to(torch.bfloat16)
           for _ in range(steps)]
    x = qkv[0].clone()

    def step():
        q_start, kv_len, slots, _, head, _ = cf.cf_kv_map(cl, nl, t, page, f, h, n)
        k, v = x[:, heads:heads + kv_heads], x[:, heads + kv_heads:]
        cf.cf_kv_write(k, v, kc, vc, slots)
        plan = cf.cf_attn_plan(q_start, kv_len, n, 1, heads, kv_heads, dim)
        return cf.cf_attn_paged(plan, x[:, :heads], kc, vc, t, lse=True), head

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()  # the first step, as every replay below redoes it: same table, slots and values
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        (out, lse), head = step()
        h.copy_(head)
        cl.add_(nl)
    for i in range(steps):
        x.copy_(qkv[i])
        g.replay()
        torch.cuda.synchronize()
        c["q"] = qkv[i][:, :heads].cpu()
        for r in range(n):
            c["ks"][r] = torch.cat([c["ks"][r], qkv[i][r:r + 1, heads:heads + kv_heads].cpu()])
            c["vs"][r] = torch.cat([c["vs"][r], qkv[i][r:r + 1, heads + kv_heads:].cpu()])
        _compare(out, lse, _want_paged(c, [a + i for a in ctx], [1] * n, dim ** -0.5, "bf16"))


# ------------------------------------------------------------------ packed prompts
def _want_prompt(q, k, v, ql, kl, causal, scale, kind, q0=0, k0=0):
    parts, a, b = [], q0, k0
    for n, m in zip(ql, kl):
        sees = [(m - n + j + 1) if causal else m for j in range(n)]
        parts.append(attn_ref.attend(q[a:a + n].float().cpu().numpy(), k[b:b + m].float().cpu().numpy(),
                                     v[b:b + m].float().cpu().numpy(), sees, scale, kind))
        a, b = a + n, b + m
    return [np.concatenate(p) for p in zip(*parts)]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("kind,heads,kv_heads,dim", [("bf16", 4, 1, 128), ("fp16", 2, 2, 64), ("bf16", 6, 2, 80),
                                                     ("fp16", 5, 1, 96), ("bf16", 2, 1, 256), ("fp16", 3, 3, 16),
                                                     ("fp16", 2, 1, 200)])
@pytest.mark.parametrize("ql,kl", [([1], [1]), ([64, 65, 1, 0, 130], None), ([3, 200, 17], [90, 64, 0]),
                                   ([127, 128, 33], [40, 300, 33])])
def test_prompt(cf, kind, heads, kv_heads, dim, causal, ql, kl):
    _say("prompt", kind, heads, kv_heads, dim, causal, ql, kl)
    kl = kl or ql
    g = torch.Generator(device="cuda").manual_seed(dim)
    q = torch.randn((sum(ql), heads, dim), generator=g, device="cuda").to(DT[kind])
    k = torch.randn((sum(kl), kv_heads, dim), generator=g, device="cuda").to(DT[kind])
    v = torch.randn((sum(kl), kv_heads, dim), generator=g, device="cuda").to(DT[kind])
    qs, ks = _i32(np.r_[0, np.cumsum(ql)]), _i32(np.r_[0, np.cumsum(kl)])
    got = cf.cf_attn_prompt(q, k, v, qs, ks, causal=causal, lse=True)
    _compare(*got, _want_prompt(q, k, v, ql, kl, causal, dim ** -0.5, kind))
    again = cf.cf_attn_prompt(q, k, v, qs, ks, causal=causal)
    assert torch.equal(got[0], again)


def test_prompt_of_many_short_sequences(cf):
    """More sequences than the search's first probes, empty ones among them."""
    rng = np.random.default_rng(3)
    ql = np.where(rng.random(300) < 0.2, 0, rng.integers(1, 9, 300)).tolist()
    g = torch.Generator(device="cuda").manual_seed(3)
    q, k, v = (torch.randn((sum(ql), h, 64), generator=g, device="cuda").to(torch.bfloat16) for h in (2, 1, 1))
    got = cf.cf_attn_prompt(q, k, v, _i32(np.r_[0, np.cumsum(ql)]), causal=True, lse=True)
    _compare(*got, _want_prompt(q, k, v, ql, ql, True, 0.125, "bf16"))


@pytest.mark.parametrize("causal", [True, False])
def test_prompt_slices_of_a_fused_projection(cf, causal):
    """Strided q, k and v, sequences that begin after the first token, NaN around them."""
    ql = [40, 100]
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn((200, 8, 64), generator=g, device="cuda").to(torch.bfloat16)
    x[:20], x[160:] = float("nan"), float("nan")
    q, k, v = x[:, :4], x[:, 4:6], x[:, 6:]
    qs = _i32([20, 60, 160])
    out, lse = cf.cf_attn_prompt(q, k, v, qs, causal=causal, lse=True)
    _compare(out[20:160], lse[20:160], _want_prompt(q, k, v, ql, ql, causal, 0.125, "bf16", 20, 20))


@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_prompt_special_values(cf, value):
    n, at = 300, [70, 71, 200]
    g = torch.Generator(device="cuda").manual_seed(7)
    q, k, v = (torch.randn((n, 2, 64), generator=g, device="cuda").to(torch.float16) for _ in range(3))
    want = _want_prompt(q, k, v, [n], [n], True, 0.125, "fp16")
    v[at, 1, 9] = value
    got = cf.cf_attn_prompt(q, k, v, _i32([0, n]), causal=True).double().cpu().numpy()
    hit = np.zeros(got.shape, bool)
    hit[min(at):, 1, 9] = True
    assert np.all(np.isnan(got[hit]) if np.isnan(value) else got[hit] == value)
    assert np.all(np.abs(got - want[0])[~hit] <= want[2][~hit])


def test_scores_of_any_size(cf):
    """Scores far apart (a running maximum that jumps) and equal ones."""
    n = 200
    g = torch.Generator(device="cuda").manual_seed(9)
    q, k, v = (torch.randn((n, 2, 64), generator=g, device="cuda").to(torch.bfloat16) for _ in range(3))
    k[50], k[150], q[10:20] = k[50] * 30, k[150] * 60, 0
    _compare(*cf.cf_attn_prompt(q, k, v, _i32([0, n]), causal=False, scale=2.0, lse=True),
             _want_prompt(q, k, v, [n], [n], False, 2.0, "bf16"))


# ------------------------------------------------------------------ enough rows for two wave groups
def _sampled(q, k, v, rows, sees, heads, scale, kind):
    """Reference of some rows and heads: q [n][H][D] of one sequence (device tensors)."""
    G = q.shape[1] // k.shape[1]
    out = []
    for h in heads:
        out.append(attn_ref.attend(q[rows][:, h:h + 1].float().cpu().numpy(),
                                   k[:, h // G:h // G + 1].float().cpu().numpy(),
                                   v[:, h // G:h // G + 1].float().cpu().numpy(), [sees[r] for r in rows], scale, kind))
    return [np.concatenate(p, axis=1) for p in zip(*out)]


@pytest.mark.parametrize("kind,dim", [("bf16", 128), ("fp16", 96), ("fp16", 128), ("bf16", 72)])
@pytest.mark.parametrize("causal", [True, False])
def test_prompt_of_many_rows(cf, kind, dim, causal):
    """3100 rows of each of 16 key/value heads, keys fewer, as many and more than the queries."""
    n, H = 3100, 16
    for m in (2900, n, 3333):
        _say("many rows", kind, dim, causal, m)
        g = torch.Generator(device="cuda").manual_seed(m)
        q = torch.randn((n, H, dim), generator=g, device="cuda").to(DT[kind])
        k, v = (torch.randn((m, H, dim), generator=g, device="cuda").to(DT[kind]) for _ in range(2))
        sees = [min(max(m - n + j + 1, 0), m) if causal else m for j in range(n)]
        rows = sorted({0, 1, 63, 64, 127, 128, 199, 200, 201, 255, 256, 300, 511, 1600, 2815, 2816, 3071, 3080, n - 2, n - 1})
        out, lse = cf.cf_attn_prompt(q, k, v, _i32([0, n]), _i32([0, m]), causal=causal, lse=True)
        heads = [0, 7, 15]
        _compare(out[rows][:, heads], lse[rows][:, heads], _sampled(q, k, v, rows, sees, heads, dim ** -0.5, kind))


@pytest.mark.parametrize("kind,ctx,new,heads,kv_heads,dim,page", [
    ("bf16", 150, 3100, 16, 16, 128, 16), ("fp16", 1, 3100, 32, 16, 96, 64), ("bf16", 40000, 3100, 16, 4, 128, 16)])
def test_paged_many_rows(cf, kind, ctx, new, heads, kv_heads, dim, page):
    """The same over a cache, the last one with its context split; NaN in the unused pages and,
    in one value past most rows' sight, an infinity."""
    _say("paged many rows", kind, ctx, new)
    kv = ctx + new
    g = torch.Generator(device="cuda").manual_seed(new)
    used = -(-kv // page)
    perm = torch.randperm(used + 9, generator=g, device="cuda")
    table = perm[:used].int()[None].contiguous()
    k, v = (torch.randn((kv, kv_heads, dim), generator=g, device="cuda").to(DT[kind]) for _ in range(2))
    q = torch.randn((new, heads, dim), generator=g, device="cuda").to(DT[kind])
    special = kv - 40
    v[special, 1, 3] = float("inf")
    kc, vc = (torch.full((used + 9, kv_heads, page, dim), float("nan"), device="cuda").to(DT[kind]) for _ in range(2))
    at = torch.arange(kv, device="cuda")
    slots = perm[at // page] * page + at % page
    cf.cf_kv_write(k, v, kc, vc, slots)
    plan = cf.cf_attn_plan(_i32([0, new]), _i32([kv]), new, new, heads, kv_heads, dim)
    out, lse = cf.cf_attn_paged(plan, q, kc, vc, table, lse=True)
    again = cf.cf_attn_paged(plan, q, kc, vc, table)
    assert torch.equal(out, again)
    rows = [0, 1, 31, 64, 255, 256, 1000, 2047, 2048, 3000, new - 42, new - 41]
    G = heads // kv_heads
    hs = [0, G, heads - 1]
    v[special, 1, 3] = 0
    _compare(out[rows][:, hs], lse[rows][:, hs],
             _sampled(q, k, v, rows, [ctx + j + 1 for j in range(new)], hs, dim ** -0.5, kind))
    seen = out[new - 40:, G:2 * G]
    assert bool(torch.isinf(seen[:, :, 3]).all()) and bool(torch.isfinite(out[:new - 40]).all())
    rest = torch.ones(dim, dtype=torch.bool, device="cuda")
    rest[3] = False
    assert bool(torch.isfinite(seen[:, :, rest]).all())


def test_plan_of_many_requests(cf):
    """More requests than one pass of the plan takes, with and without new tokens, few and many
    rows, split and whole contexts, in one step."""
    rng = np.random.default_rng(11)
    n = 1500
    new = np.where(rng.random(n) < 0.3, 0, 1)
    new[[5, 700, 1400]] = [40, 90, 17]
    kv = np.where(new > 0, rng.integers(1, 60, n) + new, rng.integers(0, 60, n))
    kv[[6, 1200]] = 9000
    new[[6, 1200]] = 1
    ctx = (kv - new).tolist()
    c = _paged_case("bf16", ctx, new.tolist(), 2, 1, 64, 16)
    want = _want_paged(c, ctx, new.tolist(), 0.125, "bf16")
    for max_new in (None, 1):
        _compare(*_run_paged(cf, c, new.tolist(), 2, 1, 64, max_new=max_new), want)


@pytest.mark.parametrize("max_new", [3100, 8])
def test_long_chunk_among_decodes(cf, max_new):
    """A chunk of 3100 tokens with running and waiting requests around it: the many-row kernel with
    two groups and the few-row kernel in one step, and with a bound on new tokens that is too low."""
    ctx, new, heads, kv_heads, dim, page = [70, 33, 20, 500, 8], [1, 3100, 0, 1, 3], 32, 16, 128, 32
    n = len(ctx)
    g = torch.Generator(device="cuda").manual_seed(2)
    kv = [c + m for c, m in zip(ctx, new)]
    pages = [-(-x // page) for x in kv]
    perm = torch.randperm(sum(pages) + 3, generator=g, device="cuda")
    table = torch.full((n, max(pages)), -1, dtype=torch.int32, device="cuda")
    kc, vc = (torch.full((sum(pages) + 3, kv_heads, page, dim), float("nan"), device="cuda").to(torch.bfloat16)
              for _ in range(2))
    ks, vs, at = [], [], 0
    for i in range(n):
        table[i, :pages[i]] = perm[at:at + pages[i]].int()
        k, v = (torch.randn((kv[i], kv_heads, dim), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
        t = torch.arange(kv[i], device="cuda")
        cf.cf_kv_write(k, v, kc, vc, perm[at + t // page] * page + t % page)
        ks.append(k)
        vs.append(v)
        at += pages[i]
    q = torch.randn((sum(new), heads, dim), generator=g, device="cuda").to(torch.bfloat16)
    starts = np.concatenate([[0], np.cumsum(new)])
    plan = cf.cf_attn_plan(_i32(starts), _i32(kv), sum(new), max_new, heads, kv_heads, dim)
    out, lse = cf.cf_attn_paged(plan, q, kc, vc, table, lse=True)
    hs = [0, 3, 31]
    for i in range(n):
        rows = [r for r in (0, 1, 2, 7, 127, 128, 1000, 2559, 2560, 3098, 3099) if r < new[i]]
        if not rows:
            continue
        o = int(starts[i])
        want = _sampled(q[o:o + new[i]], ks[i], vs[i], rows, [ctx[i] + j + 1 for j in range(new[i])], hs, dim ** -0.5,
                        "bf16")
        _compare(out[o:o + new[i]][rows][:, hs], lse[o:o + new[i]][rows][:, hs], want)
