"""Edges of the paged-cache calls against plain 64-bit forms: what rows must not see, small weights."""
import numpy as np
import pytest

from tests.test_gpu_attn import DT, _compare, _i32, _paged_case, _run_paged, _sampled, _say, _want_paged, _want_prompt

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def cf():
    from paper_2512_14098_amd import cf as _cf
    return _cf


# ------------------------------------------------------------------ infinities and NaN of later tokens
def _only_last_row(got, want, n, col):
    """All rows but the last are within their bounds; of the last only column ``col`` is not finite."""
    got = got.double().cpu().numpy()
    out, _, tol, _ = want
    hit = np.zeros(got.shape, bool)
    hit[n - 1, :, col] = True
    assert not np.isfinite(got[hit]).any()
    bad = ~(np.abs(got - out) <= tol) & ~hit
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3].tolist())


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("kind,heads,dim,ctx,new", [("bf16", 128, 64, 40, 5), ("fp16", 128, 128, 100, 3),
                                                    ("bf16", 160, 72, 9, 4), ("fp16", 136, 256, 50, 2),
                                                    ("bf16", 128, 64, 6000, 2)])
def test_last_value_is_hidden_where_a_tile_has_one_token(cf, kind, heads, dim, ctx, new, value):
    """As many heads on one key/value head as a workgroup has rows: all rows of a tile see the same
    keys, and the tile's last keys are seen by none of them."""
    _say("one token a tile", kind, heads, dim, ctx, new, value)
    c = _paged_case(kind, [ctx], [new], heads, 1, dim, 16)
    want = _want_paged(c, [ctx], [new], dim ** -0.5, kind)
    p = ctx + new - 1
    c["vc"][c["table"][0, p // 16], 0, p % 16, 3] = value
    _only_last_row(_run_paged(cf, c, [new], heads, 1, dim)[0], want, new, 3)


@pytest.mark.parametrize("value", [float("nan"), float("-inf")])
@pytest.mark.parametrize("kind,dim,ctx", [("bf16", 64, 20), ("fp16", 128, 77), ("bf16", 40, 5000)])
def test_last_value_is_hidden_whatever_max_new_says(cf, kind, dim, ctx, value):
    """Three new tokens of 16 heads on one where the bound on new tokens says one: few rows, a
    token a tile."""
    _say("bound too low", kind, dim, ctx, value)
    c = _paged_case(kind, [ctx], [3], 16, 1, dim, 32)
    want = _want_paged(c, [ctx], [3], dim ** -0.5, kind)
    p = ctx + 2
    c["vc"][c["table"][0, p // 32], 0, p % 32, 5] = value
    _only_last_row(_run_paged(cf, c, [3], 16, 1, dim, max_new=1)[0], want, 3, 5)


@pytest.mark.parametrize("kind,heads,dim,n", [("bf16", 128, 64, 70), ("fp16", 128, 128, 7), ("bf16", 144, 16, 33)])
def test_prompt_last_value_is_hidden_where_a_tile_has_one_token(cf, kind, heads, dim, n):
    _say("prompt, one token a tile", kind, heads, dim, n)
    g = torch.Generator(device="cuda").manual_seed(n)
    q, k, v = (torch.randn((n, h, dim), generator=g, device="cuda").to(DT[kind]) for h in (heads, 1, 1))
    want = _want_prompt(q, k, v, [n], [n], True, dim ** -0.5, kind)
    v[n - 1, 0, 2] = float("nan")
    _only_last_row(cf.cf_attn_prompt(q, k, v, _i32([0, n])), want, n, 2)


@pytest.mark.parametrize("paged", [True, False])
def test_last_value_is_hidden_from_256_heads(cf, paged):
    """The same with two wave groups a workgroup: 256 rows, one token a tile."""
    n, ctx, heads, dim = 200, 30 if paged else 0, 256, 72
    _say("256 heads", paged)
    g = torch.Generator(device="cuda").manual_seed(1)
    m = ctx + n
    q, k, v = (torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
               for s in ((n, heads, dim), (m, 1, dim), (m, 1, dim)))
    hs = [0, 101, 255]
    want = _sampled(q, k, v, list(range(n)), [ctx + j + 1 for j in range(n)], hs, dim ** -0.5, "bf16")
    v[m - 1, 0, 7] = float("inf")
    if paged:
        kc, vc = (torch.full((20, 1, 16, dim), float("nan"), device="cuda").to(torch.bfloat16) for _ in range(2))
        cf.cf_kv_write(k, v, kc, vc, torch.arange(m, device="cuda"))
        plan = cf.cf_attn_plan(_i32([0, n]), _i32([m]), n, n, heads, 1, dim)
        out = cf.cf_attn_paged(plan, q, kc, vc, torch.arange(20, dtype=torch.int32, device="cuda")[None])
    else:
        out = cf.cf_attn_prompt(q, k, v, _i32([0, n]))
    _only_last_row(out[:, hs], want, n, 7)


# ------------------------------------------------------------------ small weights in fp16
def _tail(n_q, heads, m, dim, seed):
    """One key with the score 17.5 and value 0 before m - 1 keys with the score 0: weights of
    e^-17.5 = 2.5e-8 of the largest, below half of fp16's least number, whose sum is 8e-4."""
    rng = np.random.default_rng(seed)
    q = np.zeros((n_q, heads, dim), np.float32)
    k = np.zeros((m, 1, dim), np.float32)
    q[:, :, 0], k[0, 0, 0] = 1.0, 17.5
    v = rng.uniform(0.5, 1.5, (m, 1, dim)).astype(np.float32)
    v[0] = 0
    return [torch.from_numpy(x).half().cuda() for x in (q, k, v)]


def _check_tail(got, q, k, v, sees):
    """As attn_ref's bound, its term for weights below the normal range smaller by the 2^7 by which
    weights are scaled at least (the largest is then 2^7 or more): 2^-32 of the largest a key."""
    pick = [0, len(sees) - 1]
    for j in pick:
        s = sees[j]
        x = k[:s, 0].double().cpu().numpy() @ q[j, 0].double().cpu().numpy()
        p = np.exp(x - x.max())
        vv = v[:s, 0].double().cpu().numpy()
        l = p.sum()
        out, A = p @ vv / l, p @ np.abs(vv) / l
        e = 17.5 * (q.shape[2] + 4) * 2.0 ** -24
        tol = (2 * 2.0 ** -11 + 2 * (2 * e + 2.0 ** -20) + (s + 64) * 2.0 ** -23) * A + 2.0 ** -32 * np.abs(vv).sum(0) / l + 2.0 ** -24
        err = np.abs(got[0][j].double().cpu().numpy() - out[None])
        assert (err <= tol[None]).all(), (j, float(err.max()), float(tol.min()), float(out.max()))
        lse = x.max() + np.log(l)
        assert abs(float(got[1][j, 0]) - lse) <= 2 * e + (s + 64) * 2.0 ** -23 + lse * 2.0 ** -22 + 2.0 ** -20


@pytest.mark.parametrize("n_q,heads,dim", [(1, 4, 64), (1, 16, 128), (3, 16, 64), (140, 2, 128), (9, 16, 256)])
def test_many_small_weights_of_a_cache(cf, n_q, heads, dim):
    """Few and many rows, the context split and whole (a second request fills the plan)."""
    m, page = 32766, 64
    _say("tail", n_q, heads, dim)
    q, k, v = _tail(n_q, heads, m, dim, n_q)
    n_pages = -(-m // page)
    kc, vc = (torch.zeros((n_pages, 1, page, dim), dtype=torch.float16, device="cuda") for _ in range(2))
    cf.cf_kv_write(k, v, kc, vc, torch.arange(m, device="cuda"))
    row = torch.arange(n_pages, dtype=torch.int32, device="cuda")
    for n in (1, 600):
        starts = _i32(np.arange(n + 1) * n_q)
        plan = cf.cf_attn_plan(starts, _i32([m] * n), n * n_q, n_q, heads, 1, dim)
        got = cf.cf_attn_paged(plan, q.repeat(n, 1, 1), kc, vc, row.repeat(n, 1), scale=1.0, lse=True)
        _check_tail([x[-n_q:] for x in got], q, k, v, [m - n_q + j + 1 for j in range(n_q)])


@pytest.mark.parametrize("n_q,heads,dim", [(1, 2, 64), (300, 2, 128), (3100, 16, 96)])
def test_many_small_weights_of_a_prompt(cf, n_q, heads, dim):
    m = 32766
    q, k, v = _tail(n_q, heads, m, dim, n_q)
    got = cf.cf_attn_prompt(q, k, v, _i32([0, n_q]), _i32([0, m]), causal=False, scale=1.0, lse=True)
    _check_tail(got, q, k, v, [m] * n_q)


# ------------------------------------------------------------------ more workgroups than a grid of 512 threads takes
def test_a_million_requests(cf):
    """1.1 million requests of one token, the bound on new tokens not known: 8.8 million workgroups
    of either kernel.  Each request sees one key, so its output is that key's value."""
    n, heads, dim, page = 1100000, 8, 72, 16
    _say("a million requests")
    g = torch.Generator(device="cuda").manual_seed(4)
    kc, vc = (torch.randn((64, heads, page, dim), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    q = torch.ones((n, heads, dim), dtype=torch.bfloat16, device="cuda")
    at = torch.arange(n, device="cuda")
    plan = cf.cf_attn_plan(torch.arange(n + 1, dtype=torch.int32, device="cuda"),
                           torch.ones(n, dtype=torch.int32, device="cuda"), n, n, heads, heads, dim)
    out = cf.cf_attn_paged(plan, q, kc, vc, (at % 64).int()[:, None].contiguous())
    for a in range(0, n, 64 * 1000):
        b = min(n, a + 64 * 1000)
        assert torch.equal(out[a:b], vc[at[a:b] % 64, :, 0]), a


# ------------------------------------------------------------------ a plan used on another stream
def test_workspace_outlives_a_call_on_another_stream(cf):
    """A plan made on one stream, used on another and dropped: its workspace is not handed out again
    while that stream has not come to the call."""
    c = _paged_case("bf16", [500], [1], 4, 2, 64, 16)
    want = _want_paged(c, [500], [1], 0.125, "bf16")
    q, kc, vc, table = c["q"].cuda(), c["kc"].cuda(), c["vc"].cuda(), _i32(c["table"])
    plan = cf.cf_attn_plan(_i32(c["q_start"]), _i32(c["kv"]), 1, 1, 4, 2, 64)
    size, at = plan.work.numel(), plan.work.data_ptr()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        got = cf.cf_attn_paged(plan, q, kc, vc, table, lse=True)
        busy = torch.cuda.Event()
        busy.record()
    del plan
    other = torch.empty(size, dtype=torch.uint8, device="cuda")
    assert not busy.query()  # the call has not run yet
    assert other.data_ptr() != at
    side.synchronize()
    _compare(*got, want)


# ------------------------------------------------------------------ scores of minus infinity
@pytest.mark.parametrize("new", [1, 40])
def test_rows_whose_scores_are_all_minus_infinity(cf, new):
    """Such rows give 0 and lse -inf, as rows that see nothing; one other key makes them its value."""
    dim = 64
    g = torch.Generator(device="cuda").manual_seed(new)
    q = torch.rand((new, 2, dim), generator=g, device="cuda").add(0.5).to(torch.bfloat16)
    k = torch.zeros((130, 1, dim), dtype=torch.bfloat16, device="cuda")
    v = torch.randn((130, 1, dim), generator=g, device="cuda").to(torch.bfloat16)
    k[:, :, 3] = float("-inf")
    kc, vc = (torch.zeros((9, 1, 16, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.arange(9, dtype=torch.int32, device="cuda")[None]
    for other in (None, 70):
        if other is not None:
            k[other] = 0
        cf.cf_kv_write(k, v, kc, vc, torch.arange(130, device="cuda"))
        plan = cf.cf_attn_plan(_i32([0, new]), _i32([130]), new, new, 2, 1, dim)
        for out, lse in (cf.cf_attn_paged(plan, q, kc, vc, table, lse=True),
                         cf.cf_attn_prompt(q, k, v, _i32([0, new]), _i32([0, 130]), causal=False, lse=True)):
            if other is None:
                assert bool((out == 0).all()) and bool(torch.isneginf(lse).all())
            else:
                assert torch.equal(out, v[other].expand_as(out)) and bool((lse == 0).all())
