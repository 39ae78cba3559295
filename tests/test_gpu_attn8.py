"""Attention over the 8-bit paged cache against the 64-bit form on the values held."""
import ctypes as C

import numpy as np
import pytest

from tests import attn_ref, kv8_ref as ref
from tests.test_gpu_attn import LENS, _compare, _i32, _say, _want_paged
from tests.test_gpu_attn_guards import BIG, SHAPES, Guarded, Step

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DT = ref.DT


@pytest.fixture(scope="module")
def cf():
    from paper_2512_14098_amd import cf as _cf
    return _cf


def _case(kind, ctx, new, heads, kv_heads, dim, page, seed=0, spread=3, poison=(0x7f, 255)):
    """Requests' keys and values in an 8-bit cache of shuffled pages, rows of different scales; cells that no
    token owns hold poison.  ks and vs are the values held."""
    rng = np.random.default_rng(seed + sum(ctx) + dim)
    kv = [c + m for c, m in zip(ctx, new)]
    used = [-(-x // page) for x in kv]
    n_pages = sum(used) + 3
    order = rng.permutation(n_pages)
    table = np.full((len(kv), max(max(used), 1)), -1, np.int64)
    codes = np.full((2, n_pages, kv_heads, page, dim), poison[0], np.uint8)
    exps = np.full((n_pages, kv_heads, 2, page), poison[1], np.uint8)
    held, at = ([], []), 0
    for i, x in enumerate(kv):
        for which in range(2):
            y = rng.standard_normal((x, kv_heads, dim))
            if which:  # keys keep their size, or the scores would be those of one key
                y = y * 2.0 ** rng.integers(-spread, spread + 1, (x, kv_heads, 1))
            code, byte = ref.quantise(torch.from_numpy(y).to(DT[kind]).double().numpy(), kind)
            for p in range(used[i]):
                table[i, p] = order[at + p]
                a, b = p * page, min((p + 1) * page, x)
                codes[which, order[at + p], :, :b - a] = code[a:b].transpose(1, 0, 2)
                exps[order[at + p], :, which, :b - a] = byte[a:b].T
            held[which].append(torch.from_numpy(ref.held(code, byte)).to(DT[kind]))
        at += used[i]
    q = torch.from_numpy((1.5 * rng.standard_normal((sum(new), heads, dim))).astype(np.float32)).to(DT[kind])
    return dict(q=q, kc=codes[0], vc=codes[1], exps=exps, table=table, ks=held[0], vs=held[1], kv=kv,
                q_start=np.concatenate([[0], np.cumsum(new)]))


def _e4m3(x):
    return torch.as_tensor(x).cuda().view(torch.float8_e4m3fn)


def _run(cf, c, new, heads, kv_heads, dim, max_new=None, scale=None, kv_len=None):
    n_tok = int(sum(new))
    plan = cf.cf_attn_plan(_i32(c["q_start"]), _i32(c["kv"] if kv_len is None else kv_len), n_tok,
                           max(new) if max_new is None else max_new, heads, kv_heads, dim)
    return cf.cf_attn_paged8(plan, c["q"].cuda(), _e4m3(c["kc"]), _e4m3(c["vc"]), torch.as_tensor(c["exps"]).cuda(),
                             _i32(c["table"]), scale=scale, lse=True)


@pytest.mark.parametrize("lens", sorted(LENS))
@pytest.mark.parametrize("kind,heads,kv_heads,dim,page", [
    ("bf16", 4, 1, 128, 16), ("fp16", 4, 2, 64, 32), ("bf16", 3, 3, 80, 64), ("fp16", 7, 1, 96, 16),
    ("bf16", 2, 2, 16, 128), ("fp16", 6, 2, 144, 16), ("bf16", 4, 2, 256, 256), ("fp16", 20, 1, 48, 16),
    ("bf16", 8, 1, 112, 64), ("fp16", 4, 1, 192, 32)])
def test_paged8(cf, kind, heads, kv_heads, dim, page, lens):
    _say("paged8", kind, heads, kv_heads, dim, page, lens)
    ctx, new = LENS[lens]
    c = _case(kind, ctx, new, heads, kv_heads, dim, page)
    want = _want_paged(c, ctx, new, dim ** -0.5, kind)
    for max_new in (None, sum(new)):
        _compare(*_run(cf, c, new, heads, kv_heads, dim, max_new), want)


@pytest.mark.parametrize("new", [1, 5, 70])
def test_split_contexts(cf, new):
    """One request, two key/value heads: joined parts are right, and the same on every call."""
    _say("split", new)
    c = _case("bf16", [9000], [new], 4, 2, 64, 16)
    a, b = _run(cf, c, [new], 4, 2, 64), _run(cf, c, [new], 4, 2, 64)
    _compare(*a, _want_paged(c, [9000], [new], 0.125, "bf16"))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
def test_as_the_16_bit_cache(cf, kind, dim):
    """Many rows: to the bit what the 16-bit cache of the values held gives."""
    ctx, new, page = [37, 0, 600], [200, 90, 70], 32
    c = _case(kind, ctx, new, 6, 2, dim, page, poison=(0, 0))
    got = _run(cf, c, new, 6, 2, dim)
    byte = torch.as_tensor(c["exps"]).double()
    kc, vc = ((torch.as_tensor(x).view(torch.float8_e4m3fn).double() * torch.exp2(byte[:, :, w] - 127)[..., None])
              .to(DT[kind]).cuda() for w, x in enumerate((c["kc"], c["vc"])))
    plan = cf.cf_attn_plan(_i32(c["q_start"]), _i32(c["kv"]), sum(new), max(new), 6, 2, dim)
    want = cf.cf_attn_paged(plan, c["q"].cuda(), kc, vc, _i32(c["table"]), lse=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("poison", [(0x7f, 255), (0x7e, 254), (0xff, 1), (0x01, 255)])
def test_masked_places_hold_anything(cf, poison):
    for ctx, new in (([17, 40], [1, 3]), ([5, 0], [60, 130])):
        c = _case("fp16", ctx, new, 4, 2, 64, 32, poison=poison)
        _compare(*_run(cf, c, new, 4, 2, 64), _want_paged(c, ctx, new, 0.125, "fp16"))


@pytest.mark.parametrize("kind,dim", [("bf16", 128), ("fp16", 64), ("bf16", 80)])
@pytest.mark.parametrize("ctx,new,at", [([60], [4], [62]), ([100], [90], [130, 150]), ([0], [200], [70, 199]),
                                        ([6000], [3], [6001]), ([6000], [40], [6003, 6039])])
@pytest.mark.parametrize("cell", [(0x7f, None), (0x38, 255)])
def test_special_values_reach_only_the_rows_that_see_them(cf, kind, dim, ctx, new, at, cell):
    """A NaN code, or a byte that is no scale, among a later token's keys or values leaves earlier rows alone."""
    _say("specials", kind, dim, ctx, new, at, cell)
    heads, page = 4, 16
    c = _case(kind, ctx, new, heads, 2, dim, page)
    out, wl, tol, ltol = _want_paged(c, ctx, new, dim ** -0.5, kind)
    code, byte = cell
    for p in at:
        pg, off = c["table"][0, p // page], p % page
        c["vc"][pg, 1, off, 5] = code
        c["kc"][pg, 0, off, 3] = 0x7f
        if byte is not None:
            c["exps"][pg, 1, 1, off] = byte
    got, lse = (x.double().cpu().numpy() for x in _run(cf, c, new, heads, 2, dim))
    sees = np.array([ctx[0] + j >= min(at) for j in range(new[0])])
    hit = np.zeros(got.shape, bool)
    if byte is None:  # only element 5 of the rows that see the value
        hit[sees, 2:, 5] = True
    else:  # a byte of 255 makes the whole row of values NaN
        hit[sees, 2:, :] = True
    hit[sees, :2, :] = True  # key/value head 0: a NaN score spoils the whole row
    assert np.all(~np.isfinite(got[hit]))
    assert np.all(np.abs(got - out)[~hit] <= tol[~hit])
    assert np.all(np.abs(lse - wl)[:, 2:] <= ltol[:, 2:])


@pytest.mark.parametrize("kind,heads,dim,ctx,new", [("bf16", 128, 64, 40, 5), ("fp16", 128, 128, 100, 3),
                                                    ("bf16", 160, 80, 9, 4), ("fp16", 136, 256, 50, 2),
                                                    ("bf16", 128, 64, 6000, 2), ("bf16", 16, 128, 77, 3)])
def test_last_value_is_hidden_where_a_tile_has_one_token(cf, kind, heads, dim, ctx, new):
    """All rows of a tile see the same keys, and the tile's last keys are seen by none of them; with 16 heads and
    a bound of one new token that is too low, in the few-row kernel."""
    _say("one token a tile", kind, heads, dim, ctx, new)
    c = _case(kind, [ctx], [new], heads, 1, dim, 16)
    out, _, tol, _ = _want_paged(c, [ctx], [new], dim ** -0.5, kind)
    p = ctx + new - 1
    c["vc"][c["table"][0, p // 16], 0, p % 16, 3] = 0xff
    got = _run(cf, c, [new], heads, 1, dim, max_new=1 if heads == 16 else None)[0].double().cpu().numpy()
    hit = np.zeros(got.shape, bool)
    hit[new - 1, :, 3] = True
    assert not np.isfinite(got[hit]).any() and (np.abs(got - out) <= tol)[~hit].all()


def test_rows_that_see_nothing(cf):
    """kv_len 0 (a refused request) and fewer keys than new tokens: zero rows, lse -inf."""
    for heads in (2, 8):
        ctx, new = [20, 33, 0], [2, 30, 40]
        c = _case("bf16", ctx, new, heads, 2, 64, 16)
        kv = [0, 10, 40]
        got = _run(cf, c, new, heads, 2, 64, kv_len=kv)
        parts, at = [], 0
        for i, m in enumerate(new):
            parts.append(attn_ref.attend(c["q"][at:at + m].float().numpy(), c["ks"][i].float().numpy(),
                                         c["vs"][i].float().numpy(), [kv[i] - m + j + 1 for j in range(m)], 0.125,
                                         "bf16"))
            at += m
        _compare(*got, [np.concatenate(p) for p in zip(*parts)])


def test_rows_whose_scores_are_all_minus_infinity(cf):
    """A query of -inf against keys that are all positive: 0 and lse -inf, few rows and many."""
    for new in (1, 40):
        c = _case("bf16", [130 - new], [new], 2, 1, 64, 16, poison=(0x38, 127))
        c["kc"][:] = 0x38  # 1.0
        c["q"][:] = 1.0
        c["q"][:, :, 7] = float("-inf")
        out, lse = _run(cf, c, [new], 2, 1, 64)
        assert bool((out == 0).all()) and bool(torch.isneginf(lse).all())


def test_pages_outside_the_cache_read_as_zeros(cf):
    ctx, new = [100, 100], [1, 40]
    c = _case("fp16", ctx, new, 4, 2, 64, 16)
    for i, bad in ((0, -5), (1, 10 ** 6)):
        c["table"][i, 2] = bad
        c["ks"][i][32:48] = 0
        c["vs"][i][32:48] = 0
    _compare(*_run(cf, c, new, 4, 2, 64), _want_paged(c, ctx, new, 0.125, "fp16"))


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
def test_scales_over_the_type_s_range(cf, kind):
    """Values next to the least and the largest numbers of the element type, exactly as held."""
    for e in ((-120, 100) if kind == "bf16" else (-14, 12)):
        ctx, new, dim = [50, 20], [2, 33], 64
        c = _case(kind, ctx, new, 4, 2, dim, 16, spread=0)
        shift = np.where(c["exps"][:, :, 1] == 255, 0, e)
        c["exps"][:, :, 1] = np.maximum(c["exps"][:, :, 1].astype(int) + shift, 1)
        for i, v in enumerate(c["vs"]):
            for t in range(c["kv"][i]):
                pg, off = c["table"][i, t // 16], t % 16
                v[t] = torch.from_numpy(ref.held(c["vc"][pg, :, off], c["exps"][pg, :, 1, off])).to(DT[kind])
        # The bound is that of the values over 2^e, whose size is 1 (an absolute term of 2^-24 is lost in
        # a sum with terms of 2^-129, and those in it), plus half a step below the type's normal range.
        c["vs"] = [v.double() * 2.0 ** -e for v in c["vs"]]
        out, _, tol, _ = _want_paged(dict(c, vs=[v.float() for v in c["vs"]]), ctx, new, 0.125, kind)
        tol = tol + 2.0 ** ((-25 if kind == "fp16" else -134) - e)
        got, lse = _run(cf, c, new, 4, 2, dim)
        assert (np.abs(got.double().cpu().numpy() * 2.0 ** -e - out) <= tol).all()


@pytest.mark.parametrize("n_q,heads,dim", [(1, 4, 64), (1, 16, 128), (3, 16, 64), (140, 2, 128), (9, 16, 256)])
def test_many_small_weights(cf, n_q, heads, dim):
    """One key with the score 18 and value 0 before keys with the score 0: weights of e^-18 of the largest, below
    half of fp16's least number, whose sum counts.  Few and many rows, the context split and whole."""
    m, page = 32766, 64
    _say("tail", n_q, heads, dim)
    rng = np.random.default_rng(n_q)
    n_pages = -(-m // page)
    q = np.zeros((n_q, heads, dim), np.float32)
    q[:, :, 0] = 1.0
    k = np.zeros((m, 1, dim))
    k[0, 0, 0] = 18.0
    v = rng.uniform(0.5, 1.5, (m, 1, dim))
    v[0] = 0
    c = [torch.zeros((n_pages, 1, page, dim), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2)]
    c.append(torch.zeros((n_pages, 1, 2, page), dtype=torch.uint8, device="cuda"))
    cf.cf_kv_write8(torch.from_numpy(k).half().cuda(), torch.from_numpy(v).half().cuda(), *c,
                    torch.arange(m, device="cuda"))
    vh = ref.held(*ref.quantise(torch.from_numpy(v).half().double().numpy(), "fp16"))
    row = torch.arange(n_pages, dtype=torch.int32, device="cuda")
    for n in (1, 600):
        plan = cf.cf_attn_plan(_i32(np.arange(n + 1) * n_q), _i32([m] * n), n * n_q, n_q, heads, 1, dim)
        out, lse = cf.cf_attn_paged8(plan, torch.from_numpy(q).half().cuda().repeat(n, 1, 1), *c, row.repeat(n, 1),
                                     scale=1.0, lse=True)
        for j in (0, n_q - 1):
            s = m - n_q + j + 1
            x = k[:s, 0, 0]
            p = np.exp(x - 18.0)
            l = p.sum()
            want, A = p @ vh[:s, 0] / l, p @ np.abs(vh[:s, 0]) / l
            e = 18.0 * (dim + 4) * 2.0 ** -24
            # attn_ref's bound; weights carry a factor of 2^7 at least, so 2^-32 of the largest a key
            tol = ((2 * 2.0 ** -11 + 2 * (2 * e + 2.0 ** -20) + (s + 64) * 2.0 ** -23) * A
                   + 2.0 ** -32 * np.abs(vh[:s, 0]).sum(0) / l + 2.0 ** -24)
            got = out[-n_q + j].double().cpu().numpy()
            assert (np.abs(got - want[None]) <= tol[None]).all(), (j, np.abs(got - want[None]).max())
            ln = 18.0 + np.log(l)
            assert abs(float(lse[-n_q + j, 0]) - ln) <= 2 * e + (s + 64) * 2.0 ** -23 + ln * 2.0 ** -22 + 2.0 ** -20


def test_strides_scale_and_stream(cf):
    """Queries out of a fused projection, another scale, work on a stream that is not the default."""
    ctx, new = [30, 5, 300], [1, 4, 50]
    c = _case("bf16", ctx, new, 4, 2, 80, 16)
    want = _want_paged(c, ctx, new, 0.3, "bf16")
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        fused = torch.zeros((sum(new), 8, 80), dtype=torch.bfloat16, device="cuda")
        fused[:, 3:7] = c["q"].cuda()
        plan = cf.cf_attn_plan(_i32(c["q_start"]), _i32(c["kv"]), sum(new), 50, 4, 2, 80)
        got = cf.cf_attn_paged8(plan, fused[:, 3:7], _e4m3(c["kc"]), _e4m3(c["vc"]), torch.as_tensor(c["exps"]).cuda(),
                                _i32(c["table"]), scale=0.3, lse=True)
    s.synchronize()
    _compare(*got, want)


def test_offsets_past_32_bits(cf):
    """A cache of more than 2^32 codes and of 2^32 exponent bytes, the request's pages at its far end."""
    for heads, dim, page, bytes_of in ((4, 128, 64, 128), (65535, 16, 16, 2)):
        n_pages = (1 << 32) // (heads * page * bytes_of) + 40
        _say("cache of", n_pages, "pages")
        new = 20 if heads == 4 else 2
        if heads == 4:
            c = _case("bf16", [500], [new], heads, heads, dim, page)
            kc, vc = (torch.empty((n_pages, heads, page, dim), dtype=torch.uint8, device="cuda") for _ in range(2))
            exps = torch.empty((n_pages, heads, 2, page), dtype=torch.uint8, device="cuda")
            small = c["kc"].shape[0]
            kc[-small:], vc[-small:] = torch.as_tensor(c["kc"]).cuda(), torch.as_tensor(c["vc"]).cuda()
            exps[-small:] = torch.as_tensor(c["exps"]).cuda()
            table = _i32(np.where(c["table"] >= 0, c["table"] + n_pages - small, -1))
            cache = kc.view(torch.float8_e4m3fn), vc.view(torch.float8_e4m3fn), exps
            plan = cf.cf_attn_plan(_i32(c["q_start"]), _i32(c["kv"]), new, new, heads, heads, dim)
            _compare(*cf.cf_attn_paged8(plan, c["q"].cuda(), *cache, table, lse=True),
                     _want_paged(c, [500], [new], dim ** -0.5, "bf16"))
        else:
            cache = [torch.empty((n_pages, heads, page, dim), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
                     for _ in range(2)] + [torch.empty((n_pages, heads, 2, page), dtype=torch.uint8, device="cuda")]
        # a write of a token there, and the way back
        k = torch.randn((1, heads, dim), device="cuda").to(torch.bfloat16)
        cf.cf_kv_write8(k, -k, *cache, torch.tensor([n_pages * page - 1], device="cuda"))
        code, byte = ref.quantise(k[0].double().cpu().numpy(), "bf16")
        assert np.array_equal(cache[0][-1, :, -1].view(torch.uint8).cpu().numpy(), code)
        assert np.array_equal(cache[2][-1, :, 0, -1].cpu().numpy(), byte)
        ko, vo = cf.cf_kv_read8(*cache, _i32([[n_pages - 1]]), _i32([0, page]), page)
        assert torch.equal(ko[-1].double().cpu(), torch.from_numpy(ref.held(code, byte))) and torch.equal(vo[-1], -ko[-1])
        del cache


def test_a_million_requests(cf):
    """1.1 million requests of one token, the bound on new tokens not known.  Each request sees one key, so its
    output is that key's value."""
    n, heads, dim, page = 1100000, 8, 80, 16
    _say("a million requests")
    g = torch.Generator(device="cuda").manual_seed(4)
    kc, vc = (torch.randint(0, 127, (64, heads, page, dim), generator=g, device="cuda", dtype=torch.uint8)
              .view(torch.float8_e4m3fn) for _ in range(2))
    exps = torch.full((64, heads, 2, page), 127, dtype=torch.uint8, device="cuda")
    q = torch.full((n, heads, dim), 2.0 ** -9, dtype=torch.bfloat16, device="cuda")
    at = torch.arange(n, device="cuda")
    plan = cf.cf_attn_plan(torch.arange(n + 1, dtype=torch.int32, device="cuda"),
                           torch.ones(n, dtype=torch.int32, device="cuda"), n, n, heads, heads, dim)
    out = cf.cf_attn_paged8(plan, q, kc, vc, exps, (at % 64).int()[:, None].contiguous())
    first = vc[:, :, 0].to(torch.bfloat16)
    for a in range(0, n, 64 * 1000):
        b = min(n, a + 64 * 1000)
        assert torch.equal(out[a:b], first[at[a:b] % 64]), a


def test_decode_step_in_a_graph(cf):
    """map, turn and write, plan and attention captured once and replayed as the requests grow."""
    heads, kv_heads, dim, page, n = 4, 2, 64, 16, 6
    ctx = [0, 15, 16, 40, 100, 31]
    c = _case("bf16", ctx, [0] * n, heads, kv_heads, dim, page)
    steps, most, n_pages = 5, 12, 80
    kc, vc = (torch.zeros((n_pages, kv_heads, page, dim), dtype=torch.uint8, device="cuda") for _ in range(2))
    exps = torch.zeros((n_pages, kv_heads, 2, page), dtype=torch.uint8, device="cuda")
    kc[:c["kc"].shape[0]], vc[:c["vc"].shape[0]] = torch.as_tensor(c["kc"]).cuda(), torch.as_tensor(c["vc"]).cuda()
    exps[:c["exps"].shape[0]] = torch.as_tensor(c["exps"]).cuda()
    kc, vc = kc.view(torch.float8_e4m3fn), vc.view(torch.float8_e4m3fn)
    table = np.full((n, most), -1, np.int64)
    table[:, :c["table"].shape[1]] = c["table"]
    free = np.setdiff1d(np.arange(n_pages), table[table >= 0])
    t, f, cl, nl, h = _i32(table), _i32(free), _i32(ctx), _i32([1] * n), _i32([0])
    g0 = torch.Generator(device="cuda").manual_seed(1)
    qkv = [torch.randn((n, heads + 2 * kv_heads, dim), generator=g0, device="cuda").to(torch.bfloat16)
           for _ in range(steps)]
    freq = torch.from_numpy(10000.0 ** (-np.arange(dim // 2) / (dim // 2))).cuda()
    x = qkv[0].clone()

    def step():
        q_start, kv_len, slots, pos, head, _ = cf.cf_kv_map(cl, nl, t, page, f, h, n)
        q = cf.cf_rope_write8(x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:], pos, freq, None, kc, vc,
                              exps, slots)
        plan = cf.cf_attn_plan(q_start, kv_len, n, 1, heads, kv_heads, dim)
        return cf.cf_attn_paged8(plan, q, kc, vc, exps, t, lse=True), head

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        (out, lse), head = step()
        h.copy_(head)
        cl.add_(nl)
    for i in range(steps):
        x.copy_(qkv[i])
        pos = _i32([a + i for a in ctx])
        g.replay()
        torch.cuda.synchronize()
        q, k = cf.cf_rope(qkv[i][:, :heads], qkv[i][:, heads:heads + kv_heads], pos, freq)
        c["q"] = q.cpu()
        for name, new in (("ks", k), ("vs", qkv[i][:, heads + kv_heads:])):
            value = torch.from_numpy(ref.held(*ref.quantise(new.double().cpu().numpy(), "bf16"))).to(torch.bfloat16)
            for r in range(n):
                c[name][r] = torch.cat([c[name][r], value[r:r + 1]])
        _compare(out, lse, _want_paged(c, [a + i for a in ctx], [1] * n, dim ** -0.5, "bf16"))


# ------------------------------------------------------------------ reads and writes inside the arrays
class Step8(Step):
    """The same through the C ABI on guarded arrays, over an 8-bit cache of any bytes."""

    def __init__(self, cf, n_seq, n_tok, max_new, heads, kv_heads, dim, page, columns, n_pages=9, seed=0):
        dim = -(-dim // 16) * 16
        super().__init__(cf, n_seq, n_tok, max_new, heads, kv_heads, dim, page, columns, n_pages, seed)
        g = torch.Generator(device="cuda").manual_seed(seed)
        n = n_pages * kv_heads * page
        noise = lambda m: Guarded(m, torch.randint(0, 256, (m,), generator=g, device="cuda", dtype=torch.uint8))
        self.kc, self.vc, self.ec = noise(n * dim), noise(n * dim), noise(2 * n)
        self.c = cf.cf_kv_cache8(self.kc.ptr(), self.vc.ptr(), self.ec.ptr(), n_pages, page, kv_heads, dim, 0)
        self.inputs = [(x, x.buf.clone()) for x in (self.kc, self.vc, self.ec, self.q, self.table)]

    def run(self):
        assert self.cf.lib().cf_attn_paged8(C.byref(self.d), C.byref(self.c), self.table.ptr(), self.columns,
                                            self.q.ptr(), self.heads * self.dim, self.dim, 0.125, self.out.ptr(),
                                            self.lse.ptr(), self.cf._stream()) == 0
        torch.cuda.synchronize()
        assert self.out.intact() and self.lse.intact() and self.work.intact()
        for x, before in self.inputs:
            assert torch.equal(x.buf, before)


@pytest.mark.parametrize("shape", SHAPES)
def test_malformed_lengths(cf, shape):
    """Starts in any order, lengths of any size, table entries outside the cache, a workspace without a plan."""
    print("malformed", shape, flush=True)
    n, n_tok = shape[0], shape[1]
    rng = np.random.default_rng(n_tok)
    s = Step8(cf, *shape)
    for starts, kv in [([n_tok, 3, -9] + [n_tok] * (n - 2), [-1, 7] + [9] * (n - 2)),
                       ([0] * n + [2 ** 31 - 1], [2 ** 31 - 1] * n), ([-2 ** 31] * (n + 1), [5] * n)] + [
                           (rng.choice(BIG, n + 1), rng.choice(BIG, n)) for _ in range(20)]:
        s.plan(starts, kv)
        s.run()
    words = s.work.n // 4
    for values in (BIG, [0, 1, 2, 3, 2 ** 27, 2 ** 28], [0, 1, 2, 4, 128, 256], None):
        x = rng.integers(-2 ** 31, 2 ** 31, words) if values is None else rng.choice(values, words)
        s.work.bytes().copy_(_i32(np.asarray(x, np.int64).astype(np.int32)).view(torch.uint8)[:s.work.n])
        s.run()


def test_rows_of_no_request_are_left(cf):
    s = Step8(cf, 3, 60, 60, 4, 2, 64, 16, 4)
    s.ec.bytes().fill_(120)
    s.inputs = [(x, x.buf.clone()) for x, _ in s.inputs]
    before = s.out.view(torch.int16).view(60, -1).clone(), s.lse.view(torch.int32).view(60, -1).clone()
    s.plan([5, 8, 8, 50], [64, 9, 2 ** 31 - 1])
    s.run()
    for got, was in zip((s.out.view(torch.int16).view(60, -1), s.lse.view(torch.int32).view(60, -1)), before):
        assert torch.equal(got[:5], was[:5]) and torch.equal(got[50:], was[50:])
        assert bool((got[5:50] != was[5:50]).any(1).all())
    first = s.out.bytes().clone()
    s.plan([5, 8, 8, 50], [64, 9, 64])
    s.run()
    assert torch.equal(first, s.out.bytes())


def test_turn_write_and_read_stay_inside(cf):
    """Rotary positions, writes and reads between guards, with slots, axes, starts and pages of any size."""
    rng = np.random.default_rng(3)
    heads, kv, dim, page, n_pages, n = 3, 2, 48, 16, 7, 90
    g = torch.Generator(device="cuda").manual_seed(1)
    x = Guarded(n * 7 * dim * 2, torch.randn((n, 7, dim), generator=g, device="cuda").to(torch.float16))
    kc, vc, ec = Guarded(n_pages * kv * page * dim), Guarded(n_pages * kv * page * dim), Guarded(2 * n_pages * kv * page)
    qo, ko, vo = Guarded(n * heads * dim * 2), Guarded(n * kv * dim * 2), Guarded(n * kv * dim * 2)
    c = cf.cf_kv_cache8(kc.ptr(), vc.ptr(), ec.ptr(), n_pages, page, kv, dim, 1)
    tok, q, k, v = 7 * dim, x.ptr(), x.ptr() + heads * dim * 2, x.ptr() + (heads + kv) * dim * 2
    freq = torch.rand(dim // 2, dtype=torch.float64, device="cuda")
    lib, s = cf.lib(), cf._stream()
    was = x.buf.clone()
    for trial in range(20):
        pos = Guarded(3 * n * 4, _i32(rng.choice(BIG, 3 * n)))
        axis = Guarded(dim * 2, _i32(rng.choice(BIG, dim // 2)))
        slots = rng.choice([-2 ** 63, -2 ** 32, -1, n_pages * page, 2 ** 31, 2 ** 32, 2 ** 63 - 1], n)
        slots[::2] = rng.permutation(n_pages * page)[:len(slots[::2])]
        sl = Guarded(8 * n, torch.as_tensor(slots).cuda())
        r = cf.cf_rope_desc(3, dim, trial % 2, 0, pos.ptr(), freq.data_ptr(), axis.ptr())
        assert lib.cf_rope_write8(C.byref(r), C.byref(c), n, heads, q, tok, dim, qo.ptr(), heads * dim, dim, k, tok, dim, v,
                                  tok, dim, sl.ptr(), s) == 0
        assert lib.cf_rope(C.byref(r), n, heads, kv, dim, 1, q, tok, dim, qo.ptr(), heads * dim, dim, k, tok, dim, ko.ptr(),
                           kv * dim, dim, s) == 0
        assert lib.cf_kv_write8(C.byref(c), n, k, tok, dim, v, tok, dim, sl.ptr(), s) == 0
        table = Guarded(4 * 5 * 4, _i32(np.where(rng.random(20) < 0.5, rng.choice(BIG, 20), rng.integers(0, n_pages, 20))))
        start = Guarded(4 * 6, _i32(rng.choice(BIG + [50, 60, 70, 90], 6)))
        assert lib.cf_kv_read8(C.byref(c), table.ptr(), 4, 5, start.ptr(), n, ko.ptr(), vo.ptr(), s) == 0
        torch.cuda.synchronize()
        assert all(y.intact() for y in (kc, vc, ec, qo, ko, vo, pos, axis, sl, table, start)) and torch.equal(x.buf, was)


def test_read_leaves_rows_of_no_request(cf):
    ko, vo = Guarded(30 * 32 * 2), Guarded(30 * 32 * 2)
    kc, vc, ec = (torch.full((2 * 16 * n,), 0x38, dtype=torch.uint8, device="cuda") for n in (32, 32, 2))
    c = cf.cf_kv_cache8(kc.data_ptr(), vc.data_ptr(), ec.data_ptr(), 2, 16, 1, 32, 0)
    start, table = _i32([4, 9, 9, 20]), _i32([[0], [1], [1]])
    assert cf.lib().cf_kv_read8(C.byref(c), table.data_ptr(), 1, 3, start.data_ptr(), 30, ko.ptr(), vo.ptr(),
                                cf._stream()) == 0
    torch.cuda.synchronize()
    for y in (ko, vo):
        got = y.view(torch.int16).view(30, 32)
        assert y.intact()
        assert bool((got[:4] == 0x5A5A).all()) and bool((got[20:] == 0x5A5A).all())
        assert bool((got[4:20] != 0x5A5A).all())
