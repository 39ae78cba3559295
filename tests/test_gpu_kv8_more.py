"""Rotary positions and the 8-bit cache: every code with every scale, and the dispatched forms that other tests leave
out (partial turns written to the cache, long reads of several heads, joins of more tiles than workgroups)."""
import numpy as np
import pytest

from tests import kv8_ref as ref
from tests.test_gpu_attn import _compare, _i32, _sampled, _say, _want_paged
from tests.test_gpu_attn8 import _case, _run
from tests.test_gpu_attn_join import Caches
from tests.test_gpu_kv8 import _cache, _cells, _dev, _rand, _slots, _turning

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DT = ref.DT


@pytest.fixture(scope="module")
def cf():
    from paper_2512_14098_amd import cf as _cf
    return _cf


# ------------------------------------------------------------------ scales
@pytest.mark.parametrize("kind", ["bf16", "fp16"])
def test_every_code_with_every_scale(cf, kind):
    """2^(byte - 127) times the code, rounded once to the type asked for; 0 is a scale like another, 255 is NaN.  The
    products are exact in 64 bits and, but for infinities, in 32, which torch's conversion goes through."""
    code = torch.arange(256, dtype=torch.uint8).repeat(256, 1).reshape(256, 1, 16, 16)  # page p: byte p
    byte = torch.arange(256, dtype=torch.uint8).reshape(256, 1, 1, 1).expand(256, 1, 2, 16).contiguous()
    c8 = code.cuda().view(torch.float8_e4m3fn)
    k, v = cf.cf_kv_read8(c8, c8.clone(), byte.cuda(), _i32(np.arange(256)[None]), _i32([0, 4096]), 4096, DT[kind])
    want = ref.held(code.numpy()[:, 0], byte.numpy()[:, 0, 0])
    want[255] = np.nan
    want = torch.from_numpy(want).to(DT[kind]).reshape(4096, 1, 16).double().numpy()
    for got in (k, v):
        assert np.array_equal(got.double().cpu().numpy(), want, equal_nan=True)


@pytest.mark.parametrize("kind,dim", [("bf16", 64), ("bf16", 128), ("fp16", 256)])
def test_attention_over_the_least_scale(cf, kind, dim):
    """Rows whose byte is 0, few and many of them: values of 2^-127 times the codes, and such keys, whose scores are
    0.  The bound is that of the values over 2^-127, whose size is the codes', plus half a step (2^-134; fp16 2^-25)
    below the type's normal range for the output."""
    for ctx, new in (([50, 3000], [1, 3]), ([20, 700], [33, 90])):
        c = _case(kind, ctx, new, 4, 2, dim, 16, spread=0)
        c["exps"][:] = np.where(c["exps"] == 255, 255, 0)
        for which, (x, codes) in enumerate(((c["ks"], c["kc"]), (c["vs"], c["vc"]))):
            for i, r in enumerate(x):
                for t in range(c["kv"][i]):
                    pg, off = c["table"][i, t // 16], t % 16
                    r[t] = torch.from_numpy(ref.held(codes[pg, :, off], c["exps"][pg, :, which, off])).to(DT[kind])
        got, lse = _run(cf, c, new, 4, 2, dim)
        big = [v.double() * 2.0 ** 127 for v in c["vs"]]
        out, wl, tol, ltol = _want_paged(dict(c, vs=[v.float() for v in big]), ctx, new, dim ** -0.5, kind)
        tol = tol + 2.0 ** (127 - (25 if kind == "fp16" else 134))
        assert (np.abs(got.double().cpu().numpy() * 2.0 ** 127 - out) <= tol).all()
        assert (np.abs(lse.double().cpu().numpy() - wl) <= ltol).all()


# ------------------------------------------------------------------ partial turns, written
@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("n", [70, 1499, 1500, 1603])
@pytest.mark.parametrize("heads,kv_heads,dim,rot,axes", [(4, 3, 128, 64, 1), (3, 5, 80, 40, 2), (2, 2, 112, 56, 1),
                                                         (5, 4, 48, 24, 3), (2, 3, 256, 240, 1), (1, 9, 32, 16, 1)])
def test_partial_turns_written(cf, kind, n, heads, kv_heads, dim, rot, axes):
    """Halves paired, some columns pass: to the bit cf_rope and cf_kv_write8, on either side of the change
    from four waves a token to one; and the codes are those of the turned keys."""
    _say("partial", kind, n, heads, kv_heads, dim, rot, axes)
    rng = np.random.default_rng(n + dim)
    t = _dev(*_turning(rng, n, rot, axes))
    x = _rand(n, (n, heads + 2 * kv_heads, dim), kind)
    q, k, v = x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:]
    n_pages = -(-n // 16) + 2
    slots = _slots(rng, n, n_pages * 16)
    a, b = _cache(n_pages, kv_heads, 16, dim), _cache(n_pages, kv_heads, 16, dim)
    qo, ko = cf.cf_rope(q, k, *t)
    cf.cf_kv_write8(ko, v, *a, torch.as_tensor(slots).cuda())
    assert torch.equal(cf.cf_rope_write8(q, k, v, *t, *b, torch.as_tensor(slots).cuda()), qo)
    want, got = _cells(*a), _cells(*b)
    for y, z in zip(want, got):
        assert np.array_equal(y, z)
    on = np.flatnonzero((slots >= 0) & (slots < 16 * n_pages))
    for which, y in enumerate((ko, v)):
        code, byte = ref.quantise(y.double().cpu().numpy()[on], kind)
        assert np.array_equal(got[which][slots[on]], code) and np.array_equal(got[2][slots[on]][:, :, which], byte)


# ------------------------------------------------------------------ long reads
@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("heads,dim,page", [(8, 128, 16), (16, 256, 32), (2, 64, 16), (3, 176, 64), (32, 128, 128)])
def test_long_reads(cf, kind, heads, dim, page):
    """Past 16384 rows with 8, 4, 16, 16 and 4 tokens a workgroup: rows before, between and after the requests as they were,
    pages outside the cache as zeros."""
    _say("long read", kind, heads, dim, page)
    rng = np.random.default_rng(dim)
    lens, lead = [9001, 0, 1, 7500, 33], 5
    n_tok = lead + sum(lens) + 3
    assert n_tok >= 16384
    n_pages = 40
    c = _cache(n_pages, heads, page, dim)
    most = -(-max(lens) // page)
    table = rng.integers(0, n_pages, (len(lens), most))
    table[rng.random(table.shape) < 0.05] = n_pages
    start = np.concatenate([[0], np.cumsum(lens)]) + lead
    k, v = cf.cf_kv_read8(*c, _i32(table), _i32(start), n_tok, DT[kind])
    req = np.repeat(np.arange(len(lens)), lens)
    pos = np.arange(sum(lens)) - (start[:-1] - lead)[req]
    pg = torch.as_tensor(table[req, pos // page]).cuda()
    on, pg, off = (pg < n_pages)[:, None, None], pg.clamp(max=n_pages - 1), torch.as_tensor(pos % page).cuda()
    for which, got in enumerate((k, v)):
        scale = torch.exp2(c[2][pg, :, which, off].double() - 127)[..., None]
        want = torch.where(on, c[which][pg, :, off].double() * scale, 0.0).to(DT[kind])
        assert torch.equal(got[lead:lead + sum(lens)], want)


# ------------------------------------------------------------------ joins
@pytest.mark.parametrize("width", [16, 8])
@pytest.mark.parametrize("kind,heads,kv_heads,dim,new,lens", [("bf16", 8, 1, 64, 8320, 40000), ("fp16", 16, 2, 48, 4170, 40001)])
def test_joined_tiles_outnumber_the_joining_workgroups(cf, width, kind, heads, kv_heads, dim, new, lens):
    """A few more tiles than run at a time, all of them split: 520 and 2 x 261.  Only heads of 64 columns or fewer
    have so many: a plan splits fewer tiles than twice the workgroups that run at a time, 512 or, of other widths with so
    many rows, 256."""
    _say("outnumber", width, kind, heads, kv_heads, dim, new, lens)
    c = Caches(cf, kind, [lens], [new], heads, kv_heads, dim)
    plan = c.plan()
    assert int(plan.work[16:20].view(torch.int32)) * kv_heads > 512  # the header's count of split tiles
    got = c.run(width, plan)
    rows, hs = [0, 1, 127, 128, new // 2, new - 130, new - 1], [0, heads // 2, heads - 1]
    want = _sampled(c.q, c.ks[0], c.vs[0], rows, [lens - new + j + 1 for j in range(new)], hs, dim ** -0.5, kind)
    _compare(*[x[rows][:, hs] for x in got], want)
    # every row: against the other width's, which holds the same values
    other = c.run(24 - width, plan)
    assert torch.equal(got[0], other[0]) and torch.equal(got[1], other[1])
    again = c.run(width, plan)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])
