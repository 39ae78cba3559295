"""Rotary positions and the 8-bit cache's writes and reads against plain 64-bit forms."""
import numpy as np
import pytest

from tests import kv8_ref as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DT = ref.DT


@pytest.fixture(scope="module")
def cf():
    from paper_2512_14098_amd import cf as _cf
    return _cf


def _say(*a):
    print(*a, flush=True)


def _i32(x):
    return torch.as_tensor(np.asarray(x, np.int32)).cuda()


def _bits(t):
    return t.contiguous().view(torch.uint8 if t.element_size() == 1 else torch.int16).cpu().numpy()


def _rand(seed, shape, kind):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(DT[kind])


def _turning(rng, n, rot, axes, far=3000):
    pos = rng.integers(-5, far, (axes, n)).astype(np.int32)
    freq = 10000.0 ** (-np.arange(rot // 2) / (rot // 2))
    axis = None if axes == 1 else rng.integers(0, axes, rot // 2).astype(np.int32)
    return pos, freq, axis


def _dev(pos, freq, axis):
    return _i32(pos), torch.from_numpy(np.asarray(freq, np.float64)).cuda(), None if axis is None else _i32(axis)


def _check_turn(got, x, pos, freq, axis, interleaved, inverse, kind):
    y, wide = ref.turn(x.double().cpu().numpy(), pos, freq, axis, interleaved, inverse)
    off = np.abs(got.double().cpu().numpy() - y)
    tol = ref.turn_bound(y, wide, kind)
    assert (off <= tol).all(), (off - tol).max()


# ------------------------------------------------------------------ rotary positions
@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("n,heads,kv_heads,dim,rot,axes", [
    (1, 1, 1, 8, 8, 1), (1, 32, 8, 128, 128, 1), (3, 5, 0, 72, 72, 2), (65, 4, 2, 64, 32, 3), (17, 7, 1, 80, 80, 2),
    (9, 3, 3, 256, 256, 3), (5, 2, 2, 136, 24, 1), (2047, 2, 1, 96, 96, 3), (2050, 3, 1, 112, 56, 1)])
def test_rope(cf, kind, interleaved, n, heads, kv_heads, dim, rot, axes):
    _say("rope", kind, interleaved, n, heads, kv_heads, dim, rot, axes)
    rng = np.random.default_rng(n + dim)
    t = _turning(rng, n, rot, axes)
    x = _rand(n, (n, heads + 2 * kv_heads, dim), kind)  # parts of a fused projection
    q, k = x[:, :heads], x[:, heads:heads + kv_heads]
    before = x.clone()
    for inverse in (False, True):
        if kv_heads:
            qo, ko = cf.cf_rope(q, k, *_dev(*t), interleaved=interleaved, inverse=inverse)
            _check_turn(ko, k, *t, interleaved, inverse, kind)
        else:
            qo = cf.cf_rope(q, None, *_dev(*t), interleaved=interleaved, inverse=inverse)
        assert qo.is_contiguous() and qo.shape == q.shape
        _check_turn(qo, q, *t, interleaved, inverse, kind)
    assert torch.equal(x, before)


@pytest.mark.parametrize("n", [33, 3000])
def test_rope_in_place(cf, n):
    rng = np.random.default_rng(n)
    t = _turning(rng, n, 96, 3)
    x = _rand(n, (n, 12, 128), "bf16")
    q, k = cf.cf_rope(x[:, :8], x[:, 8:10], *_dev(*t))
    rest = x[:, 10:].clone()
    qi, ki = x[:, :8], x[:, 8:10]
    a, b = cf.cf_rope(qi, ki, *_dev(*t), in_place=True)
    assert a is qi and b is ki
    assert torch.equal(x[:, :8], q) and torch.equal(x[:, 8:10], k) and torch.equal(x[:, 10:], rest)


def test_rope_in_place_refuses(cf):
    """Tensors that would have to be copied first, rows that overlap, one tensor for both."""
    rng = np.random.default_rng(0)
    t = _dev(*_turning(rng, 6, 64, 1))
    x = _rand(0, (6, 3, 65), "bf16")
    for q in (x[:, :, 1:], x[:, :, :64], _rand(0, (1, 3, 64), "bf16").expand(6, 3, 64),
              _rand(0, (6, 1, 64), "bf16").expand(6, 3, 64)):
        with pytest.raises(cf.CfError, match="in place"):
            cf.cf_rope(q, None, *t, in_place=True)
    y = _rand(0, (6, 3, 64), "bf16")
    with pytest.raises(cf.CfError, match="k_out_dev"):
        cf.cf_rope(y, y, *t, in_place=True)
    a, b = cf.cf_rope(y, y, *t)  # not in place: twice the same
    assert torch.equal(a, b)
    # a broadcast tensor is read as it is
    z = _rand(0, (1, 3, 64), "bf16").expand(6, 3, 64)
    assert torch.equal(cf.cf_rope(z, None, *t), cf.cf_rope(z.contiguous(), None, *t))


def test_rope_far_positions_and_missing_axes(cf):
    """Positions up to 2^31 - 1 and below 0; axes that do not exist turn nothing."""
    pos = np.array([[2 ** 31 - 1, -2 ** 31, 0, 10 ** 9, -1], [1, 2, 3, 4, 5]], np.int32)
    freq = np.array([1.0, 0.5, 1e-3, 0.0, 7.25, 1e-9, 2.0, 3.0])
    axis = np.array([0, 1, 0, 1, 2, -1, 0, 2 ** 31 - 1], np.int32)
    x = _rand(3, (5, 2, 32), "fp16")
    _check_turn(cf.cf_rope(x, None, *_dev(pos, freq, axis)), x, pos, freq, axis, False, False, "fp16")


def test_rope_inverse_is_the_gradient(cf):
    """Against the formula's transpose, and against differences of the plain form along single elements (which are
    exact but for rounding, since a turn is linear)."""
    rng = np.random.default_rng(0)
    n, dim, rot = 3, 24, 16
    pos, freq, axis = _turning(rng, n, rot, 2)
    for interleaved in (False, True):
        g = torch.from_numpy(rng.standard_normal((n, 1, dim))).to(torch.bfloat16).cuda()
        grad = cf.cf_rope(g, None, *_dev(pos, freq, axis), interleaved=interleaved, inverse=True).double().cpu().numpy()
        gd = g.double().cpu().numpy()
        x = rng.standard_normal((n, 1, dim))
        for j in range(dim):
            step = np.zeros((n, 1, dim))
            step[..., j] = 2.0 ** -10
            up, down = (ref.turn(x + d, pos, freq, axis, interleaved)[0] for d in (step, -step))
            want = ((up - down) * gd).sum(-1) / 2.0 ** -9
            # one rounding of the gradient, and 2^-50 of numbers below 8 over a step of 2^-9, dim terms
            tol = (2.0 ** -8 + 2.0 ** -20) * np.abs(want) + dim * 2.0 ** -36
            assert (np.abs(grad[..., j] - want) <= tol).all()


def test_rope_of_infinities(cf):
    """An infinity reaches its own pair alone (as NaN or infinities)."""
    x = _rand(1, (4, 2, 64), "bf16")
    y = x.clone()
    y[1, 0, 5], y[2, 1, 40] = float("inf"), float("nan")
    rng = np.random.default_rng(5)
    t = _dev(*_turning(rng, 4, 64, 1))
    a, b = cf.cf_rope(x, None, *t), cf.cf_rope(y, None, *t)
    same = torch.ones_like(x, dtype=torch.bool)
    same[1, 0, [5, 37]] = same[2, 1, [8, 40]] = False
    assert torch.equal(a[same], b[same]) and not torch.isfinite(b[~same]).any()


# ------------------------------------------------------------------ writes
def _cache(n_pages, heads, page, dim, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    k, v = (torch.randint(0, 127, (n_pages, heads, page, dim), generator=g, device="cuda", dtype=torch.uint8)
            .view(torch.float8_e4m3fn) for _ in range(2))
    return k, v, torch.randint(110, 140, (n_pages, heads, 2, page), generator=g, device="cuda", dtype=torch.uint8)


def _cells(k, v, e):
    """The cache by slot: codes of keys and values [slots][heads][dim], exponents [slots][heads][2]."""
    p, h, page, d = k.shape
    return ([np.ascontiguousarray(_bits(x).transpose(0, 2, 1, 3)).reshape(p * page, h, d) for x in (k, v)]
            + [np.ascontiguousarray(e.cpu().numpy().transpose(0, 3, 1, 2)).reshape(p * page, h, 2)])


def _check_written(before, after, k, v, slots, kind):
    want = [x.copy() for x in before]
    n_slots = len(want[0])
    for which, x in enumerate((k, v)):
        code, byte = ref.quantise(x.double().cpu().numpy(), kind)
        for t, s in enumerate(slots):
            if 0 <= s < n_slots:
                want[which][s], want[2][s, :, which] = code[t], byte[t]
    for got, w in zip(after[:2], want[:2]):  # a NaN's sign is anyone's
        nan = (w & 127) == 127
        assert np.array_equal(got[~nan], w[~nan]) and ((got[nan] & 127) == 127).all()
    assert np.array_equal(after[2], want[2])


def _slots(rng, n, n_slots):
    s = rng.permutation(n_slots)[:n]
    s[rng.random(n) < 0.1] = -1
    if n > 4:
        s[2], s[3] = n_slots, 2 ** 62
    return s


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("n,heads,dim,page", [(1, 1, 16, 16), (7, 3, 80, 32), (300, 8, 128, 16), (65, 2, 256, 256),
                                              (40, 5, 48, 64), (33, 1, 144, 16), (2100, 1, 64, 128)])
def test_write8(cf, kind, n, heads, dim, page):
    _say("write8", kind, n, heads, dim, page)
    rng = np.random.default_rng(n + dim)
    n_pages = -(-n // page) + 3
    c = _cache(n_pages, heads, page, dim)
    x = ref.rows_of_a_range(rng, n * 3 * heads, dim, kind).reshape(n, 3 * heads, dim).cuda()
    k, v = x[:, heads:2 * heads], x[:, 2 * heads:]
    slots = _slots(rng, n, n_pages * page)
    before = _cells(*c)
    cf.cf_kv_write8(k, v, *c, torch.as_tensor(slots).cuda())
    _check_written(before, _cells(*c), k, v, slots, kind)


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
def test_write8_of_infinities(cf, kind):
    """Held as NaN, without a say in the scale; every value held is one of the element type."""
    rng = np.random.default_rng(9)
    x = ref.rows_of_a_range(rng, 400, 64, kind).reshape(200, 2, 64)
    x[3, 0, 7], x[5, 1, 63], x[6, 0, 0], x[9] = float("inf"), float("-inf"), float("nan"), float("inf")
    x = x.cuda()
    c = _cache(20, 1, 16, 64)
    before = _cells(*c)
    slots = rng.permutation(320)[:200]
    cf.cf_kv_write8(x[:, :1], x[:, 1:], *c, torch.as_tensor(slots).cuda())
    after = _cells(*c)
    _check_written(before, after, x[:, :1], x[:, 1:], slots, kind)
    value = ref.held(after[0][slots], after[2][slots][:, :, 0])
    fine = np.isfinite(value)
    again = torch.from_numpy(value).to(DT[kind]).double().numpy()
    assert np.array_equal(again[fine], value[fine])
    src = x[:, :1].double().cpu().numpy()
    assert np.array_equal(fine, np.isfinite(src))
    # e4m3's half step, 2^-4, or of its smallest step, 2^-10 of the scale; 1/16 too where |x| was cut
    scale = 2.0 ** (after[2][slots][:, :, 0].astype(float) - 127)[..., None]
    off = np.abs(np.where(fine, value - np.where(fine, src, 0), 0))
    assert (off <= np.maximum(2.0 ** -4 * np.abs(np.where(fine, src, 0)), 2.0 ** -10 * scale)).all()


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("n,heads,kv_heads,dim,rot,axes,interleaved", [
    (1, 4, 1, 64, 64, 1, False), (64, 32, 8, 128, 128, 1, False), (50, 6, 2, 80, 40, 3, True),
    (2048, 2, 1, 128, 128, 3, False), (2051, 3, 3, 192, 96, 2, True), (7, 2, 2, 16, 8, 1, False)])
def test_rope_write8_is_rope_then_write(cf, kind, n, heads, kv_heads, dim, rot, axes, interleaved):
    _say("rope_write8", kind, n, heads, kv_heads, dim, rot, axes, interleaved)
    rng = np.random.default_rng(n)
    t = _dev(*_turning(rng, n, rot, axes))
    x = _rand(n, (n, heads + 2 * kv_heads, dim), kind)
    q, k, v = x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:]
    n_pages = -(-n // 16) + 2
    slots = _slots(rng, n, n_pages * 16)
    a, b = _cache(n_pages, kv_heads, 16, dim), _cache(n_pages, kv_heads, 16, dim)
    qo, ko = cf.cf_rope(q, k, *t, interleaved=interleaved)
    cf.cf_kv_write8(ko, v, *a, torch.as_tensor(slots).cuda())
    before = x.clone()
    got = cf.cf_rope_write8(q, k, v, *t, *b, torch.as_tensor(slots).cuda(), interleaved=interleaved)
    assert torch.equal(got, qo) and torch.equal(x, before)
    for y, z in zip(_cells(*a), _cells(*b)):
        assert np.array_equal(y, z)
    same = cf.cf_rope_write8(q, k, v, *t, *b, torch.as_tensor(slots).cuda(), interleaved=interleaved, in_place=True)
    assert same is q and torch.equal(q, qo) and torch.equal(x[:, heads:], before[:, heads:])


# ------------------------------------------------------------------ reads
def _check_read(cf, cache, table, lens, lead, tail, kind):
    """lead, tail: rows of no request before and after."""
    start = np.concatenate([[0], np.cumsum(lens)]) + lead
    n_tok = int(start[-1]) + tail
    cells = _cells(*cache)
    page = cache[0].shape[2]
    k, v = cf.cf_kv_read8(*cache, _i32(table), _i32(start), n_tok, DT[kind])
    assert k.shape == v.shape == (n_tok, cache[0].shape[1], cache[0].shape[3])
    for which, got in enumerate((k, v)):
        got = got.double().cpu().numpy()
        for i, m in enumerate(lens):
            for j in range(m):
                col = j // page
                p = table[i][col] if col < len(table[i]) else -1
                want = np.zeros(got.shape[1:])
                if 0 <= p < cache[0].shape[0]:
                    s = p * page + j % page
                    # exact where the cache was written in this type; these bytes are any, so rounded to it
                    want = torch.from_numpy(ref.held(cells[which][s], cells[2][s][:, which])).to(DT[kind]).double().numpy()
                assert np.array_equal(got[start[i] + j], want, equal_nan=True), (which, i, j)


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("heads,dim,page,lens", [(1, 16, 16, [1]), (2, 80, 16, [0, 33, 1, 0, 0, 17, 64]),
                                                 (8, 128, 32, [31, 32, 33]), (3, 256, 128, [130, 0]),
                                                 (16, 192, 16, [5, 6]), (1, 64, 16, [3] * 300)])
def test_read8(cf, kind, heads, dim, page, lens):
    _say("read8", kind, heads, dim, page, len(lens))
    rng = np.random.default_rng(dim)
    most = max(-(-m // page) for m in lens) + 1
    n_pages = 40
    cache = _cache(n_pages, heads, page, dim)
    table = rng.integers(0, n_pages, (len(lens), most))
    table[rng.random(table.shape) < 0.05] = rng.choice([-1, n_pages, 2 ** 31 - 1, -2 ** 31])
    _check_read(cf, cache, table, lens, 0, 0, kind)
    _check_read(cf, cache, table, lens, 3, 2, kind)


def test_read8_past_the_table(cf):
    """A request longer than its row of the table: zeros past it."""
    cache = _cache(6, 2, 16, 32)
    _check_read(cf, cache, np.array([[1, 2], [3, 4]]), [40, 20], 0, 0, "bf16")


def test_read8_many_tokens(cf):
    """Past 16384 rows, where a workgroup takes 16 of them."""
    rng = np.random.default_rng(2)
    cache = _cache(64, 1, 256, 16)
    lens = [16000, 0, 900]
    table = np.stack([rng.permutation(64) for _ in lens])
    _check_read(cf, cache, table, lens, 0, 0, "bf16")


def test_what_was_written_reads_back(cf):
    """write8 of what read8 gave changes no code and no exponent: every value held is a fixed point."""
    for kind in ("bf16", "fp16"):
        rng = np.random.default_rng(4)
        x = ref.rows_of_a_range(rng, 1000, 48, kind).reshape(500, 2, 48).cuda()
        c = _cache(32, 1, 16, 48)
        slots = torch.arange(500).cuda()
        cf.cf_kv_write8(x[:, :1], x[:, 1:], *c, slots)
        first = _cells(*c)
        k, v = cf.cf_kv_read8(*c, _i32(np.arange(32)[None]), _i32([0, 500]), 500, DT[kind])
        cf.cf_kv_write8(k, v, *c, slots)
        k2, v2 = cf.cf_kv_read8(*c, _i32(np.arange(32)[None]), _i32([0, 500]), 500, DT[kind])
        assert torch.equal(k, k2) and torch.equal(v, v2)
        # the scale may fall where the largest element was rounded down to 1.75 times a power of two or less
        assert (_cells(*c)[2] <= first[2]).all()


# ------------------------------------------------------------------ streams, graphs, empty calls
def test_empty_calls(cf):
    c = _cache(2, 2, 16, 32)
    before = _cells(*c)
    none = torch.empty((0, 2, 32), dtype=torch.bfloat16, device="cuda")
    freq = torch.ones(16, dtype=torch.float64, device="cuda")
    pos = torch.empty(0, dtype=torch.int32, device="cuda")
    slots = torch.empty(0, dtype=torch.int64, device="cuda")
    assert cf.cf_rope(none, None, pos, freq).shape == none.shape
    cf.cf_kv_write8(none, none, *c, slots)
    assert cf.cf_rope_write8(none, none, none, pos, freq, None, *c, slots).shape == none.shape
    k, v = cf.cf_kv_read8(*c, _i32([[0]]), _i32([0, 0]), 0)
    assert k.shape == v.shape == none.shape
    for a, b in zip(before, _cells(*c)):
        assert np.array_equal(a, b)


def test_in_a_graph_on_a_stream(cf):
    """A step's rotary write and a read captured once and replayed on inputs that change."""
    rng = np.random.default_rng(1)
    n, heads, kv, dim = 20, 4, 2, 64
    pos, freq, _ = _dev(*_turning(rng, n, dim, 1))
    c = _cache(8, kv, 16, dim)
    x = _rand(0, (n, heads + 2 * kv, dim), "bf16")
    slots = torch.as_tensor(rng.permutation(128)[:n]).cuda()
    table, start = _i32(np.arange(8)[None]), _i32([0, 128])

    def step(cache):
        q = cf.cf_rope_write8(x[:, :heads], x[:, heads:heads + kv], x[:, heads + kv:], pos, freq, None, *cache, slots)
        return (q,) + cf.cf_kv_read8(*cache, table, start, 128)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step(c)
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step(c)
    for i in range(4):
        x.copy_(_rand(10 + i, tuple(x.shape), "bf16"))
        pos.add_(1)
        other = tuple(t.clone() for t in c)
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, step(other)):
            assert torch.equal(a, b)
