"""In-place calls on parts of one tensor: refused where rows share elements, else as out of place."""
import numpy as np
import pytest

from tests.test_gpu_kv8 import _cache, _cells, _dev, _rand, _turning

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def cf():
    from paper_2512_14098_amd import cf as _cf
    return _cf


def test_rope_write8_in_place_refuses_shared_keys_and_values(cf):
    rng = np.random.default_rng(0)
    t = _dev(*_turning(rng, 6, 64, 1))
    x = _rand(0, (6, 12, 64), "bf16")
    before = x.clone()
    c = _cache(2, 4, 16, 64)
    cells = _cells(*c)
    slots = torch.arange(6).cuda()
    y, z = x[:, :4], x[:, 8:]
    for q, k, v in ((y, y, z), (y, z, y), (x[:, :8], x[:, 4:8], z), (x[:, 3:8], z, x[:, :4]), (y, y[2:3].expand(6, 4, 64), z)):
        with pytest.raises(cf.CfError, match="shares elements"):
            cf.cf_rope_write8(q, k, v, *t, *c, slots, in_place=True)
    assert torch.equal(x, before)
    for a, b in zip(cells, _cells(*c)):
        assert np.array_equal(a, b)
    # not in place, the keys may be the queries
    want = cf.cf_rope(y, None, *t)
    assert torch.equal(cf.cf_rope_write8(y, y, z, *t, *c, slots), want) and torch.equal(x, before)
    # keys of one token for all between the queries' rows
    cf.cf_rope_write8(y, z[1:2].expand(6, 4, 64), z, *t, *c, slots, in_place=True)
    assert torch.equal(y, want) and torch.equal(x[:, 4:], before[:, 4:])


@pytest.mark.parametrize("n", [1, 7, 1600])
def test_rope_write8_in_place_between_keys_and_values(cf, n):
    """Parts of a fused projection by head, [token][head][3][dim]: the ranges meet, the rows do not."""
    rng = np.random.default_rng(n)
    t = _dev(*_turning(rng, n, 64, 1))
    x = _rand(1, (n, 5, 3, 64), "fp16")
    before = x.clone()
    pages = -(-n // 16)
    a, b = _cache(pages, 5, 16, 64), _cache(pages, 5, 16, 64)
    slots = torch.as_tensor(rng.permutation(16 * pages)[:n]).cuda()
    want = cf.cf_rope_write8(x[:, :, 0], x[:, :, 1], x[:, :, 2], *t, *a, slots)
    q = x[:, :, 0]
    assert cf.cf_rope_write8(q, x[:, :, 1], x[:, :, 2], *t, *b, slots, in_place=True) is q
    assert torch.equal(x[:, :, 0], want) and torch.equal(x[:, :, 1:], before[:, :, 1:])
    for p, r in zip(_cells(*a), _cells(*b)):
        assert np.array_equal(p, r)


def test_rope_in_place_refuses_overlapping_queries_and_keys(cf):
    rng = np.random.default_rng(1)
    t = _dev(*_turning(rng, 5, 64, 1))
    x = _rand(2, (5, 12, 64), "bf16")
    before = x.clone()
    for q, k in ((x[:, :8], x[:, 4:10]), (x[:, 4:], x[:, :5]), (x[:, 3:4], x[:, 3:4]), (x[:, ::2], x[:, 2:6:3])):
        with pytest.raises(cf.CfError, match="q_out_dev"):
            cf.cf_rope(q, k, *t, in_place=True)
    assert torch.equal(x, before)


@pytest.mark.parametrize("n", [1, 3, 1700])
def test_rope_in_place_rows_between_rows(cf, n):
    """Parts of one tensor that share nothing: by head, by every other head, by every other token."""
    rng = np.random.default_rng(n)
    t = _dev(*_turning(rng, n, 32, 1))
    x = _rand(3, (2 * n, 6, 3, 32), "bf16")
    for part in (lambda y: (y[:n, :, 0], y[:n, :, 2]), lambda y: (y[:n, ::2, 1], y[:n, 1::2, 1]),
                 lambda y: (y[::2, :, 0], y[1::2, :, 0]), lambda y: (y[:n, :, 1], y[n:, :2, 1])):
        y = x.clone()
        q, k = part(y)
        qo, ko = cf.cf_rope(*part(x), *t)
        want = x.clone()
        for p, o in zip(part(want), (qo, ko)):
            p.copy_(o)
        a, b = cf.cf_rope(q, k, *t, in_place=True)
        assert a is q and b is k and torch.equal(y, want)


def test_rope_in_place_refuses_rows_over_one_another(cf):
    """Sliding windows and rows of other tokens' heads; [head][token][dim] and every other row are not such."""
    rng = np.random.default_rng(2)
    t = _dev(*_turning(rng, 3, 64, 1))
    base = _rand(4, (4096,), "bf16")
    before = base.clone()
    for size, strides in (((3, 4, 64), (128, 64, 1)), ((3, 3, 64), (64, 128, 1)), ((3, 1, 64), (32, 64, 1)),
                          ((3, 3, 64), (192, 96, 1))):
        with pytest.raises(cf.CfError, match="in place"):
            cf.cf_rope(base.as_strided(size, strides), None, *t, in_place=True)
    assert torch.equal(base, before)
    for size, strides in (((3, 4, 64), (64, 192, 1)), ((3, 4, 64), (512, 128, 1)), ((3, 2, 64), (128, 192, 1))):
        base.copy_(before)
        q = base.as_strided(size, strides)
        want = cf.cf_rope(q, None, *t)
        assert cf.cf_rope(q, None, *t, in_place=True) is q and torch.equal(q, want)


def test_writes_refuse_one_array_for_keys_and_values(cf):
    """Reads and attention take keys for values."""
    rng = np.random.default_rng(3)
    k, v, e = _cache(4, 2, 16, 64)
    x = _rand(5, (8, 4, 64), "bf16")
    slots = torch.arange(8).cuda()
    before = _cells(k, v, e)
    with pytest.raises(cf.CfError, match="overlap"):
        cf.cf_kv_write8(x[:, :2], x[:, 2:], k, k, e, slots)
    with pytest.raises(cf.CfError, match="overlap"):
        cf.cf_rope_write8(x, x[:, :2], x[:, 2:], *_dev(*_turning(rng, 8, 64, 1)), k, k, e, slots)
    for a, b in zip(before, _cells(k, v, e)):
        assert np.array_equal(a, b)
    table, start = torch.arange(4, dtype=torch.int32).cuda()[None], torch.tensor([0, 50], dtype=torch.int32).cuda()
    kk, _ = cf.cf_kv_read8(k, k, e, table, start, 50)
    want, _ = cf.cf_kv_read8(k, v, e, table, start, 50)
    assert torch.equal(kk, want)
