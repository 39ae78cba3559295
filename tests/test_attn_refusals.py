"""What the paged-cache calls refuse on the host, before any device work (no GPU needed)."""
import ctypes as C
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests import attn_ref  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(not os.path.exists(os.path.join(ROOT, "paper_2512_14098_amd", "libcf.so")),
                                reason="libcf.so not built")
EINVAL = -1
PTR = 1 << 20  # aligned and never dereferenced


@pytest.fixture(scope="module")
def cf():
    from paper_2512_14098_amd import cf as _cf
    return _cf


def _cache(cf, **kw):
    c = cf.cf_kv_cache()
    c.k_dev = c.v_dev = PTR
    c.n_pages, c.page, c.n_kv_heads, c.head_dim, c.dtype = 10, 16, 2, 64, 0
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _desc(cf, **kw):
    d = cf.cf_attn_desc()
    d.n_seq, d.n_tok, d.max_new, d.n_heads, d.n_kv_heads, d.head_dim = 4, 9, 5, 4, 2, 64
    d.q_start_dev = d.kv_len_dev = d.work_dev = PTR
    d.work_bytes = 1 << 40
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def _seqs(cf, **kw):
    a = cf.cf_attn_seqs()
    a.n_seq, a.n_q, a.n_k, a.n_heads, a.n_kv_heads, a.head_dim = 2, 9, 9, 4, 2, 64
    a.q_start_dev = a.k_start_dev = a.q_dev = a.k_dev = a.v_dev = PTR
    a.q_tok, a.q_head, a.k_tok, a.k_head, a.v_tok, a.v_head = 256, 64, 128, 64, 128, 64
    for k, v in kw.items():
        setattr(a, k, v)
    return a


BAD_CACHE = [dict(n_pages=-1), dict(page=8), dict(page=24), dict(page=512), dict(n_kv_heads=0), dict(head_dim=0),
             dict(head_dim=60), dict(head_dim=264), dict(dtype=2), dict(k_dev=None), dict(v_dev=PTR + 8)]


@pytest.mark.parametrize("bad", BAD_CACHE)
def test_cache(cf, bad):
    c = _cache(cf, **bad)
    assert cf.lib().cf_kv_write(C.byref(c), 3, PTR, 128, 64, PTR, 128, 64, PTR, None) == EINVAL
    assert cf.lib().cf_attn_paged(C.byref(_desc(cf)), C.byref(c), PTR, 4, PTR, 256, 64, 0.1, PTR, None, None) == EINVAL


@pytest.mark.parametrize("args", [(-1, PTR, 128, 64, PTR, 128, 64, PTR), (3, None, 128, 64, PTR, 128, 64, PTR),
                                  (3, PTR, 128, 64, None, 128, 64, PTR), (3, PTR, 128, 64, PTR, 128, 64, None),
                                  (3, PTR + 2, 128, 64, PTR, 128, 64, PTR), (3, PTR, 129, 64, PTR, 128, 64, PTR),
                                  (3, PTR, 128, 64, PTR, 128, 60, PTR)])
def test_write(cf, args):
    assert cf.lib().cf_kv_write(C.byref(_cache(cf)), *args, None) == EINVAL


def test_nothing_to_do_is_no_error(cf):
    L = cf.lib()
    assert L.cf_kv_write(C.byref(_cache(cf)), 0, None, 0, 0, None, 0, 0, None, None) == 0
    assert L.cf_attn_paged(C.byref(_desc(cf, n_tok=0)), C.byref(_cache(cf)), PTR, 4, None, 0, 0, 0.1, None, None, None) == 0
    assert L.cf_attn_prompt(C.byref(_seqs(cf, n_q=0)), 0.1, None, None, None) == 0


def test_map(cf):
    good = [3, PTR, PTR, 16, PTR, 4, PTR, 10, PTR + 4, 9, PTR, PTR, PTR, PTR, PTR, PTR, None]
    for at, value in ((0, 0), (3, 17), (3, 8), (5, 0), (7, -1), (9, -1), (1, None), (2, None), (4, None), (6, None),
                      (8, None), (10, None), (11, None), (12, None), (13, None), (14, None), (15, None),
                      (14, PTR + 4)):
        args = list(good)
        args[at] = value
        assert cf.lib().cf_kv_map(*args) == EINVAL, at


@pytest.mark.parametrize("bad", [dict(n_seq=0), dict(n_tok=-1), dict(max_new=-1), dict(n_heads=5), dict(n_heads=0),
                                 dict(n_kv_heads=0), dict(head_dim=12), dict(head_dim=512), dict(n_tok=1 << 30),
                                 dict(n_seq=1 << 24)])
def test_descriptor(cf, bad):
    n = C.c_uint64(0)
    d = _desc(cf, **bad)
    assert cf.lib().cf_attn_plan_bytes(C.byref(d), C.byref(n)) == EINVAL
    assert cf.lib().cf_attn_plan(C.byref(d), None) == EINVAL


def test_workspace(cf):
    n = C.c_uint64(0)
    assert cf.lib().cf_attn_plan_bytes(C.byref(_desc(cf)), C.byref(n)) == 0 and n.value > 0
    for bad in (dict(work_bytes=n.value - 1), dict(work_dev=None), dict(work_dev=PTR + 8), dict(q_start_dev=None),
                dict(kv_len_dev=None)):
        assert cf.lib().cf_attn_plan(C.byref(_desc(cf, **bad)), None) == EINVAL, bad


@pytest.mark.parametrize("args", [(None, 4, PTR, 256, 64, 0.1, PTR), (PTR, 0, PTR, 256, 64, 0.1, PTR),
                                  (PTR, 4, None, 256, 64, 0.1, PTR), (PTR, 4, PTR, 256, 64, 0.1, None),
                                  (PTR, 4, PTR + 4, 256, 64, 0.1, PTR), (PTR, 4, PTR, 257, 64, 0.1, PTR),
                                  (PTR, 4, PTR, 256, 64, 0.0, PTR), (PTR, 4, PTR, 256, 64, -1.0, PTR),
                                  (PTR, 4, PTR, 256, 64, float("inf"), PTR), (PTR, 4, PTR, 256, 64, float("nan"), PTR)])
def test_paged(cf, args):
    assert cf.lib().cf_attn_paged(C.byref(_desc(cf)), C.byref(_cache(cf)), *args, None, None) == EINVAL


def test_paged_cache_of_other_heads(cf):
    for kw in (dict(n_kv_heads=4), dict(head_dim=128)):
        assert cf.lib().cf_attn_paged(C.byref(_desc(cf)), C.byref(_cache(cf, **kw)), PTR, 4, PTR, 256, 64, 0.1, PTR,
                                      None, None) == EINVAL
    buf = C.create_string_buffer(256)
    cf.lib().cf_last_error(buf, 256)
    assert b"cache" in buf.value


@pytest.mark.parametrize("bad", [dict(n_seq=0), dict(n_q=-1), dict(n_k=-1), dict(n_heads=3), dict(head_dim=4),
                                 dict(dtype=5), dict(q_dev=None), dict(k_dev=None), dict(q_start_dev=None),
                                 dict(k_start_dev=None), dict(v_dev=PTR + 1), dict(v_head=63), dict(q_tok=250),
                                 dict(n_q=1 << 30), dict(n_seq=1 << 23)])
def test_prompt(cf, bad):
    assert cf.lib().cf_attn_prompt(C.byref(_seqs(cf, **bad)), 0.1, PTR, None, None) == EINVAL
    assert cf.lib().cf_attn_prompt(C.byref(_seqs(cf)), 0.0, PTR, None, None) == EINVAL
    assert cf.lib().cf_attn_prompt(C.byref(_seqs(cf)), 0.1, None, None, None) == EINVAL


def test_binding_refuses_other_types_and_shapes(cf):
    x = torch.zeros((3, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(cf.CfError):
        cf.cf_attn_prompt(x, x, x, torch.zeros(2, dtype=torch.int32))  # host tensors
    with pytest.raises(cf.CfError):
        cf.cf_kv_write(x, x, torch.zeros((2, 2, 16, 64)), torch.zeros((2, 2, 16, 64)), torch.zeros(3))


def test_reference_split_join_identity():
    """The joined parts of a split context equal the whole in 64 bits."""
    rng = np.random.default_rng(0)
    x, v = 20 * rng.standard_normal(1000), rng.standard_normal((1000, 4))
    whole = np.exp(x - x.max()) @ v / np.exp(x - x.max()).sum()
    parts = [(x[a:b].max(), np.exp(x[a:b] - x[a:b].max()).sum(), np.exp(x[a:b] - x[a:b].max()) @ v[a:b])
             for a, b in ((0, 300), (300, 301), (301, 1000))]
    m = max(p[0] for p in parts)
    got = sum(np.exp(p[0] - m) * p[2] for p in parts) / sum(np.exp(p[0] - m) * p[1] for p in parts)
    assert np.allclose(got, whole, rtol=1e-13)


def test_reference_map_by_hand():
    """Two running requests and a waiting one, pages of 16: worked out by hand."""
    w = attn_ref.kv_map([16, 5, 40], [1, 30, 0], [[7, -1, -1], [3, -1, -1], [1, 2, 4]], 16, [9, 8, 6, 5], 1, 31)
    assert w["q_start"] == [0, 1, 31, 31] and w["kv_len"] == [17, 35, 40] and w["status"] == [0, 0, 0]
    assert w["table"].tolist() == [[7, 8, -1], [3, 6, 5], [1, 2, 4]] and w["head"] == [4]
    assert w["slots"][0] == 8 * 16 and w["slots"][1] == 3 * 16 + 5 and w["slots"][12] == 6 * 16 and w["slots"][30] == 5 * 16 + 2
