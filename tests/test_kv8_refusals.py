"""What the rotary and 8-bit cache calls refuse on the host, before any device work (no GPU needed)."""
import ctypes as C
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests import kv8_ref as ref  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(not os.path.exists(os.path.join(ROOT, "paper_2512_14098_amd", "libcf.so")),
                                reason="libcf.so not built")
OK, EINVAL = 0, -1
PTR = 1 << 20  # aligned and never dereferenced


@pytest.fixture(scope="module")
def cf():
    from paper_2512_14098_amd import cf as _cf
    return _cf


def _made(s, fields, kw):
    for k, v in dict(fields, **kw).items():
        setattr(s, k, v)
    return s


def _cache(cf, **kw):
    return _made(cf.cf_kv_cache8(), dict(k_dev=PTR, v_dev=PTR, exp_dev=PTR, n_pages=10, page=16, n_kv_heads=2,
                                         head_dim=64, dtype=0), kw)


def _rope(cf, **kw):
    return _made(cf.cf_rope_desc(), dict(n_axes=3, rot_dim=64, pos_dev=PTR, freq_dev=PTR, axis_dev=PTR), kw)


def _call_rope(cf, r, n=4, heads=4, kv=2, dim=64, dtype=0, q=(PTR, 512, 64), qo=(PTR * 2, 256, 64), k=(PTR * 3, 512, 64),
               ko=(PTR * 4, 128, 64)):
    return cf.lib().cf_rope(r, n, heads, kv, dim, dtype, *q, *qo, *k, *ko, None)


def _call_write(cf, c, n=4, k=(PTR, 512, 64), v=(PTR, 512, 64), slots=PTR):
    return cf.lib().cf_kv_write8(c, n, *k, *v, slots, None)


def _call_both(cf, r, c, n=4, heads=4, q=(PTR, 512, 64), qo=(PTR * 2, 256, 64), k=(PTR, 512, 64), v=(PTR, 512, 64),
               slots=PTR):
    return cf.lib().cf_rope_write8(r, c, n, heads, *q, *qo, *k, *v, slots, None)


def _call_read(cf, c, table=PTR, most=4, n_seq=2, start=PTR, n_tok=5, k=PTR, v=PTR):
    return cf.lib().cf_kv_read8(c, table, most, n_seq, start, n_tok, k, v, None)


BAD_CACHE = [dict(n_pages=-1), dict(page=8), dict(page=24), dict(page=512), dict(n_kv_heads=0), dict(n_kv_heads=65536),
             dict(head_dim=0), dict(head_dim=72), dict(head_dim=272), dict(dtype=2), dict(k_dev=None), dict(v_dev=None),
             dict(exp_dev=None), dict(k_dev=PTR + 8), dict(v_dev=PTR + 8), dict(exp_dev=PTR + 1)]


@pytest.mark.parametrize("bad", BAD_CACHE)
def test_cache(cf, bad):
    c = C.byref(_cache(cf, **bad))
    assert _call_write(cf, c) == EINVAL
    assert _call_both(cf, C.byref(_rope(cf)), c) == EINVAL
    assert _call_read(cf, c) == EINVAL
    assert _call_write(cf, None) == _call_read(cf, None) == EINVAL


BAD_ROPE = [dict(n_axes=0), dict(n_axes=17), dict(rot_dim=0), dict(rot_dim=-8), dict(rot_dim=12), dict(rot_dim=72),
            dict(pos_dev=None), dict(freq_dev=None)]


@pytest.mark.parametrize("bad", BAD_ROPE)
def test_rotary_description(cf, bad):
    r = C.byref(_rope(cf, **bad))
    assert _call_rope(cf, r) == EINVAL
    assert _call_both(cf, r, C.byref(_cache(cf))) == EINVAL
    assert _call_rope(cf, None) == _call_both(cf, None, C.byref(_cache(cf))) == EINVAL


@pytest.mark.parametrize("bad", [
    dict(n=-1), dict(heads=0), dict(heads=65536), dict(kv=-1), dict(kv=65536), dict(dim=0), dict(dim=68), dict(dim=264),
    dict(dtype=3), dict(q=(None, 512, 64)), dict(qo=(None, 512, 64)), dict(k=(None, 512, 64)), dict(ko=(None, 512, 64)),
    dict(q=(PTR + 8, 512, 64)), dict(q=(PTR, 508, 64)), dict(qo=(PTR, 512, 68)), dict(k=(PTR + 2, 512, 64)),
    dict(ko=(PTR, 4, 64)), dict(qo=(PTR, 256, 64)), dict(ko=(PTR * 3, 512, 72)),
    dict(ko=(PTR * 2, 128, 64))])
def test_rope(cf, bad):
    assert _call_rope(cf, C.byref(_rope(cf)), **bad) == EINVAL


def test_rope_without_tokens_or_keys(cf):
    r = C.byref(_rope(cf))
    assert _call_rope(cf, r, n=0, q=(None, 0, 0), qo=(None, 0, 0), k=(None, 0, 0), ko=(None, 0, 0)) == OK
    assert _call_rope(cf, C.byref(_rope(cf, pos_dev=None)), n=0) == OK
    assert _call_write(cf, C.byref(_cache(cf)), n=0, k=(None, 0, 0), v=(None, 0, 0), slots=None) == OK
    assert _call_write(cf, C.byref(_cache(cf, n_pages=0, k_dev=None, v_dev=None, exp_dev=None))) == OK
    assert _call_both(cf, r, C.byref(_cache(cf)), n=0, q=(None, 0, 0)) == OK
    assert _call_read(cf, C.byref(_cache(cf)), n_tok=0, k=None, v=None) == OK


@pytest.mark.parametrize("bad", [dict(n=-1), dict(k=(None, 512, 64)), dict(v=(None, 512, 64)), dict(slots=None),
                                 dict(k=(PTR + 8, 512, 64)), dict(v=(PTR, 512, 60)), dict(k=(PTR, 4, 64))])
def test_write(cf, bad):
    assert _call_write(cf, C.byref(_cache(cf)), **bad) == EINVAL
    assert _call_both(cf, C.byref(_rope(cf)), C.byref(_cache(cf)), **bad) == EINVAL


@pytest.mark.parametrize("bad", [dict(heads=0), dict(heads=65536), dict(q=(None, 512, 64)), dict(qo=(None, 512, 64)),
                                 dict(q=(PTR + 4, 512, 64)), dict(qo=(PTR, 512, 65)), dict(qo=(PTR, 256, 64))])
def test_rope_write(cf, bad):
    assert _call_both(cf, C.byref(_rope(cf)), C.byref(_cache(cf)), **bad) == EINVAL


@pytest.mark.parametrize("bad", [dict(table=None), dict(most=0), dict(n_seq=0), dict(n_seq=(1 << 30) + 1), dict(start=None), dict(n_tok=-1),
                                 dict(k=None), dict(v=None), dict(k=PTR + 8), dict(v=PTR + 4)])
def test_read(cf, bad):
    assert _call_read(cf, C.byref(_cache(cf)), **bad) == EINVAL


def _desc(cf, **kw):
    return _made(cf.cf_attn_desc(), dict(n_seq=4, n_tok=9, max_new=5, n_heads=4, n_kv_heads=2, head_dim=64, q_start_dev=PTR,
                                         kv_len_dev=PTR, work_dev=PTR, work_bytes=1 << 40), kw)


def _call_paged(cf, d, c, table=PTR, most=4, q=PTR, tok=256, head=64, scale=0.1, out=PTR):
    return cf.lib().cf_attn_paged8(d, c, table, most, q, tok, head, scale, out, None, None)


@pytest.mark.parametrize("bad", BAD_CACHE + [dict(n_kv_heads=4), dict(head_dim=128)])
def test_paged_cache(cf, bad):
    assert _call_paged(cf, C.byref(_desc(cf)), C.byref(_cache(cf, **bad))) == EINVAL


@pytest.mark.parametrize("bad", [dict(n_seq=0), dict(n_tok=-1), dict(max_new=-1), dict(n_heads=3), dict(n_kv_heads=0),
                                 dict(head_dim=60), dict(q_start_dev=None), dict(kv_len_dev=None), dict(work_dev=None),
                                 dict(work_dev=PTR + 8), dict(work_bytes=10)])
def test_paged_descriptor(cf, bad):
    assert _call_paged(cf, C.byref(_desc(cf, **bad)), C.byref(_cache(cf))) == EINVAL


@pytest.mark.parametrize("bad", [dict(table=None), dict(most=0), dict(most=1 << 27), dict(q=None), dict(out=None),
                                 dict(q=PTR + 8), dict(out=PTR + 2), dict(tok=250), dict(head=63), dict(scale=0.0),
                                 dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan"))])
def test_paged(cf, bad):
    assert _call_paged(cf, C.byref(_desc(cf)), C.byref(_cache(cf)), **bad) == EINVAL
    assert _call_paged(cf, None, C.byref(_cache(cf))) == _call_paged(cf, C.byref(_desc(cf)), None) == EINVAL
    assert _call_paged(cf, C.byref(_desc(cf, n_tok=0)), C.byref(_cache(cf)), q=None, out=None) == OK


def test_binding_refuses(cf):
    """Host tensors, wrong types and shapes: errors of the binding, before the library is called."""
    bf, f8 = torch.bfloat16, torch.float8_e4m3fn
    x = torch.zeros((4, 6, 64), dtype=bf)
    cache = torch.zeros((3, 2, 16, 64), dtype=torch.uint8).view(f8)
    exps = torch.zeros((3, 2, 2, 16), dtype=torch.uint8)
    pos, freq = torch.zeros(4, dtype=torch.int32), torch.zeros(32, dtype=torch.float64)
    slots = torch.zeros(4, dtype=torch.int64)
    with pytest.raises(cf.CfError, match="device tensor"):
        cf.cf_rope(x, None, pos, freq)
    with pytest.raises(cf.CfError, match="device tensor"):
        cf.cf_kv_write8(x[:, :2], x[:, 2:4], cache, cache, exps, slots)
    with pytest.raises(cf.CfError, match="float8_e4m3fn"):
        cf.cf_kv_write8(x[:, :2], x[:, 2:4], cache.view(torch.uint8), cache, exps, slots)
    with pytest.raises(cf.CfError, match="one shape"):
        cf.cf_kv_read8(cache, cache[:2], exps, torch.zeros((1, 3), dtype=torch.int32), torch.zeros(2, dtype=torch.int32), 4)
    with pytest.raises(cf.CfError, match="exps"):
        cf.cf_kv_read8(cache, cache, exps[:, :, :1], torch.zeros((1, 3), dtype=torch.int32),
                       torch.zeros(2, dtype=torch.int32), 4)
    with pytest.raises(cf.CfError, match="bfloat16 or float16"):
        cf.cf_kv_read8(cache, cache, exps, torch.zeros((1, 3), dtype=torch.int32), torch.zeros(2, dtype=torch.int32), 4,
                       torch.float32)


# ------------------------------------------------------------------ the plain forms themselves
@pytest.mark.parametrize("kind", ["bf16", "fp16"])
def test_plain_quantiser(kind):
    """Its codes are torch's own conversion of x over the scale, its scale the smallest that fits, and what it
    holds is of the element type."""
    x = ref.rows_of_a_range(np.random.default_rng(3), 500, 32, kind)
    code, byte = ref.quantise(x.double().numpy(), kind)
    scale = torch.from_numpy(2.0 ** (byte.astype(float) - 127))[:, None]
    cut = x.double().clamp(-ref.TOP[kind], ref.TOP[kind])
    again = (cut / scale).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(again, code)
    top = cut.abs().amax(-1, keepdim=True)
    assert (top <= 448 * scale).all()
    assert ((top > 448 * scale / 2) | (scale == 2.0 ** -126)).all()
    value = torch.from_numpy(ref.held(code, byte))
    assert torch.equal(value.to(ref.DT[kind]).double(), value)


def test_plain_turn_keeps_lengths():
    rng = np.random.default_rng(0)
    x, pos, freq = rng.standard_normal((6, 2, 24)), rng.integers(0, 9999, (2, 6)), rng.random(8)
    for interleaved in (False, True):
        y, _ = ref.turn(x, pos, freq, rng.integers(0, 2, 8), interleaved)
        assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1)) and np.array_equal(y[..., 16:], x[..., 16:])
    back, _ = ref.turn(ref.turn(x, pos, freq)[0], pos, freq, inverse=True)
    assert np.allclose(back, x)
