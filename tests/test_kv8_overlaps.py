"""Calls whose outputs share elements with what they read, refused on the host (no GPU needed)."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

from tests.test_kv8_refusals import (EINVAL, OK, PTR, ROOT, _cache, _call_both, _call_read, _call_rope, _call_write,  # noqa: F401
                                     _rope, cf, pytestmark)

CSRC = os.path.join(ROOT, "paper_2512_14098_amd", "csrc")


# ------------------------------------------------------------------ the test itself, against sets of elements
@pytest.fixture(scope="module")
def host(tmp_path_factory):
    d = tmp_path_factory.mktemp("overlap")
    (d / "o.cpp").write_text("""
#include "cf_overlap.h"
extern "C" int meet(int64_t a, int64_t b, int64_t n, int64_t ha, int64_t hb, int64_t ta, int64_t tb, int64_t sa,
                    int64_t sb, int64_t d) {
  return cf::rows_meet(cf::RowSet{(void *)a, n, ha, ta, sa, d}, cf::RowSet{(void *)b, n, hb, tb, sb, d});
}
extern "C" int self(int64_t a, int64_t n, int64_t h, int64_t t, int64_t s, int64_t d) {
  return cf::rows_overlap(cf::RowSet{(void *)a, n, h, t, s, d});
}
extern "C" int bytes(int64_t p, int64_t np, int64_t q, int64_t nq) { return cf::bytes_meet((void *)p, np, (void *)q, nq); }
""")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, str(d / "o.cpp"), "-o", str(d / "o.so")])
    lib = C.CDLL(str(d / "o.so"))
    lib.meet.argtypes, lib.self.argtypes, lib.bytes.argtypes = [C.c_int64] * 10, [C.c_int64] * 6, [C.c_int64] * 4
    return lib


def _elements(p, n, heads, tok, head, d):
    rows = (p // 2 + np.arange(n)[:, None] * tok + np.arange(heads) * head).ravel()
    return {int(r) + i for r in rows for i in range(d)}


def test_rows_meet(host):
    """Against sets of elements, strides of either sign, equal and not."""
    rng = np.random.default_rng(0)
    seen = {False: 0, True: 0}
    for _ in range(8000):
        n, ha, hb, d = (int(x) for x in (rng.integers(1, 5), rng.integers(1, 5), rng.integers(1, 5), 8 * rng.integers(1, 4)))
        ta, tb, sa, sb = (int(x) * 8 for x in rng.integers(-12, 13, 4))
        if rng.random() < 0.5:
            tb = ta
        if rng.random() < 0.2:
            ta, tb = [(0, tb), (ta, 0)][rng.integers(2)]
        if rng.random() < 0.5:
            sb = sa
        a = 1 << 20
        b = a + 16 * int(rng.integers(-40, 41))
        share = bool(_elements(a, n, ha, ta, sa, d) & _elements(b, n, hb, tb, sb, d))
        assert bool(host.meet(a, b, n, ha, hb, ta, tb, sa, sb, d)) == share, (n, ha, hb, ta, tb, sa, sb, d, b - a)
        seen[share] += 1
    assert min(seen.values()) > 500


def test_rows_meet_far(host):
    """Parts of one large projection's output; strides that reach past memory; more heads than are compared."""
    q, k, tok = 1 << 30, (1 << 30) + 2 * 32 * 128, 48 * 128
    assert not host.meet(q, k, 1 << 24, 32, 8, tok, tok, 128, 128, 128)
    assert host.meet(q, k - 16, 1 << 24, 32, 8, tok, tok, 128, 128, 128)
    assert host.meet(q, k, 2, 33, 8, tok, tok, 128, 128, 128)
    assert not host.meet(q, q + 256, 1 << 20, 32, 32, 32 * 384, 32 * 384, 384, 384, 128)  # [token][head][3][128]
    assert host.meet(q, 1 << 40, 1 << 30, 1, 1, 1 << 40, 8, 8, 8, 8)
    assert host.meet(q, q + 16, 2, 65535, 65535, 1 << 30, 1 << 30, 16, 24, 8)
    assert not host.meet(q, 1 << 40, 2, 65535, 65535, 0, 0, 16, 24, 8)


def test_rows_overlap(host):
    """Of one tensor: against sets of elements, and large ones."""
    rng = np.random.default_rng(1)
    seen = {False: 0, True: 0}
    for _ in range(8000):
        n, h, d = (int(x) for x in (rng.integers(1, 6), rng.integers(1, 6), 8 * rng.integers(1, 4)))
        tok, head = (int(x) * 8 for x in rng.integers(-16, 17, 2))
        share = len(_elements(1 << 20, n, h, tok, head, d)) < n * h * d
        assert bool(host.self(1 << 20, n, h, tok, head, d)) == share, (n, h, tok, head, d)
        seen[share] += 1
    assert min(seen.values()) > 500
    assert not host.self(1 << 20, 1 << 24, 48, 6144, 128, 128) and host.self(1 << 20, 1 << 24, 49, 6144, 128, 128)
    assert not host.self(1 << 20, 32767, 32, 128, 32767 * 128, 128)  # [head][token][dim]
    assert host.self(1 << 20, 1 << 30, 2, 1 << 40, 64, 64)


def test_bytes_meet(host):
    for p, np_, q, nq in np.random.default_rng(2).integers(0, 12, (2000, 4)):
        p, np_, q, nq = (int(x) for x in (p, np_, q, nq))
        assert bool(host.bytes(p, np_, q, nq)) == bool(set(range(p, p + np_)) & set(range(q, q + nq)))
    assert not host.bytes(1 << 62, 1 << 62, 1 << 61, 1 << 61) and host.bytes(1 << 62, 1 << 62, 1 << 61, (1 << 61) + 1)


# ------------------------------------------------------------------ calls
X = PTR * 2
# 10 pages of 2 heads of 16 rows of 64: 20,480 bytes of codes each, 640 of exponents
APART = dict(k_dev=PTR, v_dev=PTR + 20480, exp_dev=PTR + 40960)


def _apart(cf, **kw):
    return C.byref(_cache(cf, **dict(APART, **kw)))


def _last(cf):
    buf = C.create_string_buffer(256)
    cf.lib().cf_last_error(buf, 256)
    return buf.value


@pytest.mark.parametrize("args", [
    dict(q=(X, 512, 64), qo=(X, 512, 64), k=(X, 512, 64)),  # in place, the keys are the queries
    dict(q=(X, 512, 64), qo=(X, 512, 64), v=(X, 512, 64)),
    dict(q=(X, 512, 64), qo=(X, 512, 64), k=(X + 3 * 128, 512, 64)),  # the last query head is the first key head
    dict(q=(X, 512, 64), qo=(X, 512, 64), v=(X + 7 * 128, 512, 64)),  # the second value head is the next token's query
    dict(qo=(X, 256, 64), k=(X + 512, 0, 64)),  # keys of one token for all, inside the output
    dict(qo=(X, 256, 64), v=(X + 1024, 512, 64)),  # another token stride
    dict(q=(X, 512, 64), qo=(PTR + 16, 256, 64))])
def test_rope_write8_output_over_keys_or_values(cf, args):
    assert _call_both(cf, C.byref(_rope(cf)), _apart(cf), **args) == EINVAL and b"k_dev or v_dev" in _last(cf)


@pytest.mark.parametrize("args", [
    dict(q=(X, 512, 64), qo=(X, 512, 64), k=(X, 512, 64)),  # queries in place, the keys are the queries
    dict(q=(X, 512, 64), k=(X, 512, 64), ko=(X, 512, 64), qo=(PTR * 3, 256, 64)),  # and the other way round
    dict(q=(X, 512, 64), qo=(X, 512, 64), k=(X + 3 * 128, 512, 64), ko=(X + 3 * 128, 512, 64)),  # shifted by heads
    dict(q=(X, 512, 64), k=(X + 7 * 128, 512, 64), qo=(PTR * 3, 256, 64), ko=(X + 7 * 128, 512, 64)),
    dict(qo=(X, 512, 64), ko=(X + 128, 512, 64)),  # outputs over each other
    dict(qo=(X, 512, 64), ko=(X + 2048, 128, 64)),
    dict(q=(X, 512, 64), qo=(X + 128, 512, 64)),  # an output a head or a token behind its input
    dict(q=(X, 512, 64), qo=(X - 1024, 512, 64)),
    dict(k=(X, 512, 64), ko=(X + 64, 512, 64), qo=(PTR * 5, 256, 64))])
def test_rope_outputs_over_other_tensors(cf, args):
    assert _call_rope(cf, C.byref(_rope(cf)), **args) == EINVAL and b"shares elements" in _last(cf)


@pytest.mark.parametrize("qo", [(X + 128, 512, 64), (X - 1024, 512, 64), (X + 16, 512, 64)])
def test_rope_write8_output_beside_its_input(cf, qo):
    assert _call_both(cf, C.byref(_rope(cf)), _apart(cf), q=(X, 512, 64), qo=qo) == EINVAL and b"with its input" in _last(cf)


@pytest.mark.parametrize("strides", [(128, 64), (64, 128), (192, 128), (0, 64), (512, 0), (512, 32), (64, 64), (-128, 64),
                                     (32, 512), (384, 192)])
def test_rows_of_an_output_over_one_another(cf, strides):
    """Four tokens of four heads of 64, in place and not."""
    r, c = C.byref(_rope(cf)), _apart(cf)
    for x in (dict(q=(X, *strides), qo=(X, *strides)), dict(q=(PTR * 8, 512, 64), qo=(X, *strides))):
        assert _call_rope(cf, r, **x, k=(PTR * 4, 512, 64), ko=(PTR * 5, 512, 64)) == EINVAL and b"rows" in _last(cf)
        assert _call_both(cf, r, c, **x) == EINVAL and b"rows" in _last(cf)
    assert _call_rope(cf, r, kv=4, k=(X, 512, 64), ko=(PTR * 5, *strides)) == EINVAL and b"rows" in _last(cf)


# ------------------------------------------------------------------ arrays of the cache, outputs of a read
@pytest.mark.parametrize("over", [dict(v_dev=PTR), dict(v_dev=PTR + 20480 - 16), dict(k_dev=PTR + 40960 - 32),
                                  dict(exp_dev=PTR + 20480 - 16), dict(exp_dev=PTR + 40960 - 16), dict(exp_dev=PTR - 624)])
def test_arrays_of_a_cache_over_one_another(cf, over):
    """Writes are refused; reads and attention may take keys for values too."""
    c = _apart(cf, **over)
    assert _call_write(cf, c) == EINVAL and b"overlap" in _last(cf)
    assert _call_both(cf, C.byref(_rope(cf)), c, q=(X, 512, 64), qo=(X, 512, 64)) == EINVAL and b"overlap" in _last(cf)
    assert _call_write(cf, c, n=0) == OK


def test_outputs_of_a_read_over_one_another(cf):
    for k, v in ((PTR, PTR), (PTR, PTR + 1280 - 16), (PTR + 1280 - 16, PTR)):  # 5 tokens of 2 heads of 64
        assert _call_read(cf, _apart(cf), k=k, v=v) == EINVAL and b"overlap" in _last(cf)


@pytest.mark.parametrize("bad,says", [
    (dict(n=-1), b"n_tok"), (dict(k=(None, 512, 64)), b"NULL"), (dict(v=(None, 512, 64)), b"NULL"), (dict(slots=None), b"NULL"),
    (dict(k=(PTR + 8, 512, 64)), b"aligned"), (dict(v=(PTR, 512, 60)), b"aligned"), (dict(k=(PTR, 4, 64)), b"aligned")])
def test_writes_into_arrays_apart(cf, bad, says):
    """What a write refuses, each for its own reason."""
    assert _call_write(cf, _apart(cf), **bad) == EINVAL and says in _last(cf)
    assert _call_both(cf, C.byref(_rope(cf)), _apart(cf), **bad) == EINVAL and says in _last(cf)


@pytest.mark.parametrize("bad,says", [
    (dict(heads=0), b"n_heads"), (dict(heads=65536), b"n_heads"), (dict(q=(None, 512, 64)), b"NULL"),
    (dict(qo=(None, 512, 64)), b"NULL"), (dict(q=(PTR + 4, 512, 64)), b"aligned"), (dict(qo=(PTR, 512, 65)), b"aligned"),
    (dict(qo=(PTR, 256, 64)), b"in place")])
def test_turned_writes_into_arrays_apart(cf, bad, says):
    assert _call_both(cf, C.byref(_rope(cf)), _apart(cf), **bad) == EINVAL and says in _last(cf)


@pytest.mark.parametrize("bad,says", [
    (dict(table=None), b"NULL"), (dict(most=0), b"max_pages"), (dict(n_seq=0), b"n_seq"), (dict(n_seq=(1 << 30) + 1), b"n_seq"),
    (dict(start=None), b"NULL"), (dict(n_tok=-1), b"n_tok"), (dict(k=None), b"NULL"), (dict(v=None), b"NULL"),
    (dict(k=PTR + 8), b"aligned"), (dict(v=PTR + 4), b"aligned")])
def test_reads_into_outputs_apart(cf, bad, says):
    assert _call_read(cf, _apart(cf), **dict(dict(v=PTR * 2), **bad)) == EINVAL and says in _last(cf)
