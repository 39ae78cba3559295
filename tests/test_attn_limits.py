"""Sizes at which the attention calls' 32-bit key numbers would overflow (no GPU needed)."""
import ctypes as C

import pytest

from tests.test_attn_refusals import EINVAL, PTR, _cache, _desc, _seqs, cf, pytestmark  # noqa: F401

MOST = 2 ** 31 - 65536


@pytest.mark.parametrize("page", [16, 256])
def test_paged_refuses_rows_of_too_many_keys(cf, page):  # noqa: F811
    """One column more than fits is refused; with as many as fit, the next check refuses."""
    d, c = _desc(cf), _cache(cf, page=page)
    args = (PTR, 256, 64, 0.1, None, None, None)
    buf = C.create_string_buffer(256)
    for columns, why in ((MOST // page, b"NULL"), (MOST // page + 1, b"too long"), (2 ** 31 - 1, b"too long")):
        assert cf.lib().cf_attn_paged(C.byref(d), C.byref(c), PTR, columns, *args) == EINVAL
        cf.lib().cf_last_error(buf, 256)
        assert why in buf.value, columns


def test_prompt_refuses_too_many_keys(cf):  # noqa: F811
    buf = C.create_string_buffer(256)
    for n_k, why in ((MOST, b"NULL"), (MOST + 1, b"n_k"), (2 ** 31 - 1, b"n_k")):
        assert cf.lib().cf_attn_prompt(C.byref(_seqs(cf, n_k=n_k)), 0.1, None, None, None) == EINVAL
        cf.lib().cf_last_error(buf, 256)
        assert why in buf.value, n_k


@pytest.mark.parametrize("heads,kv_heads", [(32, 8), (8, 1), (64, 64), (16, 16), (3, 3)])
def test_workspace_is_as_large_as_stated(cf, heads, kv_heads):  # noqa: F811
    """Up to 18 MB where no request has more than 16 rows, else 155 MB, 9 and 79 MB with 64 columns or
    fewer, and 48 bytes a tile (with its padding)."""
    G = heads // kv_heads
    for n_seq, n_tok in ((1, 1), (256, 256), (64, 10000), (1, 32767)):
        for max_new in (1, n_tok):
            for dim in (8, 64, 128, 256):
                few = min(max_new, n_tok) * G <= 16
                tiles = n_tok * G // 16 + 2 * min(n_seq, n_tok) + 8192
                most = ((9e6 if few else 79e6) if dim <= 64 else (18e6 if few else 155e6)) + 48 * tiles
                assert 0 < cf.cf_attn_plan_bytes(n_seq, n_tok, max_new, heads, kv_heads, dim) <= most
