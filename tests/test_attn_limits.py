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
