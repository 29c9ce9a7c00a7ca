"""Counting of the cache's pages at its limits.  No GPU: every call fails its checks, or launches nothing."""
import ctypes

import pytest

from paper_2512_09010_amd import binding as lv
from test_kv_host import L, cache, i32  # noqa: F401  (L is a fixture)


@pytest.mark.parametrize("length", [2 ** 63 - 1, 2 ** 63 - 15, 2 ** 63 - 16, 2 ** 62, 2 ** 31, 161])
def test_fork_of_more_tokens_than_there_are(L, length):  # noqa: F811
    """Ten pages of 16 tokens; one page free."""
    start = [1] * 9 + [0]
    refs, children = i32(*start), i32(*[-7] * 10)
    assert L.luvc_kv_fork(ctypes.byref(cache()), refs, i32(*range(10)), length, 1, children, None) == lv.LUVC_ERR_INVALID_ARG
    assert "do not fit" in lv.last_error()
    assert list(refs) == start and list(children) == [-7] * 10
