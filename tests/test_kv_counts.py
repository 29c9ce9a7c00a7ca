"""Counting of the cache's pages at its limits.  No GPU: every call fails its checks, or launches nothing."""
import ctypes

import pytest
import torch

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


def test_fork_of_a_sequence_that_holds_a_page_twice(L):  # noqa: F811
    """Every place counts; the limit of a count holds for their sum, and a refusal takes back what it has counted."""
    top, fork = 2 ** 31 - 1, lambda refs, pages, n: L.luvc_kv_fork(ctypes.byref(cache()), refs, i32(*pages), 16 * len(pages), n, i32(*[0] * 40), None)
    refs = i32(1, 1, *[0] * 8)
    assert fork(refs, [0, 1, 0, 0], 2) == lv.LUVC_OK and list(refs)[:2] == [7, 3]
    for count, n in ((top - 1, 1), (top - 3, 2), (top // 2 + 1, top // 2)):
        start = [count, 5] + [0] * 8
        refs = i32(*start)
        assert fork(refs, [1, 0, 0], n) == lv.LUVC_ERR_INVALID_ARG, (count, n)
        assert "too many" in lv.last_error() and list(refs) == start
    refs = i32(top - 2, 5, *[0] * 8)
    assert fork(refs, [1, 0, 0], 1) == lv.LUVC_OK and list(refs)[:2] == [top, 6]


def test_fork_without_a_free_page_takes_back_what_it_counted(L):  # noqa: F811
    start = [1, 2, 3] + [1] * 7
    refs = i32(*start)
    assert L.luvc_kv_fork(ctypes.byref(cache()), refs, i32(0, 1, 0, 2), 16 * 3 + 1, 1, i32(*[0] * 4), None) == lv.LUVC_ERR_WORKSPACE
    assert list(refs) == start


def test_counts_beyond_32_bits():
    """The library would see their lower 32 bits: one page, where more are asked for than memory holds."""
    refs = torch.zeros(8, dtype=torch.int32)
    for n in (2 ** 32 + 1, 2 ** 31, -2 ** 32 + 1, 2 ** 63):
        with pytest.raises(lv.LuvcError) as e:
            lv.luvc_kv_take(refs, n)
        assert e.value.status == lv.LUVC_ERR_INVALID_ARG and not refs.any()
