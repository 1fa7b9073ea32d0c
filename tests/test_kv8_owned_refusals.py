"""What dart_kv8_append_owned refuses before anything is enqueued, seen without a GPU."""
import ctypes as C

import pytest

from test_kv8_refusals import A4, _append, _cache, _pages, b  # noqa: F401


@pytest.mark.parametrize("over", [dict(ref_count=None), dict(n_pages=9), dict(page_tokens=32), dict(max_seqs=3), dict(max_pages=5), dict(page_table=A4 + 4)],
                         ids=str)
def test_other_bookkeeping_is_refused(b, over):  # noqa: F811
    L, cache, a = b.lib(), _cache(b), _append(b, max_seqs=4)
    assert L.dart_kv8_append_owned(C.byref(cache), C.byref(_pages(b, **over)), C.byref(a), None) == b.DART_ERR_INVALID_ARG


@pytest.mark.parametrize("over", [dict(batch=0), dict(k_new=None), dict(row_stride=120), dict(max_append=4), dict(first_layer=1)], ids=str)
def test_what_the_append_refuses_is_refused(b, over):  # noqa: F811
    L, cache, pages = b.lib(), _cache(b), _pages(b)
    a = _append(b, **{"max_seqs": 4, **over})
    assert L.dart_kv8_append_owned(C.byref(cache), C.byref(pages), C.byref(a), None) == b.DART_ERR_INVALID_ARG
    assert L.dart_kv8_append_owned(C.byref(cache), None, C.byref(_append(b, max_seqs=4)), None) == b.DART_ERR_INVALID_ARG
    assert L.dart_kv8_append_owned(C.byref(cache), C.byref(pages), None, None) == b.DART_ERR_INVALID_ARG
