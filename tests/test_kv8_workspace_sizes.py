"""Calls that are not cut into parts need no room for partial results (no GPU needed): a caller's small workspace stays enough."""
import ctypes as C

import pytest

from test_kv8_refusals import _cache, b  # noqa: F401


@pytest.mark.parametrize("batch,rows,heads,hkv,dim", [(1, 1, 4, 2, 64), (64, 1, 40, 8, 128), (1024, 3, 64, 8, 64), (1024, 1, 8, 8, 128)])
def test_few_rows_over_short_sequences_need_sixteen_bytes(b, batch, rows, heads, hkv, dim):  # noqa: F811
    cache = C.byref(_cache(b, n_kv_heads=hkv, head_dim=dim))
    for max_len in (0, 1, 100, 511, 512):
        assert b.lib().dart_kv8_attention_workspace_bytes(cache, batch, rows, heads, max_len) == 16
        for window, sinks in ((1, 0), (100, 4), (1 << 20, 0)):
            assert b.lib().dart_kv8_attention_window_workspace_bytes(cache, batch, rows, heads, max_len, window, sinks) == 16
    assert b.lib().dart_kv8_attention_window_workspace_bytes(cache, batch, rows, heads, 8192, 400, 64) == 16       # a short window over a long cache


@pytest.mark.parametrize("batch,hkv", [(1, 2), (31, 8), (64, 8), (200, 8)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1100, 4), (2000, 100), (4096, 4), (70000, 0)])
def test_a_window_s_workspace_holds_the_parts_of_every_smaller_bound(b, batch, hkv, window, sinks):  # noqa: F811
    cache, dim, heads = _cache(b, n_kv_heads=hkv, head_dim=128), 128, 5 * hkv
    for max_len in (513, 1200, 5000, 8192, 131001):
        room = b.lib().dart_kv8_attention_window_workspace_bytes(C.byref(cache), batch, 1, heads, max_len, window, sinks)
        for bound in sorted({1, 512, 513, 1024, 1151, 2100, 4200, max_len - 1, max_len}):
            if bound > max_len:
                continue
            out = b.DartKv8Plan()
            assert b.lib().dart_kv8_attention_window_plan(C.byref(cache), batch, 1, heads, bound, window, sinks, 1, C.byref(out)) == b.DART_OK
            assert out.many_rows == 0
            if out.max_parts > 1:
                assert room >= 16 + batch * hkv * 8 * out.max_parts * (dim + 2) * 4
            assert b.lib().dart_kv8_attention_window_workspace_bytes(C.byref(cache), batch, 1, heads, bound, window, sinks) <= room
