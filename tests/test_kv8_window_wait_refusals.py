"""What the self-test of the windowed attention's waits refuses (no GPU needed)."""
import ctypes as C

import pytest

from test_kv8_refusals import A16, A4, _attn, _cache, b  # noqa: F401


@pytest.mark.parametrize("window,limit,missing,kw", [
    (None, 100, 0, {}), ((0, 0), 100, 0, {}), ((8, -1), 100, 0, {}), ((8, 0), 0, 0, {}), ((8, 0), 100001, 0, {}), ((8, 0), 100, -1, {}),
    ((8, 0), 100, 0, dict(status=None)), ((8, 0), 100, 0, dict(rows=1)), ((8, 0), 100, 0, dict(workspace_bytes=0))], ids=str)
def test_refused(b, window, limit, missing, kw):  # noqa: F811
    w = None if window is None else C.byref(b.DartKv8Window(window[0], window[1], None))
    a = _attn(b, **{**dict(rows=60, status=A4), **kw})
    assert b.lib().dart_selftest_kv8_window_wait(C.byref(_cache(b)), C.byref(a), w, limit, missing, None) == b.DART_ERR_INVALID_ARG


def test_a_tree_and_a_chunk_are_accepted_as_far_as_the_device(b):  # noqa: F811
    for kw, positions in ((dict(mask=A16, n_rows=A4), A4), ({}, None)):
        w = b.DartKv8Window(8, 1, positions)
        got = b.lib().dart_selftest_kv8_window_wait(C.byref(_cache(b)), C.byref(_attn(b, rows=60, status=A4, **kw)), C.byref(w), 100, 0, None)
        assert got in (b.DART_ERR_CUDA, b.DART_ERR_UNSUPPORTED_ARCH)
