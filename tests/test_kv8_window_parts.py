"""Which windowed calls of a few rows are cut into parts that differ from pair to pair (no GPU needed): those that have about a wave of pairs, and
smaller ones whose windows are short."""
import ctypes as C

import pytest

from test_kv8_refusals import _cache, b  # noqa: F401


def plan(b, batch, hkv, dim, rows, group, window):  # noqa: F811
    out = b.DartKv8Plan()
    assert b.lib().dart_kv8_attention_window_plan(C.byref(_cache(b, n_kv_heads=hkv, head_dim=dim)), batch, rows, group * hkv, 8192, window, 4, 1,
                                                  C.byref(out)) == b.DART_OK
    assert out.many_rows == 0
    return out.max_parts, out.keys_per_part


def uneven(window):
    """Three parts, of which the largest has 30 32nds of the window, the sinks and what lies beside them, a 32nd in whole groups of 16 keys."""
    return 3, -(-(16 + window + 14) // 512) * 16 * 30


@pytest.mark.parametrize("batch,hkv,dim,rows,group,window", [(64, 8, 128, 1, 5, 4096), (44, 8, 128, 1, 5, 1100), (72, 8, 128, 1, 5, 2000), (60, 8, 64, 1, 4, 4096),
                                                             (32, 8, 128, 2, 5, 2000), (30, 8, 128, 1, 5, 2000), (34, 8, 128, 1, 5, 1100)])
def test_about_a_wave_of_pairs_is_cut_unevenly(b, batch, hkv, dim, rows, group, window):  # noqa: F811
    assert plan(b, batch, hkv, dim, rows, group, window) == uneven(window)


@pytest.mark.parametrize("batch,hkv,dim,rows,group,window,want", [
    (28, 8, 128, 1, 5, 4096, (4, 1152)), (40, 8, 128, 1, 5, 4096, (3, 1408)), (24, 8, 128, 2, 5, 4096, (4, 1152)),      # few pairs, long windows
    (80, 8, 128, 1, 5, 1500, (2, 768)), (100, 8, 128, 1, 5, 2000, (2, 1024)), (112, 8, 128, 1, 5, 4096, (1, 4224)), (200, 8, 128, 1, 5, 2000, (1, 2048)),
    (200, 8, 128, 1, 5, 1100, (1, 1152)), (120, 8, 64, 1, 4, 2000, (2, 1024)), (500, 2, 64, 1, 2, 4096, (2, 2176))])    # many pairs
def test_others_are_cut_into_equal_parts(b, batch, hkv, dim, rows, group, window, want):  # noqa: F811
    assert plan(b, batch, hkv, dim, rows, group, window) == want
