"""How attention calls over the paged 8-bit cache are cut (dart_kv8_attention_plan; no GPU needed), and that the shapes that
the GPU tests run cover each form: a cost model that is tuned again must not drop one unseen."""
import ctypes as C

import pytest

from kv8_plan_cases import CASES
from test_kv8_refusals import _cache, b  # noqa: F401


def plan(b, batch, rows, heads, kv_heads, dim, max_len, new=True):  # noqa: F811
    out = b.DartKv8Plan()
    rc = b.lib().dart_kv8_attention_plan(C.byref(_cache(b, n_kv_heads=kv_heads, head_dim=dim)), batch, rows, heads, max_len, int(new), C.byref(out))
    return rc, {f[0]: getattr(out, f[0]) for f in out._fields_}


@pytest.mark.parametrize("name", sorted(CASES))
def test_the_gpu_cases_are_cut_as_they_are_meant_to_be(b, name):  # noqa: F811
    rows, heads, kv_heads, dim, lens, max_len, new, _, want = CASES[name]
    rc, got = plan(b, len(lens), rows, heads, kv_heads, dim, max_len, new)
    assert rc == b.DART_OK and got["many_rows"] == 1
    assert {k: got[k] for k in want} == want
    pages = -(-max(lens) // 16)
    if "whole" in name or "chunk_in" in name and want["max_parts"] == 1:
        assert pages > 32 and got["keys_per_part"] > 4 * 128      # several windows of page ids and rounds of the rings in one CTA


def test_few_rows_and_refusals(b):  # noqa: F811
    for dim, rows in ((64, 32), (128, 24)):
        assert plan(b, 1, rows, 2, 2, dim, 1000)[1]["many_rows"] == 0 and plan(b, 1, rows + 1, 2, 2, dim, 1000)[1]["many_rows"] == 1
    for bad in ((0, 3, 4, 2, 64, 10), (2, 0, 4, 2, 64, 10), (2, 3, 5, 2, 64, 10), (2, 3, 4, 2, 64, -1), (2, 3, 4, 2, 80, 10)):
        assert plan(b, *bad)[0] == b.DART_ERR_INVALID_ARG
    assert b.lib().dart_kv8_attention_plan(C.byref(_cache(b)), 1, 1, 4, 10, 1, None) == b.DART_ERR_INVALID_ARG


@pytest.mark.parametrize("batch,rows,heads", [(1, 1, 8), (1, 60, 8), (64, 1, 8), (3, 60, 40), (2, 1001, 32), (1024, 1, 8), (1, 4096, 8)])
def test_parts_cover_the_longest_sequence_and_the_workspace_holds_them(b, batch, rows, heads):  # noqa: F811
    cache = _cache(b, n_kv_heads=8, head_dim=128)
    for max_len in (0, 1, 128, 513, 4096, 8192, 131001, 1 << 20, (1 << 31) - (1 << 21) - 16):
        rc, p = plan(b, batch, rows, heads, 8, 128, max_len)
        assert rc == b.DART_OK and p["max_parts"] * p["keys_per_part"] >= max_len and p["max_parts"] <= 65535
        partials = batch * 8 * (p["row_tiles"] * 128 if p["many_rows"] else -(-rows * heads // 8 // 8) * 8) * p["max_parts"]
        if p["max_parts"] > 1:
            assert b.lib().dart_kv8_attention_workspace_bytes(C.byref(cache), batch, rows, heads, max_len) >= partials * (128 + 2) * 4


def test_the_plan_structure_is_the_headers(b, tmp_path):  # noqa: F811
    import os
    import subprocess
    from test_kv8_refusals import ROOT
    src = tmp_path / "sz.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "dart.h"\nint main(void){printf("%zu %zu", sizeof(dart_kv8_plan), '
                   'offsetof(dart_kv8_plan, max_parts));return 0;}\n')
    exe = tmp_path / "sz"
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    assert [int(x) for x in subprocess.check_output([str(exe)]).split()] == [C.sizeof(b.DartKv8Plan), b.DartKv8Plan.max_parts.offset]
