"""What the paged 8-bit cache's C entries refuse before anything is enqueued, seen without a GPU: the pointers are
addresses that nothing reads.  (The first accepted call here would ask for the device and answer UNSUPPORTED_ARCH or
CUDA, never OK.)"""
import ctypes as C
import os
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A16, A4, ODD = 0x10000, 0x10004, 0x10002


@pytest.fixture(scope="module")
def b():
    from paper_2601_19278_b200 import build
    build.build()
    from paper_2601_19278_b200 import binding
    return binding


def _cache(b, **over):
    v = dict(format=0, n_layers=2, n_pages=8, n_kv_heads=2, page_tokens=16, head_dim=64, k_pages=A16, v_pages=A16, k_scale=A4, v_scale=A4)
    v.update(over)
    return b.DartKv8Cache(**v)


def _attn(b, **over):
    v = dict(layer=0, batch=2, rows=3, n_q_heads=4, max_seqs=2, max_pages=4, max_len=64, q=A16, k_new=A16, v_new=A16, q_stride=256, new_stride=128,
             slots=None, seq_lens=A4, page_table=A4, n_rows=None, mask=None, out=A16, workspace=A16, workspace_bytes=1 << 40, status=None)
    v.update(over)
    return b.DartKv8AttnIn(**v)


def _append(b, **over):
    v = dict(first_layer=0, n_layers=2, batch=2, rows=3, max_append=3, max_seqs=2, max_pages=4, k_new=A16, v_new=A16, row_stride=128,
             layer_stride=768, slots=None, seq_lens=A4, page_table=A4, n_append=None, row_index=None, status=None)
    v.update(over)
    return b.DartKv8AppendIn(**v)


def _pages(b, **over):
    v = dict(n_pages=8, page_tokens=16, max_seqs=4, max_pages=4, page_table=A4, seq_lens=A4, ref_count=A4)
    v.update(over)
    return b.DartKv8Pages(**v)


BAD_CACHE = [dict(format=2), dict(n_layers=0), dict(n_layers=1025), dict(n_pages=0), dict(n_pages=(1 << 24) + 1), dict(n_kv_heads=0),
             dict(n_kv_heads=257), dict(page_tokens=8), dict(page_tokens=48), dict(page_tokens=256), dict(head_dim=96), dict(head_dim=256),
             dict(k_pages=None), dict(v_pages=A4), dict(k_scale=None), dict(v_scale=ODD)]


@pytest.mark.parametrize("over", BAD_CACHE, ids=str)
def test_every_call_refuses_a_bad_pool(b, over):
    L, bad = b.lib(), _cache(b, **over)
    refused = b.DART_ERR_INVALID_ARG
    assert L.dart_kv8_attention(C.byref(bad), C.byref(_attn(b)), None) == refused
    assert L.dart_kv8_append(C.byref(bad), C.byref(_append(b)), None) == refused
    assert L.dart_kv8_reserve(C.byref(_pages(b)), C.byref(bad), A4, A4, 1, A16, 1 << 40, None, None) == refused
    assert L.dart_kv8_compact(C.byref(_pages(b)), C.byref(bad), None, A16, 1 << 40, None, None) == refused


@pytest.mark.parametrize("over", [
    dict(layer=-1), dict(layer=2), dict(batch=0), dict(batch=1025), dict(batch=3), dict(rows=0), dict(rows=4097), dict(n_q_heads=0),
    dict(n_q_heads=5), dict(n_q_heads=2 * 129, q_stride=1 << 20), dict(max_seqs=0), dict(max_pages=0), dict(max_len=-1), dict(max_len=65), dict(q=None), dict(q=A4),
    dict(q_stride=248), dict(q_stride=260), dict(k_new=None), dict(v_new=None), dict(k_new=A4), dict(new_stride=120), dict(new_stride=132),
    dict(slots=ODD), dict(seq_lens=None), dict(page_table=None), dict(n_rows=ODD), dict(mask=A16, rows=65), dict(mask=A16, k_new=None, v_new=None),
    dict(out=None), dict(out=A4), dict(workspace=None), dict(workspace=A4), dict(workspace_bytes=0), dict(status=ODD)], ids=str)
def test_attention_refuses(b, over):
    assert b.lib().dart_kv8_attention(C.byref(_cache(b)), C.byref(_attn(b, **over)), None) == b.DART_ERR_INVALID_ARG


@pytest.mark.parametrize("over", [
    dict(first_layer=-1), dict(first_layer=1), dict(n_layers=0), dict(n_layers=3), dict(batch=0), dict(batch=1025), dict(batch=3), dict(rows=0),
    dict(max_append=0), dict(max_append=4), dict(row_index=A4, max_append=(1 << 20) + 1), dict(max_seqs=0), dict(max_pages=0),
    dict(max_pages=1 << 28), dict(k_new=None), dict(v_new=A4), dict(row_stride=120), dict(row_stride=129), dict(layer_stride=-8),
    dict(layer_stride=12), dict(seq_lens=None), dict(page_table=ODD), dict(slots=ODD), dict(n_append=ODD), dict(row_index=ODD),
    dict(status=ODD)], ids=str)
def test_append_refuses(b, over):
    assert b.lib().dart_kv8_append(C.byref(_cache(b)), C.byref(_append(b, **over)), None) == b.DART_ERR_INVALID_ARG


def test_page_operations_refuse(b):
    L, refused, ws = b.lib(), b.DART_ERR_INVALID_ARG, 1 << 40
    good, cache = _pages(b), _cache(b)
    for over in (dict(n_pages=0), dict(page_tokens=17), dict(max_seqs=0), dict(max_seqs=65537), dict(max_pages=0), dict(max_pages=1 << 28),
                 dict(page_table=None), dict(seq_lens=ODD), dict(ref_count=None)):
        bad = _pages(b, **over)
        assert L.dart_kv8_fork(C.byref(bad), A4, A4, 1, None, None) == refused
        assert L.dart_kv8_release(C.byref(bad), A4, 1, None, None) == refused
        assert L.dart_kv8_reserve(C.byref(bad), C.byref(cache), A4, A4, 1, A16, ws, None, None) == refused
        assert L.dart_kv8_compact(C.byref(bad), C.byref(cache), None, A16, ws, None, None) == refused
    for n in (0, -1, 1025):
        assert L.dart_kv8_fork(C.byref(good), A4, A4, n, None, None) == refused
        assert L.dart_kv8_release(C.byref(good), A4, n, None, None) == refused
        assert L.dart_kv8_reserve(C.byref(good), C.byref(cache), A4, A4, n, A16, ws, None, None) == refused
    assert L.dart_kv8_fork(C.byref(good), None, A4, 1, None, None) == refused
    assert L.dart_kv8_fork(C.byref(good), A4, ODD, 1, None, None) == refused
    assert L.dart_kv8_release(C.byref(good), A4, 1, ODD, None) == refused
    need = L.dart_kv8_pages_workspace_bytes(C.byref(good))
    assert need > 0 and L.dart_kv8_pages_workspace_bytes(None) == 0
    for w, size in ((None, ws), (A4, ws), (A16, need - 1)):
        assert L.dart_kv8_reserve(C.byref(good), C.byref(cache), A4, A4, 1, w, size, None, None) == refused
        assert L.dart_kv8_compact(C.byref(good), C.byref(cache), None, w, size, None, None) == refused
    other = _cache(b, n_pages=9)                                         # another pool than the bookkeeping's
    assert L.dart_kv8_reserve(C.byref(good), C.byref(other), A4, A4, 1, A16, ws, None, None) == refused
    assert L.dart_kv8_compact(C.byref(good), C.byref(_cache(b, page_tokens=32)), None, A16, ws, None, None) == refused


def test_attention_workspace_size(b):
    L, cache = b.lib(), _cache(b)
    sizes = [L.dart_kv8_attention_workspace_bytes(C.byref(cache), 2, 3, 4, n) for n in (0, 100, 1000, 100000)]
    assert sizes[0] > 0 and sizes == sorted(sizes)
    for bad in ((0, 3, 4, 10), (2, 0, 4, 10), (2, 3, 5, 10), (2, 3, 4, -1), (1025, 3, 4, 10)):
        assert L.dart_kv8_attention_workspace_bytes(C.byref(cache), *bad) == 0
    assert L.dart_kv8_attention_workspace_bytes(C.byref(_cache(b, head_dim=80)), 2, 3, 4, 10) == 0


def test_struct_layouts_match_the_header(b, tmp_path):
    names = {"dart_kv8_cache": b.DartKv8Cache, "dart_kv8_attn_in": b.DartKv8AttnIn, "dart_kv8_append_in": b.DartKv8AppendIn, "dart_kv8_pages": b.DartKv8Pages}
    lines = []
    for n, s in names.items():
        lines.append(f'printf("%zu ", sizeof({n}));')
        lines += [f'printf("%zu ", offsetof({n}, {f[0]}));' for f in s._fields_]
    src = tmp_path / "sz.c"
    src.write_text("#include <stdio.h>\n#include <stddef.h>\n#include \"dart.h\"\nint main(void){" + "".join(lines) + "return 0;}\n")
    exe = tmp_path / "sz"
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    want = []
    for s in names.values():
        want += [C.sizeof(s)] + [getattr(s, f[0]).offset for f in s._fields_]
    assert [int(x) for x in subprocess.check_output([str(exe)]).split()] == want


def test_packed_arguments_are_the_structures(b):
    for packer, s in ((b._KV8_ATTN, b.DartKv8AttnIn), (b._KV8_APPEND, b.DartKv8AppendIn)):
        assert packer.size == C.sizeof(s)
        values = list(range(1, len(s._fields_) + 1))
        filled = s.from_buffer_copy(packer.pack(*values))
        assert [getattr(filled, f[0]) for f in s._fields_] == values


def test_the_binding_refuses_host_tensors(b):
    pages = torch.zeros(1, 4, 2, 16, 64, dtype=torch.int8)
    scale = torch.ones(1, 4, 2)
    with pytest.raises(ValueError, match="CUDA"):
        b.Kv8Cache(pages, pages, scale, scale)
    with pytest.raises(ValueError, match="float8_e4m3fn or int8"):
        b.Kv8Cache(pages.float(), pages, scale, scale)
    with pytest.raises(ValueError, match="CUDA"):
        b.Kv8Pages(torch.full((2, 4), -1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(4, dtype=torch.int32), 16)
