"""The bounded waits of the many-row attention with a window, made to run out as test_gpu_kv8_timeout does it: keys of the cache stop arriving at some
group of 64, beside tiles of new rows that arrive.  Nothing faults and nothing hangs; the next call gives the bits that the call before gave."""
import ctypes as C

import pytest
import torch

from paper_2601_19278_b200 import binding as b
from test_gpu_kv8 import DEV, Case, guarded, intact
from test_gpu_kv8_window import trees, windowed

pytestmark = pytest.mark.gpu


def selftest(c, q, kn, vn, max_len, window, sinks, mask, positions, limit, missing_from):
    B, R, H, d = q.shape
    out, raw_o = guarded((B, R, H, d), torch.bfloat16, 0)
    ws, raw_w = guarded((b.kv8_attention_window_workspace_bytes(c.cache, B, R, H, max_len, window, sinks),), torch.uint8)
    status, raw_s = guarded((1,), torch.int32, 0)
    ptr = lambda t: 0 if t is None else t.data_ptr()  # noqa: E731
    a = b.DartKv8AttnIn(layer=0, batch=B, rows=R, n_q_heads=H, max_seqs=c.table.shape[0], max_pages=c.table.shape[1], max_len=max_len,
                        q=ptr(q), k_new=ptr(kn), v_new=ptr(vn), q_stride=H * d, new_stride=c.hkv * d, seq_lens=ptr(c.seq_lens),
                        page_table=ptr(c.table), mask=ptr(mask), out=ptr(out), workspace=ptr(ws), workspace_bytes=ws.numel(), status=ptr(status))
    w = b.DartKv8Window(window, sinks, ptr(positions))
    rc = b.lib().dart_selftest_kv8_window_wait(c.cache.ref, C.byref(a), C.byref(w), limit, missing_from, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    intact(raw_o, raw_w, raw_s, *c.raws)
    return rc, int(status)


# trees in one row tile, in pairs and over many KV heads; chunks whose rows see the cache and one another, and some one another alone
@pytest.mark.parametrize("B,R,H,hkv,d,pt,fmt,tree", [(2, 60, 1, 1, 128, 16, "e4m3", True), (2, 60, 5, 1, 64, 64, "int8", True), (8, 60, 40, 8, 128, 32, "int8", True),
                                                     (2, 300, 4, 1, 128, 128, "e4m3", False), (2, 1001, 2, 2, 64, 16, "int8", False)])
@pytest.mark.parametrize("window,sinks,missing_from", [(150, 4, 0), (150, 4, 1), (150, 130, 3), (1500, 0, 0), (1500, 4, 3), (1500, 0, 6)])
def test_waits_that_run_out_are_reported_and_the_next_call_is_unharmed(B, R, H, hkv, d, pt, fmt, tree, window, sinks, missing_from):
    max_len = 3000
    c = Case([2900] + [700] * (B - 1), pt, fmt, hkv, d, seed=R, room=max_len - 2900)
    q, kn, vn = (c.bf16(B, R, h, d).to(DEV) for h in (H, hkv, hkv))
    mask = positions = None
    if tree:
        mask, positions = trees(c.rng, c.lens, R, [R] * B)
    kw = dict(mask=mask, positions=positions)
    good = windowed(c, q, kn, vn, max_len, window, sinks, **kw)
    on = [None if t is None else torch.as_tensor(t, dtype=dt).to(DEV) for t, dt in ((mask, torch.uint8), (positions, torch.int32))]
    for limit in (100, 400):
        assert selftest(c, q, kn, vn, max_len, window, sinks, *on, limit, missing_from) == (b.DART_OK, b.DART_ERR_TIMEOUT)
        assert torch.equal(windowed(c, q, kn, vn, max_len, window, sinks, **kw), good)
