"""The bounded waits of the many-row attention over the paged 8-bit cache, made to run out: keys stop arriving at some group of
64 and every wait has a short limit.  Nothing faults and nothing hangs: the status word says TIMEOUT, nothing outside the
buffers is written, and the next call gives the bits that the call before gave."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2601_19278_b200 import binding as b
from test_gpu_kv8 import DEV, Case, attend, guarded, intact, tree_mask

pytestmark = pytest.mark.gpu


def selftest(c, q, kn, vn, mask, max_len, limit, missing_from):
    B, R, H, d = q.shape
    out, raw_o = guarded((B, R, H, d), torch.bfloat16, 0)
    ws, raw_w = guarded((b.kv8_attention_workspace_bytes(c.cache, B, R, H, max_len),), torch.uint8)
    status, raw_s = guarded((1,), torch.int32, 0)
    ptr = lambda t: 0 if t is None else t.data_ptr()  # noqa: E731
    a = b.DartKv8AttnIn(layer=0, batch=B, rows=R, n_q_heads=H, max_seqs=c.table.shape[0], max_pages=c.table.shape[1], max_len=max_len,
                        q=ptr(q), k_new=ptr(kn), v_new=ptr(vn), q_stride=H * d, new_stride=c.hkv * d, seq_lens=ptr(c.seq_lens),
                        page_table=ptr(c.table), mask=ptr(mask), out=ptr(out), workspace=ptr(ws), workspace_bytes=ws.numel(), status=ptr(status))
    rc = b.lib().dart_selftest_kv8_wait(c.cache.ref, C.byref(a), limit, missing_from, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    intact(raw_o, raw_w, raw_s, *c.raws)
    return rc, int(status)


# one row tile; two that share key steps, whole and split; a tree; a prompt's chunk
@pytest.mark.parametrize("B,R,H,hkv,d,pt,fmt,tree,max_len", [(2, 60, 1, 1, 128, 16, "e4m3", True, 3000), (2, 4096, 1, 1, 64, 64, "int8", False, 3000),
                                                             (16, 60, 40, 8, 128, 16, "int8", True, 8192), (2, 300, 4, 1, 128, 128, "e4m3", False, 3000)])
@pytest.mark.parametrize("missing_from", [0, 1, 3, 6])
def test_waits_that_run_out_are_reported_and_the_next_call_is_unharmed(B, R, H, hkv, d, pt, fmt, tree, max_len, missing_from):
    c = Case([2900] + [700] * (B - 1), pt, fmt, hkv, d, seed=R, room=max_len - 2900)
    q, kn, vn = (c.bf16(B, R, h, d).to(DEV) for h in (H, hkv, hkv))
    mask = torch.from_numpy(np.stack([tree_mask(c.rng, R, R)] * B)).to(DEV) if tree else None
    good = attend(c, 0, q, kn, vn, max_len, mask=mask)
    for limit in (100, 400):
        assert selftest(c, q, kn, vn, mask, max_len, limit, missing_from) == (b.DART_OK, b.DART_ERR_TIMEOUT)
        assert torch.equal(attend(c, 0, q, kn, vn, max_len, mask=mask), good)


def test_the_self_test_of_calls_that_have_no_such_waits_is_refused():
    c = Case([300], 16, "e4m3", 1, 64, seed=1)
    for R, limit, missing, want in ((1, 100, 0, b.DART_ERR_INVALID_ARG), (32, 100, 0, b.DART_ERR_INVALID_ARG), (40, 0, 0, b.DART_ERR_INVALID_ARG),
                                    (40, 100001, 0, b.DART_ERR_INVALID_ARG), (40, 100, -1, b.DART_ERR_INVALID_ARG)):
        q, kn, vn = (c.bf16(1, R, 1, 64).to(DEV) for _ in range(3))
        assert selftest(c, q, kn, vn, None, 300, limit, missing) == (want, 0)
