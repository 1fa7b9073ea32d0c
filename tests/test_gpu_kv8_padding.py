"""Padded batches: entries that add nothing (count 0) name a slot that another entry of the list names too."""
import pytest
import torch

from paper_2601_19278_b200 import binding as b
from test_gpu_kv8 import DEV, Case, Server, same_pool

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("slots,counts", [([1, 1, 0, 0], [0, 3, 2, 0]), ([0, 0, 0, 0], [4, 0, 0, 0]), ([0, 0, 0, 0], [0, 0, 0, 4]),
                                          ([1, 0, 1, 0], [0, 0, 0, 0])])
def test_an_append_entry_without_rows_claims_no_slot(slots, counts, fmt):
    c = Case([5, 14], 16, fmt, 2, 64, layers=2, seed=61, room=8)
    kn, vn = c.bf16(2, 4, 4, 2, 64), c.bf16(2, 4, 4, 2, 64)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    status = i32([0])
    b.kv8_append(c.cache, 0, kn.to(DEV), vn.to(DEV), c.seq_lens, c.table, slots=i32(slots), n_append=i32(counts), status=status)
    for i, (s, n) in enumerate(zip(slots, counts)):
        for l in range(2):
            c.pool.append(l, c.pages[s], c.lens[s], kn[l, i, :n].double().numpy(), vn[l, i, :n].double().numpy())
    same_pool(c)
    assert int(status) == 0


def test_a_reserve_entry_without_positions_claims_no_slot():
    s = Server(30, 16, 4, 4, seed=62)
    s.reserve([1, 1, 0, 0, 2], [0, 20, 5, 0, 0])
    s.check()
    s.advance([0, 1], [5, 20])
    s.fork([1], [2])
    s.reserve([2, 2, 1, 1], [0, 9, 3, 0])                    # one copy: the last listed sharer keeps the page
    s.check()


def test_two_entries_with_rows_are_still_one_too_many():
    c = Case([5, 14], 16, "int8", 1, 64, seed=63, room=8)
    kn, vn = c.bf16(1, 3, 2, 1, 64), c.bf16(1, 3, 2, 1, 64)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    status = i32([0])
    b.kv8_append(c.cache, 0, kn.to(DEV), vn.to(DEV), c.seq_lens, c.table, slots=i32([0, 0, 0]), n_append=i32([0, 2, 1]), status=status)
    c.pool.append(0, c.pages[0], 5, kn[0, 1].double().numpy(), vn[0, 1].double().numpy())
    same_pool(c)
    assert int(status) == b.DART_ERR_INVALID_ARG
    s = Server(30, 16, 4, 4, seed=64)
    b.kv8_reserve(s.pages, s.cache, s.i32([0, 0, 0]), s.i32([0, 5, 40]), workspace=s.ws, status=s.status)
    s.book.reserve([0], [5])
    torch.cuda.synchronize()
    assert int(s.status) == b.DART_ERR_INVALID_ARG
    s.status.zero_()
    s.check()
