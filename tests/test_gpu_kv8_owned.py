"""An append after a reserve that did not fit, by a caller that does not look at the status in between: the table still
names pages that other sequences share, and those stay as they are, bit for bit."""
import numpy as np
import pytest
import torch

from paper_2601_19278_b200 import binding as b
from test_gpu_kv8 import DEV, Server

pytestmark = pytest.mark.gpu


def rows(s, layers, batch, n, seed, scale=30.0):
    g = torch.Generator().manual_seed(seed)
    hkv, d = s.t[0].shape[2], s.t[0].shape[4]
    return [(torch.randn(layers, batch, n, hkv, d, generator=g) * scale).to(torch.bfloat16) for _ in range(2)]


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("more", [2, 40])
def test_a_shared_page_survives_the_append_after_a_reserve_over_capacity(fmt, more):
    s = Server(5, 16, 4, 6, fmt, hkv=2, d=64, layers=2, seed=51)
    s.reserve([0], [20])
    s.advance([0], [20])
    s.fork([0], [1])
    s.reserve([2], [33])                                     # the rest of the pool
    s.advance([2], [33])
    s.check()
    assert not s.reserve([0, 1, 2], [more, more, 3])         # a copy of the shared page has no place
    kn, vn = rows(s, 2, 3, more, 1)                          # larger than what is there: a scale would grow
    counts = [more, more, 3 if more > 2 else 2]
    b.kv8_append(s.cache, 0, kn.to(DEV), vn.to(DEV), s.lens, s.table, slots=s.i32([0, 1, 2]), n_append=s.i32(counts), status=s.status, pages=s.pages)
    torch.cuda.synchronize()
    assert int(s.status) == b.DART_ERR_INVALID_ARG           # (the reserve's own error was cleared by `reserve`)
    s.status.zero_()
    for l in range(2):                                       # slot 2 owns its last page, which has room
        s.pool.append(l, s.book.table[2], 33, kn[l, 2, :counts[2]].double().numpy(), vn[l, 2, :counts[2]].double().numpy())
    s.check()


def test_the_status_of_the_reserve_stays():
    s = Server(4, 16, 3, 4, seed=52)
    s.reserve([0], [20])
    s.advance([0], [20])
    s.fork([0], [1])
    s.reserve([2], [17])
    s.advance([2], [17])
    kn, vn = rows(s, 2, 2, 1, 2)
    who, one = s.i32([0, 1]), s.i32([1, 1])
    g = torch.cuda.CUDAGraph()                               # nobody looks in between: both calls are one captured graph
    torch.cuda.synchronize()
    k, v = kn.to(DEV), vn.to(DEV)
    with torch.cuda.graph(g):
        b.kv8_reserve(s.pages, s.cache, who, one, workspace=s.ws, status=s.status)
        b.kv8_append(s.cache, 0, k, v, s.lens, s.table, slots=who, status=s.status, pages=s.pages)
    for _ in range(2):
        s.status.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert int(s.status) == b.DART_ERR_CAPACITY
        s.status.zero_()
        s.check()
    s.release([2])                                           # now there is room
    g.replay()
    s.copies(s.book.reserve([0, 1], [1, 1]))
    for l in range(2):
        for i in range(2):
            s.pool.append(l, s.book.table[i], 20, kn[l, i].double().numpy(), vn[l, i].double().numpy())
    torch.cuda.synchronize()
    assert int(s.status) == 0
    for w in (0, 1):
        np.testing.assert_array_equal(s.t[2 + w].cpu().numpy(), s.pool.scales[w].astype(np.float32))
    assert s.table.tolist() == s.book.table and s.ref.tolist() == s.book.ref


@pytest.mark.parametrize("n", [1, 3, 16, 40, 129])
def test_an_owned_append_is_the_append(n):
    """Every team size: the same bits with and without the counts."""
    out = []
    for owned in (False, True):
        s = Server(40, 128 if n > 40 else 16, 3, 12, "int8", hkv=2, d=128, seed=53)
        s.reserve([0, 1, 2], [5, 16, 0])
        s.advance([0, 1, 2], [5, 16, 0])
        s.reserve([0, 1, 2], [n, n, n])
        kn, vn = rows(s, 2, 3, n, 3)
        b.kv8_append(s.cache, 0, kn.to(DEV), vn.to(DEV), s.lens, s.table, status=s.status, pages=s.pages if owned else None)
        torch.cuda.synchronize()
        assert int(s.status) == 0
        out.append([t.clone() for t in s.t])
    assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(*out))


def test_pages_without_a_holder_and_other_tables_are_refused():
    s = Server(12, 16, 3, 4, seed=54)
    s.reserve([0], [20])
    s.advance([0], [20])
    kn, vn = rows(s, 2, 1, 2, 4)
    s.ref[s.book.table[0][1]] = 0
    s.book.ref[s.book.table[0][1]] = 0
    b.kv8_append(s.cache, 0, kn.to(DEV), vn.to(DEV), s.lens, s.table, slots=s.i32([0]), status=s.status, pages=s.pages)
    torch.cuda.synchronize()
    assert int(s.status) == b.DART_ERR_INVALID_ARG
    s.status.zero_()
    s.check()
    for table in (s.table.clone(), s.table[:2]):
        with pytest.raises((b.DartError, ValueError)):
            b.kv8_append(s.cache, 0, kn.to(DEV), vn.to(DEV), s.lens[:table.shape[0]].clone(), table, slots=s.i32([0]), pages=s.pages)
