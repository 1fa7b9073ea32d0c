"""The paged 8-bit KV cache on the GPU against the oracle: attention (single tokens, a few rows, trees, prompt chunks),
append, page operations, and a run of them together.

Tolerance of attention, per element: the bf16 output is off by at most half a step, 2^-8 |ref|.  Weights enter the second
product rounded to fp16 (2^-11 each) or are kept in fp32; a score off by e changes every weight by a factor of at most
1 + 2 e, and scores are fp32 sums of exact products (keys and queries fit fp16 once scaled by a power of two, up to
2^-25 of the row's largest element): e <= 2^-19 * sum |q_i k_i| / sqrt(d).  With A = sum p |v|: error <= 2^-8 |ref| +
(2^-10 + 2^-18 X) A, plus 2^-20 of the largest |v| for elements that fp16 cuts off."""
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import kv8 as ok
from paper_2601_19278_b200 import binding as b

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
FMT = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
GUARD = 4096          # bytes of sentinel around every buffer that a kernel writes


def guarded(shape, dtype, fill=None):
    n = math.prod(shape) * torch.empty((), dtype=dtype).element_size()
    raw = torch.full((GUARD + n + GUARD,), 0xA5, dtype=torch.uint8, device=DEV)
    t = raw[GUARD:GUARD + n].view(dtype).view(shape)
    if fill is not None:
        t.fill_(fill)
    return t, raw


def intact(*raws):
    for raw in raws:
        assert bool((raw[:GUARD] == 0xA5).all()) and bool((raw[-GUARD:] == 0xA5).all()), "a kernel wrote outside its buffer"


def random_codes(rng, shape, fmt):
    c = rng.integers(0, 256, shape).astype(np.uint8)
    c[c == (0x80 if fmt == "int8" else 0x7F)] = 0          # codes that an append never writes
    if fmt == "e4m3":
        c[c == 0xFF] = 0
    return c


class Case:
    """A pool with random codes and scales, and sequences whose pages are scattered over it."""

    def __init__(self, lens, pt, fmt, hkv, d, layers=1, seed=0, spare=2, scale_exp=(-8, -5), room=0):
        rng = self.rng = np.random.default_rng(seed)
        self.lens, self.pt, self.fmt, self.hkv, self.d, self.layers = list(lens), pt, fmt, hkv, d, layers
        need = [-(-(n + room) // pt) for n in lens]
        total = sum(need) + spare
        ids = rng.permutation(total).tolist()
        self.pages = [[ids.pop() for _ in range(k)] for k in need]
        self.cols = max(1, max(need))
        table = np.full((len(lens), self.cols), -1, np.int32)
        for i, p in enumerate(self.pages):
            table[i, :len(p)] = p
        codes = [random_codes(rng, (layers, total, hkv, pt, d), fmt) for _ in range(2)]
        scales = [(2.0 ** rng.integers(scale_exp[0], scale_exp[1] + 1, (layers, total, hkv))).astype(np.float32) for _ in range(2)]
        self.pool = ok.Pool([c.copy() for c in codes], [s.copy() for s in scales], fmt)
        self.raws, self.t = [], []
        for x, dt in ((codes[0], FMT[fmt]), (codes[1], FMT[fmt]), (scales[0], torch.float32), (scales[1], torch.float32)):
            t, raw = guarded(x.shape, dt)
            (t.view(torch.uint8) if x.dtype == np.uint8 else t).copy_(torch.from_numpy(x))
            self.t.append(t)
            self.raws.append(raw)
        self.cache = b.Kv8Cache(*self.t)
        self.table = torch.from_numpy(table).to(DEV)
        self.seq_lens = torch.tensor(self.lens, dtype=torch.int32, device=DEV)

    def bf16(self, *shape, scale=1.0):
        return torch.from_numpy((self.rng.standard_normal(shape) * scale).astype(np.float32)).to(torch.bfloat16)


def attend(c, layer, q, kn, vn, max_len, slots=None, n_rows=None, mask=None, status_want=0, seq_lens=None, table=None, cache=None):
    """One call with guarded output and workspace; returns the output."""
    B, R, H, d = q.shape
    out, raw_o = guarded((B, R, H, d), torch.bfloat16, float("nan"))
    ws, raw_w = guarded((b.kv8_attention_workspace_bytes(c.cache, B, R, H, max_len),), torch.uint8)
    status, raw_s = guarded((1,), torch.int32, 0)
    b.kv8_attention(cache or c.cache, layer, q, kn, vn, c.seq_lens if seq_lens is None else seq_lens, c.table if table is None else table, out,
                    max_len=max_len, workspace=ws, slots=slots, n_rows=n_rows, mask=mask, status=status)
    torch.cuda.synchronize()
    intact(raw_o, raw_w, raw_s)
    assert int(status) == status_want
    return out


def check(c, layer, got, q, kn, vn, slots=None, n_rows=None, mask=None, only=None):
    """Every row (or `only` these) of every batch entry against the oracle."""
    f64 = lambda t: None if t is None else t.double().cpu().numpy()  # noqa: E731
    B, R = q.shape[:2]
    for i in range(B):
        s = i if slots is None else slots[i]
        r = R if n_rows is None else n_rows[i]
        m = None if mask is None else mask[i][:r, :r]
        rows = None if only is None else [x for x in only if x < r]
        ref, absv, absx = ok.attention(c.pool, layer, c.pages[s], c.lens[s], f64(q)[i, :r], None if kn is None else f64(kn)[i, :r],
                                       None if vn is None else f64(vn)[i, :r], m, rows)
        top = max([1e-30] + [np.abs(c.pool.read(1, layer, h, c.pages[s], c.lens[s])).max(initial=0.0) for h in range(c.hkv)]
                  + ([] if vn is None or r == 0 else [float(vn[i, :r].abs().max())]))
        tol = 2.0 ** -8 * np.abs(ref) + (2.0 ** -10 + 2.0 ** -18 * absx[..., None]) * absv + 2.0 ** -20 * top * (absv > 0)
        g = f64(got)[i]
        pick = range(r) if rows is None else rows
        for x in pick:
            err = np.abs(g[x] - ref[x])
            assert np.all(err <= tol[x]), (i, x, float((err - tol[x]).max()), float(err.max()))
        assert np.all(g[r:] == 0), "rows that do not exist are zero"


def tree_mask(rng, R, used):
    m = np.zeros((R, R), np.uint8)
    for x in range(used):
        if x:
            m[x] = m[rng.integers(max(0, x - 9), x)]
        m[x, x] = 1
    return m


# ---- attention --------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("H,hkv,d", [(4, 2, 64), (5, 1, 128), (8, 1, 128), (7, 1, 64), (12, 1, 128), (16, 2, 64), (3, 3, 128)])
def test_single_tokens(fmt, H, hkv, d):
    c = Case([0, 1, 15, 16, 17, 63, 64, 65, 130, 257], 16, fmt, hkv, d, seed=H)
    q, kn, vn = c.bf16(10, 1, H, d, scale=2.0), c.bf16(10, 1, hkv, d), c.bf16(10, 1, hkv, d)
    got = attend(c, 0, q.to(DEV), kn.to(DEV), vn.to(DEV), 257)
    check(c, 0, got, q, kn, vn)


@pytest.mark.parametrize("pt", [16, 32, 64, 128])
@pytest.mark.parametrize("R,H,hkv,d,fmt", [(2, 8, 2, 64, "int8"), (3, 5, 1, 128, "e4m3"), (8, 5, 1, 128, "int8"), (8, 8, 1, 64, "e4m3"),
                                           (25, 6, 1, 128, "e4m3"), (33, 8, 2, 64, "int8")])
def test_causal_rows_over_ragged_sequences(pt, R, H, hkv, d, fmt):
    c = Case([0, 1, pt - 1, pt, pt + 1, 100, 301], pt, fmt, hkv, d, seed=R + pt)
    q, kn, vn = c.bf16(7, R, H, d), c.bf16(7, R, hkv, d, scale=3.0), c.bf16(7, R, hkv, d)
    n_rows = [R, R, 1, R - 1, 0, R, R]
    got = attend(c, 0, q.to(DEV), kn.to(DEV), vn.to(DEV), 320 if pt == 128 else 301, n_rows=torch.tensor(n_rows, dtype=torch.int32, device=DEV))
    check(c, 0, got, q, kn, vn, n_rows=n_rows)


@pytest.mark.parametrize("R,H,hkv,d,pt,fmt", [(60, 5, 1, 128, 64, "e4m3"), (60, 4, 2, 64, 16, "int8"), (16, 2, 2, 64, 32, "e4m3"), (64, 8, 1, 128, 128, "int8"),
                                              (1, 3, 1, 64, 16, "int8")])
def test_trees(R, H, hkv, d, pt, fmt):
    c = Case([333, 0, 64, 190], pt, fmt, hkv, d, seed=R)
    used = [R, max(1, R - 7), R // 2, R]
    mask = np.stack([tree_mask(c.rng, R, u) for u in used])
    mask[3, R // 2] = 0                                     # a row in the middle that sees only the cache
    if R > 2:
        mask[1, 1] = 0                                      # no cache either: an empty row
    q, kn, vn = c.bf16(4, R, H, d), c.bf16(4, R, hkv, d), c.bf16(4, R, hkv, d)
    dm = torch.from_numpy(mask).to(DEV)
    got = attend(c, 0, q.to(DEV), kn.to(DEV), vn.to(DEV), 333, mask=dm)          # unused slots: empty mask rows, cache visible
    check(c, 0, got, q, kn, vn, mask=mask)
    got = attend(c, 0, q.to(DEV), kn.to(DEV), vn.to(DEV), 333, mask=dm, n_rows=torch.tensor(used, dtype=torch.int32, device=DEV))
    check(c, 0, got, q, kn, vn, mask=mask, n_rows=used)
    if R > 2:
        assert bool((got[1, 1] == 0).all())


@pytest.mark.parametrize("R,H,hkv,d,pt,fmt", [(130, 4, 1, 128, 32, "e4m3"), (257, 7, 1, 64, 16, "int8"), (65, 8, 2, 128, 64, "int8")])
def test_prompt_chunks(R, H, hkv, d, pt, fmt):
    c = Case([0, 77, 200], pt, fmt, hkv, d, seed=R)
    q, kn, vn = c.bf16(3, R, H, d), c.bf16(3, R, hkv, d), c.bf16(3, R, hkv, d)
    n_rows = [R, R - 66 if R > 66 else 3, R]
    got = attend(c, 0, q.to(DEV), kn.to(DEV), vn.to(DEV), 200, n_rows=torch.tensor(n_rows, dtype=torch.int32, device=DEV))
    check(c, 0, got, q, kn, vn, n_rows=n_rows, only=[0, 1, 31, 63, 64, R // 2, R - 2, R - 1])


@pytest.mark.parametrize("R,H,hkv,pt,fmt", [(1, 5, 1, 64, "e4m3"), (1, 8, 1, 16, "int8"), (4, 5, 1, 128, "int8"), (60, 5, 1, 64, "e4m3")])
def test_long_sequences_are_split_and_joined(R, H, hkv, pt, fmt):
    c = Case([20011, 3], pt, fmt, hkv, 128, seed=7)
    q, kn, vn = c.bf16(2, R, H, 128), c.bf16(2, R, hkv, 128), c.bf16(2, R, hkv, 128)
    for max_len in (20011, -(-20011 // pt) * pt):
        got = attend(c, 0, q.to(DEV), kn.to(DEV), vn.to(DEV), max_len)
        check(c, 0, got, q, kn, vn, only=[0, R - 1])


@pytest.mark.parametrize("R", [1, 3, 60])
def test_rows_that_read_the_cache_alone(R):
    c = Case([50, 0, 129], 32, "e4m3", 2, 128, seed=8)
    q = c.bf16(3, R, 10, 128)
    got = attend(c, 0, q.to(DEV), None, None, 129)
    check(c, 0, got, q, None, None)
    assert bool((got[1] == 0).all())


@pytest.mark.parametrize("R", [1, 5, 60])
def test_layers_slots_and_slices_of_a_qkv_matrix(R):
    c = Case([40, 0, 90, 17], 16, "int8", 2, 64, layers=3, seed=9)
    H, d, B = 8, 64, 5
    slots = [2, 0, 2, 3, 1]                                 # a sequence may be read twice
    qkv = c.bf16(B, R, (H + 4) * d + 8).to(DEV)             # a padded row stride, offsets of 16 bytes
    q = qkv[..., :H * d].view(B, R, H, d)
    kn, vn = (qkv[..., (H + 2 * i) * d:(H + 2 * i + 2) * d].view(B, R, 2, d) for i in (0, 1))
    ds = torch.tensor(slots, dtype=torch.int32, device=DEV)
    for layer in (0, 2):
        got = attend(c, layer, q, kn, vn, 90, slots=ds)
        check(c, layer, got, q, kn, vn, slots=slots)


@pytest.mark.parametrize("R", [1, 2, 40])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_what_is_hidden_stays_hidden(R, fmt):
    """NaN and infinities behind a sequence's end, in rows that do not exist, and in rows that a row does not see."""
    c = Case([70, 16, 5], 16, fmt, 1, 64, seed=10)
    H = 6
    q, kn, vn = c.bf16(3, R, H, 64), c.bf16(3, R, 1, 64), c.bf16(3, R, 1, 64)
    clean = attend(c, 0, q.to(DEV), kn.to(DEV), vn.to(DEV), 70)
    if fmt == "e4m3":                                       # the codes behind the lengths
        for i in range(3):
            off = c.lens[i] % 16
            if off:
                for t in c.t[:2]:
                    t.view(torch.uint8)[:, c.pages[i][-1], :, off:] = 0x7F
        torch.testing.assert_close(attend(c, 0, q.to(DEV), kn.to(DEV), vn.to(DEV), 70), clean, rtol=0, atol=0)
    n_rows = torch.tensor([R, 0, max(1, R - 1)], dtype=torch.int32, device=DEV)
    want = attend(c, 0, q.to(DEV), kn.to(DEV), vn.to(DEV), 70, n_rows=n_rows)
    bad_k, bad_v = kn.clone(), vn.clone()
    for t in (bad_k, bad_v):
        t[1], t[2, max(1, R - 1):] = float("nan"), float("inf")
    torch.testing.assert_close(attend(c, 0, q.to(DEV), bad_k.to(DEV), bad_v.to(DEV), 70, n_rows=n_rows), want, rtol=0, atol=0)
    if R > 2:                                               # the last row is seen by itself alone
        bad_k, bad_v, bad_q = kn.clone(), vn.clone(), q.clone()
        bad_k[:, -1], bad_v[:, -1, :, 5], bad_v[:, -1, :, 9] = float("inf"), float("-inf"), float("nan")
        got = attend(c, 0, q.to(DEV), kn.to(DEV), bad_v.to(DEV), 70)
        torch.testing.assert_close(got[:, :-1], clean[:, :-1], rtol=0, atol=0)
        assert bool((got[:, -1, :, 5] == -math.inf).all()) and bool(got[:, -1, :, 9].isnan().all())
        torch.testing.assert_close(got[:, -1, :, 10:], clean[:, -1, :, 10:], rtol=0, atol=0)
        got = attend(c, 0, q.to(DEV), bad_k.to(DEV), vn.to(DEV), 70)
        torch.testing.assert_close(got[:, :-1], clean[:, :-1], rtol=0, atol=0)
        bad_q[:, 1] = float("nan")
        got = attend(c, 0, bad_q.to(DEV), kn.to(DEV), vn.to(DEV), 70)
        keep = [x for x in range(R) if x != 1]
        torch.testing.assert_close(got[:, keep], clean[:, keep], rtol=0, atol=0)
        assert bool(got[:, 1].isnan().all())


@pytest.mark.parametrize("R", [1, 4, 40])
def test_scales_and_magnitudes_far_apart(R):
    c = Case([300, 33], 16, "e4m3", 1, 128, seed=11, scale_exp=(-40, -4))
    for big in (2.0 ** -30, 1.0, 2.0 ** 30):
        q, kn, vn = c.bf16(2, R, 4, 128, scale=1.0), c.bf16(2, R, 1, 128), c.bf16(2, R, 1, 128, scale=big)
        q[:, :, 1] *= 2.0 ** -40                            # a flat softmax
        q[:, :, 2] *= 20.0                                  # a sharp one
        kn[:, 0] = 0
        vn[:, 0] = 0
        got = attend(c, 0, q.to(DEV), kn.to(DEV), vn.to(DEV), 300)
        check(c, 0, got, q, kn, vn)


@pytest.mark.parametrize("R", [1, 40])
def test_bad_lengths_slots_counts_and_pages_are_reported(R):
    c = Case([40, 90], 16, "e4m3", 2, 64, seed=12)
    q, kn, vn = (c.bf16(2, R, h, 64).to(DEV) for h in (4, 2, 2))
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    good = attend(c, 0, q, kn, vn, 90)
    for kw in (dict(seq_lens=i32(-1, 90)), dict(seq_lens=i32(91, 90)), dict(slots=i32(2, 1)), dict(slots=i32(-1, 1)), dict(n_rows=i32(-1, R)),
               dict(n_rows=i32(R + 1, R))):
        got = attend(c, 0, q, kn, vn, 90, status_want=b.DART_ERR_INVALID_ARG, **kw)
        assert bool((got[0] == 0).all())
        torch.testing.assert_close(got[1], good[1], rtol=0, atol=0)
    for page in (-1, c.cache.n_pages, 1 << 30):
        table = c.table.clone()
        table[0, 1] = page
        got = attend(c, 0, q, kn, vn, 90, status_want=b.DART_ERR_INVALID_ARG, table=table)
        torch.testing.assert_close(got[1], good[1], rtol=0, atol=0)
    table = c.table.clone()
    table[0, 3:] = 1 << 30                                  # columns behind the length are not read
    torch.testing.assert_close(attend(c, 0, q, kn, vn, 90, table=table), good, rtol=0, atol=0)


@pytest.mark.parametrize("R,H,hkv,big", [(400, 1, 1, 1.0), (400, 2, 2, 25.0), (300, 3, 1, 0.01)])
def test_prompt_chunks_whose_new_rows_dominate(R, H, hkv, big):
    """Key steps of new rows that whole tiles see, with scores that grow along the chunk (the reference maximum moves in
    the middle of it) and with a cache of a few keys or none."""
    c = Case([0, 3, 140], 16, "e4m3", hkv, 128, seed=R)
    q, kn, vn = c.bf16(3, R, H, 128), c.bf16(3, R, hkv, 128), c.bf16(3, R, hkv, 128)
    kn *= torch.linspace(0.1, big, R).view(1, R, 1, 1)
    vn *= torch.exp2(torch.randint(-6, 7, (1, R, 1, 1)).float())
    got = attend(c, 0, q.to(DEV), kn.to(DEV), vn.to(DEV), 140)
    check(c, 0, got, q, kn, vn, only=[0, 1, 63, 64, 127, 128, 129, 191, 192, 255, 256, 257, R - 1])


@pytest.mark.parametrize("B,R,H,hkv,d,lens", [(3, 1, 128, 1, 128, [70, 0, 300]), (2, 1, 256, 2, 64, [33, 500]), (1, 4096, 1, 1, 64, [100]),
                                              (1024, 1, 4, 2, 64, [i % 37 for i in range(1024)]), (2, 1, 256, 256, 64, [20, 40])])
def test_the_largest_shapes(B, R, H, hkv, d, lens):
    c = Case(lens, 16, "e4m3", hkv, d, seed=B + R)
    q, kn, vn = c.bf16(B, R, H, d), c.bf16(B, R, hkv, d), c.bf16(B, R, hkv, d)
    got = attend(c, 0, q.to(DEV), kn.to(DEV), vn.to(DEV), max(lens))
    check(c, 0, got, q, kn, vn, only=[0, 1, 127, 128, R // 2 + 3, R - 1] if R > 1 else None)


@pytest.mark.parametrize("R,H,hkv,d,fmt", [(17, 1, 1, 128, "e4m3"), (24, 1, 1, 128, "int8"), (20, 2, 2, 128, "e4m3"), (4, 5, 1, 128, "e4m3"),
                                           (3, 8, 1, 128, "int8"), (2, 24, 2, 64, "e4m3"), (6, 4, 1, 64, "int8"), (8, 4, 1, 64, "e4m3"),
                                           (17, 1, 1, 64, "int8"), (32, 1, 1, 64, "e4m3"), (31, 2, 2, 64, "int8"), (25, 1, 1, 128, "e4m3"),
                                           (33, 1, 1, 64, "int8")])
def test_seventeen_to_thirty_two_rows(R, H, hkv, d, fmt):
    """More new rows than one group of 16, three and four tiles of 8 rows, and the first sizes beyond them."""
    c = Case([301, 0, 16, 33, 5003], 16, fmt, hkv, d, seed=R + H + d)
    q, kn, vn = c.bf16(5, R, H, d), c.bf16(5, R, hkv, d, scale=2.0), c.bf16(5, R, hkv, d)
    n_rows = [R, R, max(1, R - 3), min(R, 16), R]
    dn = torch.tensor(n_rows, dtype=torch.int32, device=DEV)
    got = attend(c, 0, q.to(DEV), kn.to(DEV), vn.to(DEV), 5003, n_rows=dn)
    check(c, 0, got, q, kn, vn, n_rows=n_rows)
    mask = np.stack([tree_mask(c.rng, R, u) for u in n_rows])
    mask[1, R - 1] = 0                                      # an empty row
    want = attend(c, 0, q.to(DEV), kn.to(DEV), vn.to(DEV), 5003, n_rows=dn, mask=torch.from_numpy(mask).to(DEV))
    check(c, 0, want, q, kn, vn, n_rows=n_rows, mask=mask)
    assert bool((want[1, R - 1] == 0).all())
    bad_k, bad_v = kn.clone(), vn.clone()                   # what does not exist or is not seen may hold anything
    for t in (bad_k, bad_v):
        for x, n in enumerate(n_rows):
            t[x, n:] = float("nan")
        t[1, R - 1] = float("inf")
    mask[1, R - 1, :] = 0
    mask[1, :, R - 1] = 0
    got = attend(c, 0, q.to(DEV), bad_k.to(DEV), bad_v.to(DEV), 5003, n_rows=dn, mask=torch.from_numpy(mask).to(DEV))
    torch.testing.assert_close(got, want, rtol=0, atol=0)


def test_a_first_call_may_be_captured():
    """A process whose first attention calls (both kernels) lie inside a graph capture."""
    code = """
import sys; sys.path.insert(0, {root!r})
import torch
from paper_2601_19278_b200 import binding as b
dev = "cuda:0"
k, v = (torch.randint(-99, 99, (1, 9, 2, 16, 64), device=dev).to(torch.int8) for _ in range(2))
s = torch.full((1, 9, 2), 2.0 ** -6, device=dev)
c = b.Kv8Cache(k, v, s, s.clone())
table, lens = torch.arange(8, dtype=torch.int32, device=dev).view(1, 8), torch.tensor([100], dtype=torch.int32, device=dev)
calls = []
for R in (1, 20, 200):
    q, kn, vn = (torch.randn(1, R, h, 64, device=dev).bfloat16() for h in (4, 2, 2))
    out, ws = torch.zeros_like(q), torch.empty(b.kv8_attention_workspace_bytes(c, 1, R, 4, 128), dtype=torch.uint8, device=dev)
    calls.append((q, kn, vn, out, ws))
run = lambda outs: [b.kv8_attention(c, 0, q, kn, vn, lens, table, o, max_len=128, workspace=ws) for (q, kn, vn, _, ws), o in zip(calls, outs)]
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    run([x[3] for x in calls])
g.replay()
eager = [torch.zeros_like(x[3]) for x in calls]
run(eager)
torch.cuda.synchronize()
assert all(torch.equal(a, x[3]) and bool(a.any()) for a, x in zip(eager, calls))
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code.format(root=root)], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout[-2000:]


def test_append_takes_the_first_rows_without_counts():
    c = Case([3, 0], 16, "int8", 1, 64, seed=41, room=8)
    kn, vn = c.bf16(1, 2, 5, 1, 64), c.bf16(1, 2, 5, 1, 64)
    b.kv8_append(c.cache, 0, kn.to(DEV), vn.to(DEV), c.seq_lens, c.table, max_append=2)
    for i in range(2):
        c.pool.append(0, c.pages[i], c.lens[i], kn[0, i, :2].double().numpy(), vn[0, i, :2].double().numpy())
    same_pool(c)


def test_pools_past_four_gigabytes():
    """Pages whose bytes lie beyond 32-bit offsets: append into them, read them back by attention on both kernels, copy them."""
    hkv, pt, d, n_pages = 8, 64, 128, 75000                       # 4.9 GB each of K and V
    k, v = (torch.empty(1, n_pages, hkv, pt, d, dtype=torch.int8, device=DEV) for _ in range(2))
    ks, vs = (torch.full((1, n_pages, hkv), float("nan"), device=DEV) for _ in range(2))
    cache = b.Kv8Cache(k, v, ks, vs)
    rng = np.random.default_rng(0)
    ref = torch.ones(n_pages, dtype=torch.int32, device=DEV)      # everything taken but the last pages
    ref[-6:] = 0
    table = torch.full((2, 4), -1, dtype=torch.int32, device=DEV)
    lens = torch.zeros(2, dtype=torch.int32, device=DEV)
    pages = b.Kv8Pages(table, lens, ref, pt)
    ws = torch.empty(b.kv8_pages_workspace_bytes(pages), dtype=torch.uint8, device=DEV)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    status = i32(0)
    b.kv8_reserve(pages, cache, i32(0), i32(150), workspace=ws, status=status)
    assert table[0, :3].tolist() == [n_pages - 6, n_pages - 5, n_pages - 4]
    rows = [torch.from_numpy(rng.standard_normal((1, 1, 150, hkv, d)).astype(np.float32)).to(torch.bfloat16) for _ in range(2)]
    b.kv8_append(cache, 0, rows[0].to(DEV), rows[1].to(DEV), lens, table, slots=i32(0), status=status)
    lens[0] = 150
    b.kv8_fork(pages, i32(0), i32(1), status=status)
    b.kv8_reserve(pages, cache, i32(1), i32(4), workspace=ws, status=status)           # the last page is copied
    assert table[1].tolist() == [n_pages - 6, n_pages - 5, n_pages - 3, -1] and int(status) == 0
    codes = [np.zeros((1, 4, hkv, pt, d), np.uint8) for _ in range(2)]
    pool = ok.Pool(codes, [np.ones((1, 4, hkv)) for _ in range(2)], "int8")
    pool.append(0, [0, 1, 2], 0, rows[0][0, 0].double().numpy(), rows[1][0, 0].double().numpy())
    for R in (1, 20):
        q, kn, vn = (torch.from_numpy(rng.standard_normal((2, R, h, d)).astype(np.float32)).to(torch.bfloat16) for h in (2 * hkv, hkv, hkv))
        out = torch.empty(2, R, 2 * hkv, d, dtype=torch.bfloat16, device=DEV)
        w = torch.empty(b.kv8_attention_workspace_bytes(cache, 2, R, 2 * hkv, 256), dtype=torch.uint8, device=DEV)
        b.kv8_attention(cache, 0, q.to(DEV), kn.to(DEV), vn.to(DEV), lens, table, out, max_len=256, workspace=w, status=status)
        for i in range(2):
            want, absv, absx = ok.attention(pool, 0, [0, 1, 2], 150, q[i].double().numpy(), kn[i].double().numpy(), vn[i].double().numpy(), None)
            tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -10 + 2.0 ** -18 * absx[..., None]) * absv + 2.0 ** -18
            assert np.all(np.abs(out[i].double().cpu().numpy() - want) <= tol)
    ref[:-6] = 0                                                  # only the two sequences live: they move to the front
    b.kv8_compact(pages, cache, workspace=ws, status=status)
    b.kv8_attention(cache, 0, q.to(DEV), kn.to(DEV), vn.to(DEV), lens, table, out, max_len=256, workspace=w, status=status)
    assert table[0, :3].tolist() == [0, 1, 2] or sorted(table[0, :3].tolist() + [int(table[1, 2])]) == [0, 1, 2, 3]
    assert np.all(np.abs(out[1].double().cpu().numpy() - want) <= tol) and int(status) == 0


def test_other_streams_and_first_calls_inside_a_capture():
    """A call on a stream that is not the current one, and page operations captured and replayed."""
    s = Server(40, 16, 6, 6, seed=31)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    b.kv8_reserve(s.pages, s.cache, s.i32([0, 1]), s.i32([20, 30]), workspace=s.ws, status=s.status, stream=st)
    s.copies(s.book.reserve([0, 1], [20, 30]))
    st.synchronize()
    s.advance([0, 1], [20, 30])
    s.check()
    src, dst, who, more = s.i32([0, 1]), s.i32([2, 3]), s.i32([0, 1, 2, 3]), s.i32([1, 1, 1, 1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.kv8_fork(s.pages, src, dst, status=s.status)
        b.kv8_reserve(s.pages, s.cache, who, more, workspace=s.ws, status=s.status)
        b.kv8_release(s.pages, who[2:], status=s.status)
        b.kv8_compact(s.pages, s.cache, workspace=s.ws, n_live=s.n_live, status=s.status)
    for _ in range(3):
        g.replay()
        s.book.fork([0, 1], [2, 3])
        s.copies(s.book.reserve([0, 1, 2, 3], [1, 1, 1, 1]))
        s.book.release([2, 3])
        s.copies(s.book.compact())
        s.check()


def test_results_repeat_bit_for_bit():
    c = Case([5000, 1200, 77], 64, "e4m3", 2, 128, seed=13)
    for R in (1, 3, 60):
        q, kn, vn = (c.bf16(3, R, h, 128).to(DEV) for h in (10, 2, 2))
        first = attend(c, 0, q, kn, vn, 5000)
        for _ in range(3):
            assert torch.equal(attend(c, 0, q, kn, vn, 5000), first)


@pytest.mark.parametrize("R", [1, 60])
def test_captured_calls_follow_lengths_on_the_device_and_keep_apart(R):
    """Two graphs with a workspace each, replayed on two streams at once, with lengths changed between replays."""
    c = Case([3000, 900], 32, "int8", 2, 64, seed=14)
    calls = []
    for k in range(2):
        q, kn, vn = (c.bf16(2, R, h, 64).to(DEV) for h in (8, 2, 2))
        lens = c.seq_lens.clone()
        out = torch.empty(2, R, 8, 64, dtype=torch.bfloat16, device=DEV)
        ws = torch.empty(b.kv8_attention_workspace_bytes(c.cache, 2, R, 8, 3000), dtype=torch.uint8, device=DEV)
        call = lambda q=q, kn=kn, vn=vn, lens=lens, out=out, ws=ws: b.kv8_attention(c.cache, 0, q, kn, vn, lens, c.table, out, max_len=3000, workspace=ws)  # noqa: E731,E501
        call()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        calls.append((g, q, kn, vn, lens, out, torch.cuda.Stream()))
    for lens_now in ([3000, 900], [1, 0], [2047, 64]):
        for _, _, _, _, lens, _, _ in calls:
            lens.copy_(torch.tensor(lens_now, dtype=torch.int32))
        torch.cuda.synchronize()
        for _ in range(3):
            for g, _, _, _, _, _, st in calls:
                with torch.cuda.stream(st):
                    g.replay()
        torch.cuda.synchronize()
        for _, q, kn, vn, lens, out, _ in calls:
            want = attend(c, 0, q, kn, vn, 3000, seq_lens=lens)
            assert torch.equal(out, want)


def test_the_binding_refuses_wrong_tensors():
    c = Case([40, 90], 16, "e4m3", 2, 64, seed=15)
    q, kn, vn = (c.bf16(2, 3, h, 64).to(DEV) for h in (4, 2, 2))
    out = torch.empty_like(q)
    ws = torch.empty(b.kv8_attention_workspace_bytes(c.cache, 2, 3, 4, 90), dtype=torch.uint8, device=DEV)
    base = dict(cache=c.cache, layer=0, q=q, k_new=kn, v_new=vn, seq_lens=c.seq_lens, page_table=c.table, out=out, max_len=90, workspace=ws)
    b.kv8_attention(**base)
    for kw in (dict(q=q.half()), dict(q=q.cpu()), dict(q=q[0]), dict(q=q.transpose(1, 2)), dict(k_new=kn[:, :2]), dict(k_new=None), dict(v_new=None),
               dict(v_new=vn[:1]), dict(k_new=kn.float()), dict(seq_lens=c.seq_lens.long()), dict(seq_lens=c.seq_lens[:1]), dict(page_table=c.table[0]),
               dict(page_table=c.table.cpu()), dict(out=out.float()), dict(out=out[:1]), dict(workspace=ws.int()), dict(n_rows=c.seq_lens[:1]),
               dict(mask=torch.ones(2, 3, 3, device=DEV)), dict(mask=torch.ones(2, 3, 2, dtype=torch.uint8, device=DEV)),
               dict(slots=c.seq_lens.cpu()), dict(status=c.seq_lens.float())):
        with pytest.raises(ValueError):
            b.kv8_attention(**{**base, **kw})
    for kw in (dict(layer=1), dict(max_len=97), dict(max_len=-1), dict(workspace=ws[:0])):
        with pytest.raises(b.DartError):
            b.kv8_attention(**{**base, **kw})
    new = kn[None]
    b.kv8_append(c.cache, 0, new, vn[None], c.seq_lens * 0, c.table)
    for kw in (dict(k_new=new[0]), dict(v_new=new[:, :1]), dict(k_new=new.half()), dict(n_append=c.seq_lens[:1]),
               dict(row_index=torch.zeros(2, 3, dtype=torch.int64, device=DEV)), dict(row_index=torch.zeros(1, 3, dtype=torch.int32, device=DEV))):
        with pytest.raises(ValueError):
            b.kv8_append(**{**dict(cache=c.cache, first_layer=0, k_new=new, v_new=vn[None], seq_lens=c.seq_lens, page_table=c.table), **kw})
    with pytest.raises(b.DartError):
        b.kv8_append(c.cache, 1, new, vn[None], c.seq_lens, c.table)
    torch.cuda.synchronize()


# ---- append -----------------------------------------------------------------------------------------------------------
def same_pool(c):
    torch.cuda.synchronize()
    for w in (0, 1):
        np.testing.assert_array_equal(c.t[2 + w].cpu().numpy().astype(np.float64), c.pool.scales[w].astype(np.float64))
        got = ok.values(c.t[w].view(torch.uint8).cpu().numpy(), c.fmt)
        np.testing.assert_array_equal(got, ok.values(c.pool.codes[w], c.fmt))       # as values: +0 and -0 are one
    intact(*c.raws)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("pt,d,hkv", [(16, 64, 2), (32, 128, 1), (64, 128, 3), (128, 128, 2), (128, 64, 1)])
def test_append_equals_the_oracle(fmt, pt, d, hkv):
    lens = [0, 1, pt - 1, pt, 3 * pt + 5, 7]
    c = Case(lens, pt, fmt, hkv, d, layers=2, seed=pt, room=2 * pt + 3)
    R = 2 * pt + 3
    counts = [R, 1, 2, pt, 0, R - 1]
    kn, vn = (c.bf16(2, 6, R, hkv, d, scale=s) for s in (1.0, 30.0))
    kn[:, 2] *= 0.01                                        # scales that do not grow
    kn[:, 5, :, :, :3] = 0
    vn[0, 3] = 0                                            # a block of zeros: the smallest scale
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    for layers in ((0, 2), (1, 1)):
        if layers[1] == 1:
            kn, vn = kn[:1] * 3, vn[:1] * 0.25
        b.kv8_append(c.cache, layers[0], kn.to(DEV), vn.to(DEV), c.seq_lens, c.table, n_append=torch.tensor(counts, dtype=torch.int32, device=DEV),
                     status=status)
        for l in range(layers[1]):
            for i, n in enumerate(counts):
                c.pool.append(layers[0] + l, c.pages[i], lens[i], kn[l, i, :n].double().numpy(), vn[l, i, :n].double().numpy())
        same_pool(c)
    assert int(status) == 0


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_append_of_accepted_paths_token_by_token_and_strided(fmt):
    c = Case([13, 30, 0], 16, fmt, 2, 64, layers=3, seed=21, room=40)
    R, A = 20, 5
    big = c.bf16(3, 3, R, 4 * 64 + 16).to(DEV)              # K and V interleaved in one matrix with a padded row
    kn, vn = (big[..., i * 128:(i + 1) * 128].view(3, 3, R, 2, 64) for i in (0, 1))
    index = torch.tensor([[0, 3, 7, 7, 19], [2, 1, 0, 0, 0], [0, 0, 0, 0, 0]], dtype=torch.int32)
    counts = [5, 2, 1]
    for step in range(4):
        b.kv8_append(c.cache, 0, kn, vn, c.seq_lens, c.table, n_append=torch.tensor(counts, dtype=torch.int32, device=DEV), row_index=index.to(DEV),
                     slots=torch.tensor([1, 0, 2], dtype=torch.int32, device=DEV))
        for l in range(3):
            for i, slot in enumerate((1, 0, 2)):
                rows = index[i, :counts[i]].tolist()
                c.pool.append(l, c.pages[slot], c.lens[slot], kn[l, i, rows].double().cpu().numpy(), vn[l, i, rows].double().cpu().numpy())
        same_pool(c)
        for i, slot in enumerate((1, 0, 2)):
            c.lens[slot] += counts[i]
        c.seq_lens.copy_(torch.tensor(c.lens, dtype=torch.int32))
        big.mul_(1.7)                                       # the scales grow


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_append_of_extreme_values(fmt):
    c = Case([0, 3], 16, fmt, 1, 64, seed=22, room=20)
    kn, vn = c.bf16(1, 2, 20, 1, 64), c.bf16(1, 2, 20, 1, 64)
    kn[0, 0, 3, 0, 5], kn[0, 0, 4, 0, 6], kn[0, 0, 17, 0, 7] = float("inf"), float("-inf"), float("nan")
    vn[0, 0, :16] = float("nan")                            # no finite value at all
    vn[0, 1] *= 2.0 ** -100                                 # below the smallest scale
    kn[0, 1] *= 2.0 ** 100
    b.kv8_append(c.cache, 0, kn.to(DEV), vn.to(DEV), c.seq_lens, c.table)
    for i in range(2):
        c.pool.append(0, c.pages[i], c.lens[i], kn[0, i].double().numpy(), vn[0, i].double().numpy())
    same_pool(c)


def test_bad_appends_are_reported_and_touch_nothing():
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    for kw in (dict(seq_lens=i32(-1, 5)), dict(seq_lens=i32(47, 5)), dict(n_append=i32(-1, 2)), dict(n_append=i32(3, 2)), dict(slots=i32(2, 1)),
               dict(slots=i32(-1, 1)), dict(table=(0, -1)), dict(table=(0, 1 << 30))):
        c = Case([5, 5], 16, "e4m3", 1, 64, seed=23, room=40)
        kn, vn = c.bf16(1, 2, 2, 1, 64), c.bf16(1, 2, 2, 1, 64)
        table = c.table.clone()
        if "table" in kw:
            table[0, kw["table"][0]] = kw["table"][1]
        status = i32(0)
        b.kv8_append(c.cache, 0, kn.to(DEV), vn.to(DEV), kw.get("seq_lens", c.seq_lens), table, n_append=kw.get("n_append"), slots=kw.get("slots"),
                     status=status)
        assert int(status) == b.DART_ERR_INVALID_ARG
        n = 2 if "n_append" not in kw else 2
        c.pool.append(0, c.pages[1], 5, kn[0, 1, :n].double().numpy(), vn[0, 1, :n].double().numpy())
        same_pool(c)                                        # entry 1 is written, entry 0 changed nothing
    c = Case([5, 5], 16, "e4m3", 1, 64, seed=24, room=40)   # the same slot twice: the first entry counts
    kn, vn, status = c.bf16(1, 2, 2, 1, 64), c.bf16(1, 2, 2, 1, 64), i32(0)
    b.kv8_append(c.cache, 0, kn.to(DEV), vn.to(DEV), c.seq_lens, c.table, slots=i32(1, 1), status=status)
    c.pool.append(0, c.pages[1], 5, kn[0, 0].double().numpy(), vn[0, 0].double().numpy())
    same_pool(c)
    assert int(status) == b.DART_ERR_INVALID_ARG
    status = i32(0)
    index = i32(0, 2, 0, 0).view(2, 2)                      # a source row that does not exist reads row 0 and is reported
    b.kv8_append(c.cache, 0, kn.to(DEV), vn.to(DEV), c.seq_lens, c.table, row_index=index, status=status)
    torch.cuda.synchronize()
    intact(*c.raws)
    assert int(status) == b.DART_ERR_INVALID_ARG


# ---- page operations --------------------------------------------------------------------------------------------------
class Server:
    """A pool and its bookkeeping on the GPU, next to the oracle's."""

    def __init__(self, n_pages, pt, seqs, cols, fmt="int8", hkv=2, d=64, layers=2, seed=0):
        rng = np.random.default_rng(seed)
        codes = [random_codes(rng, (layers, n_pages, hkv, pt, d), fmt) for _ in range(2)]
        scales = [(2.0 ** rng.integers(-8, -4, (layers, n_pages, hkv))).astype(np.float32) for _ in range(2)]
        self.pool, self.book, self.fmt = ok.Pool(codes, scales, fmt), ok.Book(n_pages, pt, seqs, cols), fmt
        self.raws, self.t = [], []
        for x, dt in ((codes[0], FMT[fmt]), (codes[1], FMT[fmt]), (scales[0], torch.float32), (scales[1], torch.float32)):
            t, raw = guarded(x.shape, dt)
            (t.view(torch.uint8) if x.dtype == np.uint8 else t).copy_(torch.from_numpy(x))
            self.t.append(t)
            self.raws.append(raw)
        self.table, r1 = guarded((seqs, cols), torch.int32, -1)
        self.lens, r2 = guarded((seqs,), torch.int32, 0)
        self.ref, r3 = guarded((n_pages,), torch.int32, 0)
        self.status, r4 = guarded((1,), torch.int32, 0)
        self.n_live, r5 = guarded((1,), torch.int32, -1)
        self.cache, self.pages = b.Kv8Cache(*self.t), b.Kv8Pages(self.table, self.lens, self.ref, pt)
        self.ws, r6 = guarded((b.kv8_pages_workspace_bytes(self.pages),), torch.uint8)
        self.raws += [r1, r2, r3, r4, r5, r6]

    i32 = staticmethod(lambda v: torch.tensor(list(v), dtype=torch.int32, device=DEV))

    def copies(self, pairs):
        for w in (0, 1):
            for x in (self.pool.codes[w], self.pool.scales[w]):
                for s, d in pairs:
                    x[:, d] = x[:, s]

    def fork(self, src, dst):
        b.kv8_fork(self.pages, self.i32(src), self.i32(dst), status=self.status)
        self.book.fork(src, dst)

    def reserve(self, seqs, more):
        b.kv8_reserve(self.pages, self.cache, self.i32(seqs), self.i32(more), workspace=self.ws, status=self.status)
        pairs = self.book.reserve(seqs, more)
        if pairs is None:
            assert int(self.status) == b.DART_ERR_CAPACITY
            self.status.zero_()
            return False
        self.copies(pairs)
        return True

    def release(self, seqs):
        b.kv8_release(self.pages, self.i32(seqs), status=self.status)
        self.book.release(seqs)

    def compact(self):
        b.kv8_compact(self.pages, self.cache, workspace=self.ws, n_live=self.n_live, status=self.status)
        self.copies(self.book.compact())
        assert int(self.n_live) == sum(r > 0 for r in self.book.ref)

    def advance(self, seqs, more):
        for s, n in zip(seqs, more):
            self.book.lens[s] += n
        self.lens.copy_(self.i32(self.book.lens))

    def check(self, contents=True):
        torch.cuda.synchronize()
        assert int(self.status) == 0
        assert self.table.tolist() == self.book.table and self.lens.tolist() == self.book.lens and self.ref.tolist() == self.book.ref
        if contents:
            for w in (0, 1):
                np.testing.assert_array_equal(self.t[w].view(torch.uint8).cpu().numpy(), self.pool.codes[w])
                np.testing.assert_array_equal(self.t[2 + w].cpu().numpy(), self.pool.scales[w])
        intact(*self.raws)


@pytest.mark.parametrize("fmt,pt,hkv,d", [("int8", 16, 2, 64), ("e4m3", 64, 3, 128), ("int8", 128, 1, 128)])
def test_page_operations_equal_a_sequential_program(fmt, pt, hkv, d):
    s, rng = Server(60, pt, 12, 8, fmt, hkv, d, layers=3, seed=pt), np.random.default_rng(pt)
    for _ in range(60):
        used, empty = [i for i in range(12) if s.book.lens[i]], [i for i in range(12) if not s.book.lens[i] and s.book.table[i][0] == -1]
        kind = rng.integers(0, 5)
        if kind == 0 and used and len(empty) >= 2:
            a = int(rng.choice(used))
            s.fork([a, int(rng.choice(used))], empty[:2])
        elif kind in (1, 2):
            group = [int(i) for i in rng.permutation(12)[:rng.integers(1, 9)]]
            more = [int(min(rng.integers(0, 2 * pt), 8 * pt - s.book.lens[i])) for i in group]
            if s.reserve(group, more):
                s.advance(group, more)
        elif kind == 3 and used:
            s.release([int(i) for i in rng.permutation(used)[:2]])
        else:
            s.compact()
        s.check()


def test_a_pool_without_enough_pages_changes_nothing():
    s = Server(10, 16, 4, 8, seed=8)
    assert s.reserve([0, 1], [70, 60])                      # nine pages
    s.advance([0, 1], [70, 60])
    s.fork([0], [2])
    for seqs, more in (([3], [17]), ([0, 2, 3], [1, 1, 1]), ([1, 0], [20, 30])):
        assert not s.reserve(seqs, more)
        s.check()
    assert s.reserve([0, 2], [1, 1])                        # one copy: the last page
    s.check()


def test_a_reserve_of_more_than_two_to_the_31_columns_changes_nothing():
    S, M, P = 1024, (1 << 21) + 8, 32
    i32 = Server.i32
    table, lens, ref = torch.full((S, M), -1, dtype=torch.int32, device=DEV), i32([0] * S), i32([0] * P)
    pages = b.Kv8Pages(table, lens, ref, 16)
    k, v = (torch.zeros(1, P, 1, 16, 64, dtype=torch.int8, device=DEV) for _ in range(2))
    cache = b.Kv8Cache(k, v, torch.ones(1, P, 1, device=DEV), torch.ones(1, P, 1, device=DEV))
    ws, status = torch.empty(b.kv8_pages_workspace_bytes(pages), dtype=torch.uint8, device=DEV), i32([0])
    for n in (M * 16, (1 << 20) * 16):                      # 2^31 + 8192 and 2^30 columns
        status.zero_()
        b.kv8_reserve(pages, cache, i32(range(S)), i32([n] * S), workspace=ws, status=status)
        assert int(status) == b.DART_ERR_CAPACITY
        assert int(table.max()) == -1 and int(table.min()) == -1 and not ref.any() and not lens.any()
    status.zero_()
    b.kv8_reserve(pages, cache, i32(range(S)), i32([16] * P + [0] * (S - P)), workspace=ws, status=status)
    assert int(status) == 0 and table[:P, 0].tolist() == list(range(P)) and ref.tolist() == [1] * P and int(table[P:].max()) == -1


def test_many_sequences_and_pages():
    """More pages than one round of the planning scan, lists longer than a warp, sharers listed and not."""
    s = Server(20000, 16, 700, 40, hkv=1, layers=1, seed=5)
    lens = [int(x) for x in np.random.default_rng(1).integers(1, 300, 350)]
    s.reserve(range(350), lens)
    s.advance(range(350), lens)
    s.check(False)
    s.fork(range(350), range(350, 700))
    s.check(False)
    s.reserve(list(range(700))[::-1], [5] * 700)            # every partly filled page has all its sharers listed
    s.check(False)
    s.release([i for i in range(700) if i % 3])
    s.check(False)
    s.compact()
    s.check()


def test_reserve_keeps_a_shared_page_for_the_last_listed_sharer():
    s = Server(30, 16, 6, 4, seed=6)
    s.reserve([0], [20])
    s.advance([0], [20])
    s.fork([0, 0, 0], [1, 2, 3])
    s.reserve([2, 0], [3, 3])                               # sharers 1 and 3 are not listed: both copy
    s.check()
    s.reserve([3, 1], [3, 3])                               # all sharers listed: the last keeps the page
    s.check()
    s.lens[0], s.book.lens[0] = 2, 2                        # rolled back into the shared first page
    s.reserve([0], [30])
    s.check()


def test_bad_lists_are_reported_and_skipped():
    s = Server(30, 16, 6, 4, seed=7)
    s.reserve([0, 1], [20, 33])
    s.advance([0, 1], [20, 33])
    def reported():
        torch.cuda.synchronize()
        assert int(s.status) == b.DART_ERR_INVALID_ARG
        s.status.zero_()
        s.check()
    i = s.i32
    for src, dst in (([0], [1]), ([0], [0]), ([6], [2]), ([-1], [2]), ([0], [6]), ([0], [-1])):      # in use, itself, out of range
        b.kv8_fork(s.pages, i(src), i(dst), status=s.status)
        reported()
    b.kv8_fork(s.pages, i([0, 1]), i([2, 2]), status=s.status)           # a destination twice: the first pair counts
    s.book.fork([0], [2])
    reported()
    b.kv8_fork(s.pages, i([0, 3]), i([3, 4]), status=s.status)           # a source that is a destination
    s.book.fork([0], [3])
    reported()
    for seqs, more in (([0, 0], [5, 5]), ([0, 6], [5, 5]), ([0, -1], [5, 5]), ([0, 1], [5, 32]), ([0, 1], [5, -1])):
        b.kv8_reserve(s.pages, s.cache, i(seqs), i(more), workspace=s.ws, status=s.status)
        s.copies(s.book.reserve([0], [5]))
        reported()
    b.kv8_release(s.pages, i([1, 1, 7]), status=s.status)
    s.book.release([1])
    reported()
    s.release([5])                                          # an empty slot: nothing to give back
    s.check()
    with pytest.raises(ValueError):
        b.kv8_fork(s.pages, i([0]), i([1, 2]))
    with pytest.raises(ValueError):
        b.kv8_reserve(s.pages, s.cache, i([0]), i([1]).long(), workspace=s.ws)
    with pytest.raises(b.DartError):
        b.kv8_reserve(s.pages, s.cache, i([0]), i([1]), workspace=s.ws[:16])
    with pytest.raises(b.DartError):
        b.kv8_release(s.pages, i([]))


# ---- a run of them together -------------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt,pt", [("e4m3", 16), ("int8", 32)])
def test_speculative_steps_over_the_pool(fmt, pt):
    """Prompts appended, trees verified, accepted paths committed, sequences forked, finished and the pool compacted:
    after every step the attention equals the oracle's over its own pool and bookkeeping."""
    layers, hkv, H, d, R, seqs = 2, 2, 6, 64, 12, 5
    s, rng = Server(60, pt, seqs, 12, fmt, hkv, d, layers, seed=pt), np.random.default_rng(3)
    bf16 = lambda *shape: torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(torch.bfloat16)  # noqa: E731

    def commit(group, kn, vn, index, counts):
        assert s.reserve(group, counts)
        b.kv8_append(s.cache, 0, kn.to(DEV), vn.to(DEV), s.lens, s.table, slots=s.i32(group), n_append=s.i32(counts),
                     row_index=None if index is None else torch.tensor(index, dtype=torch.int32, device=DEV), status=s.status)
        for l in range(layers):
            for i, g in enumerate(group):
                rows = list(range(counts[i])) if index is None else index[i][:counts[i]]
                s.pool.append(l, s.book.table[g], s.book.lens[g], kn[l, i, rows].double().numpy(), vn[l, i, rows].double().numpy())
        s.advance(group, counts)

    prompt = [33, 7, 64]
    commit([0, 1, 2], bf16(layers, 3, 64, hkv, d), bf16(layers, 3, 64, hkv, d), None, prompt)
    for step in range(5):
        group = [i for i in range(seqs) if s.book.lens[i]]
        B = len(group)
        mask = np.stack([tree_mask(rng, R, R - i) for i in range(B)])
        q, kn, vn = bf16(layers, B, R, H, d), bf16(layers, B, R, hkv, d), bf16(layers, B, R, hkv, d)
        for l in range(layers):
            out = torch.empty(B, R, H, d, dtype=torch.bfloat16, device=DEV)
            ws = torch.empty(b.kv8_attention_workspace_bytes(s.cache, B, R, H, 12 * pt), dtype=torch.uint8, device=DEV)
            b.kv8_attention(s.cache, l, q[l].to(DEV), kn[l].to(DEV), vn[l].to(DEV), s.lens, s.table, out, max_len=12 * pt, workspace=ws,
                            slots=s.i32(group), mask=torch.from_numpy(mask).to(DEV), status=s.status)
            torch.cuda.synchronize()
            for i, g in enumerate(group):
                ref, absv, absx = ok.attention(s.pool, l, [p for p in s.book.table[g] if p >= 0], s.book.lens[g], q[l, i].double().numpy(),
                                               kn[l, i].double().numpy(), vn[l, i].double().numpy(), mask[i])
                tol = 2.0 ** -8 * np.abs(ref) + (2.0 ** -10 + 2.0 ** -18 * absx[..., None]) * absv + 2.0 ** -18
                assert np.all(np.abs(out[i].double().cpu().numpy() - ref) <= tol), (step, l, g)
        paths = [[0] + sorted(rng.permutation(np.arange(1, R))[:3].tolist()) for _ in range(B)]
        commit(group, kn, vn, paths, [int(x) for x in rng.integers(1, 5, B)])
        s.check()
        if step == 0:
            s.fork([0, 2], [3, 4])
        if step == 2:
            s.release([0, 1])
            s.compact()
        s.check()
