"""Pins of the oracle's paged 8-bit cache: code values and rounding against torch's float8 type, scales by their
definition, attention against torch's SDPA on the dequantised cache, page operations by their invariants."""
import math

import numpy as np
import pytest
import torch

from oracle import kv8 as ok


def test_e4m3_values_are_torchs():
    got = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(ok.E4M3_TABLE, got)


def test_rounding_to_codes_is_torchs():
    g = torch.Generator().manual_seed(1)
    x = torch.cat([torch.randn(20000, generator=g) * 10.0 ** torch.randint(-4, 3, (20000,), generator=g),
                   torch.from_numpy((ok.E4M3_TABLE[:126] + ok.E4M3_TABLE[1:127]) / 2).float()])     # every tie
    x = torch.cat([x, -x]).clamp(-448, 448)
    want = x.to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    got = ok.round_to_code(x.double().numpy(), ok.E4M3)
    np.testing.assert_array_equal(ok.E4M3_TABLE[got], ok.E4M3_TABLE[want])
    i = torch.linspace(-140, 140, 5601).double()
    np.testing.assert_array_equal(ok.round_to_code(i.numpy(), ok.INT8).view(np.int8), i.round().clamp(-127, 127).to(torch.int8).numpy())


def test_non_finite_inputs_have_their_codes():
    x = np.array([np.inf, -np.inf, np.nan])
    np.testing.assert_array_equal(ok.values(ok.round_to_code(x, ok.E4M3), ok.E4M3)[:2], [448, -448])
    assert math.isnan(ok.values(ok.round_to_code(x, ok.E4M3), ok.E4M3)[2])
    np.testing.assert_array_equal(ok.values(ok.round_to_code(x, ok.INT8), ok.INT8), [127, -127, 0])


@pytest.mark.parametrize("fmt", [ok.E4M3, ok.INT8])
def test_block_scale_is_the_smallest_power_of_two_that_fits(fmt):
    rng = np.random.default_rng(2)
    for m in list(rng.uniform(0, 1, 50) * 2.0 ** rng.integers(-30, 30, 50)) + [ok.QMAX[fmt], ok.QMAX[fmt] * 2, 1.0, 0.0]:
        s = ok.block_scale(np.array([m, -m / 3, np.inf, np.nan]), fmt)
        assert m <= ok.QMAX[fmt] * s and (s == ok.SCALE_FLOOR or m > ok.QMAX[fmt] * s / 2)
        assert math.frexp(s)[0] == 0.5


def _pool(fmt, pages=7, hkv=2, pt=16, d=64, seed=3):
    rng = np.random.default_rng(seed)
    codes = [rng.integers(0, 255, (1, pages, hkv, pt, d)).astype(np.uint8) for _ in range(2)]
    for c in codes:
        c[(c & 0x7F) == 0x7F] = 0
    return ok.Pool(codes, [2.0 ** rng.integers(-9, -5, (1, pages, hkv)) for _ in range(2)], fmt)


@pytest.mark.parametrize("fmt", [ok.E4M3, ok.INT8])
def test_attention_is_sdpa_on_the_dequantised_cache(fmt):
    pool, rng = _pool(fmt), np.random.default_rng(4)
    r, H, hkv, d, length, pages = 5, 4, 2, 64, 37, [4, 1, 6]
    q, kn, vn = rng.standard_normal((r, H, d)), rng.standard_normal((r, hkv, d)), rng.standard_normal((r, hkv, d))
    mask = np.tril(rng.integers(0, 2, (r, r)))
    np.fill_diagonal(mask, 1)
    for m in (None, mask):
        out, absv, absx = ok.attention(pool, 0, pages, length, q, kn, vn, m)
        vis = np.concatenate([np.ones((r, length), bool), (np.tril(np.ones((r, r))) if m is None else m).astype(bool)], 1)
        k = np.stack([np.concatenate([pool.read(0, 0, h, pages, length), kn[:, h]]) for h in range(hkv)])
        v = np.stack([np.concatenate([pool.read(1, 0, h, pages, length), vn[:, h]]) for h in range(hkv)])
        t = lambda x: torch.from_numpy(x)  # noqa: E731
        want = torch.nn.functional.scaled_dot_product_attention(t(q).transpose(0, 1), t(k).repeat_interleave(H // hkv, 0),
                                                                t(v).repeat_interleave(H // hkv, 0), attn_mask=t(vis))
        np.testing.assert_allclose(out, want.transpose(0, 1).numpy(), rtol=1e-10, atol=1e-12)
        assert (absv >= np.abs(out) - 1e-12).all() and (absx > 0).all()


def test_append_then_read_is_within_half_a_step():
    rng = np.random.default_rng(5)
    for fmt, half in ((ok.E4M3, 2.0 ** -4), (ok.INT8, None)):
        pool = _pool(fmt)
        rows = [rng.standard_normal((40, 2, 64)) * np.linspace(0.2, 3, 40)[:, None, None] for _ in range(2)]
        pool.append(0, [5, 0, 2], 0, rows[0][:9], rows[1][:9])
        pool.append(0, [5, 0, 2], 9, rows[0][9:], rows[1][9:])       # the first page's scale grows
        for w in (0, 1):
            for h in range(2):
                got = pool.read(w, 0, h, [5, 0, 2], 40)
                s = np.repeat(pool.scales[w][0, [5, 0, 2], h], 16)[:40, None]
                # one rounding each; rows re-rounded to a larger scale have had two
                bound = (2 * half * np.abs(rows[w][:, h]) * 1.07 + s * 2.0 ** -9) if half else 1.01 * s
                assert (np.abs(got - rows[w][:, h]) <= bound).all()


def test_page_operations_keep_their_invariants():
    rng = np.random.default_rng(6)
    book = ok.Book(40, 16, 8, 6)
    pool = {p: None for p in range(40)}                # what a page holds
    want = {}                                          # slot -> what its sequence should hold, per column

    def holds(s):
        return [pool[p] for p in book.table[s][:-(-book.lens[s] // 16)]]

    for step in range(200):
        free_slots = [s for s in range(8) if book.lens[s] == 0 and book.table[s][0] == -1]
        used = [s for s in range(8) if book.lens[s]]
        kind = rng.integers(0, 4)
        if kind == 0 and used and free_slots:
            s, d = int(rng.choice(used)), free_slots[0]
            book.fork([s], [d])
            want[d] = list(want[s])
        elif kind == 1:
            group = [int(s) for s in rng.permutation(8)[:3]]
            more = [int(min(rng.integers(0, 20), 96 - book.lens[s])) for s in group]
            copies = book.reserve(group, more)
            if copies is None:
                continue
            for a, b in copies:
                pool[b] = pool[a]
            for s, n in zip(group, more):              # the sequence writes its own pages
                for t in range(book.lens[s], book.lens[s] + n):
                    pool[book.table[s][t // 16]] = (s, step)
                book.lens[s] += n
                want[s] = want.get(s, [])[:] if book.lens[s] else []
                cols = -(-book.lens[s] // 16)
                first = (book.lens[s] - n) // 16
                if n:
                    want[s] = want[s][:first] + [(s, step)] * (cols - first)
        elif kind == 2 and used:
            s = int(rng.choice(used))
            book.release([s])
            want[s] = []
        else:
            for a, b in book.compact():
                pool[b] = pool[a]
            live = [p for p in range(40) if book.ref[p]]
            assert live == list(range(len(live)))
        counts = [0] * 40
        for row in book.table:
            for p in row:
                if p >= 0:
                    counts[p] += 1
        assert counts == book.ref
        for s in range(8):
            if book.lens[s]:
                assert holds(s) == want[s], (step, s)
