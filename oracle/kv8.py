"""The paged 8-bit KV cache, stated plainly in fp64 / Python integers: code values, rounding to codes, append, attention
of new rows, and the page operations as a sequential program.  (The paper leaves the target's cache to its serving
stack; Section 3 and Figure 2 fix what the verification attention computes.)"""
from __future__ import annotations

import math
from typing import List, Optional, Sequence

import numpy as np

E4M3, INT8 = "e4m3", "int8"
QMAX = {E4M3: 448.0, INT8: 127.0}
SCALE_FLOOR = 2.0 ** -64


def e4m3_value(code: int) -> float:
    """Sign, four exponent bits (bias 7), three fraction bits; no infinities, S.1111.111 is NaN."""
    sign = -1.0 if code & 0x80 else 1.0
    e, m = (code >> 3) & 15, code & 7
    if e == 15 and m == 7:
        return math.nan
    return sign * (m / 8.0 * 2.0 ** -6 if e == 0 else (1.0 + m / 8.0) * 2.0 ** (e - 7))


E4M3_TABLE = np.array([e4m3_value(c) for c in range(256)])


def values(codes: np.ndarray, fmt: str) -> np.ndarray:
    """Values of stored bytes (uint8), before the scale."""
    return E4M3_TABLE[codes] if fmt == E4M3 else codes.view(np.int8).astype(np.float64)


def round_to_code(x: np.ndarray, fmt: str) -> np.ndarray:
    """Nearest code as a byte, ties to even, saturating; NaN: e4m3's NaN / integer 0."""
    x = np.asarray(x, dtype=np.float64)
    if fmt == INT8:
        return np.clip(np.rint(np.nan_to_num(x, nan=0.0, posinf=127.0, neginf=-127.0)), -127, 127).astype(np.int8).view(np.uint8)
    mags = E4M3_TABLE[:127]                          # ascending: 0 .. 448
    a = np.minimum(np.abs(x), 448.0)
    hi = np.clip(np.searchsorted(mags, np.nan_to_num(a)), 1, 126)
    lo = hi - 1
    up, down = mags[hi] - a, a - mags[lo]
    pick = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo).astype(np.uint8)
    return np.where(np.isnan(x), np.uint8(0x7F), pick | (np.signbit(x).astype(np.uint8) << 7)).astype(np.uint8)


def block_scale(x: np.ndarray, fmt: str) -> float:
    """Smallest power of two >= 2^-64 that fits the block's largest finite value."""
    x = np.abs(x[np.isfinite(x)])
    biggest = float(x.max()) if x.size else 0.0
    s = SCALE_FLOOR
    while biggest > QMAX[fmt] * s:
        s *= 2.0
    return s


class Pool:
    """Codes [layers, pages, kv heads, page tokens, dim] (uint8) and scales [layers, pages, kv heads], K at 0 and V at 1."""

    def __init__(self, codes: Sequence[np.ndarray], scales: Sequence[np.ndarray], fmt: str):
        self.codes, self.scales, self.fmt = list(codes), list(scales), fmt
        self.pt = self.codes[0].shape[3]

    def read(self, which: int, layer: int, head: int, pages: Sequence[int], length: int) -> np.ndarray:
        d = self.codes[which].shape[4]
        out = [values(self.codes[which][layer, p, head], self.fmt) * float(self.scales[which][layer, p, head]) for p in pages]
        return np.concatenate(out).reshape(-1, d)[:length] if out else np.zeros((0, d))

    def append(self, layer: int, pages: Sequence[int], length: int, k_rows: np.ndarray, v_rows: np.ndarray) -> None:
        """k_rows, v_rows [n, kv heads, dim] to positions length .. length + n - 1 of the sequence with these pages."""
        n = k_rows.shape[0]
        for which, rows in ((0, k_rows), (1, v_rows)):
            codes, scales = self.codes[which], self.scales[which]
            j = 0
            while j < n:
                col, off = (length + j) // self.pt, (length + j) % self.pt
                take = min(n - j, self.pt - off)
                p = pages[col]
                for h in range(rows.shape[1]):
                    block = rows[j:j + take, h].astype(np.float64)
                    s = block_scale(block, self.fmt)
                    if col * self.pt < length:                  # the page already holds rows of the sequence
                        was = float(scales[layer, p, h])
                        s = max(s, was)
                        if s != was:
                            codes[layer, p, h, :off] = round_to_code(values(codes[layer, p, h, :off], self.fmt) * (was / s), self.fmt)
                    codes[layer, p, h, off:off + take] = round_to_code(block / s, self.fmt)
                    scales[layer, p, h] = s
                j += take


def attention(pool: Pool, layer: int, pages: Sequence[int], length: int, q: np.ndarray, k_new: Optional[np.ndarray],
              v_new: Optional[np.ndarray], mask: Optional[np.ndarray], only: Optional[Sequence[int]] = None):
    """Rows q [r, heads, dim] over the cache and the new rows [r, kv heads, dim] (mask [r, r], None: causal).  Returns the
    output and, for tolerances, sum p |v| and the largest sum |q_i k_i| / sqrt(d) among the visible keys.  `only`: the
    rows to compute (the others stay zero)."""
    r, H, d = q.shape
    hkv = pool.codes[0].shape[2]
    out, absv, absx = np.zeros((r, H, d)), np.zeros((r, H, d)), np.zeros((r, H))
    for h in range(hkv):
        k, v = (pool.read(w, layer, h, pages, length) for w in (0, 1))
        for j in range(h * (H // hkv), (h + 1) * (H // hkv)):
            for x in (range(r) if only is None else only):
                ks, vs = k, v
                if k_new is not None:
                    sees = [y for y in range(r) if (mask[x, y] if mask is not None else y <= x)]
                    ks, vs = np.concatenate([k, k_new[sees, h]]), np.concatenate([v, v_new[sees, h]])
                if not len(ks):
                    continue
                s = ks @ q[x, j] / math.sqrt(d)
                p = np.exp(s - s.max())
                p /= p.sum()
                out[x, j], absv[x, j] = p @ vs, p @ np.abs(vs)
                absx[x, j] = (np.abs(ks) @ np.abs(q[x, j])).max() / math.sqrt(d)
    return out, absv, absx


class Book:
    """Page bookkeeping as a sequential program.  Every operation returns the (source, destination) pages it copies."""

    def __init__(self, n_pages: int, page_tokens: int, max_seqs: int, max_pages: int):
        self.pt, self.ref = page_tokens, [0] * n_pages
        self.table: List[List[int]] = [[-1] * max_pages for _ in range(max_seqs)]
        self.lens = [0] * max_seqs

    def fork(self, src: Sequence[int], dst: Sequence[int]) -> None:
        for s, d in zip(src, dst):
            cols = -(-self.lens[s] // self.pt)
            self.table[d][:cols] = self.table[s][:cols]
            self.lens[d] = self.lens[s]
            for p in self.table[d][:cols]:
                self.ref[p] += 1

    def reserve(self, seqs: Sequence[int], n_new: Sequence[int]):
        """None (and nothing changed) if the free pages do not suffice."""
        free = iter([p for p, r in enumerate(self.ref) if r == 0])
        ref, table, copies = list(self.ref), [list(t) for t in self.table], []
        for s, n in zip(seqs, n_new):
            if n == 0:
                continue
            for col in range(self.lens[s] // self.pt, (self.lens[s] + n - 1) // self.pt + 1):
                old = table[s][col]
                if old >= 0 and ref[old] == 1:
                    continue
                page = next(free, None)
                if page is None:
                    return None
                if old >= 0:
                    ref[old] -= 1
                    copies.append((old, page))
                table[s][col], ref[page] = page, 1
        self.ref, self.table = ref, table
        return copies

    def release(self, seqs: Sequence[int]) -> None:
        for s in seqs:
            for col, p in enumerate(self.table[s]):
                if p >= 0:
                    self.ref[p] -= 1
                self.table[s][col] = -1
            self.lens[s] = 0

    def compact(self):
        n_live = sum(r > 0 for r in self.ref)
        src = [p for p, r in enumerate(self.ref) if r > 0 and p >= n_live]
        dst = [p for p, r in enumerate(self.ref) if r == 0 and p < n_live]
        to = dict(zip(src, dst))
        for a, b in zip(src, dst):
            self.ref[b], self.ref[a] = self.ref[a], 0
        self.table = [[to.get(p, p) for p in row] for row in self.table]
        return list(zip(src, dst))
