"""The many-row attention over the paged 8-bit cache in each of the forms in which a call is cut, against the oracle at a few rows
of every tile (tolerance: test_gpu_kv8)."""
import numpy as np
import pytest
import torch

from kv8_plan_cases import CASES
from paper_2601_19278_b200 import binding as b
from test_gpu_kv8 import DEV, Case, attend, check, tree_mask

pytestmark = pytest.mark.gpu


PAGES = [(16, "int8"), (128, "e4m3"), (16, "e4m3"), (64, "e4m3"), (128, "int8")]
# the largest shapes at two page sizes
RUNS = [(name, pt, fmt) for name in sorted(CASES) for pt, fmt in (PAGES[:2] if CASES[name][0] > 1000 else PAGES)]


@pytest.mark.parametrize("name,pt,fmt", RUNS)
def test_every_form_equals_the_oracle(name, pt, fmt):
    R, H, hkv, d, lens, max_len, new, tree, want = CASES[name]
    c = Case(lens, pt, fmt, hkv, d, seed=R + pt)
    B, G = len(lens), H // hkv
    plan = b.kv8_attention_plan(c.cache, B, R, H, max_len, new)
    assert {k: plan[k] for k in want} == want
    table = torch.full((B, max(c.cols, -(-max_len // pt))), -1, dtype=torch.int32, device=DEV)      # columns for max_len
    table[:, :c.cols] = c.table
    q, kn, vn = c.bf16(B, R, H, d), c.bf16(B, R, hkv, d), c.bf16(B, R, hkv, d)
    n_rows = [R - (i * 7) % max(1, R // 4) for i in range(B)]
    mask = np.stack([tree_mask(c.rng, R, n) for n in n_rows]) if tree and R <= 64 else None
    on = lambda t: t.to(DEV) if new else None  # noqa: E731
    got = attend(c, 0, q.to(DEV), on(kn), on(vn), max_len, n_rows=torch.tensor(n_rows, dtype=torch.int32, device=DEV), table=table,
                 mask=None if mask is None else torch.from_numpy(mask).to(DEV))
    edges = [128 * t // G + x for t in range(1, 3) for x in (-1, 0)]
    only = sorted({0, R // 2, R - 1 - R // 4} | {x for x in edges if 0 <= x < R})
    check(c, 0, got, q, kn if new else None, vn if new else None, n_rows=n_rows, mask=mask, only=only)
