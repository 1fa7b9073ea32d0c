"""Windowed attention of many rows where a query's size times a key's scale is nothing in fp32: hidden keys have no weight, visible ones equal weights.
Tolerance: test_gpu_kv8's, the arithmetic is the same (the scores are zero or next to it, exactly or rounded)."""
import pytest
import torch

from test_gpu_kv8 import Case
from test_gpu_kv8_window import check, trees, windowed

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("R,H,tree", [(60, 5, True), (45, 2, True), (300, 4, False), (200, 2, False)])
@pytest.mark.parametrize("key_exp,query", [(-100, 0.0), (-64, 2.0 ** -90)])
@pytest.mark.parametrize("window,sinks", [(90, 5), (150, 0)])
def test_zero_and_tiny_queries_over_small_keys(fmt, R, H, tree, key_exp, query, window, sinks):
    """Scales of 2^-100 (the smallest allowed) and 2^-64 (the smallest that an append writes), lengths that end inside a step, windows whose edge lies
    inside one; every third row is an ordinary one, which sees keys where its neighbours see none."""
    lens = [1000, 333, 40]
    c = Case(lens, 16, fmt, 1, 128, seed=R + H)
    c.t[2].fill_(2.0 ** key_exp)
    c.pool.scales[0][:] = 2.0 ** key_exp
    q, kn, vn = c.bf16(3, R, H, 128), c.bf16(3, R, 1, 128, scale=2.0 ** -100), c.bf16(3, R, 1, 128)
    for r in range(R):
        if r % 3:
            q[:, r] = q[:, r] * query
    kw = {}
    if tree:
        mask, pos = trees(c.rng, lens, R, [R] * 3)
        kw = dict(mask=mask, positions=pos)
    got = windowed(c, q, kn, vn, 1000, window, sinks, **kw)
    assert bool(torch.isfinite(got).all())
    check(c, got, q, kn, vn, window, sinks, only=None if tree else [0, 1, 2, 63, 64, 65, 88, 89, 90, 91, 92, 127, 128, R - 2, R - 1], **kw)


@pytest.mark.parametrize("R,H,tree", [(1, 5, False), (60, 5, True), (300, 4, False)])
def test_a_scale_that_is_nan_is_not_taken_for_a_small_one(R, H, tree):
    """Such a page is a fault of the caller's; the rows that see it say so, whatever the number of rows, and the other sequences are unharmed."""
    lens = [1000, 333]
    c = Case(lens, 16, "int8", 1, 128, seed=R)
    q, kn, vn = c.bf16(2, R, H, 128), c.bf16(2, R, 1, 128), c.bf16(2, R, 1, 128)
    kw = {}
    if tree:
        mask, pos = trees(c.rng, lens, R, [R] * 2)
        kw = dict(mask=mask, positions=pos)
    c.t[2][0, c.pages[0][980 // 16]] = float("nan")
    got = windowed(c, q, kn, vn, 1000, 150, 4, **kw)
    sees = R if tree else min(R, 980 // 16 * 16 + 15 - 1000 + 150)      # the page's last position is in the window of so many rows
    assert bool(got[0, :sees].isnan().all()) and bool(got[1].isfinite().all())
