"""Shapes that take each of the forms in which the many-row attention over the paged 8-bit cache cuts a call, with the plan that
each is there for (compared by the CPU tests, run against the oracle on the GPU)."""
RAGGED16 = [2600, 0, 1, 127, 128, 129, 640, 700, 255, 256, 257, 1023, 1500, 64, 63, 2047]

# name: (rows, heads, kv heads, dim, lengths, max_len, new rows, tree, plan)
CASES = {
    # a pair and a single tile, whole: two-slot rings go round, K and V buffers released by two pipelines
    "pair_and_odd_tile_whole": (60, 40, 8, 128, RAGGED16, 8192, True, True, dict(row_tiles=3, paired=1, max_parts=1)),
    "pair_and_odd_tile_whole_d64": (60, 40, 8, 64, RAGGED16, 8192, True, True, dict(row_tiles=3, paired=1, max_parts=1)),
    "pair_and_odd_tile_cache_alone": (60, 40, 8, 128, RAGGED16, 8192, False, False, dict(row_tiles=3, paired=1, max_parts=1)),
    # the same with the keys split: the single tile takes twice the keys of a pair
    "pair_and_odd_tile_split": (60, 40, 8, 128, [8192, 3001, 4300], 8192, True, True, dict(row_tiles=3, paired=1, max_parts=3)),
    "pairs_split": (100, 40, 8, 128, [6000, 8191, 17, 4225], 8192, True, False, dict(row_tiles=4, paired=1, max_parts=2)),
    # one tile over many steps: three-slot rings, steps alternating between the pipelines, page ids window by window
    "single_tile_whole": (60, 8, 8, 128, [2600] + [100, 0, 33] * 6, 8192, True, True, dict(row_tiles=1, paired=0, max_parts=1)),
    "single_tile_whole_d64": (60, 8, 8, 64, [2999] + [100, 0, 33] * 6, 3008, True, True, dict(row_tiles=1, paired=0, max_parts=1)),
    "single_tiles_split": (60, 40, 8, 128, [4096], 4096, True, True, dict(row_tiles=3, paired=0, max_parts=6)),
    # prompt chunks: cached steps, new rows that all rows of a warp see, the diagonal
    "chunk_in_pairs": (1001, 32, 8, 128, [700, 1500], 4500, True, False, dict(row_tiles=32, paired=1, max_parts=1)),
    "chunk_in_single_tiles": (300, 32, 8, 128, [1700, 900], 4500, True, False, dict(row_tiles=10, paired=0, max_parts=1)),
    "chunk_in_pairs_split": (4096, 1, 1, 64, [2100, 130], 3008, True, False, dict(row_tiles=32, paired=1, max_parts=4)),
    "chunk_pair_and_odd_tile_split": (130, 16, 8, 128, [8000, 50, 2900], 8192, True, False, dict(row_tiles=3, paired=1, max_parts=3)),
}
