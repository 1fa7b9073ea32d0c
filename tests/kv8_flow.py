"""One speculative step after another with the target's paged 8-bit cache, on the draft tree that the library itself built: reserve and
append the prompts; attention of the tree's nodes under dart_build_tree's mask and n_nodes; an accepted path out of
dart_tree_verify_inputs' retrieve rows reserved, appended and counted; the next single token.  Every attention is compared with
the oracle over its own pool (tolerance: test_gpu_kv8), every append with its codes and scales."""
import numpy as np
import torch

from oracle import kv8 as ok
from paper_2601_19278_b200 import binding as b


def verify_inputs(ses):
    B, bud, L = ses.w.batch, ses.cfg.tree_budget, ses.w.K
    i32 = lambda *shape: torch.full(shape, -9, dtype=torch.int32, device=ses.dev)  # noqa: E731
    pos, retrieve, leaves = i32(B, bud), i32(B, bud, L + 1), i32(B)
    ses.draft.verify_inputs(batch=B, max_levels=L, parents=ses.parents, depth=ses.depth, n_nodes=ses.n_nodes, root_pos=ses.inp["seq_lens"],
                            position_ids=pos, retrieve=retrieve, n_leaves=leaves)
    return retrieve, leaves


def run(ses, fmt, page_tokens, hkv, heads, dim, prompts, layers=2, steps=2, seed=0):
    """`ses`: a session whose step and tree have run.  Returns the number of comparisons made."""
    dev, B, R = ses.dev, ses.w.batch, ses.cfg.tree_budget
    cols = -(-(max(prompts) + steps * (ses.w.K + 1) + 1) // page_tokens)
    n_pages, rng, compared = B * cols, np.random.default_rng(seed), 0
    dt = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}[fmt]
    k, v = (torch.zeros(layers, n_pages, hkv, page_tokens, dim, dtype=torch.uint8, device=dev).view(dt) for _ in range(2))
    ks, vs = (torch.zeros(layers, n_pages, hkv, device=dev) for _ in range(2))
    table, lens, ref, status = (torch.full(s, x, dtype=torch.int32, device=dev) for s, x in (((B, cols), -1), ((B,), 0), ((n_pages,), 0), ((1,), 0)))
    cache, pages = b.Kv8Cache(k, v, ks, vs), b.Kv8Pages(table, lens, ref, page_tokens)
    pws = torch.empty(b.kv8_pages_workspace_bytes(pages), dtype=torch.uint8, device=dev)
    pool = ok.Pool([np.zeros((layers, n_pages, hkv, page_tokens, dim), np.uint8) for _ in range(2)], [np.zeros((layers, n_pages, hkv)) for _ in range(2)], fmt)
    book = ok.Book(n_pages, page_tokens, B, cols)
    bf16 = lambda *shape: torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(torch.bfloat16)  # noqa: E731
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
    slots = torch.arange(B, dtype=torch.int32, device=dev)

    def commit(kn, vn, counts, index):
        """Reserve, append and advance; nobody looks at the status in between."""
        b.kv8_reserve(pages, cache, slots, counts, workspace=pws, status=status)
        b.kv8_append(cache, 0, kn.to(dev), vn.to(dev), lens, table, slots=slots, n_append=counts, row_index=index, status=status, pages=pages)
        lens.index_add_(0, slots, counts)
        n = counts.tolist()
        assert book.reserve(list(range(B)), n) is not None
        for l in range(layers):
            for i in range(B):
                rows = list(range(n[i])) if index is None else index[i, :n[i]].tolist()
                pool.append(l, book.table[i], book.lens[i], kn[l, i, rows].double().numpy(), vn[l, i, rows].double().numpy())
        book.lens = [x + y for x, y in zip(book.lens, n)]
        assert table.tolist() == book.table and lens.tolist() == book.lens and ref.tolist() == book.ref and int(status) == 0
        for w, (c, s) in enumerate(((k, ks), (v, vs))):
            np.testing.assert_array_equal(s.cpu().numpy().astype(np.float64), pool.scales[w])
            np.testing.assert_array_equal(ok.values(c.view(torch.uint8).cpu().numpy(), fmt), ok.values(pool.codes[w], fmt))

    def attend(rows, mask, n_rows):
        nonlocal compared
        max_len = max(book.lens)                             # a tight bound
        ws = torch.empty(b.kv8_attention_workspace_bytes(cache, B, rows, heads, max_len), dtype=torch.uint8, device=dev)
        kn, vn = bf16(layers, B, rows, hkv, dim), bf16(layers, B, rows, hkv, dim)
        for l in range(layers):
            q, out = bf16(B, rows, heads, dim), torch.empty(B, rows, heads, dim, dtype=torch.bfloat16, device=dev)
            b.kv8_attention(cache, l, q.to(dev), kn[l].to(dev), vn[l].to(dev), lens, table, out, max_len=max_len, workspace=ws, slots=slots,
                            mask=mask, n_rows=n_rows, status=status)
            got = out.double().cpu().numpy()
            for i in range(B):
                n = rows if n_rows is None else int(n_rows[i])
                m = None if mask is None else mask[i, :n, :n].cpu().numpy()
                want, absv, absx = ok.attention(pool, l, [p for p in book.table[i] if p >= 0], book.lens[i], q[i, :n].double().numpy(),
                                                kn[l, i, :n].double().numpy(), vn[l, i, :n].double().numpy(), m)
                tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -10 + 2.0 ** -18 * absx[..., None]) * absv + 2.0 ** -18
                assert np.all(np.abs(got[i, :n] - want) <= tol) and np.all(got[i, n:] == 0)
                compared += want.size
        assert int(status) == 0
        return kn, vn

    commit(bf16(layers, B, max(prompts), hkv, dim), bf16(layers, B, max(prompts), hkv, dim), i32(prompts), None)
    retrieve, leaves = verify_inputs(ses)
    for step in range(steps):
        kn, vn = attend(R, ses.mask, ses.n_nodes)
        pick = [int(rng.integers(0, int(x))) for x in leaves]                       # the target's choice: a leaf's path, cut somewhere
        path = retrieve[torch.arange(B, device=dev), i32(pick).long()].contiguous()
        depth = (path >= 0).sum(1).tolist()
        commit(kn, vn, i32([int(rng.integers(1, x + 1)) for x in depth]), path)     # (-1 behind the counts)
        attend(1, None, None)
    return compared
