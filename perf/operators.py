"""The paged 8-bit KV cache of the target model, measured: attention of new rows over it, the append that quantises rows
into its pages, and the page operations of a server (fork, reserve with copy-on-write, release, compact).

Shapes follow the drafting workloads of this repository (`synthetic.WORKLOADS`): head layouts 4/2 x 64, 32/8, 40/8 and
64/8 x 128, prefixes 128 .. 8192, trees of 60 nodes, batches 1 .. 16, and a decoding batch of 64.
"""
import math

import torch

own = False

E4M3_MAX, INT8_MAX = 448.0, 127.0
SCALE_FLOOR = 2.0 ** -64


# ---------------------------------------------------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------------------------------------------------
def _attn(name, batch, rows, heads, kv_heads, dim, lo, hi, page, fmt, mask):
    return {"name": name, "op": "attention", "batch": batch, "rows": rows, "heads": heads, "kv_heads": kv_heads, "dim": dim, "len_lo": lo,
            "len_hi": hi, "page": page, "fmt": fmt, "mask": mask}


def _app(name, batch, rows, append, layers, kv_heads, dim, lo, hi, page, fmt, tree):
    return {"name": name, "op": "append", "batch": batch, "rows": rows, "append": append, "layers": layers, "kv_heads": kv_heads, "dim": dim,
            "len_lo": lo, "len_hi": hi, "page": page, "fmt": fmt, "tree": tree}


def _pg(name, op, seqs, forks, layers, kv_heads, dim, lo, hi, page, fmt, reserve):
    return {"name": name, "op": op, "seqs": seqs, "forks": forks, "layers": layers, "kv_heads": kv_heads, "dim": dim, "len_lo": lo, "len_hi": hi,
            "page": page, "fmt": fmt, "reserve": reserve}


def listed():
    return [
        # the smallest model of the test suite, one token of one short sequence: the latency of a call
        _attn("decode_smallest", 1, 1, 4, 2, 64, 128, 128, 16, "e4m3", "causal"),
        # a decoding batch of a serving process, one token per sequence, ragged prefixes
        _attn("decode_batch64", 64, 1, 40, 8, 128, 512, 8192, 64, "e4m3", "causal"),
        # one user with a very long context: few rows, a long axis
        _attn("decode_long", 1, 1, 64, 8, 128, 131001, 131001, 128, "int8", "causal"),
        # verification of one draft tree by the 40-head target
        _attn("tree_single", 1, 60, 40, 8, 128, 4096, 4096, 64, "e4m3", "tree"),
        # verification of a batch of trees, ragged prefixes
        _attn("tree_batch16", 16, 60, 40, 8, 128, 512, 8192, 32, "int8", "tree"),
        # a chunk of a prompt over the cached beginning of it (odd length)
        _attn("prompt_chunk", 2, 1001, 32, 8, 128, 3500, 4500, 64, "e4m3", "causal"),
        # one decoded token into the cache of one small layer: the latency of a call
        _app("append_token", 1, 1, 1, 1, 2, 64, 129, 129, 16, "e4m3", False),
        # the accepted paths of a batch of trees, committed for all layers at once
        _app("append_accepted", 16, 60, 9, 16, 8, 128, 100, 1000, 64, "int8", True),
        # prompts of a batch, one layer
        _app("append_prompt", 4, 2047, 2047, 1, 8, 128, 0, 100, 64, "e4m3", False),
        # parallel sampling: every sequence forked, all of them about to write
        _pg("fork_reserve", "fork", 16, 3, 16, 8, 128, 200, 1000, 64, "e4m3", 9),
        # a single fork of a short sequence: the latency of the calls
        _pg("fork_one", "fork", 1, 1, 1, 2, 64, 100, 100, 16, "int8", 1),
        # half the sequences finish; the survivors' pages are moved to the front of the pool
        _pg("release_compact", "compact", 64, 0, 16, 8, 128, 200, 1000, 64, "e4m3", 0),
    ]


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    most = max(_cost(c) for c in listed())
    while True:
        heads, kv_heads, dim = rng.choice([(4, 2, 64), (32, 8, 128), (40, 8, 128), (64, 8, 128), (6, 2, 64), (7, 1, 128)])
        page, fmt = rng.choice([16, 32, 64, 128]), rng.choice(["e4m3", "int8"])
        kind = rng.choice(["decode", "few", "tree", "chunk", "append", "accepted", "fork", "compact"])
        if kind in ("decode", "few", "tree", "chunk"):
            rows = 1 if kind == "decode" else rng.randint(2, 9) if kind == "few" else rng.randint(10, 60) if kind == "tree" else log(65, 1001)
            hi = log(1, 131001 if kind == "decode" else 20000)
            c = _attn("", log(1, 64 if kind in ("decode", "few") else 16), rows, heads, kv_heads, dim, rng.randint(0, hi), hi, page, fmt,
                      "tree" if kind == "tree" else "causal")
            size = c["batch"] * hi * kv_heads * dim * 2 * 5 + c["batch"] * heads * rows * (hi + rows) * 8.0   # the plain form's intermediates
        elif kind in ("append", "accepted"):
            hi = log(1, 1000)
            rows = log(1, 2047) if kind == "append" else rng.randint(2, 60)
            c = _app("", log(1, 16), rows, rows if kind == "append" else min(rows, rng.randint(1, 9)), 1 if kind == "append" else rng.randint(1, 16),
                     kv_heads, dim, rng.randint(0, hi), hi, page, fmt, kind == "accepted")
            size = c["batch"] * c["layers"] * (hi + rows + page) * kv_heads * dim * 20.0
        else:
            hi = log(2, 1000)
            n = log(2, 64)
            c = _pg("", kind, n if kind == "compact" else max(1, n // 4), 0 if kind == "compact" else rng.randint(1, 3), rng.randint(1, 16), kv_heads, dim,
                    rng.randint(1, hi), hi, page, fmt, 0 if kind == "compact" else rng.randint(1, 9))
            size = c["seqs"] * c["layers"] * (hi + page) * kv_heads * dim * 8.0
        del c["name"]
        if _cost(c) <= most and size < 30e9:
            return c


# ---------------------------------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------------------------------
def _lens(case, n):
    """Lengths from len_lo to len_hi, spread evenly, longest first: a case's work does not depend on the seed."""
    lo, hi = case["len_lo"], case["len_hi"]
    return [hi - (hi - lo) * i // max(1, n - 1) if n > 1 else hi for i in range(n)]


def _pages_of(length, page):
    return -(-length // page)


def _codes(shape, fmt, g, dev):
    """Codes as an append leaves them: N(0, 1) values, the page's largest somewhere in the format's upper half."""
    out = torch.empty(shape, dtype=torch.float8_e4m3fn if fmt == "e4m3" else torch.int8, device=dev)
    flat, step = out.view(-1), 1 << 26
    amp = 80.0 if fmt == "e4m3" else 24.0
    for i in range(0, flat.numel(), step):
        x = torch.randn(min(step, flat.numel() - i), generator=g, device=dev) * amp
        if fmt == "e4m3":
            flat[i:i + step] = x.clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
        else:
            flat[i:i + step] = x.round_().clamp_(-INT8_MAX, INT8_MAX).to(torch.int8)
    return out


def _scales(shape, fmt, g, dev):
    e = torch.randint(-1, 2, shape, generator=g, device=dev).float()
    return torch.exp2(e - (7.0 if fmt == "e4m3" else 5.0))


def _tree_parents(n, gen):
    """Parents of a draft tree's slots, parents[x] < x, slot 0 the root."""
    return [-1] + [int(torch.randint(max(0, x - 12), x, (1,), generator=gen)) for x in range(1, n)]


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed * 7 + 1)
    h = torch.Generator().manual_seed(seed * 7 + 2)
    page, fmt, hkv, d = case["page"], case["fmt"], case["kv_heads"], case["dim"]
    s = {"case": case}
    if case["op"] == "attention":
        B, R = case["batch"], case["rows"]
        lens = _lens(case, B)
        cols = max(1, max(_pages_of(n, page) for n in lens))
        total = sum(_pages_of(n, page) for n in lens) + 1
        ids = torch.randperm(total, generator=h).tolist()
        table = torch.full((B, cols), -1, dtype=torch.int32)
        for b, n in enumerate(lens):
            k = _pages_of(n, page)
            table[b, :k] = torch.tensor([ids.pop() for _ in range(k)], dtype=torch.int32)
        s["table"], s["lens"], s["max_len"] = table.to(dev), torch.tensor(lens, dtype=torch.int32, device=dev), max(lens)
        s["k"], s["v"] = (_codes((1, total, hkv, page, d), fmt, g, dev) for _ in range(2))
        s["ks"], s["vs"] = (_scales((1, total, hkv), fmt, g, dev) for _ in range(2))
        bf = lambda *shape: torch.randn(shape, generator=g, device=dev).to(torch.bfloat16)  # noqa: E731
        s["q"], s["k_new"], s["v_new"] = bf(B, R, case["heads"], d), bf(B, R, hkv, d), bf(B, R, hkv, d)
        s["n_rows"] = s["mask"] = None
        if case["mask"] == "tree":      # trees that use most of their slots; the rest has an empty mask row
            mask = torch.zeros(B, R, R, dtype=torch.uint8)
            used = [R - (i * 3) % max(1, R // 6) for i in range(B)]
            for b in range(B):
                for x, p in enumerate(_tree_parents(used[b], h)):
                    if p >= 0:
                        mask[b, x] = mask[b, p]
                    mask[b, x, x] = 1
            s["mask"], s["n_rows"] = mask.to(dev), torch.tensor(used, dtype=torch.int32, device=dev)
        s["out"] = torch.empty_like(s["q"])
        return s
    if case["op"] == "append":
        B, R, L, A = case["batch"], case["rows"], case["layers"], case["append"]
        lens = _lens(case, B)
        cnt = [max(1, A - (i * 5) % max(1, A)) for i in range(B)]      # ragged, the first sequence has the most
        need = [_pages_of(n + c, page) for n, c in zip(lens, cnt)]
        total, cols = sum(need), max(need)
        ids = torch.randperm(total, generator=h).tolist()
        table = torch.full((B, cols), -1, dtype=torch.int32)
        for b in range(B):
            table[b, :need[b]] = torch.tensor([ids.pop() for _ in range(need[b])], dtype=torch.int32)
        s["table"], s["lens"], s["cnt"] = table.to(dev), torch.tensor(lens, dtype=torch.int32, device=dev), torch.tensor(cnt, dtype=torch.int32, device=dev)
        s["k"], s["v"] = (_codes((L, total, hkv, page, d), fmt, g, dev) for _ in range(2))
        s["ks"], s["vs"] = (_scales((L, total, hkv), fmt, g, dev) for _ in range(2))
        s["k_new"], s["v_new"] = (torch.randn(L, B, R, hkv, d, generator=g, device=dev).to(torch.bfloat16) for _ in range(2))
        s["index"] = None
        if case["tree"]:                # an accepted path: ascending slots from the root on
            index = torch.zeros(B, A, dtype=torch.int32)
            for b in range(B):
                path = sorted((torch.randperm(R - 1, generator=h)[:A - 1] + 1).tolist()) if A > 1 else []
                index[b, :len(path) + 1] = torch.tensor([0] + path, dtype=torch.int32)
            s["index"] = index.to(dev)
        return s
    # page operations: `book` holds table, lengths and reference counts in one buffer, restored at the start of a pass
    N, F, L = case["seqs"], case["forks"], case["layers"]
    lens = _lens(case, N)
    slots = N * (1 + F)
    cols = _pages_of(max(lens) + case["reserve"], page)
    live = sum(_pages_of(n, page) for n in lens)
    total = live + slots * (1 + _pages_of(case["reserve"], page))
    ids = torch.randperm(total, generator=h).tolist()
    book = torch.zeros(slots * cols + slots + total, dtype=torch.int32)
    book[:slots * cols] = -1
    table, ref = book[:slots * cols].view(slots, cols), book[slots * cols + slots:]
    for b, n in enumerate(lens):
        for j in range(_pages_of(n, page)):
            table[b, j] = ids.pop()
            ref[int(table[b, j])] = 1
        book[slots * cols + b] = n
    s["pristine"], s["book"] = book.to(dev), book.to(dev)
    s["table"] = s["book"][:slots * cols].view(slots, cols)
    s["seq_lens"], s["ref"] = s["book"][slots * cols:slots * cols + slots], s["book"][slots * cols + slots:]
    s["k"], s["v"] = (_codes((L, total, hkv, page, d), fmt, g, dev) for _ in range(2))
    s["ks"], s["vs"] = (_scales((L, total, hkv), fmt, g, dev) for _ in range(2))
    as_dev = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    if case["op"] == "fork":
        s["src"], s["dst"] = as_dev([i % N for i in range(N * F)]), as_dev([N + i for i in range(N * F)])
        s["who"], s["more"] = as_dev(list(range(slots))), as_dev([case["reserve"]] * slots)
    else:
        order = torch.randperm(N, generator=h).tolist()
        s["gone"] = as_dev(sorted(order[:max(1, N // 2)]))
    return s


# ---------------------------------------------------------------------------------------------------------------------
# The plain forms
# ---------------------------------------------------------------------------------------------------------------------
def _take(codes, *at):
    """Codes of some pages, as float32 (indexing goes through bytes: it copies 8-bit floats unread)."""
    return codes.view(torch.uint8)[at].view(codes.dtype).float()


def _plain_attention(s):
    c = s["case"]
    B, R, H, hkv, d, page = c["batch"], c["rows"], c["heads"], c["kv_heads"], c["dim"], c["page"]
    table = s["table"].clamp(min=0).long()
    S = table.shape[1] * page

    def cached(codes, scales):
        x = _take(codes[0], table) * scales[0][table][..., None, None]        # [B, cols, hkv, page, d]
        return x.permute(0, 2, 1, 3, 4).reshape(B, hkv, S, d)

    n_rows = s["n_rows"] if s["n_rows"] is not None else torch.full_like(s["lens"], R)
    at, row = torch.arange(S, device=table.device), torch.arange(R, device=table.device)
    in_cache = at[None] < s["lens"][:, None]                                    # [B, S]
    is_row = row[None] < n_rows[:, None]                                        # [B, R]
    among = s["mask"].bool() if s["mask"] is not None else (row[None, :] <= row[:, None])[None].expand(B, R, R)
    among = among & is_row[:, None, :] & is_row[:, :, None]
    see = torch.cat([(in_cache[:, None, :] & is_row[:, :, None]), among], 2)[:, None, None]      # [B, 1, 1, R, S + R]
    k = torch.cat([cached(s["k"], s["ks"]), s["k_new"].float().permute(0, 2, 1, 3)], 2)
    v = torch.cat([cached(s["v"], s["vs"]), s["v_new"].float().permute(0, 2, 1, 3)], 2)
    q = s["q"].float().view(B, R, hkv, H // hkv, d).permute(0, 2, 3, 1, 4).reshape(B, hkv, H // hkv * R, d)
    x = (q @ k.transpose(2, 3)).view(B, hkv, H // hkv, R, S + R) * (1.0 / math.sqrt(d))
    x = torch.where(see, x, -math.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1)                                                           # [B, hkv, G, R]
    o = (p.view(B, hkv, H // hkv * R, S + R) @ v).view(B, hkv, H // hkv, R, d)
    o = torch.where(total[..., None] > 0, o / total[..., None], 0.0)
    return o.permute(0, 3, 1, 2, 4).reshape(B, R, H, d).to(torch.bfloat16)


def _pow2_scale(biggest, fmt):
    """The smallest power of two >= SCALE_FLOOR with biggest <= qmax * scale."""
    f, e = torch.frexp(biggest)
    top, shift = (0.875, 9) if fmt == "e4m3" else (0.9921875, 7)
    sc = torch.ldexp(torch.ones_like(biggest), e - shift + (f > top).to(e.dtype))
    return torch.where(biggest > 0, sc, 0.0).clamp(min=SCALE_FLOOR)


def _quantise(x, fmt):
    if fmt == "e4m3":
        return x.clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    return x.round().clamp(-INT8_MAX, INT8_MAX).to(torch.int8)


def _plain_append(s):
    c = s["case"]
    B, page, fmt, A = c["batch"], c["page"], c["fmt"], c["append"]
    dev = s["table"].device
    W = (A + page - 2) // page + 1                          # pages that A rows can touch
    lens, cnt = s["lens"].long(), s["cnt"].long()
    col = lens[:, None] // page + torch.arange(W, device=dev)                   # [B, W]
    touched = (col * page < (lens + cnt)[:, None]).view(-1).nonzero()[:, 0]
    b = touched // W
    first = col.view(-1)[touched] * page                                        # position of the page's first token
    pages = s["table"][b, col.view(-1)[touched]].long()                         # [T]
    at = first[:, None] + torch.arange(page, device=dev)                        # [T, page]
    j = at - lens[b][:, None]
    is_new, is_old = (j >= 0) & (j < cnt[b][:, None]), j < 0
    j = j.clamp(0, A - 1)
    rows = s["index"].long()[b[:, None], j] if s["index"] is not None else j
    for new, codes, scales in ((s["k_new"], s["k"], s["ks"]), (s["v_new"], s["v"], s["vs"])):
        x = new[:, b[:, None], rows].float().transpose(2, 3)                    # [L, T, hkv, page, d]
        here = is_new[None, :, None, :, None]
        biggest = torch.where(here, x.abs(), 0.0).amax((-1, -2))                # [L, T, hkv]
        was = torch.where((first < lens[b])[None, :, None], scales[:, pages], 0.0)
        sc = torch.maximum(_pow2_scale(biggest, fmt), was)
        now = _take(codes, slice(None), pages)
        old = _quantise(now * (was / sc)[..., None, None], fmt).float()
        got = torch.where(here, _quantise(x / sc[..., None, None], fmt).float(), torch.where(is_old[None, :, None, :, None], old, now))
        codes.view(torch.uint8)[:, pages] = _quantise(got, fmt).view(torch.uint8)
        scales[:, pages] = sc
    return {"k": s["k"], "v": s["v"], "k_scale": s["ks"], "v_scale": s["vs"]}


def _copy_pages(s, src, dst):
    for x in (s["k"].view(torch.uint8), s["v"].view(torch.uint8), s["ks"], s["vs"]):
        x[:, dst] = x[:, src]


def _plain_fork(s):
    page = s["case"]["page"]
    table, lens, ref = s["table"], s["seq_lens"], s["ref"]
    src, dst, who, more = (s[n].long() for n in ("src", "dst", "who", "more"))
    col = torch.arange(table.shape[1], device=table.device)
    held = col[None] * page < lens[src].long()[:, None]
    row = torch.where(held, table[src], -1)
    table[dst] = row
    lens[dst] = lens[src]
    ref += torch.bincount(row[held].long(), minlength=ref.numel()).to(ref.dtype)
    # reserve: the pages under positions len .. len + more - 1
    now = lens[who].long()
    wants = (col[None] >= (now // page)[:, None]) & (col[None] * page < (now + more)[:, None]) & (more > 0)[:, None]      # [n, cols]
    have = table[who]
    same = (have[:, None, :] == have[None, :, :]) & wants[:, None, :] & wants[None, :, :]                                # [n, n, cols]
    earlier = torch.ones(len(who), len(who), dtype=torch.bool, device=col.device).tril(-1)
    rank = (same & earlier[:, :, None]).sum(1)
    copies = wants & (have >= 0) & (rank < ref[have.clamp(min=0).long()] - 1)
    needs = copies | (wants & (have < 0))
    free = (ref == 0).nonzero()[:, 0]
    which = needs.nonzero()
    fresh = free[:len(which)]
    is_copy = copies[needs]
    old = have[needs].long()
    ref[fresh] = 1
    ref -= torch.bincount(old[is_copy], minlength=ref.numel()).to(ref.dtype)
    table[who[which[:, 0]], which[:, 1]] = fresh.to(table.dtype)
    _copy_pages(s, old[is_copy], fresh[is_copy])


def _plain_compact(s):
    table, lens, ref = s["table"], s["seq_lens"], s["ref"]
    gone = s["gone"].long()
    row = table[gone]
    ref -= torch.bincount(row[row >= 0].long(), minlength=ref.numel()).to(ref.dtype)
    table[gone] = -1
    lens[gone] = 0
    n_live = (ref > 0).sum()
    at = torch.arange(ref.numel(), device=ref.device)
    src = ((ref > 0) & (at >= n_live)).nonzero()[:, 0]
    dst = ((ref == 0) & (at < n_live)).nonzero()[:, 0]
    to = at.clone()
    to[src] = dst
    table.copy_(torch.where(table >= 0, to[table.clamp(min=0).long()].to(table.dtype), -1))
    ref[dst] = ref[src]
    ref[src] = 0
    _copy_pages(s, src, dst)


def run(s):
    """One pass: the plain form, or the calls that a user makes of the framework."""
    c = s["case"]
    if own:
        return _own(s)
    if c["op"] == "attention":
        return _plain_attention(s)
    if c["op"] == "append":
        return _plain_append(s)
    s["book"].copy_(s["pristine"])
    (_plain_fork if c["op"] == "fork" else _plain_compact)(s)
    return {"table": s["table"], "lens": s["seq_lens"], "ref": s["ref"], "k": s["k"], "v": s["v"], "k_scale": s["ks"], "v_scale": s["vs"]}


def _own(s):
    from paper_2601_19278_b200 import binding
    c = s["case"]
    if "cache" not in s:                # the descriptors of the pool and the workspace, which a program keeps
        s["cache"] = binding.Kv8Cache(s["k"], s["v"], s["ks"], s["vs"])
        if c["op"] == "attention":
            n = binding.kv8_attention_workspace_bytes(s["cache"], c["batch"], c["rows"], c["heads"], s["max_len"])
            s["work"] = torch.empty(n, dtype=torch.uint8, device=s["q"].device)
        elif c["op"] != "append":
            s["pages"] = binding.Kv8Pages(s["table"], s["seq_lens"], s["ref"], c["page"])
            s["work"] = torch.empty(binding.kv8_pages_workspace_bytes(s["pages"]), dtype=torch.uint8, device=s["table"].device)
    if c["op"] == "attention":
        binding.kv8_attention(s["cache"], 0, s["q"], s["k_new"], s["v_new"], s["lens"], s["table"], s["out"], max_len=s["max_len"],
                              n_rows=s["n_rows"], mask=s["mask"], workspace=s["work"])
        return s["out"]
    if c["op"] == "append":
        binding.kv8_append(s["cache"], 0, s["k_new"], s["v_new"], s["lens"], s["table"], n_append=s["cnt"], row_index=s["index"],
                           max_append=c["append"])
        return {"k": s["k"], "v": s["v"], "k_scale": s["ks"], "v_scale": s["vs"]}
    s["book"].copy_(s["pristine"])
    if c["op"] == "fork":
        binding.kv8_fork(s["pages"], s["src"], s["dst"])
        binding.kv8_reserve(s["pages"], s["cache"], s["who"], s["more"], workspace=s["work"])
    else:
        binding.kv8_release(s["pages"], s["gone"])
        binding.kv8_compact(s["pages"], s["cache"], workspace=s["work"])
    return {"table": s["table"], "lens": s["seq_lens"], "ref": s["ref"], "k": s["k"], "v": s["v"], "k_scale": s["ks"], "v_scale": s["vs"]}


# ---------------------------------------------------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------------
def work(case):
    hkv, d, page = case["kv_heads"], case["dim"], case["page"]
    if case["op"] == "attention":
        B, R, H = case["batch"], case["rows"], case["heads"]
        lens = _lens(case, B)
        among = R * (R + 1) / 2 if case["mask"] == "causal" else 6.0 * R      # a tree's nodes see their few ancestors
        return {"bytes": 2.0 * sum(lens) * hkv * d + 8.0 * sum(_pages_of(n, page) for n in lens) * hkv + 4.0 * B * R * (H + hkv) * d,
                "flops": 4.0 * d * H * sum(R * n + among for n in lens)}
    if case["op"] == "append":
        A = case["append"]
        rows = sum(max(1, A - (i * 5) % max(1, A)) for i in range(case["batch"]))
        return {"bytes": 6.0 * case["layers"] * rows * hkv * d, "flops": 0.0}
    slab = 2.0 * case["layers"] * hkv * (page * d + 4)                         # a page of all layers, K and V
    lens = _lens(case, case["seqs"])
    if case["op"] == "fork":
        copied = sum(case["forks"] for n in lens if n % page)                 # the partly filled page, once per fork
        return {"bytes": 2.0 * copied * slab + 8.0 * sum(_pages_of(n, page) for n in lens) * (1 + case["forks"]), "flops": 0.0}
    held = [_pages_of(n, page) for n in lens]
    live = sum(held) / 2.0                                                     # about half the pages survive, in random places
    total = sum(held) + case["seqs"]
    return {"bytes": 2.0 * live * max(0.0, 1 - live / total) * slab + 8.0 * total, "flops": 0.0}


# ---------------------------------------------------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def _round_e4m3(x):
    """Nearest e4m3 value, ties to even: 4 significant bits down to 2^-6, steps of 2^-9 below."""
    _, e = torch.frexp(x)
    step = torch.exp2((e.double() - 4).clamp(min=-9.0))
    return (x / step).round() * step


def exact(case, seed):
    s = prepare(case, seed)
    d, page = case["dim"], case["page"]
    if case["op"] == "attention":
        B, R, H, hkv = case["batch"], case["rows"], case["heads"], case["kv_heads"]
        if 4.0 * d * H * B * R * (case["len_hi"] + R) > 4e12:
            return None
        lens = s["lens"].tolist()
        used = s["n_rows"].tolist() if s["n_rows"] is not None else [R] * B
        out = torch.zeros(B, R, H, d, dtype=torch.float64, device=s["q"].device)
        for b in range(B):
            n, r = lens[b], used[b]
            ids = s["table"][b, :_pages_of(n, page)].long()
            for h in range(hkv):
                def whole(codes, scales, new):
                    c = _take(codes[0], ids, h).double() * scales[0, ids, h].double()[:, None, None]
                    return torch.cat([c.reshape(-1, d)[:n], new[b, :r, h].double()])
                k, v = whole(s["k"], s["ks"], s["k_new"]), whole(s["v"], s["vs"], s["v_new"])
                block = s["mask"][b, :r, :r].bool() if s["mask"] is not None else torch.ones(r, r, dtype=torch.bool, device=k.device).tril()
                hidden = ~torch.cat([torch.ones(r, n, dtype=torch.bool, device=k.device), block], 1)
                for j in range(h * (H // hkv), (h + 1) * (H // hkv)):
                    x = s["q"][b, :r, j].double() @ k.T / math.sqrt(d)
                    out[b, :r, j] = torch.softmax(x.masked_fill(hidden, -math.inf), 1) @ v
        return out
    if case["op"] == "append":
        L, A, hkv = case["layers"], case["append"], case["kv_heads"]
        if case["batch"] * (A // page + 2) > 3000:
            return None
        top = E4M3_MAX if case["fmt"] == "e4m3" else INT8_MAX
        near = _round_e4m3 if case["fmt"] == "e4m3" else torch.round
        found = {}
        for name, codes, scales, new in (("k", s["k"], s["ks"], s["k_new"]), ("v", s["v"], s["vs"], s["v_new"])):
            val, sc = codes.double(), scales.double()
            for b, (n, cnt) in enumerate(zip(s["lens"].tolist(), s["cnt"].tolist())):
                src = s["index"][b].tolist() if s["index"] is not None else list(range(A))
                j = 0
                while j < cnt:
                    first, off = n + j - (n + j) % page, (n + j) % page
                    p = int(s["table"][b, first // page])
                    rows = src[j:min(cnt, j + page - off)]
                    x = new[:, b, rows].double().transpose(1, 2)                # [L, hkv, rows, d]
                    big = x.abs().amax((2, 3))
                    want = torch.exp2(torch.ceil(torch.log2(big / top))).clamp(min=SCALE_FLOOR)
                    want = torch.where(big > want * top, want * 2, torch.where((big <= want * top / 2) & (want > SCALE_FLOOR), want / 2, want))
                    if off:
                        want = torch.maximum(want, sc[:, p])
                        val[:, p, :, :off] = near(val[:, p, :, :off] * (sc[:, p] / want)[..., None, None])
                    sc[:, p] = want
                    val[:, p, :, off:off + len(rows)] = near(x / want[..., None, None])
                    j += len(rows)
            found[name], found[name + "_scale"] = val, sc
        if case["fmt"] == "int8":       # whole numbers are compared as they are
            found["k"] = found["v"] = None
        return found
    return None                         # page operations move whole numbers
