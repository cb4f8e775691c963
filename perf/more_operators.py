"""Operators over a paged key-value cache for drafted tokens and for long contexts, as cases that can be timed.

A case is a dict of plain sizes.  `op` says which public entry point one pass calls:

  tree      fdy_tree_attention: drafted tokens of every sequence, each over the cached ones and those it goes on from
  keep      fdy_pages_keep: of a row's last tokens those that are kept move together, pages behind them are given up
  bounds    fdy_page_bounds: the smallest and largest key elements of every page that has new tokens
  select    fdy_page_select: the pages whose bounds promise most to a sequence's queries
  selected  fdy_selected_attention: one new token of every sequence over the pages that were chosen for each cache head

Where `own` is false a pass computes the same in elementary torch operations, in 32 bits (the pages' scores, which are
compared with each other, in 64), rounded once at the end.  Lengths and numbers of drafted tokens follow from the case alone;
which pages hold what, the drafted trees and everything that the operators read is drawn from the seed.
"""
import math
import zlib

import numpy as np
import torch

own = False

DEV = "cuda:0"
FLOATS = {"bf16": torch.bfloat16, "f16": torch.float16, "f8": torch.float8_e4m3fn}
WIDTH = {"bf16": 2, "f16": 2, "f8": 1}


# ---- the cases -----------------------------------------------------------------------------
def _tree(name, rows, shortest, longest, least, most, shape, heads, kv_heads, dim, page, order, type_, cache, window=0):
    return dict(name=name, op="tree", rows=rows, shortest=shortest, longest=longest, least=least, most=most, shape=shape,
                heads=heads, kv_heads=kv_heads, dim=dim, page=page, order=order, type=type_, cache=cache, window=window)


def _keep(name, rows, shortest, longest, drafts, prefix, kept, page, planes, token_bytes, pieces):
    return dict(name=name, op="keep", rows=rows, shortest=shortest, longest=longest, drafts=drafts, prefix=prefix, kept=kept,
                page=page, planes=planes, token_bytes=token_bytes, pieces=pieces)


def _bounds(name, rows, shortest, longest, fresh, kv_heads, dim, page, order, cache):
    return dict(name=name, op="bounds", rows=rows, shortest=shortest, longest=longest, fresh=fresh, kv_heads=kv_heads,
                dim=dim, page=page, order=order, cache=cache)


def _select(name, rows, shortest, longest, heads, kv_heads, dim, page, type_, cache, budget, sinks, recent):
    return dict(name=name, op="select", rows=rows, shortest=shortest, longest=longest, heads=heads, kv_heads=kv_heads,
                dim=dim, page=page, type=type_, cache=cache, budget=budget, sinks=sinks, recent=recent)


def _selected(name, rows, budget, longest, heads, kv_heads, dim, page, order, type_, cache):
    return dict(name=name, op="selected", rows=rows, budget=budget, longest=longest, heads=heads, kv_heads=kv_heads,
                dim=dim, page=page, order=order, type=type_, cache=cache)


def listed():
    return [
        # one user, a small tree over a short context: latency
        _tree("tree_one", 1, 517, 517, 8, 8, "tree", 32, 8, 128, 16, "token", "bf16", "bf16"),
        # continuous batching: contexts of every size, trees of 1 to 16 tokens, one row that drafts nothing
        _tree("tree_ragged", 33, 17, 8192, 1, 16, "tree", 32, 8, 128, 16, "token", "bf16", "bf16"),
        # wide trees over long contexts: as many operations as bytes are worth
        _tree("tree_wide", 8, 6000, 8192, 64, 64, "tree", 64, 8, 128, 32, "token", "bf16", "bf16"),
        # five tokens guessed in a row by every sequence of a large batch, an 8-bit cache, a layer that looks back 2,048 tokens
        _tree("chain_window_f8", 64, 100, 8192, 5, 5, "chain", 40, 40, 128, 32, "head", "f16", "f8", window=2048),
        # verification is over: of 26 drafted tokens a path of 5 stays, in all planes of 36 layers
        _keep("keep_path", 64, 30, 500, 26, 1, 5, 16, 72, 2048, 1),
        # rows held to a budget: the first 64 and the last 1,000 tokens stay, heads-first pages
        _keep("keep_ends", 8, 4096, 4096, 4000, 64, 1064, 32, 32, 2048, 8),
        # one new token in every row of a batch: the bounds of the last pages
        _bounds("bounds_step", 256, 1, 8192, 1, 8, 128, 16, "token", "bf16"),
        # prompts that have just been read: all their pages
        _bounds("bounds_prompt", 5, 20000, 32768, 32768, 8, 128, 64, "head", "f16"),
        # one very long context: latency of the choice
        _select("select_one", 1, 131072, 131072, 32, 8, 128, 16, "bf16", "bf16", 128, 1, 2),
        # a batch of long contexts over an 8-bit cache
        _select("select_batch_f8", 96, 1000, 65536, 64, 8, 128, 16, "bf16", "f8", 256, 1, 4),
        # the chosen pages of one context
        _selected("selected_one", 1, 128, 131072, 32, 8, 128, 16, "token", "bf16", "bf16"),
        # the chosen pages of a batch, heads-first pages
        _selected("selected_batch", 64, 64, 32768, 64, 8, 128, 64, "head", "bf16", "bf16"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


HEADS = ((32, 8), (64, 8), (40, 40), (16, 8), (28, 4), (32, 1), (12, 12), (24, 2))


def draw(rng):
    op = rng.choice(["tree", "tree", "tree", "keep", "bounds", "select", "select", "selected"])
    heads, kv_heads = rng.choice(HEADS)
    type_ = rng.choice(["bf16", "f16"])
    cache = rng.choice([type_, type_, "f8"])
    order = rng.choice(["token", "head"])
    page = rng.choice([8, 16, 32, 64, 128, 256])
    dim = rng.choice([64, 80, 96, 128, 192, 256])
    if op == "tree":
        rows, most = _log_int(rng, 1, 128), _log_int(rng, 1, 64)
        # up to about 250 MB of cache and 2^28 scores
        longest = min(65536, 250_000_000 // (rows * kv_heads * dim * 2 * WIDTH[cache]), (1 << 28) // (rows * heads * most))
        longest = _log_int(rng, most + 1, max(most + 2, longest))
        shortest = max(most, rng.choice([1, longest // 2, longest]))
        c = _tree("", rows, shortest, longest, rng.choice([1, most]), most, rng.choice(["tree", "tree", "chain"]), heads, kv_heads,
                  dim, page, order, type_, cache, rng.choice([0, 0, 0, _log_int(rng, 16, 4096)]))
    elif op == "keep":
        page, planes, pieces = rng.choice([16, 32, 64]), rng.choice([2, 8, 32, 72]), rng.choice([1, 4, 8])
        token_bytes = pieces * rng.choice([128, 256, 512])
        rows, kept = _log_int(rng, 1, 256), _log_int(rng, 1, 64)
        drafts = 2 * kept + rng.randint(0, 2 * kept)
        longest = _log_int(rng, drafts + 1, 2 * drafts + 1000)
        while rows * (longest + 2 * page) * planes * token_bytes > 1_500_000_000:
            rows, longest, planes = max(1, rows // 2), max(drafts + 1, longest // 2), planes if rows > 1 else max(2, planes // 2)
        c = _keep("", rows, max(drafts, longest // 3), longest, drafts, rng.randint(0, kept), kept, page, planes, token_bytes, pieces)
    elif op == "bounds":
        rows = _log_int(rng, 1, 256)
        longest = _log_int(rng, 2, max(3, min(65536, 500_000_000 // (rows * kv_heads * dim * WIDTH[cache]))))
        c = _bounds("", rows, rng.choice([1, max(1, longest // 2)]), longest, rng.choice([1, 1, rng.randint(1, longest), longest]),
                    kv_heads, dim, page, order, cache)
    elif op == "select":
        rows, sinks, recent = _log_int(rng, 1, 128), rng.randint(0, 4), rng.randint(1, 8)
        most = min(131072, 300_000_000 * page // (rows * kv_heads * dim * 2 * WIDTH[cache]))
        longest = _log_int(rng, page, max(2 * page, most))
        c = _select("", rows, rng.choice([1, max(1, longest // 2), longest]), longest, heads, kv_heads, dim, page, type_, cache,
                    sinks + recent + _log_int(rng, 1, 300), sinks, recent)
    else:
        rows = _log_int(rng, 1, 128)
        most = 250_000_000 // (rows * kv_heads * dim * 2 * WIDTH[cache])  # tokens
        budget = _log_int(rng, 1, max(2, min(8192, most) // page))
        longest = min(budget * page * rng.choice([1, 2, 8]), max(budget * page, most))
        c = _selected("", rows, budget, longest, heads, kv_heads, dim, page, order, type_, cache)
    del c["name"]
    return c


# ---- shapes that follow from the case alone ---------------------------------------------------
def _shape_rng(c):
    """Lengths are part of the case: the same for every seed."""
    return np.random.RandomState(zlib.crc32(repr(sorted((k, v) for k, v in c.items() if k != "name")).encode()))


def _lengths(c):
    n, lo, hi = c["rows"], c["shortest"], c["longest"]
    lens = np.exp(_shape_rng(c).uniform(math.log(lo), math.log(hi + 1), n)).astype(np.int64)
    lens = np.clip(lens, lo, hi)
    lens[0] = hi
    if n > 8 and lo == 1 and c["op"] != "tree":
        lens[n // 2] = 0  # a row whose sequence has just been given up
    return lens


def _drafts(c):
    """Drafted tokens of each sequence, the last ones of its row."""
    n = _shape_rng(c).randint(c["least"], c["most"] + 1, c["rows"])
    n[0] = c["most"]
    if c["rows"] > 8 and c["least"] < c["most"]:
        n[c["rows"] // 2] = 0  # one that drafts nothing this time
    return n


def _depths(c, rng):
    """Of every sequence a tree over its drafted tokens, as the token that each goes on from (-1: the cached ones)."""
    trees = []
    for n in _drafts(c):
        if c["shape"] == "chain":
            trees.append(np.arange(n) - 1)
        else:  # broad near the root
            trees.append(np.array([-1] + [int(rng.randint(max(0, j // 3 - 3), max(1, (j + 1) // 2))) for j in range(1, n)])[:n])
    return trees


def _fresh(c):
    return np.minimum(_lengths(c), c["fresh"])


def _chosen(c):
    """Tokens in each sequence's chosen pages."""
    rng = _shape_rng(c)
    total = rng.randint(max(1, c["longest"] // 2), c["longest"] + 1, c["rows"])
    total[0] = c["longest"]
    pages = -(-total // c["page"])
    taken = np.minimum(pages, c["budget"])
    return (taken - 1) * c["page"] + total - (pages - 1) * c["page"], taken, pages


def _kept_list(c, rng):
    """Numbers of the drafted tokens that stay, ascending: the first `prefix`, then some that lie behind all places they go to
    (so a second pass over what the first left moves the same tokens to the same places)."""
    free = c["kept"] - c["prefix"]
    if c["kept"] > 64:
        rest = np.arange(c["drafts"] - free, c["drafts"])  # a row's end
    else:
        rest = c["kept"] + np.sort(rng.permutation(c["drafts"] - c["kept"])[:free])
    return np.concatenate([np.arange(c["prefix"]), rest])


def work(c):
    if c["op"] == "keep":
        moved = c["rows"] * (c["kept"] - c["prefix"])
        pages = int((-(-_lengths(c) // c["page"]) - -(-(_lengths(c) - c["drafts"] + c["kept"]) // c["page"])).sum())
        return {"bytes": 2 * moved * c["planes"] * c["token_bytes"] + c["rows"] * (c["kept"] + 4) * 4 + pages * 12, "flops": 0}
    if c["op"] == "bounds":
        lens, fresh = _lengths(c), _fresh(c)
        first = (lens - fresh) // c["page"] * c["page"]
        read, pages = int(np.where(fresh > 0, lens - first, 0).sum()), int(np.where(fresh > 0, -(-(lens - first) // c["page"]), 0).sum())
        of_head = c["kv_heads"] * c["dim"] * WIDTH[c["cache"]]
        return {"bytes": read * of_head + pages * (2 * of_head + 4) + c["rows"] * 8, "flops": 2 * read * c["kv_heads"] * c["dim"]}
    if c["op"] == "select":
        pages = -(-_lengths(c) // c["page"])
        looked = int(np.where(pages > c["budget"], pages, 0).sum())
        taken = int(np.minimum(pages, c["budget"]).sum())
        of_page = c["kv_heads"] * c["dim"] * 2
        return {"bytes": looked * of_page * WIDTH[c["cache"]] + int(pages.sum()) * 4 + taken * c["kv_heads"] * 4
                + c["rows"] * (c["heads"] * c["dim"] * WIDTH[c["type"]] + 8), "flops": 2 * looked * of_page}
    w, cw = WIDTH[c["type"]], WIDTH[c["cache"]]
    if c["op"] == "selected":
        n, taken, _ = _chosen(c)
        seen = int(n.sum())
        return {"bytes": seen * c["kv_heads"] * 2 * c["dim"] * cw + c["rows"] * c["heads"] * (c["dim"] * 2 * w + 4)
                + int(taken.sum()) * c["kv_heads"] * 4 + c["rows"] * 4, "flops": 4 * seen * c["heads"] * c["dim"]}
    lens, drafts = _lengths(c), _drafts(c)
    past = np.minimum(lens - drafts, c["window"]) if c["window"] else lens - drafts
    read = int(np.where(drafts > 0, past + drafts, 0).sum())
    depth = (drafts + 1) / 2 if c["shape"] == "chain" else np.minimum(drafts, 2 + np.log2(np.maximum(drafts, 1)))
    pairs = int((drafts * (past + depth)).sum())
    return {"bytes": read * c["kv_heads"] * 2 * c["dim"] * cw + int(drafts.sum()) * (c["heads"] * (c["dim"] * 2 * w + 4) + 8)
            + read // c["page"] * 4 + c["rows"] * 8, "flops": 4 * pairs * c["heads"] * c["dim"]}


# ---- inputs --------------------------------------------------------------------------------------
def _pool(c, n_pages, gen):
    """One pool in the case's order, and a view of it as [page, token, head, dim]."""
    token_first = c["order"] == "token"
    shape = (n_pages, c["page"], c["kv_heads"], c["dim"]) if token_first else (n_pages, c["kv_heads"], c["page"], c["dim"])
    pool = torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16).to(FLOATS[c["cache"]])
    return pool, pool if token_first else pool.transpose(1, 2)


def _scales(c, gen):
    return [torch.rand(c["kv_heads"], generator=gen, device=DEV) * 0.8 + 0.6 if c["cache"] == "f8" else None for _ in "kv"]


def _rows_table(lens, page, rng, spare=7):
    """Rows over scattered pages: the table (-1 behind a row's pages), and the pool's pages."""
    pages = -(-lens // page)
    n_pages = int(pages.sum()) + spare
    j = np.arange(int(pages.max()) + 1)[None]
    at = np.where(j < pages[:, None], (np.cumsum(pages) - pages)[:, None] + j, -1)
    return np.where(at >= 0, rng.permutation(n_pages)[at], -1).astype(np.int32), n_pages


def _int32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(DEV)


def _attention_state(c, gen, n_pages, tokens, **more):
    pools, views = zip(*(_pool(c, n_pages, gen) for _ in "kv"))
    q = torch.randn(tokens, c["heads"], c["dim"], generator=gen, device=DEV) * 1.5
    return dict(case=dict(c), q=q.to(FLOATS[c["type"]]), pools=pools, views=views, scales=_scales(c, gen), scale=c["dim"] ** -0.5,
                out=torch.empty(q.shape, dtype=FLOATS[c["type"]], device=DEV), lse=torch.empty(tokens, c["heads"], device=DEV),
                status=torch.zeros(1, dtype=torch.int32, device=DEV), **more)


def prepare(c, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed * 7919 + 17)
    rng = np.random.RandomState((seed * 31 + 5) % (1 << 31))
    if c["op"] == "selected":
        # every cache head has a choice of its own among the pages of the sequence's row
        seen, taken, pages = _chosen(c)
        table, n_pages = _rows_table(pages * c["page"], c["page"], rng)
        lists = np.full((c["rows"], c["kv_heads"], c["budget"]), -1, np.int64)
        for s, (t, p) in enumerate(zip(taken, pages)):
            for h in range(c["kv_heads"]):
                lists[s, h, :t] = table[s, np.append(np.sort(rng.permutation(p - 1)[:t - 1]), p - 1)]
        return _attention_state(c, gen, n_pages, c["rows"], table=_int32(lists), lens=_int32(seen))
    if c["op"] == "keep":
        return _keep_state(c, gen, rng)
    lens = _lengths(c)
    table, n_pages = _rows_table(lens, c["page"], rng)
    if c["op"] == "tree":
        drafts = _drafts(c)
        first = np.concatenate([[0], np.cumsum(drafts)])
        sees = np.zeros((int(first[-1]), (c["most"] + 63) // 64), np.uint64)
        for s, parents in enumerate(_depths(c, rng)):
            for j, p in enumerate(parents):
                if p >= 0:
                    sees[first[s] + j] = sees[first[s] + p]
                sees[first[s] + j, j // 64] |= np.uint64(1 << (j % 64))
        return _attention_state(c, gen, n_pages, int(first[-1]), table=_int32(table), lens=_int32(lens), first=_int32(first),
                                sees=None if c["shape"] == "chain" else torch.from_numpy(sees.view(np.int64)).to(DEV))
    if c["op"] == "bounds":
        pool, view = _pool(c, n_pages, gen)
        return dict(case=dict(c), pool=pool, view=view, table=_int32(table), lens=_int32(lens), fresh=_int32(_fresh(c)),
                    bounds=torch.zeros(n_pages, c["kv_heads"], 2, c["dim"], dtype=FLOATS[c["cache"]], device=DEV),
                    status=torch.zeros(1, dtype=torch.int32, device=DEV))
    shape = (n_pages, c["kv_heads"], 1, c["dim"])
    middle = torch.randn(shape, generator=gen, device=DEV)
    half = torch.rand(shape, generator=gen, device=DEV) + 0.7
    bounds = torch.cat([middle - half, middle + half], 2).to(FLOATS[c["cache"]])
    q = torch.randn(c["rows"], c["heads"], c["dim"], generator=gen, device=DEV) * 1.5
    return dict(case=dict(c), q=q.to(FLOATS[c["type"]]), bounds=bounds, scales=_scales(c, gen), table=_int32(table),
                lens=_int32(lens), n_pages=n_pages, seen=torch.empty(c["rows"], dtype=torch.int32, device=DEV),
                pages=torch.empty(c["rows"], c["kv_heads"], c["budget"], dtype=torch.int32, device=DEV),
                status=torch.zeros(1, dtype=torch.int32, device=DEV))


def _keep_state(c, gen, rng):
    """Rows, the pool's books in one array, and its contents as words."""
    lens = _lengths(c)
    table, n_pages = _rows_table(lens, c["page"], rng)
    refs = np.zeros(n_pages, np.int32)
    refs[table[table >= 0]] = 1
    free = np.zeros(-(-n_pages // 64) * 64, np.uint8)
    free[:n_pages] = refs == 0
    parts = [refs, np.packbits(free, bitorder="little").view(np.int32), table.reshape(-1), lens.astype(np.int32)]
    ends = np.cumsum([-(-len(x) // 4) * 4 for x in parts])  # each on a 16-byte boundary
    starts = [int(e - -(-len(x) // 4) * 4) for e, x in zip(ends, parts)]
    saved = np.zeros(ends[-1], np.int32)
    for s, x in zip(starts, parts):
        saved[s:s + len(x)] = x
    saved = _int32(saved)
    meta = saved.clone()
    refs, bits, flat, lens = (meta[s:s + len(x)] for s, x in zip(starts, parts))
    # a page of a plane: pieces (heads) of its tokens one after the other
    planes = torch.randint(-1 << 31, (1 << 31) - 1, (c["planes"], n_pages, c["pieces"], c["page"], c["token_bytes"] // c["pieces"] // 4),
                           generator=gen, device=DEV, dtype=torch.int32)
    return dict(case=dict(c), saved=saved, meta=meta, refs=refs, bits=bits.view(torch.int64), table=flat.view(table.shape), lens=lens,
                n_pages=n_pages, planes=planes, addresses=torch.tensor([p.data_ptr() for p in planes], dtype=torch.int64, device=DEV),
                rows=torch.arange(c["rows"], dtype=torch.int32, device=DEV), drafts=_int32(np.full(c["rows"], c["drafts"])),
                keep=_int32([_kept_list(c, rng) for _ in range(c["rows"])]), kept=_int32(np.full(c["rows"], c["kept"])),
                status=torch.zeros(1, dtype=torch.int32, device=DEV))


# ---- the operators in their plain form ----------------------------------------------------------
def _stored(x):
    """Elements as integers of their width: indexing moves bits only."""
    return x.view(torch.uint8 if x.element_size() == 1 else torch.int16)


def _gathered(s, which, pages):
    """[..., token, head, dim] in 32 bits of the pages [..., page]."""
    x = _stored(s["views"][which])[pages.long().clamp(min=0)]
    return x.view(s["pools"][which].dtype).float().flatten(-4, -3)


def _softmax(x, seen, v):
    """Weighted values and the logarithm of the weights' sum; x [..., query, token], v [..., token, dim]."""
    x = torch.where(seen, x, -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    e = torch.exp(x - m)
    total = e.sum(-1, keepdim=True)
    return torch.matmul(e, v) / torch.where(total == 0, 1.0, total), (m + torch.log(total))[..., 0]


def _plain_tree(s):
    c = s["case"]
    B, H, D, M = c["rows"], c["kv_heads"], c["dim"], c["most"]
    first, lens = s["first"].long(), s["lens"].long()
    drafts = first[1:] - first[:-1]
    k, v = (_gathered(s, i, s["table"]).transpose(1, 2) for i in (0, 1))  # [row, head, token, dim]
    if s["scales"][0] is not None:
        k, v = k * s["scales"][0][:, None, None], v * s["scales"][1][:, None, None]
    j = torch.arange(M, device=DEV)
    there = j < drafts[:, None]
    token = torch.where(there, first[:-1, None] + j, 0)  # [row, draft]
    q = s["q"].float()[token].view(B, M, H, -1, D).permute(0, 2, 1, 3, 4)  # [row, head, draft, group, dim]
    at = torch.arange(k.shape[2], device=DEV)
    base = (lens - drafts)[:, None]
    i = at - base  # [row, token]: number of a token among the drafted ones
    if s["sees"] is None:
        drafted = i[:, None] <= j[:, None]
    else:
        word = torch.gather(s["sees"][token], 2, (i.clamp(0, M - 1) // 64)[:, None].expand(B, M, -1))
        drafted = (word >> (i.clamp(0, M - 1) % 64)[:, None] & 1).bool()
    seen = torch.where((i < 0)[:, None], True, drafted) & (at < lens[:, None])[:, None] & there[:, :, None]
    if c["window"]:  # the last ones of what each sees
        behind = seen.flip(2).long().cumsum(2).flip(2)
        seen &= behind <= c["window"]
    x = torch.matmul(q.flatten(2, 3), k.transpose(2, 3).contiguous()) * s["scale"]
    del k
    seen = seen[:, None, :, None].expand(B, H, M, q.shape[3], -1).flatten(2, 3)
    v = torch.where(at[:, None] < lens[:, None, None, None], v, 0.0).contiguous()
    out, lse = _softmax(x, seen, v)
    out = out.view(B, H, M, -1, D).permute(0, 2, 1, 3, 4).reshape(B, M, -1, D)
    lse = lse.view(B, H, M, -1).permute(0, 2, 1, 3).reshape(B, M, -1)
    s["out"].copy_(out[there])
    s["lse"].copy_(lse[there])
    return {"out": s["out"], "lse": s["lse"]}


def _plain_selected(s):
    c = s["case"]
    B, H, D = c["rows"], c["kv_heads"], c["dim"]
    k, v = (_gathered(s, i, s["table"]) for i in (0, 1))  # [row, list, token, head, dim]
    head = torch.arange(H, device=DEV)
    k, v = (x[:, head, :, head].transpose(0, 1) for x in (k, v))  # [row, head, token, dim]
    if s["scales"][0] is not None:
        k, v = k * s["scales"][0][:, None, None], v * s["scales"][1][:, None, None]
    q = s["q"].float().view(B, H, -1, D)
    seen = (torch.arange(k.shape[2], device=DEV) < s["lens"][:, None])[:, None, None]
    x = torch.matmul(q, k.transpose(2, 3).contiguous()) * s["scale"]
    out, lse = _softmax(x, seen, torch.where(seen.transpose(2, 3), v, 0.0).contiguous())
    s["out"].copy_(out.reshape(B, -1, D))
    s["lse"].copy_(lse.reshape(B, -1))
    return {"out": s["out"], "lse": s["lse"]}


def _plain_bounds(s):
    c = s["case"]
    pt, lens = c["page"], s["lens"].long()
    j = torch.arange(s["table"].shape[1], device=DEV)
    renewed = (j * pt < lens[:, None]) & ((j + 1) * pt > (lens - s["fresh"])[:, None]) & (s["fresh"] > 0)[:, None]
    row, j = torch.nonzero(renewed, as_tuple=True)
    page = s["table"][row, j].long()
    k = _stored(s["view"])[page].view(s["pool"].dtype).float()  # [page, token, head, dim]
    held = (j[:, None] * pt + torch.arange(pt, device=DEV) < lens[row, None])[:, :, None, None]
    low, high = torch.where(held, k, math.inf).amin(1), torch.where(held, k, -math.inf).amax(1)
    _stored(s["bounds"])[page] = _stored(torch.stack([low, high], 2).to(s["bounds"].dtype))
    return {"bounds": s["bounds"]}


def _plain_select(s):
    c = s["case"]
    B, H, pt = c["rows"], c["kv_heads"], c["page"]
    lens = s["lens"].long()
    pages = (lens + pt - 1) // pt
    q = s["q"].double().view(B, H, -1, c["dim"])
    if s["scales"][0] is not None:
        q = q * s["scales"][0].double()[:, None, None]
    up, down = q.clamp(min=0).sum(2), q.clamp(max=0).sum(2)  # [row, head, dim]
    score = []
    for row in range(B):  # a row at a time: all rows' bounds in 64 bits are large
        b = _stored(s["bounds"])[s["table"][row].long().clamp(min=0)].view(s["bounds"].dtype).double()  # [page, head, 2, dim]
        score.append((b[:, :, 1] * up[row] + b[:, :, 0] * down[row]).sum(-1))
    score = torch.stack(score).transpose(1, 2)  # [row, head, page]
    j = torch.arange(score.shape[2], device=DEV)
    n = pages[:, None, None]
    # those always taken ahead of the others, those that a row has not behind all
    rank = torch.where(j >= n, 2, torch.where((j < c["sinks"]) | (j >= n - c["recent"]), 0, 1)).expand_as(score)
    order = torch.sort(score, dim=-1, descending=True, stable=True)[1]
    order = torch.gather(order, 2, torch.sort(torch.gather(rank, 2, order), dim=-1, stable=True)[1])
    taken = torch.minimum(pages, torch.full_like(pages, c["budget"]))
    chosen = torch.zeros_like(order, dtype=torch.bool).scatter_(2, order, (j < taken[:, None, None]).expand_as(order))
    s["pages"].fill_(-1)
    row, head, page = torch.nonzero(chosen, as_tuple=True)
    place = chosen.long().cumsum(2)[row, head, page] - 1
    s["pages"][row, head, place] = s["table"][row, page]
    s["seen"].copy_(torch.where(pages > 0, (taken - pages) * pt + lens, 0))
    return {"pages": s["pages"], "seen": s["seen"]}


def _plain_keep(s):
    c = s["case"]
    pt, lens, table = c["page"], s["lens"].long(), s["table"].long()
    row = torch.arange(c["rows"], device=DEV)[:, None]
    base = (lens - s["drafts"])[:, None]
    to = base + torch.arange(c["kept"], device=DEV)
    source = base + s["keep"].long()
    from_page, to_page = table[row, source // pt], table[row, to // pt]
    s["planes"][:, to_page, :, to % pt] = s["planes"][:, from_page, :, source % pt]
    after = lens - s["drafts"] + s["kept"]
    j = torch.arange(table.shape[1], device=DEV)
    gone = (j >= ((after + pt - 1) // pt)[:, None]) & (j < ((lens + pt - 1) // pt)[:, None])
    s["refs"].index_add_(0, table[gone], torch.full_like(table[gone], -1, dtype=torch.int32))
    s["lens"].copy_(after)
    free = s["refs"] == 0
    free = torch.nn.functional.pad(free, (0, s["bits"].numel() * 64 - free.numel())).view(-1, 64).long()
    s["bits"].copy_((free << torch.arange(64, device=DEV)).sum(1))
    return {"meta": s["meta"], "planes": s["planes"]}


# ---- the library's calls --------------------------------------------------------------------------
def _handle(s):
    """Descriptor and workspace of a state, which such a program makes once and keeps beside its buffers."""
    from paper_2604_06664_amd import decode as fdd

    c = s["case"]
    h = dict(lib=fdd)
    if c["op"] == "keep":
        piece = c["token_bytes"] // c["pieces"]
        of_page = c["page"] * c["token_bytes"]
        h["desc"] = fdd.make_pages(refs=s["refs"], free_bits=s["bits"], table=s["table"], lens=s["lens"], page_tokens=c["page"],
                                   planes=s["addresses"], page_bytes=of_page, page_stride=of_page)
        h["token"] = fdd.make_token(token_stride=piece, piece_bytes=piece, pieces=c["pieces"], piece_stride=piece * c["page"])
        h["bytes"] = fdd.fdy_pages_workspace_bytes(h["desc"], c["rows"])
    elif c["op"] == "select":
        kv = fdd.make_kv(None, None, type=fdd.TYPES[c["cache"]], n_pages=s["n_pages"], page_tokens=c["page"], n_heads=c["kv_heads"],
                         head_dim=c["dim"], page_stride=0, token_stride=0, head_stride=0, k_scale=s["scales"][0])
        h["desc"] = fdd.make_select_desc(q=s["q"], bounds=s["bounds"], table=s["table"], lens=s["lens"], kv=kv, pages=s["pages"],
                                         seen=s["seen"], sinks=c["sinks"], recent=c["recent"])
        h["bytes"] = fdd.fdy_page_select_workspace_bytes(h["desc"])
    else:
        pools, view = (s["pools"], s["views"][0]) if c["op"] != "bounds" else ((s["pool"], None), s["view"])
        strides, scales = view.stride(), s.get("scales", (None, None))
        kv = fdd.make_kv(*pools, type=fdd.TYPES[c["cache"]], n_pages=pools[0].shape[0], page_tokens=c["page"],
                         n_heads=c["kv_heads"], head_dim=c["dim"], page_stride=strides[0], token_stride=strides[1],
                         head_stride=strides[2], k_scale=scales[0], v_scale=scales[1])
        if c["op"] == "bounds":
            h["desc"] = fdd.make_bounds_desc(bounds=s["bounds"], table=s["table"], lens=s["lens"], kv=kv, fresh=s["fresh"],
                                             max_fresh=c["fresh"])
        elif c["op"] == "tree":
            h["desc"] = fdd.make_draft_desc(q=s["q"], out=s["out"], lse=s["lse"], table=s["table"], lens=s["lens"], kv=kv,
                                            scale=s["scale"], first=s["first"], sees=s["sees"], max_draft=c["most"], window=c["window"])
            h["bytes"] = fdd.fdy_tree_attention_workspace_bytes(h["desc"])
        else:
            h["desc"] = fdd.make_selected_desc(q=s["q"], out=s["out"], lse=s["lse"], table=s["table"], lens=s["lens"], kv=kv,
                                               scale=s["scale"])
            h["bytes"] = fdd.fdy_selected_attention_workspace_bytes(h["desc"])
    if "bytes" in h:
        h["workspace"] = torch.zeros(h["bytes"], dtype=torch.uint8, device=DEV)
    return h


def _own(s):
    c = s["case"]
    h = s.get("handle")
    if h is None:
        h = s["handle"] = _handle(s)
    fdd = h["lib"]
    if c["op"] == "tree":
        fdd.fdy_tree_attention(h["desc"], h["workspace"], h["bytes"], s["status"])
        return {"out": s["out"], "lse": s["lse"]}
    if c["op"] == "selected":
        fdd.fdy_selected_attention(h["desc"], h["workspace"], h["bytes"], s["status"])
        return {"out": s["out"], "lse": s["lse"]}
    if c["op"] == "bounds":
        fdd.fdy_page_bounds(h["desc"], s["status"])
        return {"bounds": s["bounds"]}
    if c["op"] == "select":
        fdd.fdy_page_select(h["desc"], h["workspace"], h["bytes"], s["status"])
        return {"pages": s["pages"], "seen": s["seen"]}
    fdd.fdy_pages_keep(h["desc"], h["token"], s["rows"], s["drafts"], s["keep"], s["kept"], c["rows"], c["kept"], h["workspace"],
                       h["bytes"], s["status"])
    return {"meta": s["meta"], "planes": s["planes"]}


PLAIN = dict(tree=_plain_tree, selected=_plain_selected, bounds=_plain_bounds, select=_plain_select, keep=_plain_keep)


def run(s):
    if "saved" in s:
        s["meta"].copy_(s["saved"])  # the pool's books as they were before the call: the next pass changes them the same way
    return _own(s) if own else PLAIN[s["case"]["op"]](s)


# ---- the definitions in 64 bits ---------------------------------------------------------------------
def exact(c, seed):
    if c["op"] in ("keep", "select"):
        return None  # whole numbers
    s = prepare(c, seed)
    if c["op"] == "bounds":
        bounds = s["bounds"].double()
        for row, (n, new) in enumerate(zip(_lengths(c).tolist(), _fresh(c).tolist())):
            if new == 0:
                continue
            at = torch.arange((n - new) // c["page"] * c["page"], n, device=DEV)
            page = s["table"][row, at // c["page"]].long()
            k = _stored(s["view"])[page, at % c["page"]].view(s["pool"].dtype).double()
            for i, (worst, best) in enumerate(((math.inf, "amin"), (-math.inf, "amax"))):
                found = torch.full((len(bounds), *k.shape[1:]), worst, dtype=torch.float64, device=DEV).index_reduce_(0, page, k, best)
                bounds[page, :, i] = found[page]
        return {"bounds": bounds}
    cache = [p.double() if c["order"] == "token" else p.double().transpose(1, 2) for p in s["pools"]]
    if c["cache"] == "f8":
        cache = [x * f.double()[:, None] for x, f in zip(cache, s["scales"])]
    group, H, pt = c["heads"] // c["kv_heads"], c["kv_heads"], c["page"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    if c["op"] == "selected":
        for row, n in enumerate(_chosen(c)[0].tolist()):
            at = torch.arange(n, device=DEV)
            for h in range(H):
                page = s["table"][row, h, at // pt].long()
                k, v = (x[page, at % pt, h] for x in cache)
                heads = slice(h * group, (h + 1) * group)
                x = s["q"][row, heads].double() @ k.t().contiguous() * s["scale"]
                lse[row, heads] = torch.logsumexp(x, -1)
                out[row, heads] = torch.softmax(x, -1) @ v
        return {"out": out, "lse": lse}
    rng = np.random.RandomState((seed * 31 + 5) % (1 << 31))
    _rows_table(_lengths(c), pt, rng)  # takes from the generator what `prepare` took
    trees = _depths(c, rng)
    token = 0
    for row, n in enumerate(_lengths(c).tolist()):
        m = len(trees[row])
        if m == 0:
            continue
        # what each drafted token goes on from, by its parents
        sees = torch.zeros(m, n, dtype=torch.bool)
        sees[:, :n - m] = True
        for j in range(m):
            a = j
            while a >= 0:
                sees[j, n - m + a] = True
                a = int(trees[row][a])
            if c["window"]:
                seen = torch.nonzero(sees[j])[:, 0]
                sees[j, seen[:max(0, len(seen) - c["window"])]] = False
        at = torch.arange(n, device=DEV)
        page = s["table"][row, at // pt].long()
        k, v = (x[page, at % pt] for x in cache)  # [token, head, dim]
        q = s["q"][token:token + m].double().view(m, H, group, -1).transpose(0, 1).flatten(1, 2)  # [head, draft * group, dim]
        x = torch.bmm(q, k.permute(1, 2, 0).contiguous()) * s["scale"]
        x = x.view(H, m, group, n).masked_fill(~sees.to(DEV)[:, None], -math.inf).flatten(1, 2)
        lse[token:token + m] = torch.logsumexp(x, -1).view(H, m, group).transpose(0, 1).flatten(1, 2)
        out[token:token + m] = torch.bmm(torch.softmax(x, -1), v.transpose(0, 1).contiguous()).view(H, m, group, -1).transpose(0, 1).flatten(1, 2)
        token += m
    return {"out": out, "lse": lse}
