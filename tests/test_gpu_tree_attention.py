"""fdy_tree_attention through the C ABI against its definition in 64 bits (tolerances: tests/support/paged.py)."""
import math

import numpy as np
import pytest
import torch

import oracle.decode as od
from paper_2604_06664_amd import decode as fdd
from tests.support.paged import DEV, DTYPES, Cache, int32, near

pytestmark = pytest.mark.gpu


def tree(c, rng):
    """Ancestors and self of c drafted tokens, each going on from an earlier one or from the cached ones."""
    sees = []
    for j in range(c):
        p = int(rng.integers(-1, j)) if j else -1
        sees.append(({j} | sees[p]) if p >= 0 else {j})
    return sees


def bits_of(sees, words):
    out = np.zeros((len(sees), words), np.uint64)
    for t, who in enumerate(sees):
        for i in who:
            out[t, i // 64] |= np.uint64(1 << (i % 64))
    return torch.from_numpy(out.view(np.int64)).to(DEV)


class Drafts:
    def __init__(self, lens, drafts, Hq, H, D, kind="bf16", cache=None, window=0, seed=1, shape="tree", scale=None, most=None,
                 words=None, **kw):
        rng = np.random.default_rng(seed + 100)
        self.cache = Cache(lens, H, D, cache=cache or kind, seed=seed, **kw)
        self.kind, self.window, self.drafts, self.Hq = kind, window, list(drafts), Hq
        T = sum(drafts)
        self.scale = D ** -0.5 if scale is None else scale
        self.q = torch.from_numpy(rng.standard_normal((T, Hq, D)).astype(np.float32)).to(DTYPES[kind])
        self.most = most or max(list(drafts) + [1])
        self.sees = None if shape == "chain" else [x for c in drafts for x in tree(c, rng)]
        self.d_sees = None if self.sees is None else bits_of(self.sees, words or -(-self.most // 64))
        self.d_first = int32(np.concatenate([[0], np.cumsum(drafts)]))
        self.d_q = self.q.to(DEV)
        self.out = torch.full((T, Hq, D), 5.0, dtype=DTYPES[kind], device=DEV)
        self.lse = torch.full((T, Hq), 5.0, device=DEV)
        self.ws = None

    def desc(self, **kw):
        c = self.cache
        args = dict(q=self.d_q, out=self.out, lse=self.lse, table=c.d_table, lens=c.d_lens, kv=c.kv(), scale=self.scale,
                    first=self.d_first, sees=self.d_sees, max_draft=self.most, window=self.window)
        args.update(kw)
        return fdd.make_draft_desc(**args)

    def run(self, **kw):
        desc = self.desc(**kw)
        n = fdd.fdy_tree_attention_workspace_bytes(desc)
        if self.ws is None:
            self.ws = torch.randint(0, 256, (n,), dtype=torch.uint8, device=DEV)  # contents are irrelevant
        assert self.ws.numel() >= n
        fdd.fdy_tree_attention(desc, self.ws, n, self.cache.status)
        torch.cuda.synchronize()
        return self.out.cpu(), self.lse.cpu(), int(self.cache.status)

    def want(self, **kw):
        c = self.cache
        args = dict(q=self.q, k_view=c.views[0], v_view=c.views[1], table=c.table, lens=c.lens, scale=self.scale, drafts=self.drafts,
                    sees=self.sees, window=self.window, k_scale=c.scales[0], v_scale=c.scales[1])
        args.update(kw)
        return od.tree_attend(**args)


def check(*args, **kw):
    p = Drafts(*args, **kw)
    got = p.run()
    assert got[2] == 0
    near(got, p.want(), p.kind)
    return p, got


KINDS = [("bf16", "bf16"), ("f16", "f16"), ("bf16", "f8"), ("f16", "f8")]


@pytest.mark.parametrize("kind,cache", KINDS)
@pytest.mark.parametrize("D", [64, 128, 256, 16, 48, 80, 96, 160, 192])
def test_lengths_around_tiles(D, kind, cache):
    lens = [5, 6, 16, 17, 31, 32, 33, 37, 63, 64, 65, 70, 128, 130, 257]
    drafts = [5, 1, 2, 0, 5, 3, 5, 5, 4, 5, 1, 5, 5, 2, 5]
    check(lens, drafts, 4, 2, D, kind=kind, cache=cache)


@pytest.mark.parametrize("shape", ["tree", "chain"])
@pytest.mark.parametrize("Hq,H", [(1, 1), (3, 3), (7, 1), (16, 1), (8, 2), (33, 1)])
@pytest.mark.parametrize("drafts", [[1, 1], [2, 7], [16, 3], [33, 64], [65, 1], [130, 200]])
def test_numbers_of_drafted_tokens(drafts, Hq, H, shape):
    check([c + n for c, n in zip(drafts, (70, 0))], drafts, Hq, H, 64, shape=shape)


@pytest.mark.parametrize("kind,cache", KINDS)
@pytest.mark.parametrize("D", [64, 128, 256])
def test_many_rows_of_a_cache_head(D, kind, cache):
    """More rows than a workgroup's waves take at once, in parts."""
    check([700, 333], [70, 40], 8, 1, D, kind=kind, cache=cache)


@pytest.mark.parametrize("order", ["token", "head"])
@pytest.mark.parametrize("pt", [1, 2, 4, 8, 16, 32, 128, 1024])
def test_page_sizes(pt, order):
    check([9, 17, 40, 129, 200], [9, 4, 1, 0, 17], 4, 2, 64, pt=pt, order=order)
    check([5, 70], [5, 6], 4, 2, 128, pt=pt, order=order, kind="f16", cache="f8", shape="chain")


@pytest.mark.parametrize("window", [1, 2, 3, 16, 31, 33, 64, 100, 1000, 0xFFFFFFFF])
@pytest.mark.parametrize("shape", ["tree", "chain"])
@pytest.mark.parametrize("pt", [4, 16])
def test_windows(window, shape, pt):
    lens, drafts = [9, 30, 64, 65, 100, 333, 220], [9, 8, 4, 1, 12, 7, 90]
    check(lens, drafts, 4, 2, 64, pt=pt, window=window, shape=shape)


def test_what_lies_ahead_of_all_windows_is_not_read():
    """Its pages are given away, and hold NaN."""
    p = Drafts([333, 200], [7, 3], 4, 2, 64, window=40)
    for r, (n, c) in enumerate(zip(p.cache.lens, p.drafts)):
        for j in range((n - c - 40) // 16):
            for v in p.cache.views:
                v[p.cache.table[r, j]] = math.nan
            p.cache.table[r, j] = -7
    p.cache.upload()
    got = p.run()
    assert got[2] == 0
    near(got, p.want(), p.kind)


@pytest.mark.parametrize("lens,drafts", [([4000], [6]), ([3001, 40], [40, 2]), ([2049] * 3, [16, 0, 9])])
@pytest.mark.parametrize("D,cache", [(64, "bf16"), (128, "f8"), (256, "bf16")])
def test_rows_in_parts(lens, drafts, D, cache):
    p, got = check(lens, drafts, 8, 2, D, cache=cache)
    for _ in range(2):  # the same every time, over the same workspace
        again = p.run()
        assert torch.equal(again[0].view(torch.int16), got[0].view(torch.int16)) and torch.equal(again[1], got[1])


def test_many_sequences():
    rng = np.random.default_rng(4)
    drafts = [int(x) for x in rng.integers(0, 5, 700)]
    lens = [c + int(x) for c, x in zip(drafts, rng.integers(0, 60, 700))]
    lens[123] += 2500
    check(lens, drafts, 2, 1, 64)


def test_as_one_new_token():
    """One drafted token each is fdy_paged_attention, up to the order of sums."""
    p, got = check([5, 100, 290, 1], [1, 1, 1, 1], 8, 2, 64)
    c = p.cache
    out, lse = torch.empty_like(p.out), torch.empty_like(p.lse)
    desc = fdd.make_attend_desc(q=p.d_q, out=out, lse=lse, table=c.d_table, lens=c.d_lens, kv=c.kv(), scale=p.scale)
    ws = torch.zeros(fdd.fdy_paged_attention_workspace_bytes(desc), dtype=torch.uint8, device=DEV)
    fdd.fdy_paged_attention(desc, ws, ws.numel(), c.status)
    assert bool(((out.cpu().double() - got[0].double()).abs() <= 2 * 2.0 ** -8 * got[0].double().abs() + 2.0 ** -12).all())
    assert bool(((lse.cpu() - got[1]).abs() <= 1e-5).all())


def test_the_same_number_each():
    p = Drafts([50, 64, 9], [4, 4, 4], 4, 2, 64)
    near(p.run(first=None), p.want(), p.kind)


def test_masks_that_show_nothing():
    """Rows that see none of the drafted tokens, not even themselves; with an empty context they see nothing at all."""
    p = Drafts([40, 4, 33], [4, 4, 1], 4, 2, 64)
    for t in (0, 1, 4, 5, 8):
        p.sees[t] = set()
    p.d_sees = bits_of(p.sees, 1)
    got = p.run()
    want = p.want()
    near(got, want, p.kind)
    assert bool((want[1][4:6] == -math.inf).all())
    p.window = 1  # of the seen ones only the last
    near(p.run(window=1), p.want(), p.kind)


def test_bits_behind_the_drafted_tokens_and_wide_masks():
    p = Drafts([60, 20], [5, 3], 4, 2, 64, most=200, words=7)
    want = p.want()
    p.d_sees |= torch.tensor([~0x1F, -1, -1, -1, -1, -1, -1], device=DEV)  # all bits from 5 on
    p.d_sees[5:, 0] &= 0x7
    p.d_sees[5:, 0] |= ~0x1F
    near(p.run(), want, p.kind)


@pytest.mark.parametrize("kind,cache", KINDS)
@pytest.mark.parametrize("pt", [8, 16])
@pytest.mark.parametrize("D", [64, 128])
def test_values_of_other_branches_that_are_no_numbers(D, pt, kind, cache):
    """Infinities and NaN in keys and values of a drafted token reach those that see it, and nobody else."""
    for bad in (math.nan, math.inf):
        if cache == "f8" and bad == math.inf:
            continue
        p = Drafts([40, 70, 33], [6, 9, 20], 4, 2, D, kind=kind, cache=cache, pt=pt)
        c = p.cache

        def put(which, r, j, d):
            t = c.lens[r] - p.drafts[r] + j
            c.views[which][c.table[r, t // pt], t % pt, :, d] = bad

        put(1, 0, 3, 5), put(1, 1, 2, 0), put(1, 1, 4, D - 1), put(0, 2, 7, 3)
        c.upload()
        out, lse, status = p.run()
        o, l, spread = p.want()
        assert status == 0
        fine = torch.isfinite(o)
        assert torch.equal(torch.isfinite(out), fine)
        assert torch.equal(torch.isnan(out), torch.isnan(o)) or bad == math.inf
        spread = torch.where(torch.isfinite(spread), spread, 4.0)
        clean = fine.all(-1)
        assert bool(clean.any()) and not bool(clean.all())
        some = fine & ~clean[..., None] & torch.isfinite(l)[..., None]  # rows in which some elements are infinite
        assert bool(((out.double() - o).abs()[some] <= 4 * (2.0 ** -11 + 2.0 ** -15) + 2.0 ** -8 * o.abs()[some]).all())
        near((out[clean][None], lse[clean][None]), (o[clean][None], l[clean][None], spread[clean][None]), kind)


def test_values_ahead_of_a_window_that_are_no_numbers():
    p = Drafts([90], [4], 4, 2, 64, window=30, shape="chain")  # windows begin at tokens 57 to 60
    c = p.cache
    for t in (57, 58, 59):
        c.views[1][c.table[0, t // 16], t % 16] = math.inf
    c.upload()
    out, lse, _ = p.run()
    o, l, spread = p.want()
    assert torch.equal(torch.isfinite(out), torch.isfinite(o)) and bool(torch.isfinite(o[3]).all()) and not bool(torch.isfinite(o[0]).any())
    near((out[3:], lse[3:]), (o[3:], l[3:], spread[3:]), "bf16")


def test_rows_of_a_larger_pool_and_strides():
    p = Drafts([9, 77, 150, 40], [3, 1, 5], 4, 2, 64, pad=8)
    rows = [3, 0, 2]
    wide = torch.zeros(9, 4, 3, 64, dtype=torch.bfloat16, device=DEV)
    q = wide[:, :, 1]
    q.copy_(p.d_q)
    out = torch.full((4, 9, 72), 5.0, dtype=torch.bfloat16, device=DEV)
    _, lse, status = p.run(q=q, out=out[:, :, :64].transpose(0, 1), rows=int32(rows))
    assert status == 0
    near((out[:, :, :64].transpose(0, 1).cpu(), lse), p.want(rows=rows), "bf16")
    assert bool((out[:, :, 64:] == 5).all())


def test_queries_of_no_sequence_stay_what_they_are():
    p = Drafts([30, 50], [4, 3], 4, 2, 64)
    d_first = int32([1, 3, 6])  # token 0 and the last belong to none
    p.drafts, p.sees = [2, 3], [{0}, {0, 1}, {0}, {1}, {0, 2}]
    p.d_sees[1:6] = bits_of(p.sees, 1)
    out, lse, status = p.run(first=d_first)
    assert status == 0
    near((out[1:6], lse[1:6]), p.want(q=p.q[1:6]), "bf16")
    for x in (out, lse):
        assert bool((x[0] == 5).all()) and bool((x[6:] == 5).all())


def test_numbers_out_of_range():
    p = Drafts([100, 50, 64, 90, 30], [3, 2, 4, 1, 5], 4, 2, 64, shape="chain")
    c = p.cache
    table, lens = c.table.copy(), list(c.lens)
    table[0, 1] = c.n_pages  # a page that is none
    lens[1] = -3             # no tokens
    lens[4] = 3              # of five drafted tokens two are not there
    c.d_table.copy_(torch.from_numpy(table))
    c.d_lens.copy_(int32(lens))
    got = p.run()
    assert got[2] == od.ST_BAD_INDEX
    near(got, p.want(table=table, lens=lens), "bf16")
    for first in ([0, 3, 2, 9, 10, 15], [0, 3, 5, 9, 10, 16], [0, -1, 5, 9, 10, 15], [0, 3, 5, 9, 10, 1 << 30]):
        c.status.zero_()
        p.out.fill_(5), p.lse.fill_(5)
        out, lse, status = p.run(first=int32(first))
        assert status == od.ST_BAD_INDEX
        for s, (a, b) in enumerate(zip(first, first[1:])):
            if not (0 <= a <= b <= 15 and b - a <= 5):
                continue
            o, l, spread = p.want(q=p.q[a:b], drafts=[b - a], rows=[s], table=table, lens=lens)
            near((out[a:b], lse[a:b]), (o, l, spread), "bf16")
    c.status.zero_()
    rows = [2, 7, -1, 2, 0]
    got = p.run(rows=int32(rows))
    assert got[2] == od.ST_BAD_INDEX
    near(got, p.want(rows=rows, table=table, lens=lens), "bf16")


@pytest.mark.parametrize("scale", [-0.125, 0.0])
def test_factors_that_are_not_positive(scale):
    check([70, 20], [5, 2], 4, 2, 64, scale=scale)


def test_large_scores():
    """Two drafted tokens and a cached one share the largest score, of 2^20 and more; their weights are 1/3 or 1/2 in full."""
    p = Drafts([300, 40], [4, 4], 4, 2, 64, scale=1.75)
    c = p.cache
    p.q[:] = 0
    p.q[:, :, 0] = 2.0 ** 18
    p.d_q.copy_(p.q)
    p.sees = [{0}, {1}, {0, 1, 2}, {0, 3}] * 2
    p.d_sees = bits_of(p.sees, 1)
    for r, n in enumerate(c.lens):
        for t in range(n):
            c.views[0][c.table[r, t // 16], t % 16] = 0
            c.views[0][c.table[r, t // 16], t % 16, :, 0] = 4.0 if t in (7, n - 4, n - 3) else -3.0
    c.upload()
    out, lse, status = p.run()
    o, l, spread = p.want()
    assert status == 0
    assert bool(((out.double() - o).abs() <= 2 * 2.0 ** -8 * spread[..., None]).all())
    assert bool(((lse.double() - l).abs() <= l.abs() * 2.0 ** -21 + 1e-6).all())


@pytest.mark.parametrize("kind,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "f8")])
@pytest.mark.parametrize("drafts", [[3, 2], [20, 9]])
def test_weights_are_held_in_more_bits_than_the_type_has(kind, cache, drafts):
    """One token of 32 takes most of the weight and has the value 0, all others have one and the same score and the value 1.
    Products are exact; 2^-15 is left to the weights, 2^-16 to factor, exponential and sums, and the result is rounded once."""
    p = Drafts([300, 2111], drafts, 8, 2, 128, kind=kind, cache=cache, scale=1.0, shape="chain")
    c = p.cache
    p.q[:] = 0
    p.q[:, :, 0] = torch.linspace(1.5, 7.5, p.q.shape[0] * 8).view(-1, 8).to(p.q.dtype)
    p.d_q.copy_(p.q)
    for r, n in enumerate(c.lens):
        for t in range(n):
            page, place = c.table[r, t // 16], t % 16
            c.views[0][page, place] = 0
            c.views[0][page, place, :, 0] = 0.0 if t % 32 == 5 else -1.0
            c.views[1][page, place] = 0.0 if t % 32 == 5 else 1.0
    for s in c.scales:
        if s is not None:
            s.fill_(1.0)
    c.upload()
    out, lse, status = p.run()
    o, l, _ = p.want()
    assert status == 0
    err = float(((out.double() - o).abs() / o).max())
    assert err <= {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}[kind] + 2.0 ** -15 + 2.0 ** -16, err
    assert bool(((lse.double() - l).abs() <= 3e-5).all())


def test_batches_of_many_sizes_in_turn_over_one_workspace():
    rng = np.random.default_rng(5)
    batches = [([int(x) + 9 for x in rng.integers(0, 500, 60)] + [2800], [int(x) for x in rng.integers(0, 9, 60)] + [5]),
               ([2500, 90], [80, 9]), ([3000], [1]), ([9] * 40, [2] * 40), ([600, 50, 900], [30, 40, 0])]
    problems = [Drafts(lens, drafts, 8, 2, 64, row_pages=pages) for lens, drafts in batches for pages in (200, 4096)]
    ws = torch.zeros(max(fdd.fdy_tree_attention_workspace_bytes(p.desc()) for p in problems), dtype=torch.uint8, device=DEV)
    wants = [p.want() for p in problems]
    for i in [0, 2, 1, 4, 6, 0, 8, 3, 5, 9, 2, 7, 0]:
        problems[i].ws = ws
        near(problems[i].run(), wants[i], "bf16")


def test_offsets_behind_32_bits():
    """Pages a GiB apart: the pool's last page starts 6 GiB in."""
    for pt in (16, 8):
        small = Drafts([60], [5], 2, 1, 64, spare=0, pt=pt)
        c, n_pages, ps = small.cache, 7 if pt == 16 else 8, 1 << 29
        pools = [torch.empty(n_pages * ps // 2, dtype=torch.int32, device=DEV) for _ in "kv"]
        for src, dst in zip(c.d_pools, pools):
            flat, x = dst.view(torch.int16), src.view(-1, pt * 64)
            for j in range(len(x)):
                flat[(n_pages - 1 - j) * ps:(n_pages - 1 - j) * ps + pt * 64] = x[j]
        table = torch.from_numpy(np.where(c.table >= 0, n_pages - 1 - c.table, -1).astype(np.int32)).to(DEV)
        kv = fdd.make_kv(*pools, type=fdd.FDY_BF16, n_pages=n_pages, page_tokens=pt, n_heads=1, head_dim=64, page_stride=ps,
                         token_stride=64, head_stride=64)
        near(small.run(kv=kv, table=table), small.want(), "bf16")
        del pools


def test_replays_while_rows_and_trees_change():
    p = Drafts([900, 1500, 64], [6, 3, 8], 4, 2, 64)
    p.ws = torch.zeros(fdd.fdy_tree_attention_workspace_bytes(p.desc()), dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        p.run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fdd.fdy_tree_attention(p.desc(), p.ws, p.ws.numel(), p.cache.status)
    rng = np.random.default_rng(9)
    for lens, drafts in (([6, 3, 8], [6, 3, 8]), ([300, 1500, 64], [1, 0, 8]), ([899, 33, 9], [6, 8, 3]), ([900, 1500, 64], [0, 0, 1])):
        p.cache.lens, p.drafts = lens, drafts
        p.cache.d_lens.copy_(int32(lens))
        p.d_first.copy_(int32(np.concatenate([[0], np.cumsum(drafts)])))
        p.sees = [x for c in drafts for x in tree(c, rng)]
        p.d_sees[:len(p.sees)] = bits_of(p.sees, 1)
        T = sum(drafts)
        p.out.fill_(5)
        graph.replay()
        torch.cuda.synchronize()
        near((p.out[:T].cpu(), p.lse[:T].cpu()), p.want(q=p.q[:T]), "bf16")
        assert bool((p.out[T:] == 5).all())
        near((p.run()[0][:T], p.lse[:T].cpu()), p.want(q=p.q[:T]), "bf16")  # eager work between the replays
    assert int(p.cache.status) == 0


@pytest.mark.parametrize("kind,cache", [("bf16", "bf16"), ("f16", "f8")])
@pytest.mark.parametrize("D", [48, 64, 128, 192])
@pytest.mark.parametrize("pt", [1, 8])
def test_many_rows_over_small_pages(pt, D, kind, cache):
    """20 to 280 query rows of a cache head, over pages of fewer tokens than a tile's half, in parts and with a window."""
    check([300, 77, 70], [5, 2, 3], 4, 1, D, kind=kind, cache=cache, pt=pt)
    check([700, 333], [70, 40], 4, 1, D, kind=kind, cache=cache, pt=pt, order="head")
    check([400, 90], [12, 40], 4, 1, D, kind=kind, cache=cache, pt=pt, window=100, shape="chain")


@pytest.mark.parametrize("drafts", [[12, 3], [40, 9]])
@pytest.mark.parametrize("pt,cache", [(16, "bf16"), (16, "f8"), (4, "bf16"), (4, "f8")])
def test_pages_that_are_none_under_many_rows(pt, cache, drafts):
    p = Drafts([300, 140], drafts, 4, 1, 64, cache=cache, pt=pt, seed=3)
    c = p.cache
    table = c.table.copy()
    table[0, 0], table[0, 96 // pt], table[1, 139 // pt] = -1, c.n_pages, 1 << 30  # the first, one inside a plain tile, the last
    c.d_table.copy_(torch.from_numpy(table))
    got = p.run()
    assert got[2] == od.ST_BAD_INDEX
    near(got, p.want(table=table), "bf16")


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("drafts", [[2, 1], [40, 9]])
def test_scores_that_grow_along_the_row(drafts, kind):
    """Every tile's scores are larger than all before by half a power of two to several: the sums are brought to a new maximum, or not yet."""
    for step in (0.05, 0.3, 1.0):
        p = Drafts([400, 260], drafts, 4, 2, 64, kind=kind, scale=1.0, shape="chain")
        c = p.cache
        p.q[:] = 0
        p.q[:, :, 0] = 1
        p.d_q.copy_(p.q)
        for r, n in enumerate(c.lens):
            for t in range(n):
                c.views[0][c.table[r, t // 16], t % 16] = 0
                c.views[0][c.table[r, t // 16], t % 16, :, 0] = step * (t // 8)
        c.upload()
        got = p.run()
        assert got[2] == 0
        near(got, p.want(), kind)  # (one product a score, of at most 50: exact but for the factor's 2^-23 of it)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("drafts", [[2, 1], [40, 9]])
def test_values_near_the_end_of_the_range(drafts, kind):
    """Weights of one row add up to 1 in the result, whatever they are held as: a value of three quarters of the largest finite one, the
    same of all tokens, comes out as it is."""
    p = Drafts([100, 70], drafts, 4, 2, 64, kind=kind, scale=8.0)
    c = p.cache
    big = torch.tensor(torch.finfo(DTYPES[kind]).max * 0.75 / (128 if kind == "bf16" else 1)).to(DTYPES[kind])  # (the sum of 100 is held in 32 bits)
    for r, n in enumerate(c.lens):
        for t in range(n):
            c.views[1][c.table[r, t // 16], t % 16] = big
    c.upload()
    out, lse, status = p.run()
    assert status == 0
    assert bool(((out.double() - big.double()).abs() <= float(big) * (2.0 ** -8 + 2.0 ** -12)).all())
