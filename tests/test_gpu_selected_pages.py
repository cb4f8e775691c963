"""fdy_page_bounds, fdy_page_select and fdy_selected_attention through the C ABI: bounds and choices equal to the oracle's, attention as
tests/support/paged.py allows."""
import math

import numpy as np
import pytest
import torch

import oracle.decode as od
from paper_2604_06664_amd import decode as fdd
from tests.support.paged import DEV, DTYPES, Cache, int32, near

pytestmark = pytest.mark.gpu
TYPES = ["bf16", "f16", "f8"]


# ---- bounds -------------------------------------------------------------------------------------
def run_bounds(c, fresh, max_fresh=1 << 20, rows=None, kv=None, table=None, lens=None, n_pages=None):
    want = torch.full((n_pages or c.n_pages, c.H, 2, c.D), 7.0, dtype=torch.float64)
    bounds = want.to(DTYPES[c.cache]).to(DEV)
    od.page_bounds(want, c.views[0], c.table if table is None else table, c.lens if lens is None else lens,
                   [1] * len(c.lens) if fresh is None else fresh, max_fresh, rows)
    desc = fdd.make_bounds_desc(bounds=bounds, table=c.d_table, lens=c.d_lens, kv=kv or c.kv(), max_fresh=min(max_fresh, 1 << 20),
                                fresh=None if fresh is None else int32(fresh), rows=None if rows is None else int32(rows))
    fdd.fdy_page_bounds(desc, c.status)
    torch.cuda.synchronize()
    got = bounds.cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got, 9.0, 1e9, -1e9), torch.nan_to_num(want, 9.0, 1e9, -1e9))
    return int(c.status)


@pytest.mark.parametrize("cache", TYPES)
@pytest.mark.parametrize("D", [16, 48, 64, 80, 128, 192, 256])
def test_bounds_of_all_pages(D, cache):
    lens = [0, 1, 2, 15, 16, 17, 33, 64, 100]
    assert run_bounds(Cache(lens, 3, D, cache=cache), lens) == 0


@pytest.mark.parametrize("D", [8, 24, 136, 248])
def test_bounds_of_heads_that_are_odd_multiples_of_8(D):
    assert run_bounds(Cache([40, 9], 2, D, cache="f16"), [40, 9]) == 0


@pytest.mark.parametrize("order", ["token", "head"])
@pytest.mark.parametrize("pt", [1, 2, 4, 16, 64, 512])
def test_bounds_of_new_tokens(pt, order):
    c = Cache([1, 17, 40, 129, 200, 0, 64], 2, 64, pt=pt, order=order, pad=8)
    assert run_bounds(c, [1, 17, 3, 129, 65, 4, 0]) == 0
    assert run_bounds(c, None) == 0
    assert run_bounds(c, [2] * 7, max_fresh=2) == 0


def test_bounds_of_rows_of_a_larger_pool_and_numbers_out_of_range():
    c = Cache([40, 0, 100, 33], 2, 64)
    assert run_bounds(c, [40, 7, 33], rows=[0, 2, 3]) == 0
    assert run_bounds(c, [40, 7, 40, 3], rows=[0, 2, 0, 2]) == 0  # a row twice
    for fresh, most, rows in (([-1, 5, 9, 3], 1 << 20, None), ([40, 5, 90, 3], 10, None), ([1, 1, 1, 1], 1, [0, 4, -1, 3])):
        c.status.zero_()
        assert run_bounds(c, fresh, max_fresh=most, rows=rows) == od.ST_BAD_INDEX
    c.status.zero_()
    table, lens = c.table.copy(), [40, -5, 1 << 29, 33]
    table[0, 1] = -3
    table[3, 0] = c.n_pages
    c.d_table.copy_(torch.from_numpy(table))
    c.d_lens.copy_(int32(lens))
    assert run_bounds(c, [40, 1, 1, 33], table=table, lens=lens) == od.ST_BAD_INDEX


@pytest.mark.parametrize("cache", TYPES)
def test_bounds_of_infinities_and_no_numbers(cache):
    c = Cache([40, 33], 2, 64, cache=cache)
    k = c.views[0]
    k[c.table[0, 0], 3, 1, 5] = math.nan
    if cache != "f8":
        k[c.table[0, 1], 0, 0, 7], k[c.table[1, 0], 4, 1, 8] = math.inf, -math.inf
    c.upload()
    assert run_bounds(c, [40, 33]) == 0


def test_bounds_behind_32_bits():
    c = Cache([60], 1, 64, spare=0)
    ps, n = 1 << 29, 7
    pool = torch.empty(n * ps // 2, dtype=torch.int32, device=DEV).view(torch.int16)
    moved = torch.zeros(n, 16, 1, 64, dtype=torch.bfloat16)
    for j in range(4):
        moved[n - 1 - j] = c.views[0][j]
        pool[(n - 1 - j) * ps:(n - 1 - j) * ps + 16 * 64] = c.views[0][j].reshape(-1).view(torch.int16).to(DEV)
    c.views[0] = moved
    c.table = np.where(c.table >= 0, n - 1 - c.table, -1).astype(np.int32)
    c.d_table = torch.from_numpy(c.table).to(DEV)
    kv = fdd.make_kv(pool, None, type=fdd.FDY_BF16, n_pages=n, page_tokens=16, n_heads=1, head_dim=64, page_stride=ps, token_stride=64,
                     head_stride=64)
    assert run_bounds(c, [60], kv=kv, n_pages=n) == 0


# ---- the choice ---------------------------------------------------------------------------------
class Choice:
    def __init__(self, lens, Hq, H, D, pt=16, kind="bf16", cache=None, seed=3, row_pages=None):
        rng = np.random.default_rng(seed)
        cache = cache or kind
        pages = [-(-n // pt) for n in lens]
        P = row_pages or max(pages + [1]) + 2
        self.n_pages, self.lens, self.pt, self.H = sum(pages) + 3, list(lens), pt, H
        self.table = np.full((len(lens), P), -1, np.int32)
        order, at = rng.permutation(self.n_pages), 0
        for r, n in enumerate(pages):
            self.table[r, :n] = order[at:at + n]
            at += n
        x = torch.from_numpy(rng.standard_normal((2, self.n_pages, H, D)).astype(np.float32))
        self.bounds = torch.stack([x.amin(0), x.amax(0)], 2).to(DTYPES[cache])
        self.q = torch.from_numpy(rng.standard_normal((len(lens), Hq, D)).astype(np.float32)).to(DTYPES[kind])
        self.k_scale = torch.from_numpy(rng.uniform(0.5, 1.5, H).astype(np.float32)) if cache == "f8" else None
        self.cache, self.D = cache, D
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)

    def desc(self, budget, sinks=1, recent=1, rows=None, q=None):
        n = len(self.lens) if rows is None else len(rows)
        self.d = [self.bounds.to(DEV), torch.from_numpy(self.table).to(DEV), int32(self.lens), None if rows is None else int32(rows),
                  None if self.k_scale is None else self.k_scale.to(DEV), self.q[:n].to(DEV) if q is None else q]
        self.pages, self.seen = torch.full((n, self.H, budget), -9, dtype=torch.int32, device=DEV), torch.full((n,), -9, dtype=torch.int32, device=DEV)
        kv = fdd.make_kv(None, None, type=fdd.TYPES[self.cache], n_pages=self.n_pages, page_tokens=self.pt, n_heads=self.H, head_dim=self.D,
                         page_stride=0, token_stride=0, head_stride=0, k_scale=self.d[4])
        desc = fdd.make_select_desc(q=self.d[5], bounds=self.d[0], table=self.d[1], lens=self.d[2], kv=kv, pages=self.pages,
                                    seen=self.seen, sinks=sinks, recent=recent, rows=self.d[3])
        n = fdd.fdy_page_select_workspace_bytes(desc)
        return desc, torch.randint(0, 256, (n,), dtype=torch.uint8, device=DEV), n  # contents are irrelevant

    def check(self, budget, sinks=1, recent=1, rows=None, q=None):
        fdd.fdy_page_select(*self.desc(budget, sinks, recent, rows, q), self.status)
        torch.cuda.synchronize()
        pages, seen = od.page_select(self.q if rows is None else self.q[:len(rows)], self.bounds, self.table, self.lens, self.pt, budget,
                                     sinks, recent, rows, self.k_scale)
        assert self.seen.cpu().tolist() == seen.tolist()
        assert np.array_equal(self.pages.cpu().numpy(), pages), np.argwhere(self.pages.cpu().numpy() != pages)[:5]
        return int(self.status)


@pytest.mark.parametrize("kind,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "f8"), ("f16", "f8")])
@pytest.mark.parametrize("D", [16, 64, 80, 128, 192, 256])
def test_choices(D, kind, cache):
    c = Choice([0, 1, 16, 17, 300, 511, 512, 513, 97], 4, 2, D, kind=kind, cache=cache)
    for budget in (2, 5, 18, 33):
        assert c.check(budget) == 0


@pytest.mark.parametrize("D", [8, 24, 136])
def test_choices_for_heads_that_are_odd_multiples_of_8(D):
    assert Choice([300, 90], 3, 3, D, kind="f16").check(4) == 0


@pytest.mark.parametrize("Hq,H", [(1, 1), (7, 1), (5, 5), (24, 2), (9, 9), (40, 40), (64, 1)])
def test_choices_for_groups(Hq, H):
    assert Choice([300, 1000], Hq, H, 64).check(6) == 0
    assert Choice([300], Hq, H, 128, cache="f8").check(6) == 0


@pytest.mark.parametrize("sinks,recent,budget", [(0, 1, 1), (0, 1, 2), (3, 4, 7), (3, 4, 8), (0, 12, 13), (12, 1, 20)])
def test_pages_that_are_always_taken(sinks, recent, budget):
    assert Choice([0, 5, 100, 112, 113, 128, 400, 1111], 4, 2, 64).check(budget, sinks, recent) == 0


@pytest.mark.parametrize("pt", [1, 4, 64, 1024])
def test_choices_over_page_sizes(pt):
    assert Choice([0, 1, pt * 9 + 1, pt * 20, pt * 33 - 1], 2, 2, 64, pt=pt).check(7) == 0


@pytest.mark.parametrize("budget", [3, 1500, 2900])
def test_long_rows(budget):
    assert Choice([3000 * 4 - 1, 2049 * 4, 17], 2, 1, 16, pt=4, kind="f16").check(budget) == 0


def test_rows_of_a_wide_table():
    assert Choice([300, 40], 4, 2, 64, row_pages=5000).check(5) == 0


def test_equal_scores_go_to_the_first():
    c = Choice([16 * 40] * 3, 4, 2, 64)
    b = c.bounds.clone()
    for r, kinds in enumerate((1, 2, 3)):  # pages of so many kinds
        for j in range(40):
            b[c.table[r, j]] = b[c.table[r, (j * 7) % kinds]]
    c.bounds = b
    for budget in (2, 3, 17, 22, 39):
        assert c.check(budget) == 0
    c.q[:] = 0
    assert c.check(9) == 0


def test_scores_one_step_apart():
    """All scores within a few of the last bits of 64."""
    c = Choice([16 * 64], 1, 1, 64, kind="f16")
    c.q[:] = 0
    c.q[0, 0, 0], c.q[0, 0, 1] = 32768.0, 2.0 ** -24
    c.bounds[:] = 0
    for j in range(64):
        c.bounds[c.table[0, j], 0, 1, 0] = 32768.0
        c.bounds[c.table[0, j], 0, 1, 1] = float((j * 37) % 64) * 2.0 ** 3
    for budget in (2, 9, 30):
        assert c.check(budget) == 0


def test_infinities_and_no_numbers():
    c = Choice([16 * 40] * 5, 2, 1, 64)
    inf, b, t = math.inf, c.bounds, c.table
    b[t[0, 5], 0, 1, 3], b[t[0, 9], 0, 0, 3] = inf, -inf
    b[t[1, 7], 0, :, 4], b[t[1, 8], 0, 0, 9], b[t[1, 20], 0, 1, 9] = math.nan, math.nan, inf
    b[t[2, 3:30], 0, 1] = -inf
    b[t[2, 3:30], 0, 0] = -inf
    c.q[3, 0, 5], c.q[3, 1, 6] = math.nan, 0.0
    c.q[4, :, 7] = 0.0  # what a query does not look at does not count
    b[t[4, 11], 0, 1, 7] = inf
    for budget in (3, 4, 6, 30):
        assert c.check(budget) == 0


def test_negative_scales():
    c = Choice([16 * 40] * 2, 4, 2, 64, cache="f8")
    c.k_scale = torch.tensor([-0.7, 0.0])
    assert c.check(9) == 0


def test_numbers_out_of_range_of_the_choice():
    c = Choice([300, 400, 500, 90], 4, 2, 64)
    c.table[0, 3], c.table[1, 0], c.table[2, 31] = -4, c.n_pages, 1 << 30
    assert c.check(5) == od.ST_BAD_INDEX
    c.status.zero_()
    assert c.check(5, rows=[3, 3]) == 0
    assert c.check(5, rows=[3, 4, -1]) == od.ST_BAD_INDEX
    c.status.zero_()
    c.lens = [-1, 1 << 30, 500, 90]
    c.table[1] = c.table[1].clip(0)
    assert c.check(5) == od.ST_BAD_INDEX


def test_strided_queries():
    c = Choice([300, 400], 4, 2, 64)
    wide = torch.zeros(4, 2, 72, dtype=torch.bfloat16, device=DEV)
    q = wide.transpose(0, 1)[:, :, :64]
    q.copy_(c.q)
    assert c.check(5, q=q) == 0


def test_bounds_of_the_pool_behind_32_bits():
    """Bounds of 2^23 pages of one head of 256 elements are 8 GiB; the row's pages are the last ones."""
    c = Choice([16 * 12], 1, 1, 256)
    n = 1 << 23
    big = torch.empty(n, 1, 2, 256, dtype=torch.bfloat16, device=DEV)
    big[n - c.n_pages:] = c.bounds.to(DEV)
    desc, ws, size = c.desc(5)
    table = torch.from_numpy(np.where(c.table >= 0, c.table + n - c.n_pages, -1).astype(np.int32)).to(DEV)
    desc.bounds, desc.table, desc.kv.n_pages = big.data_ptr(), table.data_ptr(), n
    fdd.fdy_page_select(desc, ws, size, c.status)
    torch.cuda.synchronize()
    pages, seen = od.page_select(c.q, c.bounds, c.table, c.lens, 16, 5, 1, 1)
    assert np.array_equal(c.pages.cpu().numpy(), pages + n - c.n_pages) and c.seen.cpu().tolist() == seen.tolist()


def test_choices_replayed_while_rows_grow():
    c = Choice([500, 300, 64], 4, 2, 64)
    desc, ws, size = c.desc(6)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fdd.fdy_page_select(desc, ws, size, c.status)
    for lens in ([1, 0, 3], [500, 300, 64], [97, 96, 33], [500, 299, 63]):
        c.lens = lens
        c.d[2].copy_(int32(lens))
        graph.replay()
        torch.cuda.synchronize()
        pages, seen = od.page_select(c.q, c.bounds, c.table, lens, 16, 6, 1, 1)
        assert np.array_equal(c.pages.cpu().numpy(), pages) and c.seen.cpu().tolist() == seen.tolist()
        fdd.fdy_page_select(desc, ws, size, c.status)  # eager between the replays
        assert np.array_equal(c.pages.cpu().numpy(), pages)


# ---- attention over lists of pages --------------------------------------------------------------
class Selected:
    """A list of pages of its own for every cache head; entries behind it lead nowhere."""

    def __init__(self, lens, Hq, H, D, kind="bf16", cache=None, seed=5, row_pages=None, window=0, **kw):
        rng = np.random.default_rng(seed)
        self.c = c = Cache([4096], H, D, cache=cache or kind, seed=seed, **kw)
        self.kind, self.lens, self.window, self.scale = kind, list(lens), window, D ** -0.5
        pages = [-(-n // c.pt) for n in lens]
        self.table = np.full((len(lens), H, row_pages or max(pages + [1]) + 1), -1, np.int32)
        held = c.table[0, :4096 // c.pt]
        for r, n in enumerate(pages):
            for h in range(H):
                self.table[r, h, :n] = rng.permutation(held)[:n]
        self.q = torch.from_numpy(rng.standard_normal((len(lens), Hq, D)).astype(np.float32)).to(DTYPES[kind])
        self.out = torch.full((len(lens), Hq, D), 5.0, dtype=DTYPES[kind], device=DEV)
        self.lse = torch.full((len(lens), Hq), 5.0, device=DEV)
        self.ws = None

    def run(self, table=None, lens=None, **kw):
        self.held = [self.q.to(DEV), torch.from_numpy(self.table if table is None else table).to(DEV), int32(self.lens if lens is None else lens)]
        desc = fdd.make_selected_desc(q=self.held[0], out=self.out, lse=self.lse, table=self.held[1], lens=self.held[2], kv=self.c.kv(),
                                      scale=self.scale, window=self.window, **kw)
        n = fdd.fdy_selected_attention_workspace_bytes(desc)
        if self.ws is None:
            self.ws = torch.zeros(n, dtype=torch.uint8, device=DEV)
        fdd.fdy_selected_attention(desc, self.ws, n, self.c.status)
        torch.cuda.synchronize()
        return self.out.cpu(), self.lse.cpu(), int(self.c.status)

    def want(self, table=None, lens=None, rows=None):
        """One head after the other as if it had a cache of its own."""
        c, table = self.c, self.table if table is None else table
        group, parts = self.q.shape[1] // c.H, []
        for h in range(c.H):
            scales = [None if s is None else s[h:h + 1] for s in c.scales]
            parts.append(od.attend(self.q[:, h * group:(h + 1) * group], *(v[:, :, h:h + 1] for v in c.views), table[:, h],
                                   self.lens if lens is None else lens, self.scale, self.window, rows, *scales))
        return [torch.cat(x, 1) for x in zip(*parts)]


@pytest.mark.parametrize("kind,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "f8"), ("f16", "f8")])
@pytest.mark.parametrize("D", [64, 80, 128, 256])
def test_lists_around_tiles(D, kind, cache):
    p = Selected([0, 1, 15, 16, 17, 31, 32, 33, 64, 65, 130, 257], 4, 2, D, kind=kind, cache=cache)
    got = p.run()
    assert got[2] == 0
    near(got, p.want(), kind)


@pytest.mark.parametrize("order", ["token", "head"])
@pytest.mark.parametrize("pt", [1, 4, 8, 32, 256])
def test_lists_of_pages_of_many_sizes(pt, order):
    p = Selected([5, 100, 0, 300], 8, 4, 64, pt=pt, order=order)
    near(p.run(), p.want(), "bf16")


@pytest.mark.parametrize("Hq,H", [(1, 1), (12, 12), (40, 2), (64, 4), (100, 1)])
def test_lists_for_groups(Hq, H):
    for row_pages in (None, 512):
        p = Selected([1700, 5, 0, 333], Hq, H, 64, row_pages=row_pages)
        got = p.run()
        near(got, p.want(), "bf16")
        again = p.run()
        assert torch.equal(got[0].view(torch.int16), again[0].view(torch.int16)) and torch.equal(got[1], again[1])


def test_lists_and_windows():
    p = Selected([5, 100, 0, 300], 4, 2, 64, window=70)
    near(p.run(), p.want(), "bf16")


def test_lists_out_of_range():
    p = Selected([50, 100, 20, 300], 4, 2, 64)
    table, lens = p.table.copy(), [50, 100, -2, 300]
    table[0, 1, 0], table[1, 0, 3] = -5, p.c.n_pages
    got = p.run(table=table, lens=lens)
    assert got[2] == od.ST_BAD_INDEX
    near(got, p.want(table=table, lens=lens), "bf16")
    p.c.status.zero_()
    rows = [3, 4, -1, 0]
    got = p.run(rows=int32(rows))
    assert got[2] == od.ST_BAD_INDEX
    near(got, p.want(rows=rows), "bf16")


# ---- all of them --------------------------------------------------------------------------------
@pytest.mark.parametrize("cache", ["bf16", "f8"])
def test_bounds_then_choice_then_attention(cache):
    """Keys of a few pages match the query; with a budget of a quarter of the pages attention over the chosen ones is attention over
    all but for what the others weigh, which the sums of both say; with all pages it is the same attention."""
    lens, H, Hq, D = [1000, 700, 100, 0], 2, 8, 64
    c = Cache(lens, H, D, cache=cache)
    rng = np.random.default_rng(8)
    q = torch.from_numpy(rng.standard_normal((4, Hq, D)).astype(np.float32)).to(torch.bfloat16)
    for r, n in enumerate(lens):  # keys along the group's queries on three pages
        for j in (3, 7, 20):
            if (j + 1) * 16 <= n:
                for h in range(H):
                    c.views[0][c.table[r, j], :, h] = (q[r, h * 4:(h + 1) * 4].float().mean(0) * 12).to(DTYPES[cache])
    c.upload()
    bounds = torch.zeros(c.n_pages, H, 2, D, dtype=DTYPES[cache], device=DEV)
    d_q = q.to(DEV)
    fdd.fdy_page_bounds(fdd.make_bounds_desc(bounds=bounds, table=c.d_table, lens=c.d_lens, kv=c.kv(), fresh=c.d_lens, max_fresh=1000), c.status)
    full = od.attend(q, *c.views, c.table, lens, D ** -0.5, 0, None, *c.scales)
    for budget in (16, 80):
        pages, seen = torch.empty(4, H, budget, dtype=torch.int32, device=DEV), torch.empty(4, dtype=torch.int32, device=DEV)
        desc = fdd.make_select_desc(q=d_q, bounds=bounds, table=c.d_table, lens=c.d_lens, kv=c.kv(), pages=pages, seen=seen)
        ws = torch.empty(fdd.fdy_page_select_workspace_bytes(desc), dtype=torch.uint8, device=DEV)
        fdd.fdy_page_select(desc, ws, ws.numel(), c.status)
        out, lse = torch.empty(4, Hq, D, dtype=torch.bfloat16, device=DEV), torch.empty(4, Hq, device=DEV)
        at = fdd.make_selected_desc(q=d_q, out=out, lse=lse, table=pages, lens=seen, kv=c.kv(), scale=D ** -0.5)
        aw = torch.zeros(fdd.fdy_selected_attention_workspace_bytes(at), dtype=torch.uint8, device=DEV)
        fdd.fdy_selected_attention(at, aw, aw.numel(), c.status)
        torch.cuda.synchronize()
        assert int(c.status) == 0
        got = out.cpu(), lse.cpu()
        if budget == 80:
            near(got, full, "bf16")
            continue
        for r, n in enumerate(lens):
            for h in range(H):
                for j in (3, 7, 20):
                    assert (j + 1) * 16 > n or int(c.table[r, j]) in pages[r, h].tolist()
        some = full[1] > -math.inf
        missing = 1 - torch.exp(got[1].double() - full[1])[some]  # the share of the weights that was left out
        assert bool((missing >= -1e-3).all()) and float(missing.max()) < 0.9
        err = (got[0].double() - full[0]).abs().amax(-1)[some]
        assert bool((err <= 2 * missing.clamp(min=0) * full[2][some] + (2.0 ** -8 + 2.0 ** -9) * full[2][some]).all())
