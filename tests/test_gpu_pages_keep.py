"""fdy_pages_keep through the C ABI against the same on plain lists: books and contents equal to the bit."""
import numpy as np
import pytest
import torch

import oracle.decode as od
from paper_2604_06664_amd import decode as fdd
from tests.support.paged import DEV, int32

pytestmark = pytest.mark.gpu


class Pool:
    """Planes of [page][piece][token][words of a piece] (heads first) or [page][token][piece][words], and the oracle's of
    [page][token][words]."""

    def __init__(self, lens, pt=16, n_planes=3, pieces=2, words=4, order="token", pad=0, share=(), seed=1, spare=5):
        rng = np.random.default_rng(seed)
        pages = [-(-n // pt) for n in lens]
        n_pages = sum(pages) + spare
        table, refs = np.full((len(lens), max(pages + [1]) + 1), -5, np.int64), np.zeros(n_pages, int)
        order_of, at = rng.permutation(n_pages), 0
        for r, n in enumerate(pages):
            table[r, :n] = order_of[at:at + n]
            at += n
        for r, j, of in share:  # row r's page j is row of's
            table[r, j] = table[of, j]
        for r, n in enumerate(pages):
            np.add.at(refs, table[r, :n], 1)
        wide = words + pad
        self.shape = (n_planes, n_pages, pt, pieces, wide) if order == "token" else (n_planes, n_pages, pieces, pt, wide)
        raw = rng.integers(-1 << 31, 1 << 31, self.shape, dtype=np.int64).astype(np.int32)
        self.order, self.words, self.raw = order, words, raw
        self.want = od.Books(refs, table, lens, pt, self.tokens(raw))
        self.d = torch.from_numpy(raw.copy()).to(DEV)
        self.refs, self.table, self.lens = int32(refs.tolist()), torch.from_numpy(self.want.table.copy()).to(DEV), int32(list(lens))
        self.bits = torch.from_numpy(self.want.free_bits().view(np.int64).copy()).to(DEV)
        self.addr = torch.tensor([p.data_ptr() for p in self.d], dtype=torch.int64, device=DEV) if n_planes else None
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        of_page = pt * pieces * wide * 4
        self.desc = fdd.make_pages(refs=self.refs, free_bits=self.bits, table=self.table, lens=self.lens, page_tokens=pt, planes=self.addr,
                                   page_bytes=of_page, page_stride=of_page)
        token, piece = (pieces * wide * 4, wide * 4) if order == "token" else (wide * 4, pt * wide * 4)
        self.token = fdd.make_token(token_stride=token, piece_bytes=words * 4, pieces=pieces, piece_stride=piece)

    def tokens(self, raw):
        x = raw if self.order == "token" else raw.swapaxes(2, 3)
        return x[..., :self.words]

    def keep(self, rows, drafts, lists, most=None, kept=None):
        n, most = len(rows), most or max([len(x) for x in lists] + [1])
        keep = torch.full((n, most), -77, dtype=torch.int32, device=DEV)
        for i, x in enumerate(lists):
            if x:
                keep[i, :len(x)] = int32([int(k) for k in x[:most]])
        size = fdd.fdy_pages_workspace_bytes(self.desc, n)
        ws = torch.randint(0, 256, (size,), dtype=torch.uint8, device=DEV)
        fdd.fdy_pages_keep(self.desc, self.token, int32(rows), int32(drafts), keep, int32([len(x) for x in lists] if kept is None else kept),
                           n, most, ws, size, self.status)
        od.keep(self.want, rows, drafts, lists)
        self.same()

    def same(self):
        torch.cuda.synchronize()
        w = self.want
        assert self.refs.cpu().tolist() == w.refs
        assert np.array_equal(self.bits.cpu().numpy().view(np.uint64), w.free_bits())
        assert np.array_equal(self.table.cpu().numpy(), w.table) and self.lens.cpu().tolist() == w.lens
        assert int(self.status) == w.status
        if self.shape[0]:
            got = self.d.cpu().numpy()
            assert np.array_equal(self.tokens(got), w.planes)
            x, y = (v if self.order == "token" else v.swapaxes(2, 3) for v in (got, self.raw))
            assert np.array_equal(x[..., self.words:], y[..., self.words:])  # what lies between pieces


@pytest.mark.parametrize("order,pad", [("token", 0), ("token", 4), ("head", 0), ("head", 8)])
@pytest.mark.parametrize("pt", [1, 4, 16, 64])
def test_paths(pt, order, pad):
    p = Pool([40, 7, 100, 33, 64], pt=pt, order=order, pad=pad)
    p.keep([0, 1, 2, 3, 4], [26, 7, 8, 1, 20], [[0, 2, 7, 15, 16], [], [0, 1, 2], [0], [19]])
    p.keep([4, 2], [5, 95], [[1, 3, 4], [0, 94]])  # again, on what is left
    assert p.want.status == 0


@pytest.mark.parametrize("kept", [0, 1, 7, 8, 9, 16, 17, 40])
def test_numbers_that_are_kept(kept):
    rng = np.random.default_rng(kept)
    p = Pool([300, 90, 64], n_planes=2, pieces=1, words=20)
    lists = [sorted(rng.permutation(c)[:kept].tolist()) for c in (290, 90, 41)]
    p.keep([0, 1, 2], [290, 90, 41], lists)
    assert p.want.status == 0


def test_whole_rows():
    p = Pool([64, 17, 0, 5], n_planes=1)
    p.keep([0, 1, 2, 3], [64, 17, 0, 5], [list(range(64)), [], [], list(range(5))])
    assert p.want.lens == [64, 0, 0, 5] and p.want.status == 0


def test_first_and_last_tokens_of_long_rows():
    p = Pool([5000, 3001], n_planes=2, pieces=4, words=32, order="head", pt=32)
    p.keep([0, 1], [5000, 2990], [list(range(4)) + list(range(4000, 5000)), list(range(0, 2990, 3))])
    assert p.want.status == 0


def test_books_alone():
    p = Pool([40, 50], n_planes=0)
    p.keep([0, 1], [39, 20], [[3, 5], [0, 19]])
    assert p.want.status == 0


def test_shared_pages():
    """Pages ahead of the drafted tokens may be shared, and those that are given up; one that would be written to may not."""
    p = Pool([50, 50, 50], share=[(1, 0, 0), (1, 1, 0), (2, 3, 0)])
    p.keep([1, 0], [10, 3], [[4, 9], [0]])  # row 1 writes to its page 2, its own; row 0 gives up none
    assert p.want.status == 0
    p = Pool([50, 50, 50], share=[(1, 2, 0), (2, 3, 0)])
    p.keep([0, 1, 2], [10, 30, 9], [[4, 9], [3, 8], [0]])  # row 0 would write to the page 2 that it shares; row 1 writes ahead of it
    assert p.want.status == od.ST_CAPACITY and p.want.lens == [50, 22, 42]
    p = Pool([50, 50, 50], share=[(1, 2, 0), (2, 3, 0)])
    p.keep([0, 1, 2], [10, 10, 9], [[4, 9], [3, 8], [0]])  # rows 0 and 1 would write to their common page 2
    assert p.want.status == od.ST_CAPACITY and p.want.lens == [50, 50, 42]
    p = Pool([50, 50], share=[(1, 3, 0)])
    p.keep([0, 1], [10, 10], [[0], [0, 1]])  # both give up the page that they share: it is free
    assert p.want.status == 0 and p.want.lens == [41, 42]


@pytest.mark.parametrize("rows,drafts,lists,kept", [
    ([0, 3, -1], [5, 5, 5], [[1], [1], [1]], None), ([0, 0, 1], [5, 6, 5], [[1], [2], [3]], None), ([0, 1], [-1, 5], [[], [4]], None),
    ([0, 1], [51, 5], [[1], [4]], None), ([0, 1], [5, 5], [[1, 1], [4]], None), ([0, 1], [5, 5], [[3, 2], [4]], None),
    ([0, 1], [5, 5], [[-1, 2], [4]], None), ([0, 1], [5, 5], [[5], [4]], None), ([0, 1], [2, 5], [[0, 1, 2], [4]], None)])
def test_what_is_left_as_it_is(rows, drafts, lists, kept):
    p = Pool([50, 50, 9])
    p.keep(rows, drafts, lists, kept=kept)
    assert p.want.status == od.ST_BAD_INDEX


def test_counts_out_of_range():
    p = Pool([50, 50])
    for kept in ([-1, 2], [4, 2]):
        q = torch.zeros(2, 3, dtype=torch.int32, device=DEV) + int32([0, 2, 4])
        n = fdd.fdy_pages_workspace_bytes(p.desc, 2)
        ws = torch.empty(n, dtype=torch.uint8, device=DEV)
        p.status.zero_()
        fdd.fdy_pages_keep(p.desc, p.token, int32([0, 1]), int32([6, 6]), q, int32(kept), 2, 3, ws, n, p.status)
        od.keep(p.want, [1], [6], [[0, 2]])
        p.want.status = od.ST_BAD_INDEX
        p.same()


def test_page_numbers_out_of_range():
    for j, page in ((2, -1), (3, 1 << 20)):
        p = Pool([50, 50])
        p.want.table[0, j] = page
        p.table[0, j] = page
        p.keep([0, 1], [15, 3], [[4, 14], [2]])
        assert p.want.status == od.ST_BAD_INDEX and p.want.lens == [50, 48]


def test_replays():
    """Captured on a stream of its own; books and contents change between the replays."""
    p = Pool([60, 90, 31], n_planes=4)
    n = fdd.fdy_pages_workspace_bytes(p.desc, 3)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    rows, drafts, keep, kept = int32([0, 1, 2]), int32([0, 0, 0]), torch.zeros(3, 8, dtype=torch.int32, device=DEV), int32([0, 0, 0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fdd.fdy_pages_keep(p.desc, p.token, rows, drafts, keep, kept, 3, 8, ws, n, p.status)
    for c, lists in (([9, 5, 7], [[0, 3, 8], [4], [0, 1]]), ([0, 20, 1], [[], [2, 3, 19], []]), ([30, 1, 1], [[1, 2, 9, 28], [0], [0]])):
        drafts.copy_(int32(c))
        kept.copy_(int32([len(x) for x in lists]))
        for i, x in enumerate(lists):
            keep[i, :len(x)] = int32(x) if x else keep[i, :0]
        graph.replay()
        od.keep(p.want, [0, 1, 2], c, lists)
        p.same()
