"""fdy_pages_* through the C ABI against the same calls done one entry after the other on plain lists: books and contents
equal to the bit."""
import numpy as np
import pytest
import torch

import oracle.decode as od
from paper_2604_06664_amd import decode as fdd

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Pool:
    """A pool on the device and its oracle; every call is made on both and compared."""

    def __init__(self, refs, table, lens, pt, n_planes=0, page_bytes=48, stride=64, seed=0):
        rng = np.random.default_rng(seed)
        n_pages = len(refs)
        planes = rng.integers(0, 1 << 31, (n_planes, n_pages, stride // 4), dtype=np.int64).astype(np.int32) if n_planes else None
        self.page_bytes, self.stride = page_bytes, stride
        self.want = od.Books(refs, table, lens, pt, None if planes is None else planes[:, :, :page_bytes // 4])
        self.between = None if planes is None else planes[:, :, page_bytes // 4:].copy()
        self.refs = torch.from_numpy(np.array(refs, np.int32)).to(DEV)
        self.bits = torch.from_numpy(self.want.free_bits().view(np.int64).copy()).to(DEV)
        self.table = torch.from_numpy(np.array(table, np.int32)).to(DEV)
        self.lens = torch.from_numpy(np.array(lens, np.int32)).to(DEV)
        self.planes = None if planes is None else [torch.from_numpy(p.copy()).to(DEV) for p in planes]
        self.addr = None if planes is None else torch.tensor([p.data_ptr() for p in self.planes], dtype=torch.int64, device=DEV)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.desc = fdd.make_pages(refs=self.refs, free_bits=self.bits, table=self.table, lens=self.lens, page_tokens=pt,
                                   planes=self.addr, page_bytes=page_bytes, page_stride=stride)

    def ws(self, n):
        n = fdd.fdy_pages_workspace_bytes(self.desc, n)
        return torch.randint(0, 256, (n,), dtype=torch.uint8, device=DEV), n  # contents are irrelevant

    def same(self):
        torch.cuda.synchronize()
        assert self.refs.cpu().tolist() == self.want.refs
        assert np.array_equal(self.bits.cpu().numpy().view(np.uint64), self.want.free_bits())
        assert np.array_equal(self.table.cpu().numpy(), self.want.table)
        assert self.lens.cpu().tolist() == self.want.lens
        assert int(self.status) == self.want.status
        if self.planes is not None:
            words = self.page_bytes // 4
            for p, (a, b) in enumerate(zip(self.planes, self.want.planes)):
                a = a.cpu().numpy()
                assert np.array_equal(a[:, :words], b), p
                assert np.array_equal(a[:, words:], self.between[p])

    def extend(self, rows, counts, n_slots=None):
        n = len(rows) if rows is not None else len(counts) if counts is not None else len(self.want.lens)
        total = n if counts is None else sum(max(0, c) for c in counts)
        n_slots = total if n_slots is None else n_slots
        slots = torch.full((total + 1,), -9, dtype=torch.int64, device=DEV)
        pos = torch.full((total + 1,), -9, dtype=torch.int32, device=DEV)
        ws, b = self.ws(n)
        lists = [None if x is None else torch.tensor(x, dtype=torch.int32, device=DEV) for x in (rows, counts)]
        fdd.fdy_pages_extend(self.desc, *lists, n, slots, pos, n_slots, ws, b, self.status)
        s, p = self.want.extend(range(n) if rows is None else rows, counts, n_slots)
        self.same()
        k = min(total, n_slots)
        assert slots[:k].cpu().tolist() == s[:k].tolist() and pos[:k].cpu().tolist() == p[:k].tolist()
        assert bool((slots[k:] == -9).all()) and bool((pos[k:] == -9).all())
        return s

    def fork(self, src, dst):
        ws, b = self.ws(len(src))
        a, c = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (src, dst))
        fdd.fdy_pages_fork(self.desc, a, c, len(src), ws, b, self.status)
        self.want.fork(src, dst)
        self.same()

    def free(self, rows):
        fdd.fdy_pages_free(self.desc, torch.tensor(rows, dtype=torch.int32, device=DEV), len(rows), self.status)
        self.want.free(rows)
        self.same()

    def compact(self):
        to = torch.full((len(self.want.refs) + 1,), -9, dtype=torch.int32, device=DEV)
        live = torch.full((1,), -9, dtype=torch.int32, device=DEV)
        ws, b = self.ws(0)
        fdd.fdy_pages_compact(self.desc, to, live, ws, b, self.status)
        m, n = self.want.compact()
        self.same()
        assert to.cpu().tolist() == m.tolist() + [-9] and int(live) == n


def books(rng, n_pages, n_rows, row_pages, pt, shared=0.3, fill=0.6):
    """Rows of random lengths; a row goes on from the first pages of an earlier one with probability `shared`."""
    refs, table, lens = np.zeros(n_pages, int), np.full((n_rows, row_pages), -5, int), np.zeros(n_rows, int)
    free = list(rng.permutation(n_pages))
    for r in range(n_rows):
        n = int(rng.integers(0, row_pages * pt + 1)) if rng.random() < 0.9 else 0
        pages = -(-n // pt)
        k = 0
        if r and rng.random() < shared:
            o = int(rng.integers(0, r))
            have = -(-lens[o] // pt)
            if rng.random() < 0.5:
                n, pages = int(lens[o]), have
                k = have
            else:
                k = min(pages, have)
            table[r, :k] = table[o, :k]
        while pages - k > len(free) - (1 - fill) * n_pages and pages > k:
            pages -= 1
            n = min(n, pages * pt)
        for j in range(k, pages):
            table[r, j] = free.pop()
        lens[r] = n
        for j in range(-(-n // pt)):
            refs[table[r, j]] += 1
    return refs, table, lens


@pytest.mark.parametrize("n_pages", [1, 2, 63, 64, 65, 128, 200])
def test_reset(n_pages):
    p = Pool([3] * n_pages, [[0] * 4] * 7, [5] * 7, 16)
    fdd.fdy_pages_reset(p.desc)
    p.want.refs, p.want.lens = [0] * n_pages, [0] * 7
    p.same()


@pytest.mark.parametrize("seed", range(12))
def test_random_calls(seed):
    rng = np.random.default_rng(100 + seed)
    pt = [1, 2, 16, 64][seed % 4]
    n_rows, row_pages = int(rng.integers(2, 40)), int(rng.integers(1, 9))
    n_pages = int(rng.integers(20, 300))
    refs, table, lens = books(rng, n_pages, n_rows, row_pages, pt)
    page_bytes, stride = [(16, 16), (48, 64), (4096 + 16, 4128), (32, 32)][int(rng.integers(0, 4))]
    p = Pool(refs, table, lens, pt, n_planes=int(rng.integers(0, 4)), page_bytes=page_bytes, stride=stride, seed=seed)
    p.same()
    for _ in range(8):
        what = rng.integers(0, 5)
        n = int(rng.integers(1, n_rows + 1))
        some = [int(x) for x in rng.permutation(n_rows)[:n]]
        if what == 0:
            p.extend(some if rng.random() < 0.7 else None, None)
        elif what == 1:
            p.extend(some, [int(x) for x in rng.integers(0, 2 * pt + 3, n)])
        elif what == 2:
            p.fork([int(x) for x in rng.integers(0, n_rows, n)], some)
        elif what == 3:
            p.free(some[: max(1, n // 3)])
        else:
            p.compact()


def test_beams_that_share_a_last_page():
    """Four rows of one partly filled page: three copy, the last in the list keeps it; a fifth holder outside keeps all."""
    for extra in (0, 1):
        table = [[3, 1, 0], [3, 1, 0], [3, 1, 0], [3, 1, 0], [3, 1, 0]]
        lens = [20, 20, 20, 20, 20 if extra else 0]
        refs = [0, 4 + extra, 0, 4 + extra, 0, 0, 0, 0, 0]
        p = Pool(refs, table, lens, 16, n_planes=2)
        p.extend([2, 0, 3, 1], None)
        assert p.want.refs[1] == 1 and len(set(p.want.table[:4, 1])) == 4
        p.extend([0, 1, 2, 3], [1, 2, 13, 40])
        p.compact()


def test_no_pages_left():
    table = [[0, -1, -1, -1], [1, -1, -1, -1], [2, -1, -1, -1], [2, -1, -1, -1], [-1] * 4]
    p = Pool([1, 1, 2, 0, 0], table, [16, 7, 5, 5, 0], 16, n_planes=1)
    p.extend(None, [20, 1, 1, 1, 30])  # two for the first, one copy wanted, two for the last: two are there
    assert p.want.status == od.ST_CAPACITY
    p.status.zero_()
    p.want.status = 0
    p.free([0])
    p.extend(None, [0, 60, 40, 1, 16])
    p.free([0, 1, 2, 3, 4])
    p.extend([4, 3], [64, 1])


def test_lists_that_name_a_row_twice_or_none():
    rng = np.random.default_rng(5)
    for bad in ([1, 2, 1, 3], [0, -1, 2, 9], [3, 3, 3, 3]):
        refs, table, lens = books(rng, 60, 4, 5, 8, fill=0.4)
        p = Pool(refs, table, lens, 8, n_planes=1)
        p.extend(bad, None)
        p.extend(bad, [2, 3, -4, 5])
        p.fork([0, 1, 2, 3], bad)
        p.fork(bad, [2, 0, 3, 1])
        p.free(bad)
        assert p.want.status & od.ST_BAD_INDEX


def test_fewer_slots_than_tokens():
    p = Pool([0] * 50, [[-1] * 8] * 4, [0] * 4, 4)
    p.extend(None, [5, 6, 7, 8], n_slots=15)  # the third and the fourth end behind it
    assert p.want.lens == [5, 6, 0, 0] and p.want.status == od.ST_CAPACITY
    p.extend([3, 0, 1, 2], None, n_slots=3)


def test_rows_that_are_full():
    p = Pool([1, 1] + [0] * 20, [[0, -1], [1, -1]], [4, 3], 4)
    p.extend(None, [5, 5])
    assert p.want.lens == [4, 8]
    p.extend(None, [4, 1])


@pytest.mark.parametrize("src,dst", [([1, 0], [0, 1]), ([1, 2, 3, 0], [0, 1, 2, 3]), ([0, 0, 0, 0], [0, 1, 2, 3]),
                                     ([2], [2]), ([3, 3], [1, 0]), ([0, 1, 2, 3], [3, 2, 1, 0])])
def test_forks_of_rows_that_are_sources_too(src, dst):
    rng = np.random.default_rng(8)
    refs, table, lens = books(rng, 100, 5, 6, 16)
    p = Pool(refs, table, lens, 16)
    p.fork(src, dst)
    p.fork(src, dst)


def test_long_rows():
    rng = np.random.default_rng(9)
    refs, table, lens = books(rng, 60000, 9, 5000, 2, shared=0.6)
    p = Pool(refs, table, lens, 2)
    p.fork([8, 1, 2, 3], [0, 5, 3, 2])
    p.extend(None, [300] * 9)
    p.free([1, 4])
    p.compact()


def test_large_pools_and_lists():
    rng = np.random.default_rng(10)
    n_pages, n_rows = 150_001, 3000
    refs, table, lens = np.zeros(n_pages, int), np.full((n_rows, 40), -1, int), rng.integers(0, 30 * 16, n_rows)
    page = rng.permutation(n_pages)
    at = 0
    for r in range(n_rows):
        k = -(-int(lens[r]) // 16)
        table[r, :k] = page[at:at + k]
        at += k
    refs[page[:at]] = 1
    p = Pool(refs, table, lens, 16, n_planes=1, page_bytes=16, stride=16)
    p.fork([int(x) for x in rng.integers(0, n_rows, 1500)], [int(x) for x in rng.permutation(n_rows)[:1500]])
    p.extend(None, None)
    p.extend([int(x) for x in rng.permutation(n_rows)], [int(x) for x in rng.integers(0, 40, n_rows)])
    p.compact()


@pytest.mark.parametrize("refs", [[0] * 70, [1] * 70, [0] * 69 + [1], [1] + [0] * 69, [1, 0] * 35, [1]])
def test_compact_edges(refs):
    held = [p for p, c in enumerate(refs) if c]
    p = Pool(refs, [held + [-1]], [len(held) * 8 - (3 if held else 0)], 8, n_planes=3)
    p.compact()
    p.compact()


def test_numbers_out_of_range_in_the_books():
    """No access out of bounds; the good rows' results are as ever."""
    table = [[0, 1], [99, -4], [2, 3], [4, 5]]
    p = Pool([1] * 6 + [0] * 10, table, [9, 12, 1000, -8], 8, n_planes=1)
    ws, b = p.ws(4)
    slots = torch.zeros(4, dtype=torch.int64, device=DEV)
    fdd.fdy_pages_extend(p.desc, None, None, 4, slots, None, 4, ws, b, p.status)
    assert slots.cpu().tolist() == [9 + 0 * 8, -1, -1, -1] or slots.cpu().tolist()[1:] == [-1, -1, -1]
    assert int(slots[0]) == 1 * 8 + 1 and int(p.status) == od.ST_BAD_INDEX
    for call in (lambda: fdd.fdy_pages_fork(p.desc, torch.tensor([1, 2], dtype=torch.int32, device=DEV),
                                            torch.tensor([3, 0], dtype=torch.int32, device=DEV), 2, ws, b, p.status),
                 lambda: fdd.fdy_pages_compact(p.desc, None, None, ws, b, p.status),
                 lambda: fdd.fdy_pages_free(p.desc, torch.tensor([0, 1, 2, 3], dtype=torch.int32, device=DEV), 4, p.status),
                 lambda: fdd.fdy_pages_copy(p.desc, torch.tensor([1, 77], dtype=torch.int32, device=DEV),
                                            torch.tensor([-1, 3], dtype=torch.int32, device=DEV), 2, p.status)):
        p.status.zero_()
        call()
        torch.cuda.synchronize()
        assert int(p.status) == od.ST_BAD_INDEX


def test_copy_of_listed_pages():
    rng = np.random.default_rng(12)
    p = Pool([0] * 40, [[-1]], [0], 16, n_planes=5, page_bytes=8192 + 16, stride=8448)
    order = rng.permutation(40)
    src, dst = order[:20], order[20:]
    fdd.fdy_pages_copy(p.desc, *(torch.from_numpy(x.astype(np.int32)).to(DEV) for x in (src, dst)), 20, p.status)
    p.want.planes[:, dst] = p.want.planes[:, src]
    p.same()


def test_planes_wider_than_32_bits():
    """Two pages 5 GiB apart in one plane."""
    stride = 5 << 30
    plane = torch.empty((stride + 1024) // 8, dtype=torch.int64, device=DEV)
    plane[:128] = torch.arange(128, device=DEV)
    addr = torch.tensor([plane.data_ptr()], dtype=torch.int64, device=DEV)
    refs, bits = torch.tensor([2, 0], dtype=torch.int32, device=DEV), torch.tensor([2], dtype=torch.int64, device=DEV)
    table, lens = torch.zeros(2, 1, dtype=torch.int32, device=DEV), torch.tensor([3, 3], dtype=torch.int32, device=DEV)
    desc = fdd.make_pages(refs=refs, free_bits=bits, table=table, lens=lens, page_tokens=16, planes=addr, page_bytes=1024,
                          page_stride=stride)
    n = fdd.fdy_pages_workspace_bytes(desc, 2)
    slots = torch.zeros(2, dtype=torch.int64, device=DEV)
    fdd.fdy_pages_extend(desc, None, None, 2, slots, None, 2, torch.empty(n, dtype=torch.uint8, device=DEV), n)
    assert slots.cpu().tolist() == [16 + 3, 3]
    assert torch.equal(plane[stride // 8:stride // 8 + 128], torch.arange(128, device=DEV))


def test_replays():
    """extend, fork and free captured together; every replay against the same calls on the lists."""
    rng = np.random.default_rng(14)
    refs, table, lens = books(rng, 300, 12, 20, 4, fill=0.3)
    lens = np.minimum(lens, 40)
    refs = np.zeros(300, int)
    for r in range(12):
        for q in table[r, :-(-lens[r] // 4)]:
            refs[q] += 1
    p = Pool(refs, table, lens, 4, n_planes=2)
    src, dst = [0, 1, 2, 3], [5, 6, 1, 8]
    d = [torch.tensor(x, dtype=torch.int32, device=DEV) for x in (src, dst, [10])]
    ws, b = p.ws(12)
    slots, pos = torch.zeros(12, dtype=torch.int64, device=DEV), torch.zeros(12, dtype=torch.int32, device=DEV)

    def calls():
        fdd.fdy_pages_fork(p.desc, d[0], d[1], 4, ws, b, p.status)
        fdd.fdy_pages_extend(p.desc, None, None, 12, slots, pos, 12, ws, b, p.status)
        fdd.fdy_pages_free(p.desc, d[2], 1, p.status)

    kept = [x.clone() for x in (p.refs, p.bits, p.table, p.lens, *p.planes)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for x, y in zip((p.refs, p.bits, p.table, p.lens, *p.planes), kept):
        x.copy_(y)
    for _ in range(5):
        graph.replay()
        p.want.fork(src, dst)
        s, q = p.want.extend(None, [1] * 12, 12)
        p.want.free([10])
        p.same()
        assert slots.cpu().tolist() == s.tolist() and pos.cpu().tolist() == q.tolist()


@pytest.mark.parametrize("more", [0, 1500])
def test_rows_that_keep_a_page_wait_for_the_other_holders(more):
    """Pairs of rows of one partly filled page each, pages short: where the first of a pair gets no copy the second must not go
    on in the page.  `more` rows behind them have room in pages of their own (long lists are kept by another kernel)."""
    for pages_left in (0, 1, 2, 3):
        for rows in ([0, 1, 2, 3], [2, 0, 1, 3], [1, 0, 3, 2], [3, 1, 2, 0], [0, 1], [2, 3, 1]):
            own = list(range(4, 4 + more))
            table = [[0, -1], [0, -1], [1, -1], [1, -1]] + [[r - 2, -1] for r in own]
            refs = [2, 2] + [1] * more + [0] * pages_left
            p = Pool(refs, table, [5, 5, 9, 9] + [3] * more, 16, n_planes=1)
            p.extend(rows + own, None)
            p.extend(list(reversed(rows)) + own, [1 + (r == 2) for r in rows] + [2] * more)
            p.extend(own + rows, [1] * more + [12 if r == 1 else 1 for r in rows])


@pytest.mark.parametrize("seed", range(6))
def test_beams_in_a_pool_that_runs_out(seed):
    rng = np.random.default_rng(200 + seed)
    pt, beams, groups = 8, 2 + seed % 3, [6, 500][seed % 2]
    lens = np.repeat(rng.integers(1, 3 * pt, groups), beams)
    pages = -(-lens[::beams] // pt)
    table, refs = np.full((groups * beams, 6), -1, int), np.zeros(int(pages.sum()) + groups * beams // 2, int)
    order, at = rng.permutation(len(refs)), 0
    for g, k in enumerate(pages):
        table[g * beams:(g + 1) * beams, :k] = order[at:at + k]
        refs[order[at:at + k]] = beams
        at += k
    p = Pool(refs, table, lens, pt, n_planes=1, page_bytes=16, stride=16)
    for _ in range(4):
        p.extend([int(r) for r in rng.permutation(len(lens))], [int(c) for c in rng.integers(0, 3, len(lens))])
        src, dst = rng.permutation(len(lens))[:5], rng.permutation(len(lens))[:5]
        p.fork([int(x) for x in src], [int(x) for x in dst])
